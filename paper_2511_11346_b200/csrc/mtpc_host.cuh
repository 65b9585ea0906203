// What the host side of the calls beside the head shares: sizes, alignments, and whether there is a device to launch on.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mtpc.h"

namespace mtpc {

constexpr size_t kAlign = 256;
constexpr int kMaxRows = 1 << 30;
constexpr int kSms = 148;               // what grids are sized for: the results of sums that are cut by them do not depend on the device
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline size_t element(int dtype) { return dtype == MTPC_F32 ? 4 : 2; }
inline bool known(int dtype) { return dtype == MTPC_F32 || dtype == MTPC_BF16; }

// The current device is one that the library is built for.
inline int check_device() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess || major != 10) {
    cudaGetLastError();
    return MTPC_ERR_CUDA;
  }
  return MTPC_OK;
}

// Rows of a matrix of the caller: every row starts where vectors of `vec` elements may. An absent matrix allows anything.
inline bool rows_allow(const void* p, int64_t stride, size_t element_bytes, int vec, int rows) {
  return p == nullptr || (aligned(p, element_bytes * vec) && (rows <= 1 || stride % vec == 0));
}
// Rows that are read may lie anywhere, also all in one place (stride 0); rows that are written must not overlap.
inline bool input_rows(const void* p, int64_t stride, int rows) { return p == nullptr || rows <= 1 || stride >= 0; }
inline bool output_rows(const void* p, int64_t stride, int rows, int d) { return p == nullptr || rows <= 1 || stride >= d; }

inline int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }
inline int round_warp(int x) { return (x + 31) / 32 * 32; }

}  // namespace mtpc
