// How the host side launches a kernel.
#pragma once
#include <cuda_runtime.h>
#include <string.h>

#include "../../include/mtpc.h"

namespace mtpc {

inline int check_launch() { return cudaGetLastError() == cudaSuccess ? MTPC_OK : MTPC_ERR_CUDA; }

// Launch `kernel`, optionally allowed to start before the kernel ahead of it in the stream has finished (programmatic
// dependent launch): such a kernel calls grid_dependency_wait() before it touches global memory, so what overlaps is its launch and
// set-up (about 2 us a kernel). cluster > 1: in clusters of that many CTAs.
// Eight kernels do more before they wait. A kernel that lets its dependents in after its own wait (a gate) has nothing unfinished ahead of
// it, so whatever was launched before it has ended when anything behind it starts; each of the eight relies on one:
//   draft_slot_kernel, circuit_hmm_kernel and the static HMM's Eq. 6 kernel copy the head's static tables. The tables are written by a plain
//     launch (bind_parameters), and the first kernel of every call that runs one of the three is a gate (the fp32 conversion, the projection,
//     the weight pass; an acceptance call, whose first kernel may be circuit_hmm_kernel, needs a draft since the last update).
//   loss_coeff_kernel reads the targets and writes the coefficients. The projection it is launched behind is a gate (on a factored head the
//     merge), so the caller's writes and the readers of the last call's coefficients are done.
//   loss_partial_kernel, beside the last GEMM, reads the prefixes and writes its partial sums. The GEMMs are NOT gates, they let their
//     dependents in before they wait. What lies between them and the circuit is: logit_gradient_kernel, by its plain launch, or on a factored
//     head lowrank_pad_kernel. Whoever makes the one a dependent or lets the other's dependents in early breaks the loss.
//   adapted_gemm_kernel reads the rows, W and row_adaptor, and waits for the terms of low (or v) where it comes to them; ahead of it is
//     adaptor_low_kernel, a gate, or itself. It is a gate too: its epilogue's warps wait first, and they alone let its dependents in.
//   adapted_rows_kernel reads x, W, A and row_adaptor and waits for low; ahead of it is low_rows_kernel, a gate. (Where it forms low itself it
//     waits before it reads; what it does ahead of that is to ask W into L2.)
//   adaptor_grad_kernel reads the bitmaps, the terms and the rows, and writes dA, dB and their parts. Ahead of it is the product, a gate, so
//     adaptor_low_kernel has ended, and with it whatever used these buffers before the call; nothing in it needs the product. It lets its
//     dependents in at once and waits at its end. So it is NOT a gate: what is behind it waits before it touches memory, and when it has ended
//     so has the product. Without a product ahead (after_low) it waits first.
template <typename... Params, typename... Args>
void launch_clusters(void (*kernel)(Params...), int cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool dependent,
                     Args&&... args) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (dependent) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
void launch_kernel(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool dependent, Args&&... args) {
  launch_clusters(kernel, 1, grid, block, smem, st, dependent, args...);
}

}  // namespace mtpc
