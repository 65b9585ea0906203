// Host side of the calls of a training or decoding step that need no head (include/mtpc.h): embeddings, the residual norm, the gradients'
// norm. Argument checks, carving of the caller's workspace, choice of the build, launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>
#include <new>

#include "../../include/mtpc.h"
#include "mtpc_clip.cuh"
#include "mtpc_embed.cuh"
#include "mtpc_host.cuh"
#include "mtpc_launch.cuh"
#include "mtpc_norm.cuh"

namespace {

using namespace mtpc;

constexpr long long kClearBesideChunks = 32 << 20;    // bytes
constexpr long long kFewBytes = 32 << 20;

// Whether rows start off their vectors of eight elements alike in all of some matrices: then *shift and *pitch say how (SplitRow). Absent ones are left out.
struct RowsOf {
  const void* p;
  int64_t stride;
  size_t element_bytes;
};
bool rows_alike(std::initializer_list<RowsOf> all, int* shift, int* pitch) {
  bool first = true;
  for (const RowsOf& m : all) {
    if (m.p == nullptr) continue;
    const int s = static_cast<int>(reinterpret_cast<uintptr_t>(m.p) / m.element_bytes % 8), q = static_cast<int>(((m.stride % 8) + 8) % 8);
    if (!first && (s != *shift || q != *pitch)) return false;
    *shift = s;
    *pitch = q;
    first = false;
  }
  return true;
}

// ---------------------------------------------------------------- residual norm
// How the rows of a call are read: as vectors, as vectors between single elements, or element by element.
enum RowPath { kRowVectors, kRowSplit, kRowElements };
template <typename IO, bool SPLIT>
void launch_rmsnorm_vectors(const NormArgs& a, cudaStream_t st) {
  const int packs = ceil_div(a.d, 8);
  // Blocks of 256 threads on an SM: bf16 six instead of five (2005 rows of 4096 to 8 bits 14.1 for 14.4 us), where fp32 would spill (8192 rows 87 for 80).
  constexpr int kCtas = sizeof(IO) == 2 && !SPLIT ? 6 : 4;
  if (packs <= 32)
    launch_kernel(residual_rmsnorm_kernel<IO, 1, 256, 6, SPLIT>, ceil_div(a.T, 8), dim3(32, 8), 0, st, true, a);
  else if (packs <= 64)
    launch_kernel(residual_rmsnorm_kernel<IO, 2, 256, kCtas, SPLIT>, ceil_div(a.T, 8), dim3(32, 8), 0, st, true, a);
  else if (packs <= 512)
    launch_kernel(residual_rmsnorm_kernel<IO, 2, 256, kCtas, SPLIT>, a.T, round_warp(ceil_div(packs, 2)), 0, st, true, a);
  else if (packs <= 1024)
    launch_kernel(residual_rmsnorm_kernel<IO, 2, 512, 2, SPLIT>, a.T, round_warp(ceil_div(packs, 2)), 0, st, true, a);
  else
    launch_kernel(residual_rmsnorm_kernel<IO, 4, 1024, 1, SPLIT>, a.T, round_warp(ceil_div(packs, 4)), 0, st, true, a);
}
template <typename IO>
void launch_rmsnorm(const NormArgs& a, RowPath path, cudaStream_t st) {
  if (path == kRowVectors) launch_rmsnorm_vectors<IO, false>(a, st);
  else if (path == kRowSplit) launch_rmsnorm_vectors<IO, true>(a, st);
  else if (a.d <= 4096) launch_kernel(residual_rmsnorm_plain_kernel<IO, 4>, a.T, round_warp(ceil_div(a.d, 4)), 0, st, true, a);
  else launch_kernel(residual_rmsnorm_plain_kernel<IO, 32>, a.T, round_warp(ceil_div(a.d, 32)), 0, st, true, a);
}

// Blocks of the gradient kernel: as many as an SM takes, of two rows (a warp) at least where there are rows for every SM.
constexpr int kGradRows = 8;            // rows of a block whose warps have one each, d <= 256
int norm_grad_blocks(int T, int d, int vectors_a_thread = 2) {
  const int per_sm = d > 4096 ? 1 : std::max(1, std::min(16, 512 / round_warp(ceil_div(d, 8 * vectors_a_thread))));
  return std::min(T, std::max(kSms, std::min(kSms * per_sm, T / 2)));
}
// Returns the blocks launched, each of which leaves its part of d weight.
template <typename IO, typename DY, typename DX, bool SPLIT>
int launch_rmsnorm_grad_vectors(const NormGradArgs& a, cudaStream_t st) {
  const int packs = ceil_div(a.d, 8);
  // Two vectors a thread where a row ahead of them fits the registers and a warp has that many, else one; us, two / one: 8192 rows of 4096, d_out fp32,
  // all else bf16 57 / 64, fp32 sum 94 / 70, fp32 d_x 107 / 80, all fp32 124 / 86; 16384 rows, all bf16: of 2048 57 / 67, of 1024 34.6 / 36.9, of
  // 512 24.7 / 23.9; of 2047, in split rows, 68 / 64.
  constexpr bool kNarrow = !SPLIT && sizeof(IO) + sizeof(DY) + sizeof(DX) <= 8;
  const int nv = packs > 512 || (kNarrow && packs > 64) ? 2 : 1, threads = round_warp(ceil_div(packs, nv));
  int blocks = packs <= 32 ? std::min(ceil_div(a.T, kGradRows), 2 * kSms) : norm_grad_blocks(a.T, a.d, nv);
  if (SPLIT && packs > 32 && blocks < a.T) blocks = std::max(8, blocks / 8 * 8);        // a block's rows start alike
  if (packs <= 32)
    launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 1, 256, 2, SPLIT, kGradRows>, blocks, dim3(32, kGradRows), 0, st, true, a);
  else if (threads <= 256 && nv == 1)
    launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 1, 256, 2, SPLIT, 1>, blocks, threads, 0, st, true, a);
  else if (nv == 1)
    launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 1, 512, 1, SPLIT, 1>, blocks, threads, 0, st, true, a);
  else if constexpr (kNarrow) {
    if (threads <= 256) launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 2, 256, 2, SPLIT, 1>, blocks, threads, 0, st, true, a);
    else launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 2, 512, 1, SPLIT, 1>, blocks, threads, 0, st, true, a);
  } else
    launch_kernel(rmsnorm_grad_kernel<IO, DY, DX, 2, 512, 1, SPLIT, 1>, blocks, threads, 0, st, true, a);
  return blocks;
}
template <typename IO, typename DY, typename DX>
int launch_rmsnorm_grad(const NormGradArgs& a, RowPath path, cudaStream_t st) {
  const int packs = ceil_div(a.d, 8);
  if (packs <= 1024 && path != kRowElements)
    return path == kRowVectors ? launch_rmsnorm_grad_vectors<IO, DY, DX, false>(a, st) : launch_rmsnorm_grad_vectors<IO, DY, DX, true>(a, st);
  const int blocks = norm_grad_blocks(a.T, a.d);
  if (path == kRowVectors)
    launch_kernel(rmsnorm_grad_plain_kernel<IO, DY, DX, 8, 4>, blocks, round_warp(ceil_div(packs, 4)), 0, st, true, a);
  else if (a.d <= 4096)
    launch_kernel(rmsnorm_grad_plain_kernel<IO, DY, DX, 1, 4>, blocks, round_warp(ceil_div(a.d, 4)), 0, st, true, a);
  else
    launch_kernel(rmsnorm_grad_plain_kernel<IO, DY, DX, 1, 32>, blocks, round_warp(ceil_div(a.d, 32)), 0, st, true, a);
  return blocks;
}
template <typename IO, typename DY>
int launch_rmsnorm_grad(const NormGradArgs& a, int dx_dtype, RowPath path, cudaStream_t st) {
  return dx_dtype == MTPC_F32 ? launch_rmsnorm_grad<IO, DY, float>(a, path, st) : launch_rmsnorm_grad<IO, DY, __nv_bfloat16>(a, path, st);
}

// ---------------------------------------------------------------- embedding
struct EmbedPlan {
  int range;                            // tokens of a block of embed_order_kernel (0: the digits' kernels sort)
  int digits, rounds, tiles;
  int threads, chunk, chunks;           // of the sums
  size_t off_key[2], off_pos[2], off_bounds, off_hist, off_part, total;
};
void plan_embed(int T, int v, int d, EmbedPlan* p) {
  memset(p, 0, sizeof(*p));
  int bits = 1;
  while ((static_cast<int64_t>(1) << bits) <= v) ++bits;                // keys run up to v
  // Every block of the one-launch sort reads all tokens, so there is one per SM (a second one on some of them takes twice as long), until a block's tokens
  // would be too many. One digit / the one launch, the whole gradient, 320 tokens: 8192 positions of 4096 41 / 37 us, 16384 of 1024 30.4 / 30.1,
  // 32768 of 1024 36.9 / 41.2; two digits, 30000 tokens: 16000 of 512 39 / 32, 32768 of 512 47 / 46.
  if (T <= (bits <= kSortDigit ? kOrderMaxT / 2 : kOrderMaxT)) p->range = std::min(kOrderMaxRange, ceil_div(v + 1, kSms));
  p->digits = p->range ? 1 : (bits + kSortDigit - 1) / kSortDigit;
  p->rounds = ceil_div(T, static_cast<long long>(kSortTile) * kSortMaxTiles);
  p->tiles = ceil_div(T, static_cast<long long>(kSortTile) * p->rounds);
  // Chunks of 8 positions at least, as many as give every SM the four blocks that it holds, of 256 threads with four columns each.
  p->threads = std::min(kSegmentThreads, round_warp(ceil_div(d, 4)));
  p->chunk = std::max(8, ceil_div(static_cast<long long>(T) * ceil_div(d, 4 * p->threads) * p->threads, kSms * 4 * kSegmentThreads));
  p->chunks = ceil_div(T, p->chunk);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  for (int i = 0; i < 2; ++i) {
    p->off_key[i] = take(i < p->digits ? static_cast<size_t>(T) * 4 : 0);
    p->off_pos[i] = take(i < p->digits ? static_cast<size_t>(T) * 4 : 0);
  }
  p->off_bounds = take((static_cast<size_t>(v) + 1) * sizeof(int2));
  p->off_hist = take(p->range ? 0 : static_cast<size_t>(p->tiles) * kSortBins * 4);
  p->off_part = take(static_cast<size_t>(p->chunks) * 2 * d * 4);
  p->total = off;
}

// The embedding gradient's kernels may use the shared memory that they ask for: said once on each device.
constexpr int kMaxDevices = 64;
int g_embed_allowed[kMaxDevices];
int allow_embed_gradient() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return MTPC_ERR_CUDA;
  if (__atomic_load_n(&g_embed_allowed[dev], __ATOMIC_ACQUIRE)) return MTPC_OK;
  const auto allow = [](auto* kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess;
  };
  if (!allow(embed_order_kernel, order_smem_bytes(kOrderMaxT))) return MTPC_ERR_CUDA;
  __atomic_store_n(&g_embed_allowed[dev], 1, __ATOMIC_RELEASE);
  return MTPC_OK;
}

int check_embed_sizes(int T, int v, int d) {
  if (T < 0 || v < 1 || d < 1) return MTPC_ERR_SHAPE;
  if (T > kEmbedMaxT || v > kEmbedMaxV || d > kEmbedMaxD) return MTPC_ERR_UNSUPPORTED;
  return MTPC_OK;
}

template <typename TI, typename TO>
void launch_embed(const EmbedArgs& a, bool vectors, cudaStream_t st) {
  int share = 8;                        // threads to a row
  while (share < 256 && share * 8 < a.d) share <<= 1;
  const int rows = 256 / share;
  if (!vectors)
    launch_kernel(embed_split_kernel<TI, TO>, ceil_div(a.T, rows), dim3(share, rows), 0, st, true, a);
  else if (a.T >= 4 * kSms * 8)
    launch_kernel(embed_kernel<TI, TO, 8, 4>, ceil_div(a.T, rows * 4), dim3(share, rows), 0, st, true, a);
  else                                  // few rows: their columns over several blocks
    launch_kernel(embed_kernel<TI, TO, 8, 1>, dim3(ceil_div(a.T, rows), ceil_div(a.d, share * 8)), dim3(share, rows), 0, st, true, a);
}

}  // namespace

struct mtpc_gradient_list {
  const ClipChunk* chunks;              // in the workspace
  double* partial;
  int count, blocks;
};

namespace {

// What a list of gradients needs: its chunks, and the sums of the first pass's blocks.
struct ListPlan {
  long long chunks;
  int blocks;
  size_t off_partial, total;
};
bool same_place(const mtpc_gradient& e) { return e.out == e.data; }
// Elements of an entry before the first that vectors of eight may start at, for both of its addresses; -1: there is none for both.
int wide_head(const mtpc_gradient& e) {
  const int at = static_cast<int>(reinterpret_cast<uintptr_t>(e.data) / element(e.dtype) % 8);
  if (e.out && static_cast<int>(reinterpret_cast<uintptr_t>(e.out) / element(e.out_dtype) % 8) != at) return -1;
  return (8 - at) % 8;
}
int plan_list(const mtpc_gradient* entries, int32_t count, ListPlan* p) {
  if (count < 0) return MTPC_ERR_SHAPE;
  if (count > 0 && !entries) return MTPC_ERR_NULL;
  p->chunks = 0;
  for (int i = 0; i < count; ++i) {
    const mtpc_gradient& e = entries[i];
    if (e.count < 0 || e.count > (static_cast<int64_t>(1) << 40) || !known(e.dtype) || (e.out && !known(e.out_dtype))) return MTPC_ERR_SHAPE;
    if (e.count == 0) continue;
    if (!e.data) return MTPC_ERR_NULL;
    if (!aligned(e.data, element(e.dtype)) || (e.out && !aligned(e.out, element(e.out_dtype)))) return MTPC_ERR_SHAPE;
    if (e.out && same_place(e) && e.dtype != e.out_dtype) return MTPC_ERR_SHAPE;
    p->chunks += (e.count + kClipChunk - 1) / kClipChunk;
    if (p->chunks > (1 << 30)) return MTPC_ERR_UNSUPPORTED;
  }
  // One wave of blocks, or up to kClipWaves of them with 16 chunks each (the waves follow each other through the list, so that the second pass finds
  // more of what the first one left in L2: 671 MB 306 us in eight waves, 327 in one; 78 MB, where each block's sum of the others' counts, 47 and 41).
  const long long waves = std::max<long long>(1, std::min<long long>(kClipWaves, p->chunks / (16 * kClipBlocks)));
  const long long rounds = std::max<long long>(1, (p->chunks + waves * kClipBlocks - 1) / (waves * kClipBlocks));
  p->blocks = static_cast<int>(std::max<long long>(1, (p->chunks + rounds - 1) / rounds));      // every block as many chunks, but for one
  p->off_partial = align_up(static_cast<size_t>(p->chunks) * sizeof(ClipChunk));
  p->total = p->off_partial + align_up(static_cast<size_t>(p->blocks) * sizeof(double));
  return MTPC_OK;
}

// No result may lie where another result or another entry's gradient does: the passes read and write them in no order.
struct Span {
  uintptr_t begin, end;
  bool written;
};
int check_overlap(const mtpc_gradient* entries, int32_t count) {
  Span* spans = new (std::nothrow) Span[2 * static_cast<size_t>(count) + 1];
  if (!spans) return MTPC_ERR_CUDA;
  size_t n = 0;
  for (int i = 0; i < count; ++i) {
    const mtpc_gradient& e = entries[i];
    if (e.count == 0) continue;
    const uintptr_t in = reinterpret_cast<uintptr_t>(e.data), to = reinterpret_cast<uintptr_t>(e.out);
    if (!e.out || !same_place(e)) spans[n++] = {in, in + static_cast<size_t>(e.count) * element(e.dtype), false};
    if (e.out) spans[n++] = {to, to + static_cast<size_t>(e.count) * element(e.out_dtype), true};
  }
  std::sort(spans, spans + n, [](const Span& x, const Span& y) { return x.begin < y.begin; });
  uintptr_t any = 0, written = 0;       // where what lies before ends
  int rc = MTPC_OK;
  for (size_t i = 0; i < n; ++i) {
    if (spans[i].begin < (spans[i].written ? any : written)) rc = MTPC_ERR_SHAPE;
    any = std::max(any, spans[i].end);
    if (spans[i].written) written = std::max(written, spans[i].end);
  }
  delete[] spans;
  return rc;
}

}  // namespace

extern "C" {

int mtpc_embed(const int32_t* tokens, int32_t T, const void* table, int64_t table_stride, int32_t table_dtype, int32_t v, int32_t d,
               float scale, void* out, int64_t out_stride, int32_t out_dtype, uint32_t* out_status, void* stream) {
  int rc = check_embed_sizes(T, v, d);
  if (rc != MTPC_OK) return rc;
  if (!known(table_dtype) || !known(out_dtype)) return MTPC_ERR_SHAPE;
  if (T == 0) return MTPC_OK;
  if (!tokens || !table || !out) return MTPC_ERR_NULL;
  if (!input_rows(table, table_stride, v) || !output_rows(out, out_stride, T, d)) return MTPC_ERR_SHAPE;
  if (!aligned(tokens, 4) || !aligned(table, element(table_dtype)) || !aligned(out, element(out_dtype)) || !aligned(out_status, 4)) return MTPC_ERR_SHAPE;
  if ((rc = check_device()) != MTPC_OK) return rc;
  EmbedArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = tokens;
  a.table = table;
  a.out = out;
  a.status = out_status;
  a.table_stride = table_stride;
  a.out_stride = out_stride;
  a.T = T;
  a.v = v;
  a.d = d;
  a.scale = scale;
  rows_alike({{out, T > 1 ? out_stride : 0, element(out_dtype)}}, &a.shift, &a.pitch);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool vectors = d % 8 == 0 && rows_allow(table, table_stride, element(table_dtype), 8, v) && rows_allow(out, out_stride, element(out_dtype), 8, T);
  if (table_dtype == MTPC_F32) {
    if (out_dtype == MTPC_F32) launch_embed<float, float>(a, vectors, st);
    else launch_embed<float, __nv_bfloat16>(a, vectors, st);
  } else {
    if (out_dtype == MTPC_F32) launch_embed<__nv_bfloat16, float>(a, vectors, st);
    else launch_embed<__nv_bfloat16, __nv_bfloat16>(a, vectors, st);
  }
  return check_launch();
}

int mtpc_embed_backward_workspace_bytes(int32_t T, int32_t v, int32_t d, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  const int rc = check_embed_sizes(T, v, d);
  if (rc != MTPC_OK) return rc;
  EmbedPlan p;
  plan_embed(T > 0 ? T : 1, v, d, &p);
  *out_bytes = p.total;
  return MTPC_OK;
}

int mtpc_embed_backward(const int32_t* tokens, int32_t T, const void* d_out, int64_t d_out_stride, int32_t d_out_dtype, float scale,
                        int32_t v, int32_t d, float* d_table, int64_t d_table_stride, int32_t accumulate, void* workspace,
                        size_t workspace_bytes, uint32_t* out_status, void* stream) {
  int rc = check_embed_sizes(T, v, d);
  if (rc != MTPC_OK) return rc;
  if (!known(d_out_dtype)) return MTPC_ERR_SHAPE;
  if (!d_table || (T > 0 && (!tokens || !d_out || !workspace))) return MTPC_ERR_NULL;
  if (!input_rows(d_out, d_out_stride, T) || !output_rows(d_table, d_table_stride, v, d)) return MTPC_ERR_SHAPE;
  if (!aligned(tokens, 4) || !aligned(d_out, element(d_out_dtype)) || !aligned(d_table, 4) || !aligned(out_status, 4)) return MTPC_ERR_SHAPE;
  EmbedPlan p;
  plan_embed(T > 0 ? T : 1, v, d, &p);
  if (T > 0 && (workspace_bytes < p.total || !aligned(workspace, kAlign))) return MTPC_ERR_WORKSPACE;
  if (T == 0 && accumulate) return MTPC_OK;
  if ((rc = check_device()) != MTPC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (T == 0)                           // (not accumulated: the gradient is zeros)
    return cudaMemset2DAsync(d_table, static_cast<size_t>(v == 1 ? d : d_table_stride) * 4, 0, static_cast<size_t>(d) * 4, v, st) == cudaSuccess
               ? MTPC_OK : MTPC_ERR_CUDA;
  EmbedSegmentArgs a;
  memset(&a, 0, sizeof(a));
  a.key = reinterpret_cast<int*>(ws + p.off_key[0]);
  a.pos = reinterpret_cast<int*>(ws + p.off_pos[0]);
  a.bounds = reinterpret_cast<int2*>(ws + p.off_bounds);
  a.d_out = d_out;
  a.d_table = d_table;
  a.part = reinterpret_cast<float*>(ws + p.off_part);
  a.d_out_stride = d_out_stride;
  a.d_table_stride = d_table_stride;
  a.T = T;
  a.v = v;
  a.d = d;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  a.scale = scale;
  a.accumulate = accumulate != 0;
  const auto table_allows = [&](int vec) { return d % vec == 0 && rows_allow(d_table, d_table_stride, 4, vec, v); };
  a.row_vec = table_allows(8) ? 8 : table_allows(4) ? 4 : 1;
  const auto vectors = [&](int vec) {
    return table_allows(vec) && rows_allow(d_out, d_out_stride, element(d_out_dtype), vec, T);
  };
  const int vec = vectors(4) ? 4 : 1;
  // One launch for few positions, but where most of its time would be clearing (one launch / three, us: 128 positions, 5000 rows of 512 6.5 / 12.4,
  // 32768 rows 24 / 18.6), which it does row after row.
  if (T <= kFewT && (accumulate ? v <= 32768 : static_cast<long long>(v) * d * 4 <= kFewBytes)) {
    const int threads = std::min(kFewThreads, round_warp(ceil_div(d, vec)));
    const dim3 grid(std::min(v, kSms * 16), ceil_div(d, threads * vec));
    if (d_out_dtype == MTPC_F32)
      launch_kernel(vec == 4 ? embed_few_kernel<float, 4, 8> : embed_few_kernel<float, 1, 8>, grid, threads, 0, st, true, tokens, a, out_status);
    else
      launch_kernel(vec == 4 ? embed_few_kernel<__nv_bfloat16, 4, 8> : embed_few_kernel<__nv_bfloat16, 1, 8>, grid, threads, 0, st, true, tokens, a,
                    out_status);
    return check_launch();
  }
  if ((rc = allow_embed_gradient()) != MTPC_OK) return rc;
  EmbedSortArgs s;
  memset(&s, 0, sizeof(s));
  s.tokens = tokens;
  s.key_a = reinterpret_cast<int*>(ws + p.off_key[0]);
  s.pos_a = reinterpret_cast<int*>(ws + p.off_pos[0]);
  s.key_b = reinterpret_cast<int*>(ws + p.off_key[1]);
  s.pos_b = reinterpret_cast<int*>(ws + p.off_pos[1]);
  s.bounds = reinterpret_cast<int2*>(ws + p.off_bounds);
  s.hist = reinterpret_cast<uint2*>(ws + p.off_hist);
  s.status = out_status;
  s.d_out = d_out;
  s.d_out_stride = d_out_stride;
  s.T = T;
  s.v = v;
  s.d = d;
  s.range = p.range;
  s.digits = p.digits;
  s.tiles = p.tiles;
  s.rounds = p.rounds;
  s.d_out_bytes = static_cast<int>(element(d_out_dtype));
  if (p.range) {
    launch_kernel(embed_order_kernel, ceil_div(v + 1, p.range), kOrderThreads, order_smem_bytes(T), st, true, s);
  } else {
    for (int digit = 0; digit < p.digits; ++digit) {
      launch_kernel(embed_count_kernel, p.tiles + (digit == 0 ? kSms : 0), kSortThreads, 0, st, true, s, digit);
      launch_kernel(embed_scatter_kernel, p.tiles, kSortThreads, 0, st, true, s, digit);
    }
    if (p.digits > 1) launch_kernel(embed_bounds_kernel, std::min(ceil_div(T, 256), kSms * 8), 256, 0, st, true, s);
  }
  // Rows without positions are cleared beside the chunks where they are many, as much as the chunks take to run; the others beside the join, whose
  // blocks are short: in the chunks' launch the last ones would be theirs.
  const auto clear_blocks = [&]() { return std::min(ceil_div(a.clear_end - a.clear_begin, kClearRows), kSms * 256); };
  const long long table_bytes = static_cast<long long>(v) * d * 4;
  a.clear_end = accumulate || (p.chunks > 1 && table_bytes < 2 * kClearBesideChunks) ? 0 : p.chunks == 1 ? v : static_cast<int>(kClearBesideChunks / (d * 4LL));
  const int threads = std::min(p.threads, round_warp(ceil_div(d, vec)));
  a.slabs = ceil_div(d, threads * vec);
  auto* segment = d_out_dtype == MTPC_F32 ? (vec == 4 ? embed_segment_kernel<float, 4, 8> : embed_segment_kernel<float, 1, 8>)
                                          : (vec == 4 ? embed_segment_kernel<__nv_bfloat16, 4, 8> : embed_segment_kernel<__nv_bfloat16, 1, 8>);
  launch_kernel(segment, p.chunks * a.slabs + clear_blocks(), threads, 0, st, true, a);
  if (p.chunks > 1) {
    a.clear_begin = a.clear_end;
    a.clear_end = accumulate ? a.clear_begin : v;
    const int join_vec = vec == 1 ? 1 : 4;
    launch_kernel(join_vec == 4 ? embed_join_kernel<4> : embed_join_kernel<1>,
                  ceil_div(p.chunks, kJoinWarps) * ceil_div(d, 32 * join_vec) + clear_blocks(), 32 * kJoinWarps, 0, st, true, a);
  }
  return check_launch();
}

int mtpc_residual_rmsnorm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                          int32_t weight_dtype, int32_t T, int32_t d, int32_t io_dtype, float eps, void* out_sum, int64_t sum_stride,
                          void* out, int64_t out_stride, uint8_t* out_codes, int64_t codes_stride, float* out_scales,
                          int32_t scale_group, void* stream) {
  if (T < 0 || T > kMaxRows || d < 1 || !known(io_dtype) || !known(weight_dtype) || !(eps > 0.f) || isinf(eps)) return MTPC_ERR_SHAPE;
  if (d > kNormMaxWidth) return MTPC_ERR_UNSUPPORTED;
  if (scale_group != 0 && scale_group != 32 && scale_group != 64 && scale_group != 128) return MTPC_ERR_UNSUPPORTED;
  if (T == 0) return MTPC_OK;
  if (!x || (!out && !out_codes) || (out_codes != nullptr) != (out_scales != nullptr)) return MTPC_ERR_NULL;
  if (!input_rows(x, x_stride, T) || !input_rows(residual, residual_stride, T) || !output_rows(out_sum, sum_stride, T, d) ||
      !output_rows(out, out_stride, T, d) || !output_rows(out_codes, codes_stride, T, d))
    return MTPC_ERR_SHAPE;
  const size_t e = element(io_dtype);
  if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, element(weight_dtype)) || !aligned(out_sum, e) || !aligned(out, e) ||
      !aligned(out_scales, 4))
    return MTPC_ERR_SHAPE;
  int rc = check_device();
  if (rc != MTPC_OK) return rc;
  if (out && out == out_sum) return MTPC_ERR_SHAPE;          // one would be written over the other
  NormArgs a;
  memset(&a, 0, sizeof(a));
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.sum = out_sum;
  a.out = out;
  a.codes = out_codes;
  a.scales = out_scales;
  a.x_stride = x_stride;
  a.residual_stride = residual_stride;
  a.sum_stride = sum_stride;
  a.out_stride = out_stride;
  a.codes_stride = codes_stride;
  a.T = T;
  a.d = d;
  a.group = scale_group;
  a.groups = scale_group ? ceil_div(d, scale_group) : 1;
  while ((1 << a.group_shift) < scale_group) ++a.group_shift;
  a.weight_f32 = weight_dtype == MTPC_F32;
  a.eps = eps;
  a.width = static_cast<float>(d);
  a.inv_width = 1.f / a.width;
  const bool vectors = d % 8 == 0 && rows_allow(x, x_stride, e, 8, T) && rows_allow(residual, residual_stride, e, 8, T) &&
                       rows_allow(weight, 0, element(weight_dtype), 8, 1) && rows_allow(out_sum, sum_stride, e, 8, T) &&
                       rows_allow(out, out_stride, e, 8, T) && rows_allow(out_codes, codes_stride, 1, 8, T);
  const bool alike = (!out_codes || scale_group == 0) && rows_alike({{x, T > 1 ? x_stride : 0, e}, {residual, T > 1 ? residual_stride : 0, e},
      {out_sum, T > 1 ? sum_stride : 0, e}, {out, T > 1 ? out_stride : 0, e}, {out_codes, T > 1 ? codes_stride : 0, 1}}, &a.shift, &a.pitch);
  const RowPath path = vectors ? kRowVectors : alike ? kRowSplit : kRowElements;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (io_dtype == MTPC_F32) launch_rmsnorm<float>(a, path, st);
  else launch_rmsnorm<__nv_bfloat16>(a, path, st);
  return check_launch();
}

int mtpc_residual_rmsnorm_backward_workspace_bytes(int32_t T, int32_t d, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  if (T < 0 || T > kMaxRows || d < 1) return MTPC_ERR_SHAPE;
  if (d > kNormMaxWidth) return MTPC_ERR_UNSUPPORTED;
  *out_bytes = align_up(static_cast<size_t>(norm_grad_blocks(T > 0 ? T : 1, d)) * d * 4);
  return MTPC_OK;
}

int mtpc_residual_rmsnorm_backward(const void* sum, int64_t sum_stride, int32_t io_dtype, const void* weight, int32_t weight_dtype,
                                   int32_t T, int32_t d, float eps, const void* d_out, int64_t d_out_stride, int32_t d_out_dtype,
                                   const void* d_sum, int64_t d_sum_stride, void* d_x, int64_t d_x_stride, int32_t d_x_dtype,
                                   float* d_weight, void* workspace, size_t workspace_bytes, void* stream) {
  if (T < 0 || T > kMaxRows || d < 1 || !known(io_dtype) || !known(weight_dtype) || !known(d_out_dtype) || !known(d_x_dtype) ||
      !(eps > 0.f) || isinf(eps))
    return MTPC_ERR_SHAPE;
  if (d > kNormMaxWidth) return MTPC_ERR_UNSUPPORTED;
  if (T > 0 && (!sum || !d_out || !d_x || (d_weight && !workspace))) return MTPC_ERR_NULL;
  if (!input_rows(sum, sum_stride, T) || !input_rows(d_out, d_out_stride, T) || !input_rows(d_sum, d_sum_stride, T) ||
      !output_rows(d_x, d_x_stride, T, d))
    return MTPC_ERR_SHAPE;
  if (!aligned(sum, element(io_dtype)) || !aligned(weight, element(weight_dtype)) || !aligned(d_out, element(d_out_dtype)) ||
      !aligned(d_sum, element(d_x_dtype)) || !aligned(d_x, element(d_x_dtype)) || !aligned(d_weight, 4))
    return MTPC_ERR_SHAPE;
  const int blocks = norm_grad_blocks(T, d);
  if (d_weight && T > 0 && (workspace_bytes < align_up(static_cast<size_t>(blocks) * d * 4) || !aligned(workspace, kAlign))) return MTPC_ERR_WORKSPACE;
  if (T == 0 && !d_weight) return MTPC_OK;
  int rc = check_device();
  if (rc != MTPC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  NormGradArgs a;
  memset(&a, 0, sizeof(a));
  int parts = 0;                        // of d weight
  if (T > 0) {
    a.sum = sum;
    a.weight = weight;
    a.d_out = d_out;
    a.d_stream = d_sum;
    a.d_x = d_x;
    a.partial = d_weight ? static_cast<float*>(workspace) : nullptr;
    a.sum_stride = sum_stride;
    a.d_out_stride = d_out_stride;
    a.d_stream_stride = d_sum_stride;
    a.d_x_stride = d_x_stride;
    a.T = T;
    a.d = d;
    a.weight_f32 = weight_dtype == MTPC_F32;
    a.eps = eps;
    a.width = static_cast<float>(d);
    a.inv_width = 1.f / a.width;
    const bool vectors = d % 8 == 0 && rows_allow(sum, sum_stride, element(io_dtype), 8, T) && rows_allow(weight, 0, element(weight_dtype), 8, 1) &&
                         rows_allow(d_out, d_out_stride, element(d_out_dtype), 8, T) &&
                         rows_allow(d_sum, d_sum_stride, element(d_x_dtype), 8, T) && rows_allow(d_x, d_x_stride, element(d_x_dtype), 8, T);
    const auto rows = [&](const void* p, int64_t stride, int dtype) { return RowsOf{p, T > 1 ? stride : 0, element(dtype)}; };
    const bool alike = rows_alike({rows(sum, sum_stride, io_dtype), rows(d_out, d_out_stride, d_out_dtype), rows(d_sum, d_sum_stride, d_x_dtype),
                                   rows(d_x, d_x_stride, d_x_dtype)}, &a.shift, &a.pitch);
    const RowPath path = vectors ? kRowVectors : alike ? kRowSplit : kRowElements;
    if (io_dtype == MTPC_F32)
      parts = d_out_dtype == MTPC_F32 ? launch_rmsnorm_grad<float, float>(a, d_x_dtype, path, st)
                                      : launch_rmsnorm_grad<float, __nv_bfloat16>(a, d_x_dtype, path, st);
    else
      parts = d_out_dtype == MTPC_F32 ? launch_rmsnorm_grad<__nv_bfloat16, float>(a, d_x_dtype, path, st)
                                      : launch_rmsnorm_grad<__nv_bfloat16, __nv_bfloat16>(a, d_x_dtype, path, st);
  }
  if (d_weight)
    launch_kernel(norm_weight_grad_kernel, ceil_div(d, 32), dim3(32, 32), 0, st, true, static_cast<const float*>(a.partial), parts, d, d_weight);
  return check_launch();
}

int mtpc_gradient_list_workspace_bytes(const mtpc_gradient* entries, int32_t count, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  ListPlan p;
  const int rc = plan_list(entries, count, &p);
  if (rc != MTPC_OK) return rc;
  *out_bytes = p.total;
  return MTPC_OK;
}

int mtpc_create_gradient_list(const mtpc_gradient* entries, int32_t count, void* workspace, size_t workspace_bytes, void* stream,
                              mtpc_gradient_list** out) {
  if (!out) return MTPC_ERR_NULL;
  *out = nullptr;
  ListPlan p;
  int rc = plan_list(entries, count, &p);
  if (rc != MTPC_OK) return rc;
  if (!workspace) return MTPC_ERR_NULL;
  if (workspace_bytes < p.total || !aligned(workspace, kAlign)) return MTPC_ERR_WORKSPACE;
  if ((rc = check_overlap(entries, count)) != MTPC_OK) return rc;
  if ((rc = check_device()) != MTPC_OK) return rc;
  mtpc_gradient_list* list = new (std::nothrow) mtpc_gradient_list;
  ClipChunk* chunks = new (std::nothrow) ClipChunk[static_cast<size_t>(p.chunks) + 1];
  if (!list || !chunks) {
    delete list;
    delete[] chunks;
    return MTPC_ERR_CUDA;
  }
  size_t n = 0;
  for (int i = 0; i < count; ++i) {
    const mtpc_gradient& e = entries[i];
    const int head = wide_head(e);
    // Chunks of equal length, but that the first has the elements before the first vector too: the others then start on one.
    for (int64_t at = 0; at < e.count;) {
      ClipChunk& c = chunks[n++];
      const int own_head = at == 0 && head > 0 ? head : 0;
      const int64_t take = std::min<int64_t>(e.count - at, kClipChunk + own_head);
      c.g = static_cast<const uint8_t*>(e.data) + static_cast<size_t>(at) * element(e.dtype);
      c.out = e.out ? static_cast<uint8_t*>(e.out) + static_cast<size_t>(at) * element(e.out_dtype) : nullptr;
      c.count = static_cast<int>(take);
      c.pad[0] = c.pad[1] = 0;
      c.kind = (e.dtype == MTPC_F32 ? kClipF32 : 0u) | ((e.out ? e.out_dtype : e.dtype) == MTPC_F32 ? kClipOutF32 : 0u);
      if (head >= 0 && own_head < take) c.kind |= kClipWide | (own_head == 0 && take == kClipChunk ? kClipFull : 0u) | static_cast<unsigned>(own_head) << 8;
      at += take;
    }
  }
  list->chunks = static_cast<const ClipChunk*>(workspace);
  list->partial = reinterpret_cast<double*>(static_cast<uint8_t*>(workspace) + p.off_partial);
  list->count = static_cast<int>(n);
  list->blocks = p.blocks;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool ok = n == 0 || cudaMemcpyAsync(workspace, chunks, n * sizeof(ClipChunk), cudaMemcpyHostToDevice, st) == cudaSuccess;
  ok = cudaStreamSynchronize(st) == cudaSuccess && ok;       // the host's copy goes away
  delete[] chunks;
  if (!ok) {
    cudaGetLastError();
    delete list;
    return MTPC_ERR_CUDA;
  }
  *out = list;
  return MTPC_OK;
}

int mtpc_clip_gradients(mtpc_gradient_list* list, float max_norm, float* out_norm, void* stream) {
  if (!list || !out_norm) return MTPC_ERR_NULL;
  if (!(max_norm > 0.f) || !aligned(out_norm, 4)) return MTPC_ERR_SHAPE;
  const int rc = check_device();
  if (rc != MTPC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  launch_kernel(gradient_square_kernel, list->blocks, kClipThreads, 0, st, true, list->chunks, list->count, list->partial);
  launch_kernel(gradient_scale_kernel, list->blocks, kClipThreads, 0, st, true, list->chunks, list->count, static_cast<const double*>(list->partial),
                list->blocks, max_norm, out_norm);
  return check_launch();
}

int mtpc_destroy_gradient_list(mtpc_gradient_list* list) {
  if (!list) return MTPC_ERR_NULL;
  delete list;
  return MTPC_OK;
}

}  // extern "C"
