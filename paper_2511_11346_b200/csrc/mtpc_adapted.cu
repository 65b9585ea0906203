// Host side of the projection with low-rank adaptors (include/mtpc.h): argument checks, tensor maps, carving of the caller's workspace, choice of
// the build, launches.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "../../include/mtpc.h"
#include "mtpc_adapted.cuh"
#include "mtpc_host.cuh"
#include "mtpc_launch.cuh"

namespace {

using namespace mtpc;

constexpr int kSmemLimit = 232448;      // 227 KB of dynamic shared memory per CTA on sm_100
// Rows that are dealt with each by itself (as the N of MMAs whose M are W's rows) rather than as tiles of 128. There every row costs time by its rank, in tiles every adaptor
// that occurs does. 4096 x 4096, rows in random order, graph replays with the operands in L2, us by rows / in tiles: k = 16, one adaptor 64 rows 10.1 / 12.1, 96 rows 13.4 / 12.2; eight 96 rows 13.5, 128
// rows 15.7 / 13.9; 32 adaptors 128 rows 16.0 / 28.1 (129 rows); k = 64, one 16 rows 10.3, 32 rows 13.9 / 12.2; four 32 rows 14.9, 48 rows 19.5 / 14.7; eight 64 rows 24.2, 96
// rows 37.7 / 21.2; 32 adaptors 128 rows 44.5 / 60.8 (129 rows).
// S counts the adaptors that there are, since which of them occur is known on the device alone. Where fewer do, tiles would be faster: 128 rows of one of 64 adaptors 15.7 / 12.4
// (k = 16), 41.6 / 12.6 (k = 64).
bool few_rows(int T, int k, int S) { return T <= std::min(128, 640 / std::max(k, 8) + 8 * S); }
constexpr int kMaxAdaptors = 4096, kMaxWidth = 1 << 17, kMaxBatch = 1 << 24;
constexpr size_t kControl = 1024 + sizeof(GemmControl);
constexpr int kRowsShared = sizeof(RowsShared) + 16;
std::atomic<uint64_t> g_wait_limit_ns{kWaitLimitNs};      // of every pipeline wait (a test may shorten it)

// ---------------------------------------------------------------- tensor maps
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = []() -> EncodeTiledFn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}
// bf16 rows of `cols` adjacent elements, `pitch` apart, of `matrices` matrices one behind the other (0: a map of two axes): boxes of box_cols (16, 32 or 64) columns x
// box_rows, swizzled over the bytes of a box's row, zeros outside.
int map_rows(CUtensorMap* tm, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, uint64_t matrices = 0, uint32_t box_cols = 64) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return MTPC_ERR_CUDA;
  const cuuint64_t dims[3] = {cols, rows, matrices}, strides[2] = {pitch * 2, rows * pitch * 2};
  const cuuint32_t box[3] = {box_cols, box_rows, 1}, each[3] = {1, 1, 1};
  const CUtensorMapSwizzle swizzle = box_cols == 16 ? CU_TENSOR_MAP_SWIZZLE_32B : box_cols == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
  const CUresult r = fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, matrices ? 3 : 2, const_cast<void*>(base), dims, strides, box, each,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? MTPC_OK : MTPC_ERR_CUDA;
}

// ---------------------------------------------------------------- sizes
int check_sizes(int T, int d, int m, int k, int S) {
  if (T < 0 || d < 1 || m < 1 || k < 1 || S < 1) return MTPC_ERR_SHAPE;
  if (T > kMaxBatch || d > kMaxWidth || m > kMaxWidth || k > kMaxRank || S > kMaxAdaptors) return MTPC_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(S) * k * std::max(d, m) > (static_cast<int64_t>(1) << 34)) return MTPC_ERR_UNSUPPORTED;
  return MTPC_OK;
}
int up8(int x) { return (x + 7) / 8 * 8; }
int rank16(int k) { return (k + 15) / 16 * 16; }
int pieces_of(int k) { return (k + kPieceRank - 1) / kPieceRank; }

struct ForwardPlan {
  size_t off_low, off_two, off_x, off_x_low, off_W, off_A, off_B, total;
};
void plan_forward(int T, int d, int m, int k, int S, bool copies, ForwardPlan* p) {
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  const size_t rows = T, dp = up8(d);
  const bool few = few_rows(T, k, S), own_low = static_cast<int64_t>(T) * k <= kOwnLow;
  p->off_low = take(few && !own_low ? rows * k * 4 : 0);
  p->off_two = take(few ? 0 : rows * pieces_of(k) * 128);
  p->off_x = take(copies ? rows * dp * 2 : 0);
  p->off_x_low = take(copies && !few ? rows * dp * 2 : 0);
  p->off_W = take(copies ? m * dp * 2 : 0);
  p->off_A = take(copies && !few ? static_cast<size_t>(S) * m * up8(k) * 2 : 0);
  p->off_B = take(copies && !few ? static_cast<size_t>(S) * k * dp * 2 : 0);
  p->total = off;
}

// Runs of row blocks that the adaptors' gradients are cut into: what takes least, in us: 0.45 a block, a run being its blocks and about four more for its start and end; 3 for
// the launch that adds the runs up, 0.12 a run, and their parts' bytes, which are written and read (8192 rows, 4096 to 1024 columns, k = 64, eight adaptors: one run 90 us, eleven,
// which share the work more evenly, 140). An adaptor's rows lie beside each other, so that up to S runs cut few adaptors' rows (n: runs that have rows).
int grad_splits(int tiles, int S, int blocks, int k16) {
  int best = 1;
  double least = 0.0;
  const double parts = static_cast<double>(S) * tiles * (kBlockM * 4 * 2) * k16 / 5e6;
  for (int s = 1; s <= 32 && s <= std::max(1, blocks / 4); ++s) {
    const int n = std::max(s, S);
    const double cost =
        ceil_div(static_cast<long long>(tiles) * n, kSms * grad_ctas(k16)) * (static_cast<double>(blocks) / n + 4.0) * 0.45 + (s > 1 ? 3.0 + s * (0.12 + parts) : 0.0);
    if (s == 1 || cost < least * 0.97) best = s, least = cost;
  }
  return best;
}
struct BackwardPlan {
  int splits;
  size_t off_two, off_low3, off_v3, off_present, off_grad, off_x, off_W, off_A, off_B, off_g, total;
};
void plan_backward(int T, int d, int m, int k, int S, bool copies, BackwardPlan* p) {
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  const size_t rows = T, dp = up8(d), k16 = rank16(k);
  const int blocks = ceil_div(T, 64), tiles = ceil_div(d, kBlockM) + ceil_div(m, kBlockM);
  p->splits = grad_splits(tiles, S, blocks, static_cast<int>(k16));
  p->off_two = take(rows * pieces_of(k) * 128);
  p->off_low3 = take(rows * 3 * k16 * 2);
  p->off_v3 = take(rows * 3 * k16 * 2);
  p->off_present = take(static_cast<size_t>(ceil_div(blocks, 32)) * S * 8);
  p->off_grad = take(p->splits > 1 ? static_cast<size_t>(p->splits) * S * tiles * kBlockM * k16 * 4 : 0);
  p->off_x = take(copies ? rows * dp * 2 : 0);
  p->off_W = take(copies ? m * dp * 2 : 0);
  p->off_A = take(copies ? static_cast<size_t>(S) * m * up8(k) * 2 : 0);
  p->off_B = take(copies ? static_cast<size_t>(S) * k * dp * 2 : 0);
  p->off_g = take(copies ? rows * up8(m) * 2 : 0);
  p->total = off;
}

// ---------------------------------------------------------------- operands
struct Rows {
  const __nv_bfloat16* p;
  int64_t stride;
};
// Whether tensor maps can address rows as they lie.
bool mappable(const void* p, int64_t stride, int64_t rows, int cols) { return aligned(p, 16) && (rows <= 1 || (stride % 8 == 0 && stride >= cols)); }

// Copies of what is not mappable, up to four of them in one launch.
struct Copier {
  CopyParams c;
  int n = 0;
  cudaStream_t st;
  explicit Copier(cudaStream_t stream) : st(stream) { memset(&c, 0, sizeof(c)); }
  Rows rows(const void* p, int64_t stride, int64_t rows, int cols, void* to) {
    Rows r{static_cast<const __nv_bfloat16*>(p), rows > 1 ? stride : up8(cols)};
    if (p == nullptr || mappable(p, stride, rows, cols)) return r;
    CopyRows& m = c.m[n];
    m.src = r.p;
    m.dst = static_cast<__nv_bfloat16*>(to);
    m.stride = stride;
    m.rows = rows;
    m.cols = cols;
    m.pitch = up8(cols);
    ++n;
    c.begin[n] = c.begin[n - 1] + rows * (m.pitch / 8);
    r = Rows{m.dst, m.pitch};
    if (n == 4) launch_now();           // (which clears m)
    return r;
  }
  void launch_now() {
    if (n == 0) return;
    for (int i = n + 1; i <= 4; ++i) c.begin[i] = c.begin[n];
    launch_kernel(copy_rows_kernel, ceil_div(c.begin[4], 256), 256, 0, st, true, c);
    memset(&c, 0, sizeof(c));
    n = 0;
  }
};

constexpr int kMaxDevices = 64;
int g_allowed[kMaxDevices];
// The kernels may use the shared memory that they ask for: said once on each device.
int allow_shared_memory() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return MTPC_ERR_CUDA;
  if (__atomic_load_n(&g_allowed[dev], __ATOMIC_ACQUIRE)) return MTPC_OK;
  const auto allow = [](auto* kernel, int bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess; };
  bool ok = allow(adaptor_low_kernel<false>, kSmemLimit) && allow(adaptor_low_kernel<true>, kSmemLimit);
  const auto allow_rows = [&](auto* s1, auto* s2, auto* s4, auto* s8) { ok = ok && allow(s1, kSmemLimit) && allow(s2, kSmemLimit) && allow(s4, kSmemLimit) && allow(s8, kSmemLimit); };
  allow_rows(adapted_rows_kernel<1, true, 4>, adapted_rows_kernel<2, true, 4>, adapted_rows_kernel<4, true, 4>, adapted_rows_kernel<8, true, 4>);
  allow_rows(adapted_rows_kernel<1, false, 4>, adapted_rows_kernel<2, false, 4>, adapted_rows_kernel<4, false, 4>, adapted_rows_kernel<8, false, 4>);
  allow_rows(adapted_rows_kernel<1, false, 8>, adapted_rows_kernel<2, false, 8>, adapted_rows_kernel<4, false, 8>, adapted_rows_kernel<8, false, 8>);
  ok = ok && allow(adapted_gemm_kernel<false, 256, 2>, kSmemLimit) && allow(adapted_gemm_kernel<true, 256, 2>, kSmemLimit);
  ok = ok && allow(adapted_gemm_kernel<false, 128, 1>, kSmemLimit) && allow(adapted_gemm_kernel<true, 128, 1>, kSmemLimit);
  ok = ok && allow(adapted_gemm_kernel<false, 64, 1>, kSmemLimit) && allow(adapted_gemm_kernel<true, 64, 1>, kSmemLimit);
  ok = ok && allow(adaptor_grad_kernel<16>, kSmemLimit) && allow(adaptor_grad_kernel<32>, kSmemLimit) && allow(adaptor_grad_kernel<48>, kSmemLimit) &&
       allow(adaptor_grad_kernel<64>, kSmemLimit);
  if (!ok) return MTPC_ERR_CUDA;
  __atomic_store_n(&g_allowed[dev], 1, __ATOMIC_RELEASE);
  return MTPC_OK;
}
// Stages fill an SM's shared memory, or half of it for kernels that take 256 columns of tensor memory at most: whatever CTAs meet on an SM, of calls on several streams too, have
// 512 columns together, so that none in a cluster waits for columns that another one holds.
int stages_of(int stage_bytes, int ctas_per_sm = 1, int beside = 0) {
  return std::min(kMaxStages, static_cast<int>((kSmemLimit / ctas_per_sm - (ctas_per_sm > 1 ? 1024 : 0) - kControl - beside) / stage_bytes));
}

// ---------------------------------------------------------------- launches
// low or v: rows [T, K] times the factors, if rows are given, and what else p asks for.
// product_ctas: those of the product behind it, or 0.
int launch_low(LowParams& p, const Rows& rows, const Rows& factors, bool mn, const int* which, int T, int K, int k, int S, int product_ctas, unsigned* status,
               cudaStream_t st) {
  p.which = which;
  p.status = status;
  p.wait_limit_ns = g_wait_limit_ns.load(std::memory_order_relaxed);
  p.T = T;
  p.S = S;
  p.k = k;
  p.k16 = rank16(k);
  p.pieces = pieces_of(k);
  p.split = 1;
  p.group = mn ? 64 / factor_columns(p.k16) : kMaxRank / p.k16;
  p.stage_bytes = kABytes + kMaxRank * kBlockK * 2;
  p.stages = stages_of(p.stage_bytes, 2);
  p.tiles = ceil_div(T, kBlockM);
  if (rows.p) {
    int rc = map_rows(&p.tm_a, rows.p, T, K, rows.stride, kBlockM);
    if (rc == MTPC_OK) rc = mn ? map_rows(&p.tm_f, factors.p, K, k, factors.stride, 64, S, factor_columns(p.k16)) : map_rows(&p.tm_f, factors.p, k, K, factors.stride, rank16(k), S);
    if (rc != MTPC_OK) return rc;
    p.kblocks = ceil_div(K, kBlockK);
    // CTAs that share a tile's K: four (two to eight, K = 4096, us: 8192 rows 191 / 183 / 183, 2005 rows to 4096 columns 35.3 / 32.3 / 36.0 at rank 64), since clusters of eight
    // find few places, but for three tiles and less (129 rows 28.6 / 19.7 / 15.9). Where the product's last round leaves SMs free, and one pass over the rows gives low, no more
    // than those: the product starts beside them (gradients of 1024 x 4096, 4096 columns 33.9 / 40.4 / 39.0).
    const int spare = product_ctas == 0 ? kSms : (kSms - product_ctas % kSms) % kSms;
    int most = p.tiles <= 3 ? 8 : 4;
    if (p.group >= 4 && p.tiles * 2 <= spare) most = std::min(most, spare / p.tiles);
    while (p.split * 2 <= most && p.split * 4 <= p.kblocks && p.tiles * p.split <= kSms) p.split *= 2;
    p.chunk_blocks = std::min(kChunkBlocks, ceil_div(p.kblocks, p.split));
    p.chunks = ceil_div(p.kblocks, p.chunk_blocks);
  }
  p.present_blocks = p.present ? ceil_div(T, 32 * 64) : 0;
  const int beside = ceil_div(p.present_blocks, p.split) * p.split;
  const size_t smem = kControl + static_cast<size_t>(p.stages) * p.stage_bytes;
  launch_clusters(mn ? adaptor_low_kernel<true> : adaptor_low_kernel<false>, p.split, p.tiles * p.split + beside, kLowThreads, smem, st, true, p);
  return check_launch();
}

template <bool B_MN, int TN, int CTAS>
int launch_gemm(AdaptedParams& p, const Rows& a, const Rows& b, const __nv_bfloat16* two, const Rows& f, int K, cudaStream_t st) {
  constexpr int kBCols = TN / CTAS;
  int rc = MTPC_OK;
  if (p.kblocks > 0) {
    rc = map_rows(&p.tm_a, a.p, p.T, K, a.stride, kBlockM);
    if (rc == MTPC_OK) rc = B_MN ? map_rows(&p.tm_b, b.p, K, p.N, b.stride, 64) : map_rows(&p.tm_b, b.p, p.N, K, b.stride, kBCols);
  }
  if (rc == MTPC_OK && p.pieces > 0) {
    rc = map_rows(&p.tm_u, two, p.T, p.pieces * 64, p.pieces * 64, kBlockM);
    if (rc == MTPC_OK) rc = B_MN ? map_rows(&p.tm_f, f.p, p.k, p.N, f.stride, 64, p.S) : map_rows(&p.tm_f, f.p, p.N, p.k, f.stride, kBCols, p.S);
  }
  if (rc != MTPC_OK) return rc;
  p.m_units = ceil_div(p.T, kBlockM * CTAS);
  p.n_tiles = ceil_div(p.N, TN);
  p.stage_bytes = kABytes + kBCols * kBlockK * 2;
  const int staging = p.store == 2 ? kStoreBytes : 0;
  p.stages = stages_of(p.stage_bytes, 1, staging);
  const size_t smem = kControl + staging + static_cast<size_t>(p.stages) * p.stage_bytes;
  const int workers = std::min(p.m_units * p.n_tiles, kSms / CTAS);
  launch_clusters(adapted_gemm_kernel<B_MN, TN, CTAS>, CTAS, workers * CTAS, kAdaptedThreads, smem, st, true, p);
  return check_launch();
}
// The tiles of a product of T rows and N columns over kb K blocks: their columns, and the CTAs that a tile has.
struct ProductTile {
  int columns, ctas, count;             // count: of tiles
};
// Cycles that a K block of a tile takes and that its rest does, by the bytes that an SM gets from L2 and its MMAs' time, whichever is longer; rows that lie across lines of L2
// cost the smaller tiles, which read more, half as much again. 4096 x 4096, us for pairs / 128 / 64 columns: 256 rows 28 / 18 / 16, 512 27 / 19 / 25, 768 28 / 36 / 38.
ProductTile product_tile(int T, int N, int kb, const Rows& a, const Rows& b) {
  const bool across = a.stride % 64 != 0 || b.stride % 64 != 0;
  const int pairs = ceil_div(T, 256) * ceil_div(N, 256), wides = ceil_div(T, 128) * ceil_div(N, 128), narrows = ceil_div(T, 128) * ceil_div(N, 64);
  const double pair = ceil_div(pairs, kSms / 2) * (kb * 560.0 + 2000), wide = ceil_div(wides, kSms) * (kb * (across ? 700.0 : 450.0) + 1500);
  const double narrow = ceil_div(narrows, kSms) * (kb * (across ? 550.0 : 350.0) + 1200);
  if (pair <= wide && pair <= narrow) return ProductTile{256, 2, pairs};
  return wide <= narrow ? ProductTile{128, 1, wides} : ProductTile{64, 1, narrows};
}
int k_blocks(int K, bool shared, int k, bool adaptors) { return (shared ? ceil_div(K, kBlockK) : 0) + (adaptors ? 2 * pieces_of(k) : 0); }
// rows [T, K] times W (N rows of K, or with b_mn K rows of N), plus two terms of low times the factors; shared false: these alone.
int launch_product(const Rows& a, const Rows& b, const __nv_bfloat16* two, const Rows& f, bool b_mn, const int* which, int T, int K, int N, int k, int S,
                   bool shared, bool adaptors, void* out, int64_t out_stride, unsigned* status, cudaStream_t st) {
  AdaptedParams p;
  memset(&p, 0, sizeof(p));
  p.which = which;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.out_stride = out_stride;
  p.status = status;
  p.wait_limit_ns = g_wait_limit_ns.load(std::memory_order_relaxed);
  p.T = T;
  p.S = S;
  p.N = N;
  p.k = k;
  p.pieces = adaptors ? pieces_of(k) : 0;
  p.kblocks = shared ? ceil_div(K, kBlockK) : 0;
  p.store = rows_allow(out, out_stride, 2, 16, T) ? 32 : rows_allow(out, out_stride, 2, 8, T) ? 16 : 2;
  const int columns = product_tile(T, N, k_blocks(K, shared, k, adaptors), a, b).columns;
  if (columns == 256) return b_mn ? launch_gemm<true, 256, 2>(p, a, b, two, f, K, st) : launch_gemm<false, 256, 2>(p, a, b, two, f, K, st);
  if (columns == 128) return b_mn ? launch_gemm<true, 128, 1>(p, a, b, two, f, K, st) : launch_gemm<false, 128, 1>(p, a, b, two, f, K, st);
  return b_mn ? launch_gemm<true, 64, 1>(p, a, b, two, f, K, st) : launch_gemm<false, 64, 1>(p, a, b, two, f, K, st);
}

int launch_few_rows(const Rows& x, const Rows& W, const void* x_low, int64_t x_low_stride, const void* A, const void* B, const float* scale, const int* which,
                    int T, int d, int m, int k, int S, void* out, int64_t out_stride, float* low, float* user_low, unsigned* status, cudaStream_t st) {
  LowRowsParams l;
  memset(&l, 0, sizeof(l));
  l.x = static_cast<const __nv_bfloat16*>(x_low);
  l.B = static_cast<const __nv_bfloat16*>(B);
  l.x_stride = T > 1 ? x_low_stride : 0;
  l.which = which;
  l.scale = scale;
  l.low = low;
  l.status = status;
  l.T = T;
  l.d = d;
  l.k = k;
  l.S = S;
  l.wide = d % 8 == 0 && rows_allow(x_low, x_low_stride, 2, 8, T) && aligned(B, 16);
  const bool own_low = T * k <= kOwnLow;
  if (!own_low) launch_kernel(low_rows_kernel, dim3(T, ceil_div(k, 4)), 128, 0, st, true, l);

  RowsParams p;
  memset(&p, 0, sizeof(p));
  p.tokens = (T + 15) / 16 * 16;
  int rc = map_rows(&p.tm_w, W.p, m, d, W.stride, kBlockM);
  if (rc == MTPC_OK) rc = map_rows(&p.tm_x, x.p, T, d, x.stride, p.tokens);
  if (rc != MTPC_OK) return rc;
  p.A = static_cast<const __nv_bfloat16*>(A);
  p.low = low;
  p.which = which;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.out_stride = out_stride;
  p.status = status;
  p.wait_limit_ns = g_wait_limit_ns.load(std::memory_order_relaxed);
  p.T = T;
  p.S = S;
  p.N = m;
  p.k = k;
  p.kblocks = ceil_div(d, kBlockK);
  const int tiles = ceil_div(m, kBlockM);
  // K is cut into up to four parts until the CTAs are as many as the device holds at once, two on an SM; one row by itself and more than 32 into eight, the latter where each
  // still has an SM of its own (4096 x 4096, k = 16, two / four / eight parts, us: one row 17.5 / 13.2 / 10.3, 16 rows 12.3 / 11.5 / 13.4, 64 rows 19.0 / 14.3 / 17.4; 1024 rows
  // of W: 64 rows 13.0 / 7.9 / 7.5), or where reading their adaptors' factors, for which more CTAs have more loads in flight, takes longer than that costs (four / eight parts, operands in L2:
  // k = 32, 64 rows 14.2 / 16.0, 128 rows 33.4 / 24.1; k = 48, 48 rows 18.6 / 14.8; k = 64, 64 rows 39.2 / 24.5, 128 rows 75.4 / 44.4).
  int split = 1;
  while (split < (own_low || T > 32 ? 8 : 4) && split * 2 <= p.kblocks && tiles * split * (split < 4 || own_low || T * k > 2048 ? 1 : 2) <= kSms) split *= 2;
  p.stage_bytes = kABytes + p.tokens * kBlockK * 2;
  const int shared = kRowsShared + (own_low ? 0 : ceil_div(T, split) * k * 4);       // (32 KB at most: two stages are left of the longest, and hold the sums)
  p.stages = stages_of(p.stage_bytes, 2, shared);
  p.wide = k % 8 == 0 && aligned(A, 16);
  p.store4 = rows_allow(out, out_stride, 2, 4, T);
  p.own = l;
  p.own.low = user_low;
  const size_t smem = kControl + shared + static_cast<size_t>(p.stages) * p.stage_bytes;
  const bool many = ceil_div(T, 2 * split) > 4 && k <= 16;           // rows of a thread; behind sixteen of rank their loads are not ahead (128 rows, k = 64: 49.2 / 44.4 us)
  const auto pick = [&](auto* s1, auto* s2, auto* s4, auto* s8) { return split == 8 ? s8 : split == 4 ? s4 : split == 2 ? s2 : s1; };
  auto* kernel = own_low ? pick(adapted_rows_kernel<1, true, 4>, adapted_rows_kernel<2, true, 4>, adapted_rows_kernel<4, true, 4>, adapted_rows_kernel<8, true, 4>)
                 : many  ? pick(adapted_rows_kernel<1, false, 8>, adapted_rows_kernel<2, false, 8>, adapted_rows_kernel<4, false, 8>, adapted_rows_kernel<8, false, 8>)
                         : pick(adapted_rows_kernel<1, false, 4>, adapted_rows_kernel<2, false, 4>, adapted_rows_kernel<4, false, 4>, adapted_rows_kernel<8, false, 4>);
  launch_clusters(kernel, split, tiles * split, kRowsThreads, smem, st, true, p);
  return check_launch();
}

}  // namespace

extern "C" {

int mtpc_debug_set_adapted_wait_limit_ns(uint64_t limit_ns) {
  g_wait_limit_ns.store(limit_ns == 0 ? kWaitLimitNs : limit_ns, std::memory_order_relaxed);
  return MTPC_OK;
}

int mtpc_adapted_projection_workspace_bytes(int32_t T, int32_t d, int32_t m, int32_t k, int32_t S, int32_t aligned_rows, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  const int rc = check_sizes(T, d, m, k, S);
  if (rc != MTPC_OK) return rc;
  ForwardPlan p;
  plan_forward(T, d, m, k, S, aligned_rows == 0, &p);
  *out_bytes = p.total;
  return MTPC_OK;
}

int mtpc_adapted_projection(const void* x, int64_t x_stride, const void* x_low, int64_t x_low_stride, const void* W, int64_t W_stride, const void* A,
                            const void* B, const float* scale, const int32_t* row_adaptor, int32_t T, int32_t d, int32_t m, int32_t k, int32_t S, void* out,
                            int64_t out_stride, float* out_low, void* workspace, size_t workspace_bytes, uint32_t* out_status, void* stream) {
  int rc = check_sizes(T, d, m, k, S);
  if (rc != MTPC_OK) return rc;
  if (T == 0) return MTPC_OK;
  if (!x || !W || !A || !B || !out) return MTPC_ERR_NULL;
  if (!x_low) {
    x_low = x;
    x_low_stride = x_stride;
  }
  if (!input_rows(x, x_stride, T) || !input_rows(x_low, x_low_stride, T) || !input_rows(W, W_stride, m) || !output_rows(out, out_stride, T, m)) return MTPC_ERR_SHAPE;
  for (const void* q : {x, x_low, W, A, B, static_cast<const void*>(out)})
    if (!aligned(q, 2)) return MTPC_ERR_SHAPE;
  for (const void* q : {static_cast<const void*>(scale), static_cast<const void*>(row_adaptor), static_cast<const void*>(out_low), static_cast<const void*>(out_status)})
    if (!aligned(q, 4)) return MTPC_ERR_SHAPE;
  const bool few = few_rows(T, k, S);
  const bool copies = !mappable(x, x_stride, T, d) || !mappable(W, W_stride, m, d) ||
                      (!few && (!mappable(x_low, x_low_stride, T, d) || !mappable(A, k, 2, k) || !mappable(B, d, 2, d)));
  ForwardPlan plan;
  plan_forward(T, d, m, k, S, copies, &plan);
  if (plan.total > 0 && !workspace) return MTPC_ERR_NULL;
  if (workspace_bytes < plan.total || !aligned(workspace, kAlign)) return MTPC_ERR_WORKSPACE;
  if ((rc = check_device()) != MTPC_OK || (rc = allow_shared_memory()) != MTPC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Copier copy(st);
  const Rows xr = copy.rows(x, x_stride, T, d, ws + plan.off_x), Wr = copy.rows(W, W_stride, m, d, ws + plan.off_W);
  if (few) {
    copy.launch_now();
    float* low = out_low ? out_low : reinterpret_cast<float*>(ws + plan.off_low);
    return launch_few_rows(xr, Wr, x_low, x_low_stride, A, B, scale, row_adaptor, T, d, m, k, S, out, out_stride, low, out_low, out_status, st);
  }
  const Rows Ar = copy.rows(A, k, static_cast<int64_t>(S) * m, k, ws + plan.off_A), Br = copy.rows(B, d, static_cast<int64_t>(S) * k, d, ws + plan.off_B);
  const Rows lr = x_low == x && x_low_stride == x_stride ? xr : copy.rows(x_low, x_low_stride, T, d, ws + plan.off_x_low);
  copy.launch_now();
  LowParams l;
  memset(&l, 0, sizeof(l));
  l.scale = scale;
  l.low = out_low;
  l.two = reinterpret_cast<__nv_bfloat16*>(ws + plan.off_two);
  const ProductTile tile = product_tile(T, m, k_blocks(d, true, k, true), xr, Wr);
  if ((rc = launch_low(l, lr, Br, false, row_adaptor, T, d, k, S, tile.count * tile.ctas, out_status, st)) != MTPC_OK) return rc;
  return launch_product(xr, Wr, l.two, Ar, false, row_adaptor, T, d, m, k, S, true, true, out, out_stride, out_status, st);
}

int mtpc_adapted_projection_backward_workspace_bytes(int32_t T, int32_t d, int32_t m, int32_t k, int32_t S, int32_t aligned_rows, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  const int rc = check_sizes(T, d, m, k, S);
  if (rc != MTPC_OK) return rc;
  BackwardPlan p;
  plan_backward(T, d, m, k, S, aligned_rows == 0, &p);
  *out_bytes = p.total;
  return MTPC_OK;
}

int mtpc_adapted_projection_backward(const void* x_low, int64_t x_low_stride, const void* W, int64_t W_stride, const void* A, const void* B,
                                     const float* scale, const int32_t* row_adaptor, const float* low, int32_t T, int32_t d, int32_t m, int32_t k, int32_t S,
                                     const void* d_out, int64_t d_out_stride, void* d_x, int64_t d_x_stride, void* d_x_low, int64_t d_x_low_stride,
                                     float* dA, float* dB, void* workspace, size_t workspace_bytes, uint32_t* out_status, void* stream) {
  int rc = check_sizes(T, d, m, k, S);
  if (rc != MTPC_OK) return rc;
  if (T > 0 && (!workspace || !d_out || !A || !B || (d_x && !W) || (dA && !low) || (dB && !x_low))) return MTPC_ERR_NULL;
  if (!input_rows(x_low, x_low_stride, T) || !input_rows(W, W_stride, m) || !input_rows(d_out, d_out_stride, T) || !output_rows(d_x, d_x_stride, T, d) ||
      !output_rows(d_x_low, d_x_low_stride, T, d))
    return MTPC_ERR_SHAPE;
  for (const void* q : {x_low, W, A, B, d_out, static_cast<const void*>(d_x), static_cast<const void*>(d_x_low)})
    if (!aligned(q, 2)) return MTPC_ERR_SHAPE;
  for (const void* q : {static_cast<const void*>(scale), static_cast<const void*>(row_adaptor), static_cast<const void*>(low), static_cast<const void*>(dA),
                        static_cast<const void*>(dB), static_cast<const void*>(out_status)})
    if (!aligned(q, 4)) return MTPC_ERR_SHAPE;
  const bool copies = (dB && !mappable(x_low, x_low_stride, T, d)) || (d_x && !mappable(W, W_stride, m, d)) || !mappable(A, k, 2, k) || !mappable(B, d, 2, d) ||
                      !mappable(d_out, d_out_stride, T, m);
  BackwardPlan plan;
  plan_backward(T, d, m, k, S, copies, &plan);
  if (workspace_bytes < plan.total || !aligned(workspace, kAlign)) return MTPC_ERR_WORKSPACE;
  if ((rc = check_device()) != MTPC_OK || (rc = allow_shared_memory()) != MTPC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if ((dA && cudaMemsetAsync(dA, 0, static_cast<size_t>(S) * m * k * 4, st) != cudaSuccess) ||
        (dB && cudaMemsetAsync(dB, 0, static_cast<size_t>(S) * k * d * 4, st) != cudaSuccess))
      return MTPC_ERR_CUDA;
    return MTPC_OK;
  }
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Copier copy(st);
  const Rows gr = copy.rows(d_out, d_out_stride, T, m, ws + plan.off_g);
  const Rows Ar = copy.rows(A, k, static_cast<int64_t>(S) * m, k, ws + plan.off_A), Br = copy.rows(B, d, static_cast<int64_t>(S) * k, d, ws + plan.off_B);
  const Rows Wr = d_x ? copy.rows(W, W_stride, m, d, ws + plan.off_W) : Rows{nullptr, 0};
  const Rows xr = dB ? copy.rows(x_low, x_low_stride, T, d, ws + plan.off_x) : Rows{nullptr, 0};
  copy.launch_now();

  LowParams l;
  memset(&l, 0, sizeof(l));
  l.scale = scale;
  __nv_bfloat16* two = reinterpret_cast<__nv_bfloat16*>(ws + plan.off_two);
  __nv_bfloat16* low3 = reinterpret_cast<__nv_bfloat16*>(ws + plan.off_low3);
  __nv_bfloat16* v3 = reinterpret_cast<__nv_bfloat16*>(ws + plan.off_v3);
  if (d_x || d_x_low) l.two = two;
  if (dB) l.three = v3;
  if (dA) {
    l.given = low;
    l.given_three = low3;
  }
  if (dA || dB) {
    l.present = reinterpret_cast<uint32_t*>(ws + plan.off_present);
    l.whole = l.present + static_cast<size_t>(ceil_div(T, 32 * 64)) * S;
  }
  const bool sums = d_x || d_x_low || dB;
  const ProductTile tile = d_x ? product_tile(T, d, k_blocks(m, true, k, d_x_low == nullptr), gr, Wr) : ProductTile{0, 0, 0};
  if ((sums || dA) && (rc = launch_low(l, sums ? gr : Rows{nullptr, 0}, Ar, true, row_adaptor, T, m, k, S, tile.count * tile.ctas, out_status, st)) != MTPC_OK)
    return rc;
  if (d_x && (rc = launch_product(gr, Wr, two, Br, true, row_adaptor, T, m, d, k, S, true, d_x_low == nullptr, d_x, d_x_stride, out_status, st)) != MTPC_OK) return rc;
  if (d_x_low && (rc = launch_product(gr, Rows{nullptr, 0}, two, Br, true, row_adaptor, T, m, d, k, S, false, true, d_x_low, d_x_low_stride, out_status, st)) != MTPC_OK)
    return rc;
  if (!dA && !dB) return MTPC_OK;
  GradParams p;
  memset(&p, 0, sizeof(p));
  p.which = row_adaptor;
  p.present = l.present;
  p.whole = l.whole;
  p.after_low = !d_x && !d_x_low;
  p.wide_a = k % 8 == 0 && aligned(dA, 32);
  p.out[0] = dA;
  p.out[1] = dB;
  p.part = reinterpret_cast<float*>(ws + plan.off_grad);
  p.status = out_status;
  p.wait_limit_ns = g_wait_limit_ns.load(std::memory_order_relaxed);
  p.T = T;
  p.S = S;
  p.k = k;
  p.cols[0] = m;
  p.cols[1] = d;
  p.tiles[0] = dA ? ceil_div(m, kBlockM) : 0;
  p.tiles[1] = dB ? ceil_div(d, kBlockM) : 0;
  p.blocks = ceil_div(T, 64);
  p.splits = plan.splits;
  const int k16 = rank16(k);
  for (int q = 0; q < 2; ++q) {
    if (!p.tiles[q]) continue;
    const Rows& r = q ? xr : gr;
    const __nv_bfloat16* terms = q ? v3 : low3;
    if ((rc = map_rows(&p.tm_rows[q], r.p, T, p.cols[q], r.stride, 64)) != MTPC_OK || (rc = map_rows(&p.tm_terms[q], terms, T, 3 * k16, 3 * k16, 64)) != MTPC_OK)
      return rc;
  }
  p.stage_bytes = kABytes + ceil_div(3 * k16, 64) * static_cast<int>(kMnBoxBytes);
  p.stages = stages_of(p.stage_bytes, grad_ctas(k16), kGradWords * 8);
  const size_t smem = kControl + kGradWords * 8 + static_cast<size_t>(p.stages) * p.stage_bytes;
  auto* kernel = k16 == 16 ? adaptor_grad_kernel<16> : k16 == 32 ? adaptor_grad_kernel<32> : k16 == 48 ? adaptor_grad_kernel<48> : adaptor_grad_kernel<64>;
  const long long items = static_cast<long long>(p.tiles[0] + p.tiles[1]) * S * p.splits;
  launch_kernel(kernel, static_cast<int>(std::min<long long>(items, grad_ctas(k16) * kSms)), kGradThreads, smem, st, true, p);
  if (p.splits > 1) {
    const long long quads = static_cast<long long>(S) * (p.tiles[0] + p.tiles[1]) * kBlockM * (k16 / 4);
    launch_kernel(adaptor_grad_join_kernel, ceil_div(quads, 256), 256, 0, st, true, p, k16);
  }
  return check_launch();
}

}  // extern "C"
