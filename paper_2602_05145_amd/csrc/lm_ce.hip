// Softmax cross-entropy of the LM head from the hidden states, z = y W^T, without keeping logits:
//   forward    lse_r = log sum_v exp(z_rv),  loss_r = lse_r - z[r, token_r]
//   backward   dz_rv = weight_r (exp(z_rv - lse_r) - [v = token_r]),  dy = scale dz W,  dW = scale dz^T y
// bf16: the forward product's tiles never leave their CU; what does is the maximum and the sum of exponentials of every row over
// a tile's 256 columns (3 % of the logits' bytes), and a small kernel joins them.  The backward pass goes through the vocabulary in
// pieces: a piece's logits are made again from y and W, leave their product's epilogue as dz (bf16, up to 1 GiB of it), and feed
// both gradients before the next piece takes their place.  dW is written once, a piece at a time; dy gathers its pieces in fp32.
// fp32: pieces of logits in both directions, with a pass over each.
// Rows without loss are left out: the others are copied into a dense array first, so that whatever stands in the rest (NaN as
// well) touches nothing, and their number stays on the device.
// Bound by the matrix pipes: [27853 kept of 32768, 128256], width 4096, bf16: forward 21.2 ms, backward 62.6 ms, 1.39 PFLOP/s over the four products that run.
#include <algorithm>
#include <cstring>

#include "kernels.h"
#include "prof.h"
#include "row_stats.h"

namespace tide {

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The vocabulary in pieces, the last one first.  A piece's columns are the contraction of dy: bf16 products take a multiple
// of 8 of them.  Where the vocabulary is not one, the last piece reaches back over up to 7 columns of the one before, with
// gradients of zero there: they add nothing to dy, and the rows of dW that come out zero are written again, right, by the
// piece that they belong to.
struct Piece { int64_t n0, n; int zero; };   // columns [n0, n0 + n), the first `zero` of them another piece's
struct Pieces { int64_t V, width; int count; bool by8; };
// Elements that a piece's array has room for: rows x the vocabulary up to 1 GiB, and at least 256 columns.  Never falls as the rows grow.
int64_t piece_elems(int64_t rows, int64_t V, int dtype) {
  const int64_t budget = ((int64_t)1 << 30) / (int64_t)dtype_size(dtype);
  return std::max(rows * 256, std::min(rows * (int64_t)align_up((size_t)V, 256), budget));
}
constexpr int64_t kMostColumns = ((int64_t)1 << 21) - 256;   // bf16 products take rows of fewer than 2^21 elements
Pieces plan_pieces(int64_t rows, int64_t V, int dtype) {
  const bool by8 = dtype == kBF16;
  const int64_t room = piece_elems(rows, V, dtype) / rows / 256 * 256, most = by8 ? std::min(room, kMostColumns) : room, count = (V + most - 1) / most;
  if (count == 1 && by8 && V % 8) return Pieces{V, V / 8 * 8, 2, by8};        // and the rest, at most 7 columns, as a piece of 8
  const int64_t width = (int64_t)align_up((size_t)((V + count - 1) / count), 256);   // (at most `most`)
  return Pieces{V, width, (int)((V + width - 1) / width), by8};
}
Piece piece_at(const Pieces& p, int i) {   // i = 0: the last one
  const int64_t at = p.count - 1 - i, n0 = at * p.width, n = std::min(p.width, p.V - n0);
  const int back = p.by8 && n % 8 ? (int)(8 - n % 8) : 0;
  return Piece{n0 - back, n + back, back};
}
// elements between two rows of a piece
int64_t piece_ld(const Pieces& p) { return (int64_t)align_up((size_t)p.width, 64); }

constexpr int64_t kCountRows = 1024, kDirectRows = 8192;   // see lm_begin_kernel

struct LmCePlan {
  size_t counts, cnt, kept_idx, row_pos, tokens_c, rows_c, y_c;
  size_t z, acc, dy_c, split, split_bytes;   // z: a piece (bf16: of dz), or the forward pass's statistics
  size_t total;
};

GemmArgs product(int layout, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, int in_dtype,
                 int out_dtype) {
  GemmArgs g;
  std::memset(&g, 0, sizeof(g));
  g.layout = layout; g.M = M; g.N = N; g.K = K;
  g.A = A; g.lda = lda; g.B = B; g.ldb = ldb; g.C = C; g.ldc = ldc;
  g.alpha = 1.f; g.in_dtype = in_dtype; g.out_dtype = out_dtype;
  return g;
}

LmCePlan make_plan(int64_t rows, int64_t V, int64_t d, int dtype) {
  LmCePlan p;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
  const size_t T = (size_t)rows, es = dtype_size(dtype);
  const Pieces pc = plan_pieces(rows, V, dtype);
  p.counts = take((T + kCountRows - 1) / kCountRows * 4);
  p.cnt = take(64);
  p.kept_idx = take(T * 4);
  p.row_pos = take(T * 4);
  p.tokens_c = take(T * 4);
  p.rows_c = take(T * sizeof(LmRow));
  p.y_c = take(T * d * es);
  p.z = take(std::max((size_t)piece_elems(rows, V, dtype) * es, dtype == kBF16 ? T * (size_t)((V + kLmColumns - 1) / kLmColumns) * sizeof(float2) : 0));
  p.acc = pc.count > 1 && dtype == kBF16 ? take(T * d * 4) : 0;
  // fp32: as many sums of it as the product leaves (see gemm_fp32_parts), within a bound that does not fall as rows grow
  p.dy_c = take(dtype == kF32 ? std::max(T * d, std::min(kMaxFp32Parts * T * d, (size_t)2 * kFp32PartsTiles * 4096)) * es : T * d * es);
  if (dtype == kF32 || pc.count == 1) p.acc = p.dy_c;
  p.split_bytes = 0;
  if (dtype == kBF16) {
    void* any = (void*)256;   // alignment only
    for (const int out : {kBF16, kF32}) {
      p.split_bytes = std::max(p.split_bytes, gemm_splitk_scratch_bound(product(kNN, rows, d, (int64_t)align_up((size_t)V, 8), any, 2 * 64, any, d, any, d, dtype, out)));
      p.split_bytes = std::max(p.split_bytes, gemm_splitk_scratch_bound(product(kTN, (int64_t)align_up((size_t)V, 8), d, rows, any, 2 * 64, any, d, any, d, dtype, out)));
    }
  }
  p.split = take(p.split_bytes);
  p.total = off;
  return p;
}

// fp32: a compact row's running maximum, sum and label logit
struct RowState { float m, s, z; };
static_assert(sizeof(RowState) <= sizeof(LmRow), "one array for either");

}  // namespace

__device__ __forceinline__ bool kept(const int32_t* tokens, const uint8_t* mask, int64_t t, int V) {
  const int tk = tokens[t];
  return mask[t] != 0 && tk >= 0 && tk < V;
}
__device__ __forceinline__ int block_count(int n, int* red) {   // of 256 threads; every thread gets the sum
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}
// kept rows of every kCountRows
__global__ __launch_bounds__(256) void lm_count_kernel(const int32_t* __restrict__ tokens, const uint8_t* __restrict__ mask, int64_t T, int V,
                                                       int* __restrict__ counts) {
  __shared__ int red[4];
  int n = 0;
  for (int64_t t = blockIdx.x * kCountRows + threadIdx.x; t < min(T, (blockIdx.x + 1) * kCountRows); t += 256) n += kept(tokens, mask, t, V) ? 1 : 0;
  n = block_count(n, red);
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// The dense array of the kept rows, in order, with everything that a call needs of each: its hidden state, label, place in the batch, and
// either a fresh RowState (fp32's forward) or its LmRow (backward).  Four rows per block, one per wave (eight: 90 x 4096 15.7 us, 3400 x 4096 22.9,
// 27853 x 4096 87.7; four: 11.4, 17.7, 83.0).  The rows kept before a
// block's are counted by the block itself up to kDirectRows (at most 32 rows per thread), beyond from the counts of
// kCountRows each: one launch (of 5 us next to nothing in it) instead of three, or two.
enum : int { kBeginForward = 0, kBeginForwardFp32 = 1, kBeginBackward = 2 };
struct LmBegin {
  const void* y; const int32_t* tokens; const uint8_t* mask; const float* weights;
  float *lse, *loss_rows;
  void* y_c; int32_t *tokens_c, *kept_idx, *row_pos; int* cnt; void* rows_c;
  const int* counts;
  int64_t T;
  int V, d, mode;
};
template <typename T>
__global__ __launch_bounds__(256) void lm_begin_kernel(LmBegin a) {
  constexpr int ROWS = 4;
  __shared__ int red[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t0 = (int64_t)blockIdx.x * ROWS;
  int before = 0;
  int64_t from = 0;
  if (a.counts) {
    from = t0 / kCountRows * kCountRows;
    for (int64_t i = threadIdx.x; i < t0 / kCountRows; i += 256) before += a.counts[i];
  }
#pragma unroll 4
  for (int64_t t = from + threadIdx.x; t < t0; t += 256) before += kept(a.tokens, a.mask, t, a.V) ? 1 : 0;
  before = block_count(before, red);
  const bool mine = lane < ROWS && t0 + lane < a.T && kept(a.tokens, a.mask, t0 + lane, a.V);
  const uint32_t keep = (uint32_t)__ballot(mine);
  if (t0 + ROWS >= a.T && threadIdx.x == 0) *a.cnt = before + __popc(keep);
  const int r = wave;
  const int64_t t = t0 + r;
  if (t >= a.T) return;
  if (!((keep >> r) & 1)) {
    if (lane == 0) {
      a.row_pos[t] = -1;
      if (a.mode != kBeginBackward) a.lse[t] = a.loss_rows[t] = 0.f;
    }
    return;
  }
  const int pos = before + __popc(keep & ((1u << r) - 1));
  if (lane == 0) {
    const int token = a.tokens[t];
    a.row_pos[t] = pos;
    a.kept_idx[pos] = (int32_t)t;
    a.tokens_c[pos] = token;
    if (a.mode == kBeginBackward) reinterpret_cast<LmRow*>(a.rows_c)[pos] = LmRow{a.lse[t], a.weights ? a.weights[t] : 1.f, token};
    else if (a.mode == kBeginForwardFp32) reinterpret_cast<RowState*>(a.rows_c)[pos] = RowState{-INFINITY, 0.f, 0.f};
  }
  const T* src = (const T*)a.y + (size_t)t * a.d;
  T* dst = (T*)a.y_c + (size_t)pos * a.d;
  if (a.d % 8 == 0) {
#pragma unroll 8
    for (int c = lane * 8; c < a.d; c += 64 * 8) {
      float v[8];
      ld8(src, c, v);
      st8(dst, c, v);
    }
  } else {
    for (int c = lane; c < a.d; c += 64) dst[c] = src[c];
  }
}

// fp32: one block per row, a piece's columns join the row's statistics; with the last piece they are complete
__global__ __launch_bounds__(256) void lm_stats_kernel(const float* __restrict__ z, int64_t ldz, int n0, int n, const int32_t* __restrict__ tokens,
                                                       const int* __restrict__ cnt, RowState* __restrict__ st, int last, const int32_t* __restrict__ kept_idx,
                                                       float* __restrict__ lse, float* __restrict__ loss_rows) {
  __shared__ Online sm[4];
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const float* zr = z + (size_t)row * ldz;
  Online x = online_block<256>(row_stats<float, 256>(zr, n, kLog2e), kLog2e, sm);
  if (threadIdx.x == 0) {
    const RowState o = st[row];
    const int t = tokens[row] - n0;
    const float m = fmaxf(x.m, o.m);
    const float s = (x.m == -INFINITY ? x.s : x.s * expf(x.m - m)) + (o.m == -INFINITY ? o.s : o.s * expf(o.m - m));
    const RowState all{m, s, t >= 0 && t < n ? zr[t] : o.z};
    if (last) {
      const float log_s = logf(all.s);
      const int at = kept_idx[row];
      lse[at] = all.m + log_s;
      loss_rows[at] = log_s + (all.m - all.z);
    } else {
      st[row] = all;
    }
  }
}

// bf16: a row's statistics of all tiles as one.  Sixteen rows per block (their pairs lie side by side), 64 threads each, four pairs at a time.
__global__ __launch_bounds__(1024) void lm_join_kernel(const float2* __restrict__ part, int64_t part_ld, int tiles, const float* __restrict__ label,
                                                       const int32_t* __restrict__ kept_idx, const int* __restrict__ cnt,
                                                       float* __restrict__ lse, float* __restrict__ loss_rows) {
  constexpr int U = 4, BY = 64;
  __shared__ float2 st[16][17];
  const int r = threadIdx.x & 15, by = threadIdx.x >> 4;
  const int64_t i = (int64_t)blockIdx.x * 16 + r;
  const int n = *cnt;
  if ((int64_t)blockIdx.x * 16 >= n) return;   // whole block
  float2 o = make_float2(-INFINITY, 0.f);
  auto scaled = [](float2 x, float m) { return m > -INFINITY ? x.y * __builtin_amdgcn_exp2f((x.x - m) * kLog2e) : x.y; };   // (below any number: 0, or NaN)
  auto join = [&](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    return make_float2(m, scaled(a, m) + scaled(b, m));
  };
  if (i < n) {
    for (int t = by; t < tiles; t += U * BY) {
      float2 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = t + u * BY < tiles ? part[(size_t)(t + u * BY) * part_ld + i] : make_float2(-INFINITY, 0.f);
      float m = o.x;
#pragma unroll
      for (int u = 0; u < U; ++u) m = fmaxf(m, x[u].x);
      o.y = scaled(o, m);
#pragma unroll
      for (int u = 0; u < U; ++u) o.y += scaled(x[u], m);
      o.x = m;
    }
  }
#pragma unroll
  for (int d = 16; d < 64; d *= 2) o = join(o, make_float2(__shfl_xor(o.x, d, 64), __shfl_xor(o.y, d, 64)));
  if ((threadIdx.x & 63) < 16) st[threadIdx.x >> 6][r] = o;
  __syncthreads();
  if (threadIdx.x < 16 && i < n) {
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = fmaxf(m, st[k][r].x);
#pragma unroll
    for (int k = 0; k < 16; ++k) s += scaled(st[k][r], m);
    const float log_s = logf(s);
    const int at = kept_idx[i];
    lse[at] = m + log_s;
    loss_rows[at] = log_s + (m - label[i]);
  }
}

// fp32: a piece's logits become their gradient (and what is behind a row's last column up to the next multiple of eight, something)
__global__ __launch_bounds__(256) void lm_grad_kernel(float* z, int64_t ldz, int n0, int n, const int* __restrict__ cnt, const LmRow* __restrict__ rows) {
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const LmRow o = rows[row];
  const int t = o.token - n0;
  float* zr = z + (size_t)row * ldz;
  const int first = (blockIdx.y * 256 + threadIdx.x) * 8, step = (int)gridDim.y * 2048;
  for (int c = first; c < n; c += step) {
    float v[8];
    ld8(zr, c, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = o.weight * (expf(v[j] - o.lse) - (c + j == t ? 1.f : 0.f));
    st8(zr, c, v);
  }
}

// fp32, up to kFewRows rows of a wide head: dy and dW in one pass over W.  A wave takes 256 columns and every so many-th four entries of the vocabulary: it reads
// their weights, adds them to dy by the rows' dz (scalars), and writes dW = scale dz^T y from the rows of y that it holds.  The waves of a block
// add their dy in LDS; a block's sum is one of the parts that lm_scatter_kernel joins.  Bound by memory where there are blocks enough (d / 256 x 32): this kernel
// alone 836 us at 1 x 128256 x 4008 (4.9 TB/s, 512 blocks), 358 at 2048 wide (5.9 TB/s), 236 at 1024 (4.4), 199 at 256 (1.3: 32 blocks).  With more rows on few blocks
// it is bound by its own arithmetic, and the two products are faster.  Both gradients, whole calls, us, two products / this: 1 x 128256 x 256
// 245 / 233, x 512 321 / 262, x 2048 926 / 563, x 4096 1781 / 1139; 2 x 128256 x 512 322 / 339, x 1024 536 / 398; 4 x 128256 x 256 250 / 473, x 1024 539 / 557, x 2048 942 / 696,
// x 4096 1823 / 1107; dy alone 2 x 128256 x 512 221 / 275, x 1024 319 / 328; 4 x 128256 x 1024 327 / 465, x 2048 558 / 568, x 4096 1122 / 827; over 32000 entries in the same
// places.  Hence from 512 columns a row on.  (With room for 16 rows 14 x 98922 x 2800 took 896, the products 829.)
constexpr int kFewRows = 4;
template <bool DW>
__global__ __launch_bounds__(256) void lm_few_kernel(const float* __restrict__ z, int64_t ldz, int n, const float* __restrict__ w, const float* __restrict__ y,
                                                     int d, const int* __restrict__ cnt, float scale, float* __restrict__ dy, int64_t stride,
                                                     float* __restrict__ dw) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  __shared__ f32x4_t sm[3][kFewRows][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = min(__builtin_amdgcn_readfirstlane(*cnt), kFewRows);
  const int col = ((int)blockIdx.x * 64 + lane) * 4, c = min(col, d - 4);   // (d is a multiple of 4)
  const bool in = col < d;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t acc[kFewRows], ym[DW ? kFewRows : 1];
#pragma unroll
  for (int m = 0; m < kFewRows; ++m) {
    acc[m] = zero;
    if constexpr (DW) ym[m] = m < rows ? *reinterpret_cast<const f32x4_t*>(y + (size_t)m * d + c) : zero;
  }
  const int fours = (n + 3) / 4, step = (int)gridDim.y * 4;
  auto fetch = [&](f32x4_t (&x)[4], int v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(w + (size_t)min(v + i, n - 1) * d + c));
  };
  f32x4_t next[4] = {zero, zero, zero, zero};
  int q = (int)blockIdx.y * 4 + wave;
  if (q < fours) fetch(next, q * 4);
  for (; q < fours; q += step) {
    const int v = q * 4;
    f32x4_t k[kFewRows], x[4], g[4] = {zero, zero, zero, zero};
#pragma unroll
    for (int m = 0; m < kFewRows; ++m) k[m] = *reinterpret_cast<const f32x4_t*>(z + (size_t)max(min(m, rows - 1), 0) * ldz + v);   // (a row is padded to whole 16 bytes)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = next[i];
    if (q + step < fours) fetch(next, (q + step) * 4);
#pragma unroll
    for (int m = 0; m < kFewRows; ++m) {
      if (m < rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ki = v + i < n ? k[m][i] : 0.f;
          acc[m] += ki * x[i];
          if constexpr (DW) g[i] += ki * ym[m];
        }
      }
    }
    if constexpr (DW) {
      if (in) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v + i < n) __builtin_nontemporal_store(scale * g[i], reinterpret_cast<f32x4_t*>(dw + (size_t)(v + i) * d + c));
      }
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int m = 0; m < kFewRows; ++m) sm[wave - 1][m][lane] = acc[m];
  }
  __syncthreads();
  if (wave == 0 && in) {
    float* out = dy + (size_t)blockIdx.y * stride;
#pragma unroll
    for (int m = 0; m < kFewRows; ++m)
      if (m < rows) *reinterpret_cast<f32x4_t*>(out + (size_t)m * d + c) = scale * (((acc[m] + sm[0][m][lane]) + sm[1][m][lane]) + sm[2][m][lane]);
  }
}

// compact rows back to their places, zeros elsewhere.  A row is the sum of `parts`, `stride` elements apart.
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void lm_scatter_kernel(const TI* __restrict__ src, TO* __restrict__ dst, int d, const int32_t* __restrict__ row_pos, int parts, int64_t stride) {
  const size_t t = blockIdx.x;
  const int i = row_pos[t];
  TO* b = dst + t * (size_t)d;
  const TI* a = src + (size_t)max(i, 0) * d;
  if (d % 8 == 0) {
    for (int c = threadIdx.x * 8; c < d; c += 256 * 8) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (i >= 0) ld8(a, c, v);
      if constexpr (sizeof(TI) == 4 && sizeof(TO) == 4) {
#pragma unroll 4
        for (int q = 1; q < parts && i >= 0; ++q) {
          float x[8];
          ld8(a + q * stride, c, x);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += x[j];
        }
      }
      st8(b, c, v);
    }
  } else {
    for (int c = threadIdx.x; c < d; c += 256) {
      float v = i < 0 ? 0.f : ldf(a, c);
      for (int q = 1; q < parts && i >= 0; ++q) v += ldf(a + q * stride, c);
      stf(b, c, v);
    }
  }
}

size_t lm_ce_workspace_bytes(int64_t rows, int64_t V, int64_t d, int dtype) { return make_plan(rows, V, d, dtype).total; }

namespace {
#define LM_TRY(call) do { const hipError_t e__ = (call); if (e__ != hipSuccess) return e__; } while (0)

struct LmCe {
  const LmCeArgs& a;
  LmCePlan p;
  Pieces pc;
  char* ws;
  hipStream_t s;
  LmCe(const LmCeArgs& args, hipStream_t stream)
      : a(args), p(make_plan(args.rows, args.V, args.d, args.dtype)), pc(plan_pieces(args.rows, args.V, args.dtype)), ws((char*)args.ws), s(stream) {}
  template <typename T> T* at(size_t off) const { return (T*)(ws + off); }
  const int* cnt() const { return at<const int>(p.cnt); }

  hipError_t begin(bool backward) {
    ProfScope ps("lm_ce_begin", 0, 2.0 * (double)a.rows * a.d * dtype_size(a.dtype), s);
    const bool direct = a.rows <= kDirectRows;
    if (!direct) {
      hipLaunchKernelGGL(lm_count_kernel, dim3((unsigned)((a.rows + kCountRows - 1) / kCountRows)), dim3(256), 0, s, a.tokens, a.mask, a.rows, (int)a.V, at<int>(p.counts));
      LM_TRY(hipGetLastError());
    }
    const LmBegin b{a.y, a.tokens, a.mask, a.row_weights, a.lse, a.loss_rows, ws + p.y_c, at<int32_t>(p.tokens_c), at<int32_t>(p.kept_idx),
                    at<int32_t>(p.row_pos), at<int>(p.cnt), ws + p.rows_c, direct ? nullptr : at<int>(p.counts), a.rows, (int)a.V, (int)a.d,
                    backward ? kBeginBackward : a.dtype == kF32 ? kBeginForwardFp32 : kBeginForward};
    const dim3 grid((unsigned)((a.rows + 3) / 4)), blk(256);
    if (a.dtype == kBF16) hipLaunchKernelGGL(lm_begin_kernel<bf16_t>, grid, blk, 0, s, b);
    else hipLaunchKernelGGL(lm_begin_kernel<float>, grid, blk, 0, s, b);
    return hipGetLastError();
  }
  const char* piece_w(const Piece& q) const { return (const char*)a.w + (size_t)q.n0 * a.d * dtype_size(a.dtype); }
  // y_c times the piece's rows of W, transposed
  GemmArgs logits(const Piece& q) const {
    GemmArgs g = product(kNT, a.rows, q.n, a.d, ws + p.y_c, a.d, piece_w(q), a.d, ws + p.z, piece_ld(pc), a.dtype, a.dtype);
    g.m_dev = cnt();
    return g;
  }
  hipError_t with_scratch(GemmArgs g) const {
    if (p.split_bytes) { g.scratch = ws + p.split; g.scratch_bytes = p.split_bytes; }
    return launch_gemm(g, s);
  }
};
}  // namespace

hipError_t launch_lm_ce_fwd(const LmCeArgs& a, hipStream_t s) {
  LmCe c(a, s);
  LM_TRY(c.begin(false));
  if (a.dtype == kBF16) {
    GemmArgs g = c.logits(Piece{0, a.V, 0});
    g.ldc = a.V;
    const int tiles = (int)((a.V + kLmColumns - 1) / kLmColumns);
    float* label = c.at<float>(c.p.rows_c);
    LmTarget t{c.at<int32_t>(c.p.tokens_c), c.at<float2>(c.p.z), a.rows, label, nullptr, 0, 0};
    LM_TRY(launch_gemm_lm_stats(g, t, s));
    ProfScope ps("lm_ce_join", 0, 8.0 * (double)a.rows * tiles, s);
    prof_dynamic(c.cnt(), 0, a.rows);
    hipLaunchKernelGGL(lm_join_kernel, dim3((unsigned)((a.rows + 15) / 16)), dim3(1024), 0, s, t.part, t.part_ld, tiles, label,
                       c.at<int32_t>(c.p.kept_idx), c.cnt(), a.lse, a.loss_rows);
    return hipGetLastError();
  }
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    LM_TRY(launch_gemm_fp32_few(c.logits(q), s));
    ProfScope ps("lm_ce_stats_fp32", 0, 8.0 * (double)a.rows * q.n, s);
    prof_dynamic(c.cnt(), 0, a.rows);
    hipLaunchKernelGGL(lm_stats_kernel, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), piece_ld(c.pc), (int)q.n0, (int)q.n,
                       c.at<int32_t>(c.p.tokens_c), c.cnt(), c.at<RowState>(c.p.rows_c), i + 1 == c.pc.count ? 1 : 0, c.at<int32_t>(c.p.kept_idx),
                       a.lse, a.loss_rows);
    LM_TRY(hipGetLastError());
  }
  return hipSuccess;
}

hipError_t launch_lm_ce_bwd(const LmCeArgs& a, hipStream_t s) {
  LmCe c(a, s);
  LM_TRY(c.begin(true));
  const int64_t ld = piece_ld(c.pc);
  const bool bf16 = a.dtype == kBF16, to_acc = bf16 && c.pc.count > 1;
  const LmRow* rows = c.at<LmRow>(c.p.rows_c);
  // very few rows (a single piece then) of a wide head: one pass over W; else each gradient as a product
  const bool few = !bf16 && a.rows <= kFewRows && a.d % 4 == 0 && a.d >= 512 * a.rows && a.d <= 16384;
  const int parts = bf16 ? 1 : few ? (int)std::min<int64_t>(kMaxFp32Parts, (a.V + 63) / 64) : gemm_fp32_parts(a.rows, a.d, c.pc.width);
  const int64_t part_stride = a.rows * a.d;
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    if (bf16) {
      LM_TRY(launch_gemm_lm_grad(c.logits(q), LmTarget{nullptr, nullptr, 0, nullptr, rows, (int)q.n0, q.zero}, s));
    } else {
      LM_TRY(launch_gemm_fp32_few(c.logits(q), s));
      ProfScope ps("lm_ce_grad_fp32", 0, 8.0 * (double)a.rows * q.n, s);
      prof_dynamic(c.cnt(), 0, a.rows);
      hipLaunchKernelGGL(lm_grad_kernel, dim3((unsigned)a.rows, (unsigned)std::min<int64_t>((q.n + 2047) / 2048, 64)), dim3(256), 0, s, c.at<float>(c.p.z), ld, (int)q.n0, (int)q.n, c.cnt(), rows);
      LM_TRY(hipGetLastError());
    }
    if (few) {
      ProfScope ps("lm_ce_few_fp32", 2.0 * (a.dw ? 2 : 1) * a.rows * q.n * a.d, 4.0 * (a.dw ? 2 : 1) * q.n * a.d, s);
      const dim3 grid((unsigned)((a.d + 255) / 256), (unsigned)parts);
      const float *z = c.at<float>(c.p.z), *y = c.at<float>(c.p.y_c);
      if (a.dw) hipLaunchKernelGGL(lm_few_kernel<true>, grid, dim3(256), 0, s, z, ld, (int)q.n, (const float*)a.w, y, (int)a.d, c.cnt(), a.scale, c.at<float>(c.p.acc), part_stride, (float*)a.dw);
      else hipLaunchKernelGGL(lm_few_kernel<false>, grid, dim3(256), 0, s, z, ld, (int)q.n, (const float*)a.w, y, (int)a.d, c.cnt(), a.scale, c.at<float>(c.p.acc), part_stride, nullptr);
      LM_TRY(hipGetLastError());
      break;
    }
    GemmArgs g = product(kNN, a.rows, a.d, q.n, c.ws + c.p.z, ld, c.piece_w(q), a.d, c.ws + c.p.acc, a.d, a.dtype, to_acc ? kF32 : a.dtype);
    g.m_dev = c.cnt();
    g.alpha = a.scale;
    g.accumulate = i > 0;
    if (bf16) LM_TRY(c.with_scratch(g));
    else LM_TRY(launch_gemm_fp32_parts(g, parts, part_stride, s));
    if (a.dw) {
      GemmArgs w = product(kTN, q.n, a.d, a.rows, c.ws + c.p.z, ld, c.ws + c.p.y_c, a.d, (char*)a.dw + (size_t)q.n0 * a.d * dtype_size(a.dw_dtype), a.d,
                           a.dtype, a.dw_dtype);
      w.k_dev = c.cnt();
      w.alpha = a.scale;
      LM_TRY(c.with_scratch(w));
    }
  }
  ProfScope ps("lm_ce_scatter", 0, (double)a.rows * a.d * (dtype_size(a.dtype) + (to_acc ? 4.0 : dtype_size(a.dtype))), s);
  const dim3 grid((unsigned)a.rows), blk(256);
  const int32_t* row_pos = c.at<int32_t>(c.p.row_pos);
  if (to_acc) hipLaunchKernelGGL((lm_scatter_kernel<float, bf16_t>), grid, blk, 0, s, c.at<float>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos, parts, part_stride);
  else if (bf16) hipLaunchKernelGGL((lm_scatter_kernel<bf16_t, bf16_t>), grid, blk, 0, s, c.at<bf16_t>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos, parts, part_stride);
  else hipLaunchKernelGGL((lm_scatter_kernel<float, float>), grid, blk, 0, s, c.at<float>(c.p.acc), (float*)a.dy, (int)a.d, row_pos, parts, part_stride);
  return hipGetLastError();
}

}  // namespace tide
