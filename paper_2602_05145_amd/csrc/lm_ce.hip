// Softmax cross-entropy of the LM head from the hidden states, z = y W^T, without keeping logits:
//   forward    lse_r = log sum_v exp(z_rv),  loss_r = lse_r - z[r, token_r]
//   backward   dz_rv = weight_r (exp(z_rv - lse_r) - [v = token_r]),  dy = scale dz W,  dW = scale dz^T y
// A logit exists only inside a piece of the vocabulary: the backward pass makes every piece again from y, W and lse, turns
// it into its gradient, and feeds that to both products before the next piece takes its place.  Rows without loss are left
// out: the others are copied into a dense array first, so that whatever stands in the rest (NaN as well) touches nothing.
#include <algorithm>
#include <cstring>

#include "kernels.h"
#include "prof.h"
#include "tide_common.h"

namespace tide {

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The vocabulary in pieces, the last one first.  A piece's columns are the contraction of dy: bf16 products take a multiple
// of 8 of them.  Where the vocabulary is not one, the last piece reaches back over up to 7 columns of the one before, with
// gradients of zero there: they add nothing to dy, and the rows of dW that come out zero are written again, right, by the
// piece that they belong to.
struct Piece { int64_t n0, n; int zero; };   // columns [n0, n0 + n), the first `zero` of them another piece's
struct Pieces { int64_t V, width; int count; bool by8; };
// Elements that a piece's array has room for: rows x the vocabulary up to the budget, and at least 256 columns.  Never falls as the rows grow.
int64_t piece_elems(int64_t rows, int64_t V, int dtype) {
  const int64_t budget = dtype == kBF16 ? (int64_t)1 << 27 : (int64_t)1 << 28;
  return std::max(rows * 256, std::min(rows * (int64_t)align_up((size_t)V, 256), budget));
}
Pieces plan_pieces(int64_t rows, int64_t V, int dtype) {
  const bool by8 = dtype == kBF16;
  int64_t width = piece_elems(rows, V, dtype) / rows / 256 * 256;
  int64_t count = (V + width - 1) / width;
  if (count == 1 && by8 && V % 8) {
    width = V / 8 * 8;       // and the rest, at most 7 columns, as a piece of 8
    count = 2;
  }
  return Pieces{V, width, (int)count, by8};
}
Piece piece_at(const Pieces& p, int i) {   // i = 0: the last one
  const int64_t at = p.count - 1 - i, n0 = at * p.width, n = std::min(p.width, p.V - n0);
  const int back = p.by8 && n % 8 ? (int)(8 - n % 8) : 0;
  return Piece{n0 - back, n + back, back};
}
// elements between two rows of a piece
int64_t piece_ld(const Pieces& p) { return (int64_t)align_up((size_t)p.width, 64); }

struct LmCePlan {
  size_t plan_cnt, scal, cnt, status, kept_idx, row_pos, mask_eff, mask_c, tokens_c, rows_c, y_c;
  size_t z, dz, acc, dy_c, split, split_bytes;
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
  p.plan_cnt = take(plan_rows_scratch_bytes(rows));
  p.scal = take(64);
  p.cnt = take(64);
  p.status = take(64);
  p.kept_idx = take(T * 4);
  p.row_pos = take(T * 4);
  p.mask_eff = take(T);
  p.mask_c = take(T);
  p.tokens_c = take(T * 4);
  p.rows_c = take(T * 12);
  p.y_c = take(T * d * es);
  const size_t elems = (size_t)piece_elems(rows, V, dtype);
  p.z = take(elems * 4);
  p.dz = dtype == kBF16 ? take(elems * 2) : p.z;
  p.acc = pc.count > 1 && dtype == kBF16 ? take(T * d * 4) : 0;
  p.dy_c = take(T * d * es);
  if (dtype == kF32 || pc.count == 1) p.acc = p.dy_c;
  p.split_bytes = 0;
  p.split = off;
  p.total = off;
  return p;
}

// per compact row: running maximum, sum and label logit (forward); log-sum-exp and weight (backward)
struct RowState { float a, b, c; };

}  // namespace

__global__ __launch_bounds__(256) void lm_rows_kernel(const float* __restrict__ lse, const float* __restrict__ weights, const int32_t* __restrict__ kept_idx,
                                                      const int* __restrict__ cnt, RowState* __restrict__ st, int backward) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= *cnt) return;
  if (backward) {
    const int r = kept_idx[i];
    st[i] = RowState{lse[r], weights ? weights[r] : 1.f, 0.f};
  } else {
    st[i] = RowState{-INFINITY, 0.f, 0.f};
  }
}

// one block per row: a piece's columns join the row's statistics
__global__ __launch_bounds__(256) void lm_stats_kernel(const float* __restrict__ z, int64_t ldz, int n0, int n, int zero, const int32_t* __restrict__ tokens,
                                                       const int* __restrict__ cnt, RowState* __restrict__ st) {
  __shared__ float sm[4];
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const float* zr = z + (size_t)row * ldz;
  float m = -INFINITY;
  for (int c = zero + threadIdx.x; c < n; c += 256) m = fmaxf(m, zr[c]);
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const RowState o = st[row];
  m = fmaxf(m, o.a);
  float s = 0.f;
  for (int c = zero + threadIdx.x; c < n; c += 256) s += expf(zr[c] - m);
  __shared__ float red[17];
  s = block_sum(s, red);
  if (threadIdx.x == 0) {
    const int t = tokens[row] - n0;
    st[row] = RowState{m, (o.a == -INFINITY ? o.b : o.b * expf(o.a - m)) + s, t >= zero && t < n ? zr[t] : o.c};
  }
}

__global__ __launch_bounds__(256) void lm_loss_kernel(int64_t T, const int32_t* __restrict__ row_pos, const RowState* __restrict__ st, float* __restrict__ lse,
                                                      float* __restrict__ loss_rows) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= T) return;
  const int i = row_pos[t];
  if (i < 0) {
    lse[t] = 0.f;
    loss_rows[t] = 0.f;
    return;
  }
  const RowState o = st[i];
  const float log_s = logf(o.b);
  lse[t] = o.a + log_s;
  loss_rows[t] = log_s + (o.a - o.c);
}

template <typename T>
__global__ __launch_bounds__(256) void lm_grad_kernel(const float* z, T* dz, int64_t ldz, int n0, int n, int zero, const int32_t* __restrict__ tokens,
                                                      const int* __restrict__ cnt, const RowState* __restrict__ st) {
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const RowState o = st[row];
  const int t = tokens[row] - n0;
  for (int c = threadIdx.x; c < n; c += 256) {
    const float p = expf(z[(size_t)row * ldz + c] - o.a) - (c == t ? 1.f : 0.f);
    stf(dz, (size_t)row * ldz + c, c < zero ? 0.f : o.b * p);
  }
}

template <typename TI, typename TO>
__global__ __launch_bounds__(256) void lm_scatter_kernel(const TI* __restrict__ src, TO* __restrict__ dst, int d, const int32_t* __restrict__ row_pos) {
  const size_t t = blockIdx.x;
  const int i = row_pos[t];
  TO* b = dst + t * (size_t)d;
  for (int c = threadIdx.x; c < d; c += 256) stf(b, c, i < 0 ? 0.f : ldf(src, (size_t)i * d + c));
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
    LM_TRY(launch_plan_rows(a.tokens, a.mask, a.rows, (int)a.V, 0, at<float>(p.scal), at<int>(p.cnt), at<int32_t>(p.kept_idx), at<int32_t>(p.row_pos),
                            nullptr, 0, 0, at<uint8_t>(p.mask_eff), at<int>(p.status), at<int>(p.plan_cnt), nullptr, 0, 0, 0.f, nullptr, s));
    LM_TRY(launch_gather_rows(a.rows, (int)a.d, a.y, ws + p.y_c, 0, nullptr, nullptr, a.tokens, a.mask, at<int32_t>(p.kept_idx), cnt(),
                              at<int32_t>(p.tokens_c), at<uint8_t>(p.mask_c), a.dtype, s));
    hipLaunchKernelGGL(lm_rows_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a.lse, a.row_weights, at<int32_t>(p.kept_idx), cnt(),
                       at<RowState>(p.rows_c), backward ? 1 : 0);
    return hipGetLastError();
  }
  const char* piece_w(const Piece& q) const { return (const char*)a.w + (size_t)q.n0 * a.d * dtype_size(a.dtype); }
  hipError_t logits(const Piece& q) {
    GemmArgs g = product(kNT, a.rows, q.n, a.d, ws + p.y_c, a.d, piece_w(q), a.d, ws + p.z, piece_ld(pc), a.dtype, kF32);
    g.m_dev = cnt();
    return launch_gemm(g, s);
  }
};
}  // namespace

hipError_t launch_lm_ce_fwd(const LmCeArgs& a, hipStream_t s) {
  LmCe c(a, s);
  LM_TRY(c.begin(false));
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    LM_TRY(c.logits(q));
    hipLaunchKernelGGL(lm_stats_kernel, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), piece_ld(c.pc), (int)q.n0, (int)q.n, q.zero,
                       c.at<int32_t>(c.p.tokens_c), c.cnt(), c.at<RowState>(c.p.rows_c));
    LM_TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(lm_loss_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a.rows, c.at<int32_t>(c.p.row_pos),
                     c.at<RowState>(c.p.rows_c), a.lse, a.loss_rows);
  return hipGetLastError();
}

hipError_t launch_lm_ce_bwd(const LmCeArgs& a, hipStream_t s) {
  LmCe c(a, s);
  LM_TRY(c.begin(true));
  const int64_t ld = piece_ld(c.pc);
  const bool bf16 = a.dtype == kBF16, to_acc = bf16 && c.pc.count > 1;
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    LM_TRY(c.logits(q));
    if (bf16) hipLaunchKernelGGL(lm_grad_kernel<bf16_t>, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), c.at<bf16_t>(c.p.dz), ld, (int)q.n0, (int)q.n, q.zero, c.at<int32_t>(c.p.tokens_c), c.cnt(), c.at<RowState>(c.p.rows_c));
    else hipLaunchKernelGGL(lm_grad_kernel<float>, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), c.at<float>(c.p.dz), ld, (int)q.n0, (int)q.n, q.zero, c.at<int32_t>(c.p.tokens_c), c.cnt(), c.at<RowState>(c.p.rows_c));
    LM_TRY(hipGetLastError());
    GemmArgs g = product(kNN, a.rows, a.d, q.n, c.ws + c.p.dz, ld, c.piece_w(q), a.d, c.ws + c.p.acc, a.d, a.dtype, to_acc ? kF32 : a.dtype);
    g.m_dev = c.cnt();
    g.alpha = a.scale;
    g.accumulate = i > 0;
    LM_TRY(launch_gemm(g, s));
    if (a.dw) {
      GemmArgs w = product(kTN, q.n, a.d, a.rows, c.ws + c.p.dz, ld, c.ws + c.p.y_c, a.d, (char*)a.dw + (size_t)q.n0 * a.d * dtype_size(a.dw_dtype), a.d,
                           a.dtype, a.dw_dtype);
      w.k_dev = c.cnt();
      w.alpha = a.scale;
      LM_TRY(launch_gemm(w, s));
    }
  }
  const dim3 grid((unsigned)a.rows), blk(256);
  const int32_t* row_pos = c.at<int32_t>(c.p.row_pos);
  if (to_acc) hipLaunchKernelGGL((lm_scatter_kernel<float, bf16_t>), grid, blk, 0, s, c.at<float>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos);
  else if (bf16) hipLaunchKernelGGL((lm_scatter_kernel<bf16_t, bf16_t>), grid, blk, 0, s, c.at<bf16_t>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos);
  else hipLaunchKernelGGL((lm_scatter_kernel<float, float>), grid, blk, 0, s, c.at<float>(c.p.acc), (float*)a.dy, (int)a.d, row_pos);
  return hipGetLastError();
}

}  // namespace tide
