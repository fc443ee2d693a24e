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
// Bound by the matrix pipes: [27853 kept of 32768, 128256], width 4096, bf16: forward 21.5 ms, backward 64.7 ms, 1.36 PFLOP/s over the four products that run.
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
// Elements that a piece's array has room for: rows x the vocabulary up to 1 GiB, and at least 256 columns.  Never falls as the rows grow.
int64_t piece_elems(int64_t rows, int64_t V, int dtype) {
  const int64_t budget = ((int64_t)1 << 30) / (int64_t)dtype_size(dtype);
  return std::max(rows * 256, std::min(rows * (int64_t)align_up((size_t)V, 256), budget));
}
Pieces plan_pieces(int64_t rows, int64_t V, int dtype) {
  const bool by8 = dtype == kBF16;
  const int64_t most = piece_elems(rows, V, dtype) / rows / 256 * 256, count = (V + most - 1) / most;
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

struct LmCePlan {
  size_t plan_cnt, scal, cnt, status, kept_idx, row_pos, mask_eff, mask_c, tokens_c, rows_c, y_c;
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
  p.plan_cnt = take(plan_rows_scratch_bytes(rows));
  p.scal = take(64);
  p.cnt = take(64);
  p.status = take(64);
  p.kept_idx = take(T * 4);
  p.row_pos = take(T * 4);
  p.mask_eff = take(T);
  p.mask_c = take(T);
  p.tokens_c = take(T * 4);
  p.rows_c = take(T * sizeof(LmRow));
  p.y_c = take(T * d * es);
  // (statistics of 128 columns each are fewer bytes than the whole vocabulary's dz, which is what the array holds where tiles are that small)
  p.z = take(std::max((size_t)piece_elems(rows, V, dtype) * es, dtype == kBF16 ? T * (size_t)((V + 255) / 256) * sizeof(float2) : 0));
  p.acc = pc.count > 1 && dtype == kBF16 ? take(T * d * 4) : 0;
  p.dy_c = take(T * d * es);
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

// what the products need of every compact row: the log-sum-exp, its weight and its label (backward; fp32's forward: nothing seen yet)
__global__ __launch_bounds__(256) void lm_rows_kernel(const float* __restrict__ lse, const float* __restrict__ weights, const int32_t* __restrict__ tokens_c,
                                                      const int32_t* __restrict__ kept_idx, const int* __restrict__ cnt, void* __restrict__ rows, int backward) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= *cnt) return;
  if (backward) {
    const int r = kept_idx[i];
    reinterpret_cast<LmRow*>(rows)[i] = LmRow{-lse[r] * 1.4426950408889634f, weights ? weights[r] : 1.f, tokens_c[i], lse[r]};
  } else {
    reinterpret_cast<RowState*>(rows)[i] = RowState{-INFINITY, 0.f, 0.f};
  }
}

// fp32: one block per row, a piece's columns join the row's statistics
__global__ __launch_bounds__(256) void lm_stats_kernel(const float* __restrict__ z, int64_t ldz, int n0, int n, const int32_t* __restrict__ tokens,
                                                       const int* __restrict__ cnt, RowState* __restrict__ st) {
  __shared__ float sm[4];
  __shared__ float red[17];
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const float* zr = z + (size_t)row * ldz;
  float m = -INFINITY;
  for (int c = threadIdx.x; c < n; c += 256) m = fmaxf(m, zr[c]);
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const RowState o = st[row];
  m = fmaxf(m, o.m);
  float s = 0.f;
  for (int c = threadIdx.x; c < n; c += 256) s += expf(zr[c] - m);
  s = block_sum(s, red);
  if (threadIdx.x == 0) {
    const int t = tokens[row] - n0;
    st[row] = RowState{m, (o.m == -INFINITY ? o.s : o.s * expf(o.m - m)) + s, t >= 0 && t < n ? zr[t] : o.z};
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
  const float log_s = logf(o.s);
  lse[t] = o.m + log_s;
  loss_rows[t] = log_s + (o.m - o.z);
}

// bf16: a row's statistics of all tiles as one.  Sixteen rows per block (their pairs lie side by side), sixteen threads each.
__global__ __launch_bounds__(256) void lm_join_kernel(int64_t T, const float2* __restrict__ part, int64_t part_ld, int tiles, const float* __restrict__ label,
                                                      const int32_t* __restrict__ kept_idx, const int32_t* __restrict__ row_pos, const int* __restrict__ cnt,
                                                      float* __restrict__ lse, float* __restrict__ loss_rows) {
  __shared__ float2 st[16][17];
  const int r = threadIdx.x & 15, by = threadIdx.x >> 4;
  const int64_t i = (int64_t)blockIdx.x * 16 + r;
  const int n = *cnt;
  if (by == 0 && i < T && row_pos[i] < 0) {   // (as a row of the batch, not of the compact array)
    lse[i] = 0.f;
    loss_rows[i] = 0.f;
  }
  float2 o = make_float2(-INFINITY, 0.f);
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    if (m > -INFINITY) a.y = a.y * expf(a.x - m) + b.y * expf(b.x - m);
    else a.y += b.y;                          // 0, or NaN
    a.x = m;
    return a;
  };
  if (i < n) {
#pragma unroll 4
    for (int t = by; t < tiles; t += 16) o = join(o, part[(size_t)t * part_ld + i]);
  }
  st[by][r] = o;
  __syncthreads();
  if (by == 0 && i < n) {
    for (int k = 1; k < 16; ++k) o = join(o, st[k][r]);
    const float log_s = logf(o.y);
    const int at = kept_idx[i];
    lse[at] = o.x + log_s;
    loss_rows[at] = log_s + (o.x - label[i]);
  }
}

// fp32: a piece's logits become their gradient
__global__ __launch_bounds__(256) void lm_grad_kernel(float* z, int64_t ldz, int n0, int n, const int* __restrict__ cnt, const LmRow* __restrict__ rows) {
  const int row = blockIdx.x;
  if (row >= *cnt) return;
  const LmRow o = rows[row];
  const int t = o.token - n0;
  float* zr = z + (size_t)row * ldz;
  for (int c = threadIdx.x; c < n; c += 256) zr[c] = o.weight * (expf(zr[c] - o.lse) - (c == t ? 1.f : 0.f));
}

// compact rows back to their places, zeros elsewhere
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void lm_scatter_kernel(const TI* __restrict__ src, TO* __restrict__ dst, int d, const int32_t* __restrict__ row_pos) {
  const size_t t = blockIdx.x;
  const int i = row_pos[t];
  TO* b = dst + t * (size_t)d;
  const TI* a = src + (size_t)max(i, 0) * d;
  if (d % 8 == 0) {
    for (int c = threadIdx.x * 8; c < d; c += 256 * 8) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (i >= 0) ld8(a, c, v);
      st8(b, c, v);
    }
  } else {
    for (int c = threadIdx.x; c < d; c += 256) stf(b, c, i < 0 ? 0.f : ldf(a, c));
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
    LM_TRY(launch_plan_rows(a.tokens, a.mask, a.rows, (int)a.V, 0, at<float>(p.scal), at<int>(p.cnt), at<int32_t>(p.kept_idx), at<int32_t>(p.row_pos),
                            nullptr, 0, 0, at<uint8_t>(p.mask_eff), at<int>(p.status), at<int>(p.plan_cnt), nullptr, 0, 0, 0.f, nullptr, s));
    LM_TRY(launch_gather_rows(a.rows, (int)a.d, a.y, ws + p.y_c, 0, nullptr, nullptr, a.tokens, a.mask, at<int32_t>(p.kept_idx), cnt(),
                              at<int32_t>(p.tokens_c), at<uint8_t>(p.mask_c), a.dtype, s));
    if (!backward && a.dtype == kBF16) return hipSuccess;
    ProfScope ps("lm_ce_rows", 0, 32.0 * (double)a.rows, s);
    hipLaunchKernelGGL(lm_rows_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a.lse, a.row_weights, at<int32_t>(p.tokens_c),
                       at<int32_t>(p.kept_idx), cnt(), (void*)(ws + p.rows_c), backward ? 1 : 0);
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
    const int columns = gemm_lm_stat_columns(g), tiles = (int)((a.V + columns - 1) / columns);
    float* label = c.at<float>(c.p.rows_c);
    LmTarget t{c.at<int32_t>(c.p.tokens_c), c.at<float2>(c.p.z), a.rows, label, nullptr, 0, 0};
    LM_TRY(launch_gemm_lm_stats(g, t, s));
    ProfScope ps("lm_ce_join", 0, 8.0 * (double)a.rows * tiles, s);
    prof_dynamic(c.cnt(), 0, a.rows);
    hipLaunchKernelGGL(lm_join_kernel, dim3((unsigned)((a.rows + 15) / 16)), dim3(256), 0, s, a.rows, t.part, t.part_ld, tiles, label,
                       c.at<int32_t>(c.p.kept_idx), c.at<int32_t>(c.p.row_pos), c.cnt(), a.lse, a.loss_rows);
    return hipGetLastError();
  }
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    LM_TRY(launch_gemm(c.logits(q), s));
    ProfScope ps("lm_ce_stats_fp32", 0, 8.0 * (double)a.rows * q.n, s);
    prof_dynamic(c.cnt(), 0, a.rows);
    hipLaunchKernelGGL(lm_stats_kernel, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), piece_ld(c.pc), (int)q.n0, (int)q.n,
                       c.at<int32_t>(c.p.tokens_c), c.cnt(), c.at<RowState>(c.p.rows_c));
    LM_TRY(hipGetLastError());
  }
  ProfScope ps("lm_ce_loss", 0, 24.0 * (double)a.rows, s);
  hipLaunchKernelGGL(lm_loss_kernel, dim3((unsigned)((a.rows + 255) / 256)), dim3(256), 0, s, a.rows, c.at<int32_t>(c.p.row_pos),
                     c.at<RowState>(c.p.rows_c), a.lse, a.loss_rows);
  return hipGetLastError();
}

hipError_t launch_lm_ce_bwd(const LmCeArgs& a, hipStream_t s) {
  LmCe c(a, s);
  LM_TRY(c.begin(true));
  const int64_t ld = piece_ld(c.pc);
  const bool bf16 = a.dtype == kBF16, to_acc = bf16 && c.pc.count > 1;
  const LmRow* rows = c.at<LmRow>(c.p.rows_c);
  for (int i = 0; i < c.pc.count; ++i) {
    const Piece q = piece_at(c.pc, i);
    if (bf16) {
      LM_TRY(launch_gemm_lm_grad(c.logits(q), LmTarget{nullptr, nullptr, 0, nullptr, rows, (int)q.n0, q.zero}, s));
    } else {
      LM_TRY(launch_gemm(c.logits(q), s));
      ProfScope ps("lm_ce_grad_fp32", 0, 8.0 * (double)a.rows * q.n, s);
      prof_dynamic(c.cnt(), 0, a.rows);
      hipLaunchKernelGGL(lm_grad_kernel, dim3((unsigned)a.rows), dim3(256), 0, s, c.at<float>(c.p.z), ld, (int)q.n0, (int)q.n, c.cnt(), rows);
      LM_TRY(hipGetLastError());
    }
    GemmArgs g = product(kNN, a.rows, a.d, q.n, c.ws + c.p.z, ld, c.piece_w(q), a.d, c.ws + c.p.acc, a.d, a.dtype, to_acc ? kF32 : a.dtype);
    g.m_dev = c.cnt();
    g.alpha = a.scale;
    g.accumulate = i > 0;
    LM_TRY(c.with_scratch(g));
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
  if (to_acc) hipLaunchKernelGGL((lm_scatter_kernel<float, bf16_t>), grid, blk, 0, s, c.at<float>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos);
  else if (bf16) hipLaunchKernelGGL((lm_scatter_kernel<bf16_t, bf16_t>), grid, blk, 0, s, c.at<bf16_t>(c.p.acc), (bf16_t*)a.dy, (int)a.d, row_pos);
  else hipLaunchKernelGGL((lm_scatter_kernel<float, float>), grid, blk, 0, s, c.at<float>(c.p.acc), (float*)a.dy, (int)a.d, row_pos);
  return hipGetLastError();
}

}  // namespace tide
