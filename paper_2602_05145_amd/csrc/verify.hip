// Drafted tokens verified against the target's logits: include/tide_draft.h has the formulas.
//
// Whether a token is accepted, and which one a cumulated distribution gives at a number, is decided at a border: with a vocabulary of 10^5 columns, sums that are
// off by 1e-7 pick another token for one number in forty.  So exponentials and sums are in 64 bits, off by 1e-12 at most.
#include <algorithm>

#include "kernels.h"
#include "prof.h"
#include "row_stats.h"

namespace tide {
namespace {

constexpr int kStep = 2048;       // columns that a block of 256 threads takes at a time, eight a thread
constexpr int kMaxPicks = 64;     // parts of a row that weights are summed over: one lane each
constexpr double kLog2eD = 1.4426950408889634074;

struct Part { double sum; float top; int32_t at; };   // sum of exp((z - top) / tau); the first column that holds the top (without sampling)

// 2^t for -1200 <= t <= 1: n = round(t), and on the rest f in [-1/2, 1/2] the polynomial 1 + f r(f) of least relative error (8.1e-13) with seven degrees
// in r, by exchange of its extreme points.  2^0 is 1.
__device__ __forceinline__ double pow2(double t) {
  const double n = rint(t), f = t - n;
  double r = 1.3178933490506645e-06;
  r = fma(r, f, 1.530915617496178e-05);
  r = fma(r, f, 0.00015403825462319016);
  r = fma(r, f, 0.0013333454860569847);
  r = fma(r, f, 0.009618128616124717);
  r = fma(r, f, 0.05550410935266197);
  r = fma(r, f, 0.2402265069811059);
  r = fma(r, f, 0.6931471805482124);
  return ldexp(fma(r, f, 1.0), (int)n);
}
// exp((z - top) / tau) of numbers z <= top as 2^(slope z + shift): one fused step, and what its rounded shift leaves, the same for all, in `fix`.  From |c top| = 2^40
// on, where next to the largest value the next smaller fp32 number lies 2^16 and more below in the exponent, a power of two takes the place of c: its shift is exact, the
// largest value gives 1 and all others 0, as they should.
struct Scale {
  double slope, shift, fix;
  __device__ __forceinline__ Scale(double c, double top) : slope(c), shift(-c * top), fix(1.0) {
    if (fabs(shift) < 0x1p40) {
      fix = pow2(-fma(c, top, shift));
    } else {
      int e;
      frexp(top, &e);
      slope = ldexp(1.0, 41 - e);
      shift = -slope * top;
    }
  }
  __device__ __forceinline__ double of(float z) const { return pow2(fmax(fma((double)z, slope, shift), -1200.0)); }
};
__device__ __forceinline__ double beside(float z, float top, double c) { return pow2(fmax(((double)z - (double)top) * c, -1200.0)); }   // z <= top, not both infinite
__device__ __forceinline__ bool usable(float top) { return fabsf(top) < INFINITY; }   // (a NaN is not)

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The rows of request b: `rows` of the target, of which the last has no drafted token, and drafts from draft row `first`.  Offsets that are out of order are cut to
// what is there.
struct View { int64_t row0; int64_t first; int n; bool any; };
__device__ __forceinline__ View view_of(const int32_t* cu, int b, int64_t rows, int64_t drafted) {
  const int64_t s0 = min(max((int64_t)cu[b], (int64_t)0), rows), s1 = min(max((int64_t)cu[b + 1], s0), rows);
  View v{s0, s0 - b, (int)(s1 - s0) - 1, s1 > s0};
  if (v.first < 0 || v.n < 0) v.n = 0;
  v.n = (int)min((int64_t)v.n, max(drafted - v.first, (int64_t)0));
  return v;
}
// tau of a request: 0 without sampling, NaN where it is no temperature
__device__ __forceinline__ float tau_of(const float* temperature, int b) {
  const float t = temperature ? temperature[b] : 1.f;
  return t >= 0.f && t < INFINITY ? t : __uint_as_float(0x7FC00000u);
}

template <typename T>
__device__ __forceinline__ void load_row8(const T* row, int64_t col, int64_t V, float (&z)[8]) {   // -inf behind the last column
  if (col < V) ld8(row, (size_t)col, z);
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] = col + j < V ? z[j] : -INFINITY;
}

// Of U * 2048 columns of one row: the largest value and the sum of exponentials beside it.
template <typename T, int U>
__global__ __launch_bounds__(256) void verify_stats_kernel(const VerifyArgs a, int parts, Part* __restrict__ stats, int* __restrict__ tickets) {
  __shared__ double sums[4];
  __shared__ float tops[4];
  __shared__ int places[4];
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.requests; i += (int64_t)gridDim.x * 256) tickets[i] = 0;
  const int64_t unit = blockIdx.x / parts;
  const int part = (int)(blockIdx.x % parts);
  const bool of_target = unit < a.rows;
  const int64_t row = of_target ? unit : unit - a.rows;
  const T* base = of_target ? (const T*)a.target + row * a.ldt : (const T*)a.draft + row * a.ldd;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (int64_t)part * (U * kStep) + threadIdx.x * 8;
  Raw8<T> raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u].load(base, (size_t)min(col + u * kStep, (a.V - 1) / 8 * 8));
  int b = a.requests;   // the first request that ends behind the row
  for (int b0 = 0; b0 < a.requests; b0 += 64) {
    const int k = b0 + lane;
    const unsigned long long ends = __ballot(k < a.requests && (int64_t)a.cu[min(k, a.requests - 1) + 1] - (of_target ? 0 : k + 1) > row);
    if (ends) {
      b = b0 + __ffsll(ends) - 1;
      break;
    }
  }
  if (b >= a.requests) return;
  const float tau = tau_of(a.temperature, b);
  if (!(tau >= 0.f) || (tau == 0.f && !of_target)) return;
  float z[U][8], top = -INFINITY;
  bool odd = false;   // holds a NaN
#pragma unroll
  for (int u = 0; u < U; ++u) {
    raw[u].get(z[u]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[u][j] = col + u * kStep + j < a.V ? z[u][j] : -INFINITY;
      odd |= z[u][j] != z[u][j];
      top = fmaxf(top, z[u][j]);
    }
  }
  top = __ballot(odd) ? __uint_as_float(0x7FC00000u) : fast_max(top);
  Part* out = stats + unit * parts + part;
  if (tau == 0.f) {
    int at = 0x7FFFFFFF;
#pragma unroll
    for (int u = U - 1; u >= 0; --u)
#pragma unroll
      for (int j = 7; j >= 0; --j) at = z[u][j] == top ? (int)(col + u * kStep + j) : at;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
    if (lane == 0) tops[wave] = top, places[wave] = at;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 4; ++w) {
        if (!(top == top)) break;
        if (!(tops[w] <= top)) top = tops[w], at = places[w];
        else if (tops[w] == top) at = min(at, places[w]);
      }
      *out = Part{0.0, top, at};
    }
    return;
  }
  const double c = kLog2eD / (double)tau;
  double sum = 0.0;
  if (usable(top)) {
    const Scale e(c, (double)top);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += e.of(z[u][j]);
    sum = wave_sum(sum) * e.fix;
  }
  if (lane == 0) sums[wave] = sum, tops[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    float m = tops[0];
    for (int w = 1; w < 4; ++w) m = !(tops[w] <= m) ? tops[w] : m;   // (a NaN stays: nothing is at least it)
    for (int w = 0; w < 4; ++w)
      if (!(tops[w] == tops[w])) m = tops[w];
    sum = 0.0;
    if (usable(m))
      for (int w = 0; w < 4; ++w) sum += tops[w] == -INFINITY ? 0.0 : sums[w] * beside(tops[w], m, c);
    *out = Part{sum, m, 0};
  }
}

// A whole row from its parts, by one wave: `ok` where it has a distribution
struct Row { double sum; float top; int at; bool ok; };
__device__ __forceinline__ Row join_row(const Part* p, int parts, double c, bool sampled, int lane) {
  float top = -INFINITY;
  bool odd = false;
  for (int k = lane; k < parts; k += 64) odd |= p[k].top != p[k].top, top = fmaxf(top, p[k].top);
  top = fast_max(top);
  Row r{0.0, top, 0x7FFFFFFF, !__ballot(odd) && usable(top)};
  if (!r.ok) return r;
  for (int k = lane; k < parts; k += 64) {
    if (p[k].top == -INFINITY) continue;
    if (sampled) r.sum += p[k].sum * beside(p[k].top, top, c);
    else if (p[k].top == top) r.at = min(r.at, p[k].at);
  }
  if (sampled) r.sum = wave_sum(r.sum);
  else
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r.at = min(r.at, __shfl_xor(r.at, o, 64));
  return r;
}

// Each of a request's blocks finds out how many drafted tokens are accepted and sums the weights of its columns for the token behind them; the last one to finish
// picks that token.
template <typename T>
__global__ __launch_bounds__(256) void verify_pick_kernel(const VerifyArgs a, int parts, int picks, int64_t span, const Part* __restrict__ stats,
                                                          double* __restrict__ weights, int* __restrict__ tickets) {
  __shared__ int stop, ended, finishes, last_seen, chosen;
  __shared__ Row joined[2];
  __shared__ double partial[4];
  __shared__ double before_s, border_s;
  __shared__ int64_t begin_s;
  const int b = blockIdx.x / picks, pick = blockIdx.x % picks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t drafted = a.rows - a.requests, V = a.V;
  const View v = view_of(a.cu, b, a.rows, drafted);
  if (!v.any) {
    if (pick == 0 && threadIdx.x == 0) a.accepted[b] = 0;
    return;
  }
  const float tau = tau_of(a.temperature, b);
  const bool sampled = tau > 0.f;
  const double c = kLog2eD / (double)tau;
  const Part* of_target = stats + v.row0 * parts;
  const Part* of_draft = a.draft ? stats + (a.rows + v.first) * parts : nullptr;
  const T* z_target = (const T*)a.target + v.row0 * a.ldt;
  const T* z_draft = a.draft ? (const T*)a.draft + v.first * a.ldd : nullptr;
  if (threadIdx.x == 0) stop = tau == tau ? v.n : 0, ended = 0x7FFFFFFF;
  __syncthreads();
  // a token is accepted if u q(x) < p(x); one that is no token ends the draft
  if (tau == tau)
    for (int i = wave; i < v.n; i += 4) {
      const int x = a.tokens[v.first + i];
      const bool token = x >= 0 && x < V;
      const Row p = join_row(of_target + (int64_t)i * parts, parts, c, sampled, lane);
      bool takes = token && p.ok;
      if (!sampled) takes = takes && x == p.at;
      else if (takes) {
        const double px = beside(ldf(z_target, (size_t)(i * a.ldt + x)), p.top, c) / p.sum;
        double qx = 1.0;
        if (a.draft) {
          const Row q = join_row(of_draft + (int64_t)i * parts, parts, c, true, lane);
          qx = q.ok ? beside(ldf(z_draft, (size_t)(i * a.ldd + x)), q.top, c) / q.sum : __builtin_nan("");
        }
        takes = (double)a.uniforms[v.row0 + i] * qx < px;
      }
      if (!takes && lane == 0) {
        atomicMin(&stop, i);
        if (!token) atomicMin(&ended, i);
      }
    }
  __syncthreads();
  const int j = stop;
  const bool refused = j < v.n && ended != j;   // a token was: what it was drawn from is taken off
  if (wave < 2) {
    Row r{0.0, 0.f, -1, false};
    if (tau == tau) {
      if (wave == 0) r = join_row(of_target + (int64_t)j * parts, parts, c, sampled, lane);
      else if (refused && sampled && a.draft) r = join_row(of_draft + (int64_t)j * parts, parts, c, true, lane);
    }
    if (lane == 0) joined[wave] = r;
  }
  __syncthreads();
  const Row p = joined[0], q = joined[1];
  auto tell = [&](int token) {   // by the whole block
    for (int64_t i = threadIdx.x; i <= v.n; i += 256) a.out[v.row0 + i] = i < j ? a.tokens[v.first + i] : i == j ? token : -1;
    if (threadIdx.x == 0) a.accepted[b] = j;
  };
  if (!sampled || !p.ok) {
    if (pick == 0) tell(p.ok ? p.at : -1);
    return;
  }
  const Scale ep(c, (double)p.top), eq(c, q.ok ? (double)q.top : 0.0);
  const double ip = ep.fix / p.sum, iq = q.ok ? eq.fix / q.sum : 0.0;
  const T* zp = z_target + (int64_t)j * a.ldt;
  const T* zq = q.ok ? z_draft + (int64_t)j * a.ldd : nullptr;
  const int64_t taken = refused && !a.draft ? a.tokens[v.first + j] : -1;
  auto weigh = [&](int64_t col, bool alone, double (&w)[8]) {   // of eight columns; alone: the target's probabilities
    float z[8], y[8];
    load_row8(zp, col, V, z);
    if (zq && !alone) load_row8(zq, col, V, y);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      w[k] = ep.of(z[k]) * ip;
      if (zq && !alone) w[k] = fmax(w[k] - eq.of(y[k]) * iq, 0.0);
      else if (!alone && col + k == taken) w[k] = 0.0;
    }
  };
  double sum = 0.0;
  const int64_t from = pick * span, to = min(from + span, V);
  for (int64_t base = from; base < to; base += kStep) {
    const int64_t col = base + threadIdx.x * 8;
    if (col >= V) continue;
    double w[8];
    weigh(col, false, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += w[k];
  }
  sum = wave_sum(sum);
  if (lane == 0) partial[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    __hip_atomic_store(weights + (int64_t)b * kMaxPicks + pick, partial[0] + partial[1] + partial[2] + partial[3], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // released with the ticket, so that whoever sees it sees the sum
    finishes = __hip_atomic_fetch_add(tickets + b, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == picks - 1;
  }
  __syncthreads();
  if (!finishes) return;
  // the first part whose cumulated weight goes over the border; none: the last that weighs anything
  bool alone = false;
  if (wave == 0) {
    double mine = lane < picks ? __hip_atomic_load(weights + (int64_t)b * kMaxPicks + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0, upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(upto, o, 64);
      if (lane >= o) upto += x;
    }
    const double all = __shfl(upto, 63, 64);
    const double border = fmax((double)a.uniforms[v.row0 + v.n] * all, 0.0);
    const unsigned long long over = __ballot(upto > border), some = __ballot(mine > 0.0);
    const int at = over ? __ffsll(over) - 1 : some ? 63 - __clzll(some) : -1;
    const double front = __shfl(upto - mine, max(at, 0), 64);
    if (lane == 0) {
      // nothing weighs anything (a number of 1 and more refused what both distributions agree on): from the target's alone
      begin_s = at < 0 ? -1 : at * span;
      before_s = at < 0 ? 0.0 : front;
      border_s = at < 0 ? fmax((double)a.uniforms[v.row0 + v.n], 0.0) : border;
      chosen = 0x7FFFFFFF, last_seen = -1;
    }
  }
  __syncthreads();
  alone = begin_s < 0;
  const int64_t begin = alone ? 0 : begin_s, finish = alone ? V : min(begin + span, V);
  double before = before_s;
  const double border = border_s;
  for (int64_t base = begin; base < finish; base += kStep) {
    const int64_t col = base + threadIdx.x * 8;
    double w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (col < V) weigh(col, alone, w);
    double mine = 0.0;
    int top = -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      mine += w[k];
      top = w[k] > 0.0 ? (int)(col + k) : top;
    }
    double upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(upto, o, 64);
      if (lane >= o) upto += x;
    }
    if (lane == 63) partial[wave] = upto;
    if (top >= 0) atomicMax(&last_seen, top);
    __syncthreads();
    double front = before;
    for (int k = 0; k < wave; ++k) front += partial[k];
    double run = front + (upto - mine);
    if (front + upto > border) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        run += w[k];
        if (run > border && w[k] > 0.0) {
          atomicMin(&chosen, (int)(col + k));
          break;
        }
      }
    }
    before += partial[0] + partial[1] + partial[2] + partial[3];
    __syncthreads();
    if (chosen != 0x7FFFFFFF) break;
  }
  tell(chosen != 0x7FFFFFFF ? chosen : last_seen);
}

int64_t parts_of(int64_t V, int u) { return (V + (int64_t)u * kStep - 1) / ((int64_t)u * kStep); }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t verify_workspace_bytes(int64_t rows, int requests, int64_t V) {
  return up256((size_t)(2 * rows - requests) * (size_t)parts_of(V, 1) * sizeof(Part)) + up256((size_t)requests * kMaxPicks * sizeof(double)) +
         up256((size_t)requests * sizeof(int));
}

hipError_t launch_verify(const VerifyArgs& a, int dtype, hipStream_t s) {
  char* ws = (char*)a.workspace;
  double* weights = (double*)ws;
  int* tickets = (int*)(ws + up256((size_t)a.requests * kMaxPicks * sizeof(double)));
  Part* stats = (Part*)((char*)tickets + up256((size_t)a.requests * sizeof(int)));
  const int64_t units = a.rows + (a.draft ? a.rows - a.requests : 0);
  const int u = units * parts_of(a.V, 4) >= 2048 ? 4 : units * parts_of(a.V, 2) >= 2048 ? 2 : 1;
  const int64_t parts = parts_of(a.V, u);
  {
    ProfScope ps("verify_stats", 4.0 * (double)units * a.V, (double)units * a.V * dtype_size(dtype), s);
    const dim3 grid((unsigned)(units * parts)), block(256);
#define TIDE_VERIFY(T, U) hipLaunchKernelGGL((verify_stats_kernel<T, U>), grid, block, 0, s, a, (int)parts, stats, tickets)
    if (dtype == kBF16) { if (u == 4) TIDE_VERIFY(bf16_t, 4); else if (u == 2) TIDE_VERIFY(bf16_t, 2); else TIDE_VERIFY(bf16_t, 1); }
    else { if (u == 4) TIDE_VERIFY(float, 4); else if (u == 2) TIDE_VERIFY(float, 2); else TIDE_VERIFY(float, 1); }
#undef TIDE_VERIFY
    if (const hipError_t e = hipGetLastError()) return e;
  }
  // enough blocks for the chip, and no part below one step
  const int64_t steps = parts_of(a.V, 1), wanted = std::min<int64_t>({steps, kMaxPicks, std::max<int64_t>(1, 1024 / a.requests)});
  const int64_t span = (steps + wanted - 1) / wanted * kStep;
  const int picks = (int)((a.V + span - 1) / span);
  ProfScope ps("verify_pick", 0, 2.0 * (double)a.requests * a.V * dtype_size(dtype), s);
  const dim3 grid((unsigned)((int64_t)a.requests * picks)), block(256);
  if (dtype == kBF16) hipLaunchKernelGGL(verify_pick_kernel<bf16_t>, grid, block, 0, s, a, (int)parts, picks, span, stats, weights, tickets);
  else hipLaunchKernelGGL(verify_pick_kernel<float>, grid, block, 0, s, a, (int)parts, picks, span, stats, weights, tickets);
  return hipGetLastError();
}

}  // namespace tide
