// What a served target's logits leave to train on, and the loss that is trained on it:
//   topk_logits   the k largest logits of every row, in order, with the row's log-sum-exp
//   distill       KL divergence of a student's logits from a teacher's top logits, and its gradient
// Both pass over [rows, vocab] arrays of logits that do not fit any cache: what bounds them is memory.
#include "kernels.h"
#include "prof.h"
#include "tide_common.h"

namespace tide {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Order of the logits: a key that ascends as the values do, with every NaN above +inf and one zero.  Together with the
// complement of the index it is unique in a row and says "larger value first, equal values by ascending index".
constexpr uint32_t kNanKey = 0xFFFFFFFEu;   // (a pair of all ones is larger than every element's)
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return kNanKey;
  const uint32_t b = __float_as_uint(v + 0.f);   // -0 + 0 = +0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == kNanKey) return __uint_as_float(0x7FC00000u);
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
__device__ __forceinline__ uint64_t order_pair(float v, int idx) { return ((uint64_t)order_key(v) << 32) | (uint32_t)~idx; }

// Running (max, sum of 2^(c (z - max))) over eight more values.  The difference comes first: it is 0 for the largest value whatever
// that is, also where c times it has no number (columns masked with the type's lowest value).
struct Online { float m, s; };
__device__ __forceinline__ void online_add8(Online& o, const float (&v)[8], float c) {
  float cm = v[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) cm = fmaxf(cm, v[j]);
  const float nm = fmaxf(o.m, cm);
  const float sh = nm == -INFINITY ? 0.f : nm;      // nothing but -inf so far: every term is 0
  float part = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) part += __builtin_amdgcn_exp2f((v[j] - sh) * c);
  o.s = (o.m == -INFINITY ? o.s : o.s * __builtin_amdgcn_exp2f((o.m - nm) * c)) + part;   // (before any number: 0, or NaN)
  o.m = nm;
}
__device__ __forceinline__ Online online_join(const Online& a, const Online& b, float c) {
  const float nm = fmaxf(a.m, b.m);
  const float sa = a.m == -INFINITY ? a.s : a.s * __builtin_amdgcn_exp2f((a.m - nm) * c);   // (a NaN in the sum stays)
  const float sb = b.m == -INFINITY ? b.s : b.s * __builtin_amdgcn_exp2f((b.m - nm) * c);
  return Online{nm, sa + sb};
}
// of a block of NT threads; every thread gets the result.  sm: NT / 64 pairs.  Two barriers.
template <int NT>
__device__ __forceinline__ Online online_block(Online o, float c, Online* sm) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const Online x{__shfl_xor(o.m, d, 64), __shfl_xor(o.s, d, 64)};
    o = online_join(o, x, c);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = o;
  __syncthreads();
  o = sm[0];
  for (int i = 1; i < NT / 64; ++i) o = online_join(o, sm[i], c);
  return o;
}
template <typename T>
__device__ __forceinline__ void load_tail8(const T* zr, int c, int V, float (&v)[8]) {
  if (c + 8 <= V) {
    ld8(zr, c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < V ? ldf(zr, c + j) : -INFINITY;
  }
}
// log-sum-exp of a row's values over the temperature, from their largest one and the sum beside it
__device__ __forceinline__ float row_lse(const Online& o, float tau) {
  if (o.m == -INFINITY || o.m == INFINITY) return o.s != o.s && o.m == -INFINITY ? o.s : o.m;
  return o.m / tau + logf(o.s);
}

}  // namespace

// ----------------------------------------------------------------------------------------------
// The k largest logits of a row and its log-sum-exp, in one read of the row.
//
// A block walks its row in rounds of NT x U chunks of eight columns.  What it remembers are chunks, by (largest value, index):
// an element of the k largest lies in one of the k first chunks in that order, because any chunk before its own holds an
// element before it (larger, or as large with a smaller index).  A threshold T that k chunks reach keeps almost every
// chunk out after a comparison with its maximum, which is taken anyway; the others go to a list in LDS, and when that holds
// more than k + 16 + k / 4 of them, a wave finds the k-th largest key bit by bit (a ballot per 64 keys and bit), which is the new T, and
// drops the rest.  Rows of random order pass about k chunks per doubling of what has been seen.  The order of a row
// can fill a round, never the list: it has room for one.  At the end the eight elements of each chunk left are read again
// (a few hundred of 128256) and ranked by counting.
// Sum of exponentials: against a shift that a wave keeps to itself and raises only where a chunk passes T (it is never below
// T, so what does not pass cannot exceed it): per element one conversion, half a maximum, one fused step, the exponential and
// one addition.  The first round has no T yet: each wave takes the k-th largest of its own 64 U chunk maxima, and the
// largest of those serves all.
// Bound by memory: [8192, 128256] bf16, k = 32: 327 us, 6.4 TB/s (k = 1: 321, k = 128: 365).
// ----------------------------------------------------------------------------------------------
namespace {

__device__ __forceinline__ void lds_barrier() {   // orders LDS only: loads of the next round stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// largest of eight, NaN if one is NaN
__device__ __forceinline__ float max8(const float (&v)[8]) {
  auto max3 = [](float a, float b, float c) {
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
  };
  const float m = max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), v[6]);
  return max3(m, v[7], v[7]);
}
template <typename T> struct Raw8Once : Raw8<T> {   // loads past the caches: nothing is read again
  __device__ __forceinline__ void load_once(const T* p, size_t i) {
    typedef unsigned u32x4_nt __attribute__((ext_vector_type(4)));
    const u32x4_nt* q = reinterpret_cast<const u32x4_nt*>(p + i);
    if constexpr (sizeof(T) == 2) {
      const u32x4_nt x = __builtin_nontemporal_load(q);
      this->a = make_uint4(x.x, x.y, x.z, x.w);
    } else {
      const u32x4_nt x = __builtin_nontemporal_load(q), y = __builtin_nontemporal_load(q + 1);
      this->a = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
      this->b = make_float4(__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w));
    }
  }
};

// chunks that a list may hold at the start of a round beyond the k that it needs
__host__ __device__ constexpr int list_slack(int k) { return 16 + k / 4; }
constexpr int kListKept = kMaxTeacher + list_slack(kMaxTeacher);

// By one wave, on the n > k pairs of a list: the largest 16-bit prefix that the keys of k of them reach, as a key (the whole k-th pair
// where too many share that prefix).  Pairs below it leave the list; returns what is left, at most k + list_slack(k).
struct ListCut { int n; uint32_t key; };
template <int NI>
__device__ __forceinline__ uint32_t cut_prefix(const uint64_t* list, int n, int k, int lane, int& left) {
  uint32_t key[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) key[i] = lane + 64 * i < n ? (uint32_t)(list[lane + 64 * i] >> 32) : 0u;
  uint32_t t = 0;
  left = n;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t u = t | (1u << bit);
    int c = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) c += __popcll(__ballot(key[i] >= u));
    if (c >= k) { t = u; left = c; }
  }
  return t;
}
__device__ __forceinline__ ListCut list_cut(uint64_t* list, int n, int k, int lane) {
  int left = n;
  uint64_t t;
  if (n <= 128) {
    t = (uint64_t)cut_prefix<2>(list, n, k, lane, left) << 32;
  } else if (n <= 256) {
    t = (uint64_t)cut_prefix<4>(list, n, k, lane, left) << 32;
  } else if (n <= 512) {
    t = (uint64_t)cut_prefix<8>(list, n, k, lane, left) << 32;
  } else if (n <= 1024) {
    t = (uint64_t)cut_prefix<16>(list, n, k, lane, left) << 32;
  } else {
    t = 0;
    for (int bit = 63; bit >= 48; --bit) {
      const uint64_t u = t | (1ull << bit);
      int c = 0;
      for (int i = 0; i < n; i += 64) c += __popcll(__ballot(i + lane < n && list[i + lane] >= u));
      if (c >= k) { t = u; left = c; }
    }
  }
  const uint32_t key = (uint32_t)(t >> 32);
  if (left > k + list_slack(k))
    for (int bit = 47; bit >= 0; --bit) {
      const uint64_t u = t | (1ull << bit);
      int c = 0;
      for (int i = 0; i < n; i += 64) c += __popcll(__ballot(i + lane < n && list[i + lane] >= u));
      if (c >= k) t = u;
    }
  int out = 0;
  for (int i = 0; i < n; i += 64) {   // (a pair moves down or stays: what is written has been read)
    const uint64_t p = i + lane < n ? list[i + lane] : 0;
    const uint64_t kept = __ballot(i + lane < n && p >= t);
    if (i + lane < n && p >= t) list[out + __popcll(kept & ((1ull << lane) - 1))] = p;
    out += __popcll(kept);
  }
  return ListCut{out, key};
}

}  // namespace

// (256 threads in 89 registers, five blocks on a CU: 365 us where seven take 327)
template <typename T, int NT, int U, int D>
__global__ __launch_bounds__(NT, NT == 256 ? 7 : 4) void topk_logits_kernel(const T* __restrict__ z, int64_t ldz, int V, int k, float tau,
                                                         int32_t* __restrict__ ids, float* __restrict__ values,
                                                         float* __restrict__ lse) {
  constexpr int NW = NT / 64, ROUND = NT * U * 8;
  constexpr int CAP = NT * U + kListKept > kListKept * 8 ? NT * U + kListKept : kListKept * 8;
  __shared__ uint64_t list[CAP];
  __shared__ uint32_t chunk_of[kListKept];
  __shared__ int added[3];
  __shared__ uint32_t first_key, cut_key, top_key;
  __shared__ int cut_n, found_n;
  __shared__ Online sm[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t row = blockIdx.x;
  const T* zr = z + row * (size_t)ldz;
  const float c = kLog2e / tau;
  const int last = (V - 1) / 8 * 8;                 // the last chunk: whole in memory, since rows are multiples of eight apart
  if (threadIdx.x < 3) added[threadIdx.x] = 0;
  if (threadIdx.x == 3) { first_key = 0; found_n = 0; }
  lds_barrier();

  Raw8Once<T> ring[D][U];                           // the next D rounds
  auto load = [&](Raw8Once<T> (&raw)[U], int base) {
    if (base < V) {
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u].load_once(zr, (size_t)min(base + (int)(threadIdx.x + u * NT) * 8, last));
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) load(ring[d], d * ROUND);
  int n = 0;                                        // pairs in the list
  float T_v = __uint_as_float(0x7FC00000u);         // chunks pass unless their maximum is at most this: all, so far
  float m = -INFINITY, s = 0.f;                     // the wave's shift, the lane's sum
  float shift = 0.f;                                // -c m, 0 before any number
  bool wide = false;                                // whether that is too large to be added to
  auto raise = [&](float to) {                      // the same in the whole wave
    to = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(to)));
    if (to > m) {
      s *= m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);   // (before any number the sum is 0, or NaN)
      m = to;
      shift = -m * c;
      wide = !(fabsf(shift) < 1e30f);
    }
  };
  auto columns = [&](const Raw8Once<T>& raw, int col, bool tail, float (&v)[8]) {
    raw.get(v);
    if (tail) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = col + j < V ? v[j] : -INFINITY;
    }
  };
  int r = 0;                                        // the round, modulo 3
  auto round = [&](Raw8Once<T> (&cur)[U], int base) {
    const bool tail = base + ROUND > V;
    if (base == 0) {
      uint32_t key[U];
      float all = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int col = (threadIdx.x + u * NT) * 8;
        float v[8];
        columns(cur[u], col, tail, v);
        const float cm = max8(v);
        key[u] = col < V ? order_key(cm) : 0u;
        all = fmaxf(all, cm);
      }
      uint32_t t = 0;
      for (int bit = 31; bit >= 16; --bit) {
        const uint32_t x = t | (1u << bit);
        int count = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) count += __popcll(__ballot(key[u] >= x));
        if (count >= k) t = x;
      }
      if (lane == 0 && t) atomicMax(&first_key, t);
      raise(wave_max(all));
      lds_barrier();
      t = first_key;
      if (t > 2) T_v = key_value(t - 2);            // k chunks have keys of at least t; two steps, for the two zeros
      raise(T_v);
    }
    uint64_t who[U];
    float top[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = base + (threadIdx.x + u * NT) * 8;
      float v[8];
      columns(cur[u], col, tail, v);
      const float cm = max8(v);
      const bool pass = col < V && !(cm <= T_v);
      who[u] = __ballot(pass);
      top[u] = cm;
      if (who[u] && __any(cm > m)) raise(wave_max(fmaxf(cm, m)));
      float part = 0.f;
      if (wide) {
#pragma unroll
        for (int j = 0; j < 8; ++j) part += __builtin_amdgcn_exp2f((v[j] - m) * c);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) part += __builtin_amdgcn_exp2f(fmaf(v[j], c, shift));
      }
      s += part;
    }
    int mine = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) mine += __popcll(who[u]);
    if (mine) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&added[r], mine);
      at = n + __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if ((who[u] >> lane) & 1)
          list[at + __popcll(who[u] & ((1ull << lane) - 1))] = ((uint64_t)order_key(top[u]) << 32) | (uint32_t)~((base >> 3) + threadIdx.x + u * NT);
        at += __popcll(who[u]);
      }
    }
    lds_barrier();
    n += added[r];
    if (threadIdx.x == 0) added[r == 0 ? 2 : r - 1] = 0;   // read by all before this barrier, used again behind the next
    if (n > k + list_slack(k) || (base + ROUND >= V && n > k)) {
      if (wave == 0) {
        const ListCut cut = list_cut(list, n, k, lane);
        if (lane == 0) { cut_n = cut.n; cut_key = cut.key; }
      }
      lds_barrier();
      n = cut_n;
      T_v = key_value(cut_key);
      raise(T_v);
    }
    r = r == 2 ? 0 : r + 1;
    load(cur, base + D * ROUND);
  };
  for (int base = 0; base < V; base += D * ROUND) {
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (base + d * ROUND < V) round(ring[d], base + d * ROUND);
  }

  // the elements of the chunks left, of which k reach the last threshold
  const uint32_t least = n >= k && T_v == T_v ? order_key(T_v) : 0u;
  if (threadIdx.x < n) chunk_of[threadIdx.x] = ~(uint32_t)list[threadIdx.x];
  lds_barrier();
  for (int e = threadIdx.x; e < n * 8; e += NT) {
    const int col = (int)(chunk_of[e >> 3] * 8u) + (e & 7);
    if (col < V) {
      const uint64_t p = order_pair(ldf(zr, (size_t)col), col);
      if ((uint32_t)(p >> 32) >= least) list[atomicAdd(&found_n, 1)] = p;
    }
  }
  lds_barrier();
  const int found = found_n;
  for (int i = threadIdx.x; i < found; i += NT) {
    const uint64_t p = list[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < found; ++j) rank += list[j] > p ? 1 : 0;
    if (rank < k) {
      ids[row * (size_t)k + rank] = (int32_t)~(uint32_t)p;
      values[row * (size_t)k + rank] = key_value((uint32_t)(p >> 32));
      if (rank == 0) top_key = (uint32_t)(p >> 32);
    }
  }
  if (lse) {
    const Online o = online_block<NT>(Online{m, s}, c, sm);
    if (threadIdx.x == 0) {
      const float top = key_value(top_key);         // -inf, +inf and NaN have no sum: the row's log-sum-exp is its largest element
      lse[row] = fabsf(top) < INFINITY ? o.m / tau + logf(o.s) : top;
    }
  }
}

hipError_t launch_topk_logits(int64_t rows, int V, const void* z, int64_t ldz, int k, float tau, int32_t* ids, float* values, float* lse,
                              int dtype, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  ProfScope ps("topk_logits", 0, (double)rows * ((double)V * dtype_size(dtype) + 8.0 * k), s);
  const dim3 grid((unsigned)rows);
  // Up to a row per CU, all of a CU's threads on it, and four rounds requested at a time; two rows, half of them; beyond, four waves a row
  // (us, 1024 / 512 / 256 threads, [rows, 128256] bf16, k = 32: 61 rows 27 / 29 / 43, 256 30 / 32 / 44, 512 57 / 39 / 49,
  // 1024 108 / 72 / 59).
  const int nt = rows <= 256 ? 1024 : rows <= 512 ? 512 : 256;
#define TIDE_TOPK(T, NT, U, D) hipLaunchKernelGGL((topk_logits_kernel<T, NT, U, D>), grid, dim3(NT), 0, s, (const T*)z, ldz, V, k, tau, ids, values, lse)
  if (dtype == kBF16) {
    if (nt == 1024) TIDE_TOPK(bf16_t, 1024, 4, 4);
    else if (nt == 512) TIDE_TOPK(bf16_t, 512, 4, 2);
    else TIDE_TOPK(bf16_t, 256, 4, 2);
  } else {
    if (nt == 1024) TIDE_TOPK(float, 1024, 2, 4);
    else if (nt == 512) TIDE_TOPK(float, 512, 2, 2);
    else TIDE_TOPK(float, 256, 2, 2);
  }
#undef TIDE_TOPK
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------------------
// Distillation.  With a = t / tau over the teacher's valid entries, p = exp(a - L) (L their log-sum-exp, or the given one),
// P = sum p, q = softmax(z / tau):
//   loss = tau^2 sum_j p_j (log p_j - log q_{id_j})      dz_v = tau (P q_v - sum_{j: id_j = v} p_j)
// ----------------------------------------------------------------------------------------------
namespace {

// A row's teacher, in LDS: entry j's column (-1: none), probability and student logit.
struct Teacher {
  int id[kMaxTeacher];
  float p[kMaxTeacher], z[kMaxTeacher];
  float mass, loss;     // P, and sum_j p_j log p_j
  int any;              // whether an entry says anything
};

// By one wave: everything of the row's teacher that the student's statistics do not enter.  The student's logits at its
// columns are read here, before anything of the row can be overwritten.
template <typename T>
__device__ __forceinline__ void teacher_load(Teacher& te, const T* zr, int V, int k, const int32_t* ids, const float* t, const float* lse, size_t row,
                                             float tau, int lane) {
  constexpr int PER = kMaxTeacher / 64;
  int id[PER];
  float a[PER], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 64 * i;
    id[i] = j < k ? ids[row * (size_t)k + j] : -1;
    if (id[i] >= V) id[i] = -1;
    a[i] = id[i] >= 0 ? t[row * (size_t)k + j] / tau : -INFINITY;
    if (id[i] < 0) id[i] = -1;
    m = fmaxf(m, a[i]);
  }
  bool any = false, nan = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    any |= a[i] > -INFINITY;
    nan |= a[i] != a[i];
  }
  any = __any(any || nan);
  m = wave_max(m);
  float L;
  if (lse) {
    L = lse[row];
  } else {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) s += id[i] >= 0 && any ? expf(a[i] - m) : 0.f;
    L = m + logf(wave_sum(s));
  }
  float mass = 0.f, ent = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 64 * i;
    const float p = id[i] >= 0 && any ? expf(a[i] - L) : 0.f;
    mass += p;
    ent += p != 0.f ? p * (a[i] - L) : 0.f;
    te.id[j] = id[i];
    te.p[j] = p;
    te.z[j] = id[i] >= 0 ? ldf(zr, (size_t)id[i]) : 0.f;
  }
  mass = wave_sum(mass);
  ent = wave_sum(ent);
  if (lane == 0) { te.mass = mass; te.loss = ent; te.any = any ? 1 : 0; }
}
// by one wave: sum_j p_j (log p_j - log q_j), with log q_j = (z_j - M) / tau - log S
__device__ __forceinline__ float teacher_loss(const Teacher& te, int k, const Online& o, float tau, int lane) {
  const float log_s = logf(o.s);
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxTeacher / 64; ++i) {
    const int j = lane + 64 * i;
    if (j < k && te.p[j] != 0.f) x += te.p[j] * ((te.z[j] - o.m) / tau - log_s);
  }
  return te.loss - wave_sum(x);
}
// gradient at a teacher's column: all of the row's probability on it
__device__ __forceinline__ float teacher_grad(const Teacher& te, int k, int j, float q_mass, float tau) {
  float p = 0.f;
  for (int i = 0; i < k; ++i) p += te.id[i] == te.id[j] ? te.p[i] : 0.f;
  return tau * (q_mass - p);
}

}  // namespace

// A block owns a row and reads it twice, for the statistics and for the gradient.  The columns of the teacher's entries are
// written over by the thread that wrote their eight columns before.
template <typename T, bool GRAD>
__global__ __launch_bounds__(512) void distill_kernel(DistillArgs a) {
  constexpr int NT = 512;
  __shared__ Teacher te;
  __shared__ Online sm[NT / 64];
  const size_t row = blockIdx.x;
  const T* zr = (const T*)a.z + row * (size_t)a.ldz;
  const float c = kLog2e / a.tau;
  const int V = a.V, lane = threadIdx.x & 63;
  if (threadIdx.x < 64) teacher_load(te, zr, V, a.k, a.ids, a.t, a.tlse, row, a.tau, lane);
  Online o{-INFINITY, 0.f};
  for (int i = threadIdx.x * 8; i < V; i += NT * 8) {
    float v[8];
    load_tail8(zr, i, V, v);
    online_add8(o, v, c);
  }
  o = online_block<NT>(o, c, sm);
  const bool keep = a.mask[row] != 0 && te.any;
  if (threadIdx.x < 64) {
    const float loss = keep ? a.tau * a.tau * teacher_loss(te, a.k, o, a.tau, lane) : 0.f;
    if (lane == 0) { a.lse[row] = row_lse(o, a.tau); a.loss_rows[row] = loss; }
  }
  if constexpr (GRAD) {
    T* dr = (T*)a.dz + row * (size_t)a.ldz;
    const float f = te.mass / o.s;
    for (int i = threadIdx.x * 8; i < a.ldz; i += NT * 8) {
      float v[8];
      if (keep) {
        load_tail8(zr, i, V, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < V ? a.tau * f * __builtin_amdgcn_exp2f((v[j] - o.m) * c) : 0.f;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
      }
      st8(dr, i, v);
    }
    if (keep)
      for (int j = 0; j < a.k; ++j)
        if (te.id[j] >= 0 && (te.id[j] >> 3) % NT == (int)threadIdx.x)
          stf(dr, (size_t)te.id[j], teacher_grad(te, a.k, j, f * __builtin_amdgcn_exp2f((te.z[j] - o.m) * c), a.tau));
  }
}

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const bool grad = a.dz != nullptr;
  ProfScope ps(grad ? "distill_train" : "distill_eval", 0, (double)a.rows * dtype_size(dtype) * (a.V + (grad ? (double)a.ldz : 0.0)), s);
  const dim3 grid((unsigned)a.rows), blk(512);
  if (dtype == kBF16) {
    if (grad) hipLaunchKernelGGL((distill_kernel<bf16_t, true>), grid, blk, 0, s, a);
    else hipLaunchKernelGGL((distill_kernel<bf16_t, false>), grid, blk, 0, s, a);
  } else {
    if (grad) hipLaunchKernelGGL((distill_kernel<float, true>), grid, blk, 0, s, a);
    else hipLaunchKernelGGL((distill_kernel<float, false>), grid, blk, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace tide
