// What a served target's logits leave to train on, and the loss that is trained on it:
//   topk_logits   the k largest logits of every row, in order, with the row's log-sum-exp
//   distill       KL divergence of a student's logits from a teacher's top logits, and its gradient
// Both pass over [rows, vocab] arrays of logits that do not fit any cache: what bounds them is memory.
#include <type_traits>

#include "kernels.h"
#include "prof.h"
#include "row_stats.h"

namespace tide {

namespace {

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

// log-sum-exp of a row's values over the temperature, from their largest one and the sum beside it: NaN before +inf before all others
__device__ __forceinline__ float row_lse(const Online& o, float tau) {
  if (o.s != o.s || o.m == INFINITY) return o.s;
  return o.m == -INFINITY ? o.m : o.m / tau + logf(o.s);
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
// one addition.  The first round has no T yet: k chunks of one wave reach the k-th largest of its maxima, and k of several waves the least
// of their largest, second largest ...: what is enough for k.
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
#pragma unroll 1
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t u = t | (1u << bit);
    int c = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) c += __popcll(__ballot(key[i] >= u));
    if (c >= k) { t = u; left = c; }
  }
  return t;
}
__device__ __noinline__ ListCut list_cut(uint64_t* list, int n, int k, int lane) {
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
#pragma unroll 1
    for (int bit = 63; bit >= 48; --bit) {
      const uint64_t u = t | (1ull << bit);
      int c = 0;
      for (int i = 0; i < n; i += 64) c += __popcll(__ballot(i + lane < n && list[i + lane] >= u));
      if (c >= k) { t = u; left = c; }
    }
  }
  const uint32_t key = (uint32_t)(t >> 32);
  if (left > k + list_slack(k))
#pragma unroll 1
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

// How many of a list's n <= NT pairs are larger than pair i, which is the thread's own: as many neighbouring threads share a pair as there
// are threads for, up to 16.
template <int CTRL>
__device__ __forceinline__ int dpp_int(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false); }
template <int NT>
__device__ __forceinline__ int list_rank(const uint64_t* list, int n, int& i, uint64_t& pair) {
  const int log = n <= NT / 16 ? 4 : n <= NT / 8 ? 3 : n <= NT / 4 ? 2 : n <= NT / 2 ? 1 : 0;
  i = (int)threadIdx.x >> log;
  pair = i < n ? list[i] : ~0ull;
  int rank = 0;
#pragma unroll 4
  for (int j = threadIdx.x & ((1 << log) - 1); j < n; j += 1 << log) rank += list[j] > pair ? 1 : 0;
  if (log > 0) rank += dpp_int<0xB1>(rank);    // the neighbour, the neighbouring pair, the other four, the other eight
  if (log > 1) rank += dpp_int<0x4E>(rank);
  if (log > 2) rank += dpp_int<0x141>(rank);
  if (log > 3) rank += dpp_int<0x140>(rank);
  return rank;
}

}  // namespace

// (256 threads in 89 registers, five blocks on a CU: 365 us where seven take 327)
template <typename T, int NT, int U, int D>
__global__ __launch_bounds__(NT, NT == 256 ? (D == 1 ? 8 : 7) : 4) void topk_logits_kernel(const T* __restrict__ z, int64_t ldz, int V, int k, float tau,
                                                         int32_t* __restrict__ ids, float* __restrict__ values,
                                                         float* __restrict__ lse) {
  constexpr int NW = NT / 64, ROUND = NT * U * 8;
  constexpr bool RANKS = NT > 256;   // cut by ranks, by the whole block at once: less waiting, more work
  constexpr int CAP = NT * U + kListKept > kListKept * 8 ? NT * U + kListKept : kListKept * 8;
  __shared__ uint64_t list[CAP];
  __shared__ uint32_t chunk_of[kListKept];
  __shared__ int added[3];
  __shared__ uint32_t first_any, first_all, cut_key, top_key;
  __shared__ float first[NW];
  __shared__ int cut_n, found_n;
  __shared__ Online sm[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t row = blockIdx.x;
  const T* zr = z + row * (size_t)ldz;
  const float c = scalar(kLog2e / tau);
  if (threadIdx.x < 3) added[threadIdx.x] = 0;
  if (threadIdx.x == 3) { first_any = 0; first_all = ~0u; found_n = 0; }
  lds_barrier();

  Raw8Once<T> ring[D][U];                           // the next D rounds
  // (a buffer's loads take one addition each, and give zeros behind the row)
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(zr), 0, (int)((uint32_t)ldz * (uint32_t)sizeof(T)), 0x00020000);
  const int lane_at = (int)(threadIdx.x * 8 * sizeof(T));
  auto load = [&](Raw8Once<T> (&raw)[U], int base) {
    if (base < V) {
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u].load_buffer(rs, lane_at + (base + u * NT * 8) * (int)sizeof(T));
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) load(ring[d], d * ROUND);
  int n = 0;                                        // pairs in the list
  float T_v = __uint_as_float(0x7FC00000u);         // chunks pass unless their maximum is at most this: all, so far
  float m = -INFINITY, s = 0.f;                     // the wave's shift, the lane's sum
  float shift = 0.f;                                // -c m, 0 before any number
  bool wide = false;                                // whether its rounding is too large to stand in the sum: more than 2^-2 of an exponent
  auto raise = [&](float to) {                      // the same in the whole wave
    to = scalar(to);
    if (to > m) {
      s *= m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);   // (before any number the sum is 0, or NaN)
      m = to;
      shift = -m * c;
      wide = !(fabsf(shift) < 0x1p22f);
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
  auto round = [&](auto FIRST, Raw8Once<T> (&cur)[U], int base) {   // FIRST: whether this can be the row's first round
    const bool tail = base + ROUND > V;
    if (decltype(FIRST)::value && base == 0) {
      uint32_t key[U];
      float all = -INFINITY;                        // the lane's largest number
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int col = (threadIdx.x + u * NT) * 8;
        float v[8];
        columns(cur[u], col, tail, v);
        const float cm = max8(v);
        key[u] = col < V ? order_key(cm) : 0u;
        all = fmaxf(all, cm);
      }
      const int share = (k + NW - 1) / NW;
      float t = fast_max(all);
      raise(t);
      if constexpr (RANKS) {
        // `share` lanes of a wave reach its share-th largest, and k chunks that of enough waves
        const int waves = (k + share - 1) / share;
        float left = all;
#pragma unroll 1
        for (int i = 1; i < share; ++i) {
          if (lane == __builtin_ctzll(__ballot(left == t) | (1ull << 63))) left = -INFINITY;
          t = fast_max(left);
        }
        if (lane == 0) first[wave] = t;
        lds_barrier();
        const float mine = first[lane % NW];
        int rank = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) rank += first[i] > mine || (first[i] == mine && i < lane) ? 1 : 0;
        const uint64_t at = __ballot(lane < NW && rank == waves - 1);
        t = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), __builtin_ctzll(at | (1ull << 63))));
        if (at && t > -INFINITY) T_v = scalar(key_value(order_key(t) - 2));   // (two steps below: the zeros are one)
      } else {
        // prefixes that k of the wave's chunks reach, and as many as make k of all waves together (the form above takes five registers
        // more than seven blocks on a CU have: [8192, 128256] bf16 387 us where this takes 325)
        uint32_t ta = 0, tb = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 16; --bit) {
          const uint32_t xa = ta | (1u << bit), xb = tb | (1u << bit);
          int na = 0, nb = 0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            na += __popcll(__ballot(key[u] >= xa));
            nb += __popcll(__ballot(key[u] >= xb));
          }
          if (na >= k) ta = xa;
          if (nb >= share) tb = xb;
        }
        if (lane == 0) {
          atomicMax(&first_any, ta);
          atomicMin(&first_all, tb);
        }
        lds_barrier();
        const uint32_t reached = max(first_any, first_all);
        if (reached > 2) T_v = scalar(key_value(reached - 2));
      }
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
      who[u] = __ballot(!(cm <= T_v));
      if (tail) who[u] &= __ballot(col < V);
      top[u] = cm;
      if (who[u] && __any(cm > m)) raise(fast_max(cm));
      float part = 0.f;
      if (wide) {   // (no factor as power_of's: every later raise would meet another rounding)
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
    n += __builtin_amdgcn_readfirstlane(added[r]);
    if (threadIdx.x == 0) added[r == 0 ? 2 : r - 1] = 0;   // read by all before this barrier, used again behind the next
    if (n > k + list_slack(k) || (base + ROUND >= V && n > k)) {
      if (!RANKS || n > NT) {
        if (wave == 0) {
          const ListCut cut = list_cut(list, n, k, lane);
          if (lane == 0) { cut_n = cut.n; cut_key = cut.key; }
        }
        lds_barrier();
        n = __builtin_amdgcn_readfirstlane(cut_n);
        T_v = scalar(key_value(cut_key));
      }
      if (RANKS && n > k) {
        int i;
        uint64_t pair;
        const int rank = list_rank<NT>(list, n, i, pair);
        lds_barrier();
        if (i < n && rank < k) list[rank] = pair;
        lds_barrier();
        n = k;
        T_v = scalar(key_value((uint32_t)(list[k - 1] >> 32)));
      }
      raise(T_v);
    }
    r = r == 2 ? 0 : r + 1;
    load(cur, base + D * ROUND);
  };
  for (int base = 0; base < V; base += D * ROUND) {
    round(std::true_type{}, ring[0], base);
#pragma unroll
    for (int d = 1; d < D; ++d)
      if (base + d * ROUND < V) round(std::false_type{}, ring[d], base + d * ROUND);
  }

  // the elements of the chunks left, of which k reach the last threshold
  const uint32_t least = n >= k && T_v == T_v ? order_key(T_v) : 0u;
  if (threadIdx.x < n) chunk_of[threadIdx.x] = ~(uint32_t)list[threadIdx.x];
  s = fast_sum(s);                                  // (the shift is the wave's)
  if (lane == 0) sm[wave] = Online{m, s};
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
  auto put = [&](int rank, uint64_t pair) {
    ids[row * (size_t)k + rank] = (int32_t)~(uint32_t)pair;
    values[row * (size_t)k + rank] = key_value((uint32_t)(pair >> 32));
    if (rank == 0) top_key = (uint32_t)(pair >> 32);
  };
  if (RANKS && found <= NT) {
    int i;
    uint64_t pair;
    const int rank = list_rank<NT>(list, found, i, pair);
    if (i < found && rank < k) put(rank, pair);   // (threads that share a pair write the same)
  } else {
    for (int i = threadIdx.x; i < found; i += NT) {
      const uint64_t pair = list[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < found; ++j) rank += list[j] > pair ? 1 : 0;
      if (rank < k) put(rank, pair);
    }
  }
  if (lse) {
    lds_barrier();
    if (wave == 0) {
      const Online x = lane < NW ? sm[lane] : Online{-INFINITY, 0.f};
      const float all = fast_max(x.m), sum = fast_sum(x.m == -INFINITY ? x.s : x.s * __builtin_amdgcn_exp2f((x.m - all) * c));
      const float top = key_value(top_key);         // -inf, +inf and NaN have no sum: the row's log-sum-exp is its largest element
      if (lane == 0) lse[row] = fabsf(top) < INFINITY ? all / tau + logf(sum) : top;
    }
  }
}

hipError_t launch_topk_logits(int64_t rows, int V, const void* z, int64_t ldz, int k, float tau, int32_t* ids, float* values, float* lse,
                              int dtype, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  ProfScope ps("topk_logits", 0, (double)rows * ((double)V * dtype_size(dtype) + 8.0 * k), s);
  const dim3 grid((unsigned)rows);
  // Up to half a row per CU, as many threads as share a CU on it, and four rounds requested at a time; up to two, half of them; beyond, four
  // waves a row (us, 1024 / 512 / 256 threads, [rows, 128256] bf16, k = 32: 61 rows 20.7 / 22.6 / 37.7, 256 25.7 / 24.2 / 39.8, 384 45.8 / 31.8 / 42.9,
  // 512 49.5 / 32.7 / 43.8, 768 72.8 / 50.4 / 48.8, 1024 95.9 / 60.5 / 55.1).
  // (Eight blocks a CU in fp32, without a round requested ahead, against seven with one: [1999, 32001] 57 / 61 us; bf16 [8192, 128256] 334 / 326.)
  const int nt = rows <= 128 ? 1024 : rows <= 512 ? 512 : 256;
#define TIDE_TOPK(T, NT, U, D) hipLaunchKernelGGL((topk_logits_kernel<T, NT, U, D>), grid, dim3(NT), 0, s, (const T*)z, ldz, V, k, tau, ids, values, lse)
  if (dtype == kBF16) {
    if (nt == 1024) TIDE_TOPK(bf16_t, 1024, 4, 4);
    else if (nt == 512) TIDE_TOPK(bf16_t, 512, 4, 2);
    else TIDE_TOPK(bf16_t, 256, 4, 2);
  } else {
    if (nt == 1024) TIDE_TOPK(float, 1024, 2, 4);
    else if (nt == 512) TIDE_TOPK(float, 512, 2, 2);
    else TIDE_TOPK(float, 256, 2, 1);
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

// A row's teacher, in LDS: entry j's column (-1: none), probability and student logit, the probability of all entries on that
// column, and (from teacher_finish on) the gradient there.
struct Teacher {
  alignas(16) int id[kMaxTeacher];
  float p[kMaxTeacher], z[kMaxTeacher], at[kMaxTeacher], grad[kMaxTeacher];
  float mass, loss;     // P, and sum_j p_j log p_j
  int any;              // whether an entry says anything
};

// One wave's part of it, in three steps: the entries are requested, then the student's logits at their columns (before anything
// of the row can be overwritten), and then everything is computed that the student's statistics do not enter.
constexpr int kTeacherPer = kMaxTeacher / 64;
struct TeacherRegs { int id[kTeacherPer]; float t[kTeacherPer], z[kTeacherPer], lse; };
__device__ __forceinline__ void teacher_fetch(TeacherRegs& r, const DistillArgs& a, size_t row, int lane) {
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) {
    const int j = lane + 64 * i;
    r.id[i] = j < a.k ? a.ids[row * (size_t)a.k + j] : -1;
    r.t[i] = j < a.k ? a.t[row * (size_t)a.k + j] : 0.f;
  }
  r.lse = a.tlse ? a.tlse[row] : 0.f;
}
template <typename T>
__device__ __forceinline__ void teacher_logits(TeacherRegs& r, const T* zr, int V) {
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) {
    if (r.id[i] < 0 || r.id[i] >= V) r.id[i] = -1;
    r.z[i] = r.id[i] >= 0 ? ldf(zr, (size_t)r.id[i]) : 0.f;
  }
}
__device__ __forceinline__ void teacher_load(Teacher& te, const TeacherRegs& r, const DistillArgs& args, int lane) {
  // a = t / tau less what a row's entries share: their largest one (the difference comes first: it is exact where it is small, whatever the
  // quotients would be rounded to), or the given log-sum-exp
  float a[kTeacherPer], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) m = fmaxf(m, r.id[i] >= 0 ? r.t[i] : -INFINITY);
  m = fast_max(m);
  bool says = false;
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) {
    says |= r.id[i] >= 0 && !(r.t[i] == -INFINITY);
    a[i] = r.id[i] < 0 ? -INFINITY : args.tlse ? r.t[i] / args.tau - r.lse : (r.t[i] - m) / args.tau;
  }
  const bool any = __any(says);
  // p = exp(a) over `sum`: its logarithm taken off a would be rounded to a step of a's size
  float sum = 1.f;
  if (!args.tlse) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kTeacherPer; ++i) s += r.id[i] >= 0 && any ? expf(a[i]) : 0.f;
    sum = fast_sum(s);
  }
  const float log_sum = logf(sum);
  float mass = 0.f, ent = 0.f;
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) {
    const int j = lane + 64 * i;
    const float p = r.id[i] >= 0 && any ? expf(a[i]) / sum : 0.f;
    mass += p;
    ent += p != 0.f ? p * (a[i] - log_sum) : 0.f;
    te.id[j] = r.id[i];
    te.p[j] = p;
    te.z[j] = r.z[i];
  }
  mass = fast_sum(mass);
  ent = fast_sum(ent);
  if (lane == 0) { te.mass = mass; te.loss = ent; te.any = any ? 1 : 0; }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float at[kTeacherPer] = {};
#pragma unroll 2
  for (int j = 0; j < args.k; ++j) {
    const int id = te.id[j];
    const float p = te.p[j];
#pragma unroll
    for (int i = 0; i < kTeacherPer; ++i) at[i] += id == r.id[i] ? p : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kTeacherPer; ++i) te.at[lane + 64 * i] = at[i];
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
  return te.loss - fast_sum(x);
}

// What a block knows of its row after the statistics, and what remains but for the dense part of the gradient: the loss, and the
// gradient at the teacher's columns, all of the row's probability on a column in each of its entries.  One barrier.
struct RowGrad { bool keep; float scale; };   // dz = scale 2^(c (z - max)) off the teacher's columns
__device__ __forceinline__ RowGrad teacher_finish(Teacher& te, const DistillArgs& a, size_t row, bool masked, Online o, float c, bool grad) {
  const bool keep = !masked && te.any;
  const float lse = row_lse(o, a.tau);
  if (o.m == INFINITY) o.s = NAN;   // no softmax
  const float f = te.mass / o.s;
  if (threadIdx.x < 64) {
    const float loss = keep ? a.tau * a.tau * teacher_loss(te, a.k, o, a.tau, threadIdx.x) : 0.f;
    if (threadIdx.x == 0) { a.lse[row] = lse; a.loss_rows[row] = loss; }
  }
  if (grad) {
    const int j = (int)threadIdx.x - 64;   // (the second wave on)
    if (j >= 0 && j < a.k) te.grad[j] = a.tau * (f * __builtin_amdgcn_exp2f((te.z[j] - o.m) * c) - te.at[j]);
    __syncthreads();
  }
  return RowGrad{keep, a.tau * f};
}
// the teacher's columns, each by the thread that has stored its chunk of E before (a thread's stores to one address stay in order)
template <typename T, int NT, int E>
__device__ __forceinline__ void teacher_store(const Teacher& te, int k, T* dr) {
#pragma unroll 1
  for (int j = 0; j < k; j += 4) {
    const int4 id = *reinterpret_cast<const int4*>(&te.id[j]);   // (entries from k on are -1)
    if (id.x >= 0 && (id.x / E) % NT == (int)threadIdx.x) stf(dr, (size_t)id.x, te.grad[j]);
    if (id.y >= 0 && (id.y / E) % NT == (int)threadIdx.x) stf(dr, (size_t)id.y, te.grad[j + 1]);
    if (id.z >= 0 && (id.z / E) % NT == (int)threadIdx.x) stf(dr, (size_t)id.z, te.grad[j + 2]);
    if (id.w >= 0 && (id.w / E) % NT == (int)threadIdx.x) stf(dr, (size_t)id.w, te.grad[j + 3]);
  }
}

__device__ __forceinline__ void store_once8(bf16_t* p, const float (&v)[8]) {
  typedef unsigned u32x4_nt __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4_nt{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])}, reinterpret_cast<u32x4_nt*>(p));
}
__device__ __forceinline__ void store_once8(float* p, const float (&v)[8]) {
  typedef float f32x4_nt __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(f32x4_nt{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_nt*>(p));
  __builtin_nontemporal_store(f32x4_nt{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_nt*>(p) + 1);
}

// the gradient of a row that is read from memory a second time
template <typename T, int NT>
__device__ __forceinline__ void row_grad(const T* zr, T* dr, int V, int64_t ldz, const RowGrad& g, float m, float c) {
  constexpr int U = sizeof(T) == 2 ? 4 : 2, STEP = NT * 8;
  const int last = (int)ldz - 8;
  for (int base = 0; base < ldz; base += U * STEP) {
    Raw8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u].load(zr, (size_t)min(base + u * STEP + (int)threadIdx.x * 8, last));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = base + u * STEP + threadIdx.x * 8;
      float v[8];
      raw[u].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = g.keep && col + j < V ? g.scale * __builtin_amdgcn_exp2f((v[j] - m) * c) : 0.f;
      if (col < ldz) store_once8(dr + col, v);
    }
  }
}

}  // namespace

template <typename T, bool GRAD>
__global__ __launch_bounds__(512) void distill_kernel(DistillArgs a) {
  constexpr int NT = 512;
  __shared__ Teacher te;
  __shared__ Online sm[NT / 64];
  const size_t row = blockIdx.x;
  const T* zr = (const T*)a.z + row * (size_t)a.ldz;
  const float c = kLog2e / a.tau;
  const bool masked = a.mask[row] == 0;
  TeacherRegs regs;
  if (threadIdx.x < 64) {
    teacher_fetch(regs, a, row, threadIdx.x);
    teacher_logits(regs, zr, a.V);
  }
  Online o = row_stats<T, NT, !GRAD>(zr, a.V, c);
  if (threadIdx.x < 64) teacher_load(te, regs, a, threadIdx.x);
  o = online_block<NT>(o, c, sm);
  const RowGrad g = teacher_finish(te, a, row, masked, o, c, GRAD);
  if constexpr (GRAD) {
    T* dr = (T*)a.dz + row * (size_t)a.ldz;
    row_grad<T, NT>(zr, dr, a.V, a.ldz, g, o.m, c);
    if (g.keep) teacher_store<T, NT, 8>(te, a.k, dr);
  }
}

// The training call with the row held on its CU between the statistics and the gradient: read once, written once.  A thread
// keeps the 16-byte chunks t, t + 512, ... of its block's row: the first NREG in registers, all of them wholly below V, the n_lds
// others in LDS, where padded columns are turned into -inf.  Two passes of exponentials, each one fused step and 2^x per
// element; 128256 columns of bf16 are 24 chunks in registers and 8 in LDS, 66 KB
// with the teacher's entries, so that two rows share a CU and the arithmetic of one hides behind the memory traffic of the other.
// Bound by memory: [8192, 128256] bf16, k = 32: 750 us, 5.6 TB/s (k = 128: 795; read twice: 1210).
template <typename T, int NREG>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4, 4))) void distill_resident_kernel(DistillArgs a, int n_lds) {
  constexpr int NT = 512, E = 16 / (int)sizeof(T), STEP = NT * E;
  typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
  extern __shared__ u32x4_t distill_row_lds[];                 // n_lds x NT chunks
  __shared__ Teacher te;
  __shared__ float red[NT / 64], sums[NT / 64];
  const size_t row = blockIdx.x;
  const T* zr = (const T*)a.z + row * (size_t)a.ldz;
  T* dr = (T*)a.dz + row * (size_t)a.ldz;
  const float c = kLog2e / a.tau;
  const int V = a.V, c0 = threadIdx.x * E;
  u32x4_t* mine = distill_row_lds + threadIdx.x;
  const int bytes = (int)((uint32_t)a.ldz * (uint32_t)sizeof(T));
  const __amdgpu_buffer_rsrc_t rz = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(zr), 0, bytes, 0x00020000);
  const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(dr, 0, bytes, 0x00020000);
  auto fetch = [&](int col, int soff) { return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rz, (uint32_t)col * sizeof(T), soff, 2)); };
  auto store = [&](u32x4_t v, int col, int soff) { __builtin_amdgcn_raw_buffer_store_b128(v, rd, (uint32_t)col * sizeof(T), soff, 2); };
  const bool masked = a.mask[row] == 0;
  // Where the row's chunks leave no registers, the teacher's entries are done with before they are requested; else they are requested
  // before and worked on while the chunks arrive.
  constexpr bool EARLY = NREG >= 24;
  TeacherRegs regs;
  if (threadIdx.x < 64) {
    teacher_fetch(regs, a, row, threadIdx.x);
    if constexpr (EARLY) {
      teacher_logits(regs, zr, V);
      teacher_load(te, regs, a, threadIdx.x);
    }
  }
  u32x4_t buf[NREG > 0 ? NREG : 1];
#pragma unroll
  for (int i = 0; i < NREG; ++i) buf[i] = fetch(c0, i * STEP * (int)sizeof(T));
  if constexpr (!EARLY)
    if (threadIdx.x < 64) teacher_logits(regs, zr, V);
  for (int i = 0; i < n_lds; ++i) {
    const int col = c0 + (NREG + i) * STEP, nv = V - col;
    u32x4_t v = fetch(col, 0);
    if (nv < E) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) v[k] = 2 * k + 1 < nv ? v[k] : 2 * k < nv ? ((v[k] & 0xFFFFu) | 0xFF800000u) : 0xFF80FF80u;
        else v[k] = k < nv ? v[k] : 0xFF800000u;
      }
    }
    mine[i * NT] = v;
  }
  if constexpr (!EARLY)
    if (threadIdx.x < 64) teacher_load(te, regs, a, threadIdx.x);

  // each pass takes the register chunks strictly one after the other, so that no pass keeps their unpacked values
  auto turn = [&](int i, float& running) { asm volatile("" : "+v"(running), "+v"(buf[i])); };
  auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
  auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
  auto max3 = [](float x, float y, float z) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
  };
  auto chunk_max = [&](u32x4_t v, float m) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) m = max3(m, lo(v[k]), hi(v[k]));
    } else {
      m = max3(m, __uint_as_float(v[0]), __uint_as_float(v[1]));
      m = max3(m, __uint_as_float(v[2]), __uint_as_float(v[3]));
    }
    return m;
  };
  auto power = [&](float x, float slope, float sh) { return __builtin_amdgcn_exp2f(fmaf(x, slope, sh)); };
  auto chunk_sum = [&](u32x4_t v, float slope, float sh) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) s += power(lo(v[k]), slope, sh) + power(hi(v[k]), slope, sh);
      else s += power(__uint_as_float(v[k]), slope, sh);
    }
    return s;
  };
  auto chunk_grad = [&](u32x4_t v, float slope, float sh, float f) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) v[k] = f2bf2(f * power(lo(v[k]), slope, sh), f * power(hi(v[k]), slope, sh));
      else v[k] = __float_as_uint(f * power(__uint_as_float(v[k]), slope, sh));
    }
    return v;
  };

  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NREG; ++i) {
    turn(i, m);
    m = chunk_max(buf[i], m);
  }
  for (int i = 0; i < n_lds; ++i) m = chunk_max(mine[i * NT], m);
  m = fast_max(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fast_max(red[threadIdx.x % (NT / 64)]);
  const Power pw = power_of(m, c);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NREG; ++i) {
    turn(i, s);
    s += chunk_sum(buf[i], pw.slope, pw.shift);
  }
  for (int i = 0; i < n_lds; ++i) s += chunk_sum(mine[i * NT], pw.slope, pw.shift);
  s = fast_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  const Online o{m, pw.fix * fast_sum((threadIdx.x & 63) < NT / 64 ? sums[threadIdx.x & 63] : 0.f)};
  const RowGrad g = teacher_finish(te, a, row, masked, o, c, true);
  if (!g.keep) {
    const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < NREG; ++i) store(zero, c0, i * STEP * (int)sizeof(T));
    for (int i = 0; i < n_lds; ++i) store(zero, c0 + (NREG + i) * STEP, 0);
    return;
  }
  float sh = pw.shift;
  const float f = g.scale * pw.fix;
#pragma unroll
  for (int i = 0; i < NREG; ++i) {
    turn(i, sh);
    buf[i] = chunk_grad(buf[i], pw.slope, sh, f);
    store(buf[i], c0, i * STEP * (int)sizeof(T));
  }
  for (int i = 0; i < n_lds; ++i) {
    const int col = c0 + (NREG + i) * STEP, nv = V - col;
    u32x4_t v = chunk_grad(mine[i * NT], pw.slope, sh, f);
    if (nv < E) {   // padded columns are 0 also where the row's sums are not numbers
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) v[k] = 2 * k + 1 < nv ? v[k] : 2 * k < nv ? v[k] & 0xFFFFu : 0u;
        else v[k] = k < nv ? v[k] : 0u;
      }
    }
    store(v, col, 0);
  }
  teacher_store<T, NT, E>(te, a.k, dr);
}

namespace {
constexpr int kDistillMaxLds = 17;   // chunks of a thread in LDS: 8 KB of the block's row each, beside the teacher's entries
// The resident kernel for rows that fit a CU; false where they do not.
template <typename T>
bool launch_distill_resident(const DistillArgs& a, hipStream_t s, hipError_t& e) {
  constexpr int STEP = 512 * 16 / (int)sizeof(T);
  const int64_t chunks = (a.ldz + STEP - 1) / STEP, whole = a.V / STEP;
  static const int kRegs[] = {24, 20, 16, 12, 8, 7, 6, 4, 2, 1, 0};
  int nreg = 0;
  for (int r : kRegs)
    if (r <= whole) { nreg = r; break; }
  const int64_t n_lds = chunks - nreg;
  if (n_lds > kDistillMaxLds) return false;
  const size_t lds = (size_t)n_lds * 512 * 16;
  const void* kernel = nullptr;
#define TIDE_DISTILL(R) case R: kernel = (const void*)distill_resident_kernel<T, R>; break
  switch (nreg) {
    TIDE_DISTILL(24); TIDE_DISTILL(20); TIDE_DISTILL(16); TIDE_DISTILL(12); TIDE_DISTILL(8);
    TIDE_DISTILL(7); TIDE_DISTILL(6); TIDE_DISTILL(4); TIDE_DISTILL(2); TIDE_DISTILL(1); TIDE_DISTILL(0);
  }
#undef TIDE_DISTILL
  e = hipSuccess;
  if (lds > 65536 - 4096) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kDistillMaxLds * 512 * 16);
  if (e != hipSuccess) return true;
  DistillArgs args = a;
  int n = (int)n_lds;
  void* params[] = {&args, &n};
  e = hipLaunchKernel(kernel, dim3((unsigned)a.rows), dim3(512), params, lds, s);
  return true;
}
}  // namespace

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const bool grad = a.dz != nullptr;
  ProfScope ps(grad ? "distill_train" : "distill_eval", 0, (double)a.rows * dtype_size(dtype) * (a.V + (grad ? (double)a.ldz : 0.0)), s);
  hipError_t e;
  if (grad && (dtype == kBF16 ? launch_distill_resident<bf16_t>(a, s, e) : launch_distill_resident<float>(a, s, e))) return e;
  const dim3 grid((unsigned)a.rows), blk(512);
  // LDS that goes unused holds the gradient's rows in flight to two per CU, so that the second read finds them in the last cache: us with / without,
  // fp32 [4096, 128256] 1070 / 1277, [4096, 100001] 804 / 935.
  const size_t pad = 52 * 1024;
  if (dtype == kBF16) {
    if (grad) hipLaunchKernelGGL((distill_kernel<bf16_t, true>), grid, blk, pad, s, a);
    else hipLaunchKernelGGL((distill_kernel<bf16_t, false>), grid, blk, 0, s, a);
  } else {
    if (grad) hipLaunchKernelGGL((distill_kernel<float, true>), grid, blk, pad, s, a);
    else hipLaunchKernelGGL((distill_kernel<float, false>), grid, blk, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace tide
