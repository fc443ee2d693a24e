// Embedding of tokens and its gradient: include/tide_draft.h has the formulas.
#include <algorithm>

#include "kernels.h"
#include "loose.h"
#include "prof.h"

namespace tide {
namespace {

constexpr int kCols = 512;        // columns of a wave: eight a lane
constexpr int kChunk = 2048;      // rows that a block sorts
constexpr int kWays = 16;         // sorted runs that a pass joins
constexpr int kIdBits = 21;       // ids are below 2^21, and a chunk's place takes the 11 bits behind them
constexpr uint32_t kNone = (1u << kIdBits) - 1;   // id of a row without a token; no vocabulary reaches it
static_assert(kIdBits + 11 == 32 && kChunk == 1 << 11);

// One wave copies kCols columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void embed_fwd_kernel(int64_t rows, int vocab, int d, int tiles, const int32_t* __restrict__ ids, const T* __restrict__ table,
                                                        float scale, T* __restrict__ out) {
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row = w / tiles;
  if (row >= rows) return;
  const int c = (int)(w % tiles) * kCols + (threadIdx.x & 63) * 8, count = min(8, d - c);
  if (count <= 0) return;
  const int id = ids[row];
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (id >= 0 && id < vocab) {
    load_some(table + (size_t)id * d + c, count, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= scale;
  }
  store_some(out + (size_t)row * d + c, count, x);
}

// The first `chunks` blocks sort kChunk ids each, with their places, by id and then by place; the others clear the gradient, where it is written and not
// added to, while they do.
__global__ __launch_bounds__(1024) void embed_sort_kernel(int64_t rows, int vocab, int chunks, const int32_t* __restrict__ ids, uint32_t* __restrict__ sid,
                                                          int32_t* __restrict__ pos, uint32_t* __restrict__ clear, size_t head, size_t words, int tail) {
  if (blockIdx.x >= chunks) {
    // `head` bytes up to a multiple of 16, then 16-byte words, then `tail` bytes
    uint8_t* bytes = reinterpret_cast<uint8_t*>(clear);
    const size_t at = (size_t)(blockIdx.x - chunks) * 1024 + threadIdx.x, step = (size_t)(gridDim.x - chunks) * 1024;
    u32x4* body = reinterpret_cast<u32x4*>(bytes + head);
    for (size_t i = at; i < words; i += step) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, body + i);
    if (at < head) bytes[at] = 0;
    if (at < (size_t)tail) bytes[head + words * 16 + at] = 0;
    return;
  }
  __shared__ uint32_t key[kChunk];
  const int64_t base = (int64_t)blockIdx.x * kChunk;
  for (int i = threadIdx.x; i < kChunk; i += 1024) {
    const int64_t row = base + i;
    const int id = row < rows ? ids[row] : -1;
    key[i] = id >= 0 && id < vocab ? (uint32_t)id << 11 | (uint32_t)i : kNone << 11 | (uint32_t)i;
  }
  // bitonic: no two keys are alike, so that the order is the one order there is
  for (int k = 2; k <= kChunk; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      __syncthreads();
      const int i = 2 * threadIdx.x - (threadIdx.x & (j - 1)), o = i + j;
      const uint32_t a = key[i], b = key[o];
      if ((a > b) == ((i & k) == 0)) key[i] = b, key[o] = a;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < kChunk; i += 1024) sid[base + i] = key[i] >> 11, pos[base + i] = (int32_t)(base + (key[i] & (kChunk - 1)));
}

// Joins kWays sorted runs of `run` each: a row's place is its own and, of every other run, how many come before it (equal ids: those of earlier runs).
__global__ __launch_bounds__(256) void embed_merge_kernel(int64_t total, int64_t run, const uint32_t* __restrict__ sid, const int32_t* __restrict__ pos,
                                                          uint32_t* __restrict__ sid_out, int32_t* __restrict__ pos_out) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  const int64_t group = e / (run * kWays) * (run * kWays);
  const int own = (int)((e - group) / run);
  const uint32_t id = sid[e];
  int64_t found[kWays];
#pragma unroll
  for (int s = 0; s < kWays; ++s) found[s] = 0;
  for (int64_t half = run; half > 0; half /= 2)   // (a power of two)
#pragma unroll
    for (int s = 0; s < kWays; ++s) {
      const int64_t first = group + s * run, length = min(run, total - first), next = found[s] + half;
      if (s == own || next > length) continue;   // (the last run may be short or missing)
      const uint32_t other = sid[first + next - 1];
      if (s < own ? other <= id : other < id) found[s] = next;
    }
  int64_t to = e - own * run;
#pragma unroll
  for (int s = 0; s < kWays; ++s) to += found[s];
  sid_out[to] = id, pos_out[to] = pos[e];
}

template <typename T> struct Row8;   // eight elements as loaded
template <> struct Row8<bf16_t> {
  u32x4 a;
  __device__ __forceinline__ void load(const bf16_t* p, int count) {
    if (count >= 8) { a = LDX(u32x4_of_halves, p); return; }
    a = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) a[j / 2] |= (uint32_t)p[j] << (16 * (j % 2));
  }
  __device__ __forceinline__ void add(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[2 * j] += __uint_as_float(a[j] << 16), x[2 * j + 1] += __uint_as_float(a[j] & 0xFFFF0000u);
  }
};
template <> struct Row8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p, int count) {
    if (count >= 8) { a = LDX(f32x4_of_floats, p), b = LDX(f32x4_of_floats, p + 4); return; }
    a = b = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < count) a[j] = p[j];
      if (4 + j < count) b[j] = p[4 + j];
    }
  }
  __device__ __forceinline__ void add(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += a[j], x[4 + j] += b[j];
  }
};

template <typename G>
__device__ __forceinline__ void finish(G* to, int count, float scale, bool accumulate, const float (&sum)[8]) {
  float x[8], old[8];
  if (accumulate) load_some(to, count, old);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = accumulate ? fmaf(scale, sum[j], old[j]) : scale * sum[j];
  store_some(to, count, x);
}

// A wave adds up kCols columns of `piece` rows that follow each other in the order of their tokens.  A token whose rows all lie in the piece is done;
// of one that goes on in front of or behind it, what lies here is left as a part: parts[2 p] for the first token, parts[2 p + 1] for the last (the first, where there is but
// one and it goes on in front).
template <typename T, typename G>
__global__ __launch_bounds__(256) void embed_sum_kernel(int64_t total, int piece, int d, int tiles, const uint32_t* __restrict__ sid, const int32_t* __restrict__ pos,
                                                        const T* __restrict__ dy, float scale, G* __restrict__ dtable, int accumulate, float* __restrict__ parts) {
  constexpr int U = 8;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t p = w / tiles, first = p * piece;
  if (first >= total) return;
  const int lane = threadIdx.x & 63;
  const int c = (int)(w % tiles) * kCols + lane * 8, count = min(8, d - c);
  const int64_t mine = first + min(lane, piece - 1);   // (total is a multiple of every piece)
  const uint32_t my_id = sid[mine];
  const int my_row = pos[mine];
  const uint32_t before = first > 0 ? sid[first - 1] : kNone, behind = first + piece < total ? sid[first + piece] : kNone;
  uint32_t id = __builtin_amdgcn_readlane(my_id, 0);
  if (id == kNone) return;
  bool open = before == id;     // whether the token at hand goes on in front of the piece
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto leave = [&](bool goes_on) {
    if (count > 0) {
      if (open || goes_on) store_some(parts + (size_t)(2 * p + (open ? 0 : 1)) * d + c, count, sum);
      else finish(dtable + (size_t)id * d + c, count, scale, accumulate, sum);
    }
    open = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  };
  for (int k0 = 0; k0 < piece; k0 += U) {
    Row8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = __builtin_amdgcn_readlane(my_id, k0 + u);
      const T* row = dy + (size_t)__builtin_amdgcn_readlane(my_row, k0 + u) * d + c;
      if (at == kNone) continue;   // (uniform)
      raw[u].load(row, count);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = __builtin_amdgcn_readlane(my_id, k0 + u);
      if (at != id) {
        leave(false);
        id = at;
      }
      if (at == kNone) return;   // what follows has no token either
      raw[u].add(sum);
    }
  }
  leave(behind == id);
}

// Adds up the parts of a token that reaches over pieces, from the piece it begins in.
template <typename G>
__global__ __launch_bounds__(256) void embed_join_kernel(int64_t total, int piece, int d, int tiles, const uint32_t* __restrict__ sid, float scale, G* __restrict__ dtable,
                                                         int accumulate, const float* __restrict__ parts) {
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t p = w / tiles, end = (p + 1) * piece;
  if (end >= total) return;   // nothing goes on behind the last one
  const uint32_t id = sid[end - 1];
  if (id == kNone || sid[end] != id) return;
  if (p > 0 && sid[p * piece - 1] == id) return;   // begins before
  // how many pieces it reaches into: the first place behind it, by steps that double and then halve
  int64_t lo = end, step = 1;   // sid[lo] == id
  while (lo + step < total && sid[lo + step] == id) lo += step, step *= 2;
  for (; step > 0; step /= 2)
    if (lo + step < total && sid[lo + step] == id) lo += step;
  const int64_t last = lo / piece;
  const int c = (int)(w % tiles) * kCols + (threadIdx.x & 63) * 8, count = min(8, d - c);
  if (count <= 0) return;
  float sum[8];
  load_some(parts + (size_t)(2 * p + 1) * d + c, count, sum);
  for (int64_t q = p + 1; q <= last; q += 4) {
    float x[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (q + u <= last) load_some(parts + (size_t)(2 * (q + u)) * d + c, count, x[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (q + u <= last) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += x[u][j];
      }
  }
  finish(dtable + (size_t)id * d + c, count, scale, accumulate, sum);
}

struct Plan {
  int64_t total, pieces;   // rows up to a whole chunk
  int piece, tiles;
  size_t ids[2], parts, bytes;
};
constexpr int64_t kWaves = 4096;   // waves that the sums are spread over at least, where there are rows for it

Plan make_plan(int64_t rows, int64_t d) {
  Plan p;
  p.total = (rows + kChunk - 1) / kChunk * kChunk;
  p.tiles = (int)((d + kCols - 1) / kCols);
  p.piece = 8;
  while (p.piece < 64 && (rows + p.piece - 1) / p.piece * p.tiles > kWaves) p.piece *= 2;
  p.pieces = (rows + p.piece - 1) / p.piece;
  // room for the most pieces that this many rows or fewer have, so that the size never falls as rows grow
  const int64_t cap = std::max<int64_t>(1, kWaves / p.tiles);
  const int64_t most = (rows + 7) / 8 <= cap ? (rows + 7) / 8 : std::max(cap, (rows + 63) / 64);
  const size_t list = (size_t)p.total * 8;
  p.ids[0] = 0, p.ids[1] = list, p.parts = 2 * list;
  p.bytes = (p.parts + (size_t)most * 2 * (size_t)d * 4 + 255) / 256 * 256;
  return p;
}

template <typename T, typename G>
hipError_t sums(const EmbedBwdArgs& a, const Plan& p, const uint32_t* sid, const int32_t* pos, float* parts, hipStream_t s) {
  const unsigned blocks = (unsigned)((p.pieces * p.tiles + 3) / 4);
  {
    ProfScope ps("embed_sum", (double)a.rows * a.d, (double)a.rows * a.d * sizeof(T), s);
    hipLaunchKernelGGL((embed_sum_kernel<T, G>), dim3(blocks), dim3(256), 0, s, p.total, p.piece, (int)a.d, p.tiles, sid, pos, (const T*)a.dy, a.scale, (G*)a.dtable,
                       a.accumulate, parts);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (p.pieces < 2) return hipSuccess;
  ProfScope ps("embed_join", 0, 0, s);
  hipLaunchKernelGGL((embed_join_kernel<G>), dim3(blocks), dim3(256), 0, s, p.total, p.piece, (int)a.d, p.tiles, sid, a.scale, (G*)a.dtable, a.accumulate, parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed_fwd(int64_t rows, int vocab, int d, const int32_t* ids, const void* table, float scale, void* out, int dtype, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const int tiles = (d + kCols - 1) / kCols;
  const unsigned blocks = (unsigned)((rows * tiles + 3) / 4);
  ProfScope ps("embed_fwd", 0, 2.0 * (double)rows * d * dtype_size(dtype), s);
  if (dtype == kBF16) hipLaunchKernelGGL(embed_fwd_kernel<bf16_t>, dim3(blocks), dim3(256), 0, s, rows, vocab, d, tiles, ids, (const bf16_t*)table, scale, (bf16_t*)out);
  else hipLaunchKernelGGL(embed_fwd_kernel<float>, dim3(blocks), dim3(256), 0, s, rows, vocab, d, tiles, ids, (const float*)table, scale, (float*)out);
  return hipGetLastError();
}

size_t embed_bwd_workspace_bytes(int64_t rows, int64_t d) { return make_plan(std::max<int64_t>(rows, 1), d).bytes; }

hipError_t launch_embed_bwd(const EmbedBwdArgs& a, hipStream_t s) {
  const Plan p = make_plan(std::max<int64_t>(a.rows, 1), a.d);
  char* ws = (char*)a.workspace;
  const int chunks = a.rows > 0 ? (int)(p.total / kChunk) : 0;
  const size_t bytes = a.accumulate ? 0 : (size_t)a.vocab * (size_t)a.d * dtype_size(a.table_dtype);
  const size_t head = std::min(bytes, (16 - ((uintptr_t)a.dtable & 15)) & 15), words = (bytes - head) / 16;
  const int tail = (int)(bytes - head - words * 16);
  const int clear = bytes ? (int)std::min<size_t>((words + 4095) / 4096 + 1, 2048) : 0;
  uint32_t* sid[2];
  int32_t* pos[2];
  for (int k = 0; k < 2; ++k) sid[k] = (uint32_t*)(ws + p.ids[k]), pos[k] = (int32_t*)(sid[k] + p.total);
  if (chunks + clear == 0) return hipSuccess;
  {
    ProfScope ps("embed_sort", 0, (double)bytes, s);
    hipLaunchKernelGGL(embed_sort_kernel, dim3(chunks + clear), dim3(1024), 0, s, a.rows, a.vocab, chunks, a.ids, sid[0], pos[0], (uint32_t*)a.dtable, head, words, tail);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (a.rows <= 0) return hipSuccess;
  int at = 0;
  for (int64_t run = kChunk; run < p.total; run *= kWays, at ^= 1) {
    ProfScope ps("embed_merge", 0, 0, s);
    hipLaunchKernelGGL(embed_merge_kernel, dim3((unsigned)(p.total / 256)), dim3(256), 0, s, p.total, run, sid[at], pos[at], sid[at ^ 1], pos[at ^ 1]);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  float* parts = (float*)(ws + p.parts);
  const bool wide = a.table_dtype == kF32;
  if (a.dtype == kBF16) return wide ? sums<bf16_t, float>(a, p, sid[at], pos[at], parts, s) : sums<bf16_t, bf16_t>(a, p, sid[at], pos[at], parts, s);
  return sums<float, float>(a, p, sid[at], pos[at], parts, s);
}

}  // namespace tide
