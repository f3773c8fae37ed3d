// The largest entries of a row of logits, in order, while a workgroup streams it.
#pragma once
#include "score_shared.h"

namespace adwin {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// ---- order of the alternatives --------------------------------------------------------
// One 64-bit word per entry, larger for the larger logit and then for the lower index (-0 counts as 0).
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_key(float x, int i) {
  return ((uint64_t)order_bits(x) << 32) | (uint32_t)~i;
}
__device__ __forceinline__ int key_index(uint64_t k) { return ~(int)(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t b = (uint32_t)(k >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

// fmaxf without the two instructions that quiet its operands
__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
  return m;
}

// Part of a row: vectors [v0, v1), and the row's edge entries with the first part.
template <typename T, typename Row = RowSpan<T>>
struct Piece {
  Row row;
  int v0, v1, edge;
  __device__ __forceinline__ Piece(const T* p, int n, int piece, int pieces) : row(p, n) {
    v0 = (int)((int64_t)row.vecs * piece / pieces);
    v1 = (int)((int64_t)row.vecs * (piece + 1) / pieces);
    edge = piece == 0 ? row.edge : 0;
  }
};

constexpr int kPart = 384;         // keys that a wave can list: some 90 pass the bounds at top = 64 and V = 151,936
constexpr int kFound = kWaves * kPart;
constexpr int kDense = 512;        // ... and that can be ranked

struct Select {                    // in the LDS
  uint64_t kept[ADWIN_MAX_TOP];    // the result: sorted, zeros behind the last
  uint64_t found[kFound];
  uint64_t dense[kDense];
  uint64_t best[kThreads + 1];
  uint32_t most[kThreads];         // the threads' largest entries, as order_bits >> 16
  uint32_t bounds[kWaves];         // of the waves' maxima (lanes_bound)
  int listed[kWaves];
  int count;
};

// A lower bound of the `top`-th largest of the 256 numbers in `most`, exact in 16 bits, by every wave: the bits from the
// highest on, a bit stays where at least `top` numbers reach it.  0 where fewer than `top` are above 0.
__device__ __forceinline__ uint32_t wave_bound(const volatile uint32_t* most, int top) {
  const int lane = threadIdx.x & 63;
  uint32_t v[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v[w] = most[64 * w + lane];
  uint32_t at = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t t = at | (1u << bit);
    int n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n += __popcll(__ballot(v[w] >= t));
    if (n >= top) at = t;
  }
  return at;
}
// The same of a wave's 64 numbers: a quarter of the work.  Where each of the four waves has top / 4 threads whose largest entry reaches a
// number, `top` entries do: the least of the waves' numbers is a bound as well, and little below the exact one unless the
// waves, which take 512 entries in turn, see different rows.
__device__ __forceinline__ uint32_t lanes_bound(uint32_t mine, int n) {
  uint32_t at = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t t = at | (1u << bit);
    if (__popcll(__ballot(mine >= t)) >= n) at = t;
  }
  return at;
}
constexpr uint32_t kFinite = 0x0080u;               // order_bits >> 16 of the lowest finite number; -inf has 0x007f
__device__ __forceinline__ uint32_t least_bound(const volatile uint32_t* bounds) {
  uint32_t at = bounds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) { const uint32_t b = bounds[w]; at = b < at ? b : at; }
  return at;
}
// Where some wave has too few finite entries for its share (short rows, masks), the least is no bound, and the exact one is taken of what the
// threads wrote into `most` (8,192 rows of 1,000 bf16 entries, 20 alternatives, 87 -> 51 us; 1,000 rows of 151,936, 500 of them finite, 503 -> 65 us).
__device__ __forceinline__ uint32_t some_bound(const Select& l, int top) {
  const uint32_t at = least_bound(l.bounds);
  return __builtin_expect(at < kFinite, false) ? wave_bound(l.most, top) : at;
}
// the smallest logit whose order_bits reach at << 16, a finite one: masked entries are not listed
__device__ __forceinline__ float bound_value(uint32_t at) {
  const uint32_t b = (at < kFinite ? kFinite : at) << 16;
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

// keys[0, n): the `top` largest of them into `kept`, by counting the larger ones.  Keys differ.
__device__ __forceinline__ void rank_keys(Select& l, const uint64_t* keys, int n, int top) {
  for (int q = threadIdx.x; q < n; q += kThreads) {
    const uint64_t v = keys[q];
    int r = 0, j = 0;
    for (; j + 8 <= n; j += 8) {                   // eight reads of the LDS at a time
#pragma unroll
      for (int i = 0; i < 8; ++i) r += keys[j + i] > v;
    }
    for (; j < n; ++j) r += keys[j] > v;
    if (r < top) l.kept[r] = v;
  }
  if ((int)threadIdx.x >= n && (int)threadIdx.x < top) l.kept[threadIdx.x] = 0;
}

// The `top` largest keys of a piece for any input, where more entries pass the bounds than can be listed (ties, rows in
// rising order).  Round by round over 256 vectors: a thread's largest key is ranked among the threads', the
// top-th of these is a bound that at most `top` threads pass, and what passes it and the last of the kept ones is ranked
// together with those.
template <typename T, typename Row>
__device__ __forceinline__ void select_slowly(const Piece<T, Row>& p, int top, Select& l) {
  constexpr int N = Entry<T>::kPerVec;
  const int tid = threadIdx.x;
  int have = 0;
  const int rounds = (p.v1 - p.v0 + kThreads - 1) / kThreads;
  for (int k = p.edge ? -1 : 0; k < rounds; ++k) {             // the edge first
    uint64_t key[N];
    const int i = p.v0 + k * kThreads + tid;
#pragma unroll
    for (int e = 0; e < N; ++e) key[e] = 0;
    if (k < 0) {
      if (tid < p.edge) key[0] = order_key(Entry<T>::one(p.row.p + p.row.edge_index(tid)), p.row.edge_index(tid));
    } else if (i < p.v1) {
      float x[N];
      Entry<T>::unpack(p.row.vec(i), x);
#pragma unroll
      for (int e = 0; e < N; ++e) key[e] = order_key(x[e], p.row.index(i) + e);
    }
    uint64_t mine = key[0];
#pragma unroll
    for (int e = 1; e < N; ++e) mine = key[e] > mine ? key[e] : mine;
    if (!__syncthreads_or(have < top || mine > l.kept[top - 1])) continue;
    l.best[tid] = mine;
    if (tid == 0) { l.count = 0; l.best[kThreads] = 0; }
    __syncthreads();
    int rank = 0;
    for (int j = 0; j < kThreads; ++j) rank += l.best[j] > mine;
    if (rank == top - 1 && mine) l.best[kThreads] = mine;      // keys differ, but for the zeros of idle threads
    __syncthreads();
    uint64_t bound = l.best[kThreads];
    if (have == top && l.kept[top - 1] > bound) bound = l.kept[top - 1] + 1;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (key[e] && key[e] >= bound) l.found[atomicAdd(&l.count, 1)] = key[e];     // at most top * N
    if (tid < have) l.found[kFound - 1 - tid] = l.kept[tid];
    __syncthreads();
    const int n = l.count;
    if (tid < have) l.found[n + tid] = l.found[kFound - 1 - tid];
    __syncthreads();
    rank_keys(l, l.found, n + have, top);
    have = have + n < top ? have + n : top;
    __syncthreads();
  }
  if (tid >= have && tid < top) l.kept[tid] = 0;
  __syncthreads();
}

// What the waves have listed (`listed` keys of this one) and reaches the bound of the threads' largest entries, ranked.  Every
// wave has written its bound; `again`: since the one was taken that the listed keys reach.  False where more was found
// than could be listed or can be ranked, or fewer than `top` of the piece's `entries`: masked ones belong to them.
__device__ __forceinline__ bool select_found(Select& l, int listed, int top, int entries, bool again) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) l.listed[wave] = listed;
  if (threadIdx.x == 0) l.count = 0;
  __syncthreads();
  bool fits = true;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) fits = fits && l.listed[w] <= kPart;
  if (!fits) return false;
  const uint64_t bound = again ? (uint64_t)some_bound(l, top) << 48 : 0;
  uint64_t key[kPart / 64];
  int n = 0;
#pragma unroll
  for (int u = 0; u < kPart / 64; ++u) {
    const int q = 64 * u + lane;
    key[u] = q < listed ? l.found[wave * kPart + q] : 0;
    if (key[u] < bound) key[u] = 0;
    n += __popcll(__ballot(key[u] != 0));
  }
  int at = 0;
  if (lane == 0) at = atomicAdd(&l.count, n);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int u = 0; u < kPart / 64; ++u) {
    const uint64_t which = __ballot(key[u] != 0);
    const int q = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(which >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)which, 0));
    if (key[u] && q < kDense) l.dense[q] = key[u];
    at += __popcll(which);
  }
  __syncthreads();
  if (l.count > kDense || (l.count < top && l.count < entries)) return false;
  rank_keys(l, l.dense, l.count, top);
  __syncthreads();
  return true;
}

// Lists, in the wave's part, what entry x of index i is of the lanes where `is`.  No lane waits for an answer of the LDS.
__device__ __forceinline__ void list_entry(Select& l, int& listed, bool is, float x, int i) {
  const uint64_t which = __ballot(is);
  if (which == 0) return;
  const int q = listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(which >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)which, 0));
  if (is && q < kPart) l.found[(threadIdx.x >> 6) * kPart + q] = order_key(x, i);
  listed += __popcll(which);
}
// Entries of vector v that reach the bound, in the lanes where `is`; `first`: the index of the vector's first one.
template <typename T>
__device__ __forceinline__ void list_entries(Select& l, int& listed, bool is, const uint4& v, int first, float bound) {
  float x[Entry<T>::kPerVec];
  Entry<T>::unpack(v, x);
#pragma unroll
  for (int e = 0; e < Entry<T>::kPerVec; ++e) list_entry(l, listed, is && x[e] >= bound, x[e], first + e);
}

}  // namespace adwin
