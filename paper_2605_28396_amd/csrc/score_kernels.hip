// Log-probabilities of given tokens with entropy and top alternatives, and their gradient.
//
// With x_j = z_j / temperature, m = max z, s = sum_j exp((z_j - m) / temperature):
//   log p_j = (z_j - m) / temperature - log s,   H = log s - (1/s) sum_j e_j (z_j - m) / temperature.
// Exponentials are taken to the base 2: d_j = c z_j - r, one fma, with c = log2(e) / temperature and a thread's own reference r.
#include "score_shared.h"

namespace adwin {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct LogpArgs {
  const void* z; int64_t ld; int64_t T;
  int32_t V, G, top;
  int32_t pieces;                   // workgroups per row; their sums and keys in `part`, `keys` where there are several
  float* part;                      // [T][pieces][4] m, s, t, 0
  uint64_t* keys;                   // [T][pieces][top]
  float temperature, c;             // c = log2(e) / temperature
  const int32_t* ids;
  float* logp; float* entropy; float* norm; int32_t* top_ids; float* top_logp; int32_t* row_status;
};

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

// Running sums of one thread, relative to its reference r (in units of the exponent to the base 2).
struct Sums { float r, s, t, m; };      // s = sum 2^d, t = sum 2^d d, m = largest logit
// The least reference, and that of no entries.  A reference is a whole number next to some c z, which fp32 gives to a half only as long
// as |c z| is at most 2^24: beyond, c z - r at the reference's own entry can pass the range of the exponential.  What lies lower
// (masks of large finite values) is summed as 0 relative to this; pieces whose largest logit lies outside are read again (piece_sums).
constexpr float kNoRef = -16777216.f;
// d may reach this before the reference moves.  Exponentials bear more (2^16 is far from the end of fp32), but the largest
// term's d is rounded where it is summed into t and cancels only there: with 16 the entropy of rows with one likely token was off by 2.6e-6
// at most (fp32 7.1e-6) where it is 8e-7 (1.3e-6) with 4.
constexpr float kSlack = 4.f;
// References are whole numbers, so that moving and merging sums multiplies by exact powers of two (with the threads' largest
// exponents themselves, the roundings of their differences were the same for all terms of a thread).
__device__ __forceinline__ float ref_of(float m, float c) { return ceilf(m * c); }
__device__ __forceinline__ Sums no_sums() { return {kNoRef, 0.f, 0.f, -INFINITY}; }

__device__ __forceinline__ void move_ref(Sums& a, float r) {
  const float by = a.r - r, f = fast_exp2(by);
  a.t = f * fmaf(a.s, fmaxf(by, kNegBig), a.t);
  a.s *= f;
  a.r = r;
}
// fmaxf without the two instructions that quiet its operands
__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
  return m;
}
// Returns the largest of x.  The terms of a vector are summed first: bf16 logits and whole-number references give few different terms, whose
// roundings in one sum per thread, 594 terms long at V = 151,936, were the same in all threads and did not average out: s was off by 8.8e-6
// at most where all logits are equal, by 3.3e-6 where a likely token comes early, and is by 1.1e-6 and 4.5e-7 so (fp32 2.2e-6, 7.3e-7).
template <int N>
__device__ __forceinline__ float add_entries(Sums& a, const float (&x)[N], float c) {
  float m = x[0];
  if constexpr (N > 1) m = max3(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i + 1 < N; i += 2) m = max3(m, x[i], x[i + 1]);
  if constexpr (N > 1) m = max3(m, x[N - 1], x[N - 1]);
  a.m = max3(a.m, m, m);
  if (m * c > a.r + kSlack) move_ref(a, ref_of(m, c));
  float e[N], t = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = fmaf(x[i], c, -a.r);
    e[i] = fast_exp2(d);
    t = fmaf(e[i], fmaxf(d, kNegBig), t);            // a masked entry is 0 times something finite
  }
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) e[i] += e[i + n];
  a.s += e[0];
  a.t += t;
  return m;
}
// Sums over the workgroup.  All move to the largest reference first, which multiplies them by powers of two.
__device__ __forceinline__ Sums wave_sums(Sums a) {
  move_ref(a, wave_max(a.r));
  return {a.r, wave_sum(a.s), wave_sum(a.t), wave_max(a.m)};
}
__device__ __forceinline__ Sums block_sums(const Sums& mine, float (*part)[4]) {
  Sums a = wave_sums(mine);
  if ((threadIdx.x & 63) == 0) {
    float* q = part[threadIdx.x >> 6];
    q[0] = a.r; q[1] = a.s; q[2] = a.t; q[3] = a.m;
  }
  __syncthreads();
  float r = part[0][0];
  a.m = part[0][3];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) { r = fmaxf(r, part[w][0]); a.m = fmaxf(a.m, part[w][3]); }
  a.r = r; a.s = 0.f; a.t = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sums b = {part[w][0], part[w][1], part[w][2], 0.f};
    move_ref(b, r);
    a.s += b.s;
    a.t += b.t;
  }
  return a;
}

// Part of a row: vectors [v0, v1), and the row's edge entries with the first part.
template <typename T>
struct Piece {
  RowSpan<T> row;
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
template <typename T>
__device__ __forceinline__ void select_slowly(const Piece<T>& p, int top, Select& l) {
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

// The sums relative to the piece's largest logit: 1 <= s, and the entropy log s - t / s has no terms larger than need be.
// Pieces whose references do not hold (kNoRef: logits or 1 / temperature of millions, rows at a mask's finite value) are read again,
// differences first.
template <typename T>
__device__ __forceinline__ Sums piece_sums(const Piece<T>& p, const Sums& mine, float c, float (*part)[4]) {
  Sums a = block_sums(mine, part);
  const bool far = fabsf(a.m * c) > -kNoRef && fabsf(a.m) < INFINITY;
  if (a.m == -INFINITY) return a;                    // nothing but masked entries (s = 0) and NaN
  if (!far) {
    const float by = -fmaf(a.m, c, -a.r), f = fast_exp2(by);
    a.t = f * fmaf(a.s, by, a.t);
    a.s *= f;
    return a;
  }
  __syncthreads();
  Sums b = {0.f, 0.f, 0.f, a.m};
  auto add = [&](float z, float& s, float& t) {
    const float d = (z - a.m) * c, e = fast_exp2(d);
    s += e;
    t = fmaf(e, fmaxf(d, kNegBig), t);
  };
  if ((int)threadIdx.x < p.edge) add(Entry<T>::one(p.row.p + p.row.edge_index(threadIdx.x)), b.s, b.t);
  for (int i = p.v0 + threadIdx.x; i < p.v1; i += kThreads) {
    float x[Entry<T>::kPerVec], s = 0.f, t = 0.f;
    Entry<T>::unpack(p.row.vec(i), x);
#pragma unroll
    for (int e = 0; e < Entry<T>::kPerVec; ++e) add(x[e], s, t);
    b.s += s;
    b.t += t;
  }
  return block_sums(b, part);
}

// Whether some id of the row is scored (or G = 0), and whether one is beyond V: every wave looks for itself.
struct RowIds { bool live, bad; };
__device__ __forceinline__ RowIds row_ids(const int32_t* ids, int G, int V, int64_t row) {
  RowIds is{G == 0, false};
  for (int g0 = 0; g0 < G; g0 += 64) {
    const int g = g0 + (threadIdx.x & 63);
    const int id = g < G ? ids[row * G + g] : -1;
    is.live = is.live || __ballot(id >= 0 && id < V) != 0;
    is.bad = is.bad || __ballot(id >= V) != 0;
  }
  return is;
}

// The logit of thread g's given token, g < G; masked where it is not scored.
template <typename T>
__device__ __forceinline__ float given_logit(const LogpArgs& a, int64_t row, bool* scored) {
  const int id = (int)threadIdx.x < a.G ? a.ids[row * a.G + threadIdx.x] : -1;
  *scored = id >= 0 && id < a.V;
  return *scored ? Entry<T>::one((const T*)a.z + row * a.ld + id) : -INFINITY;
}

__device__ __forceinline__ void finish_row(const LogpArgs& a, int64_t row, const Sums& sum, const uint64_t* kept, RowIds is,
                                           float given, bool scored) {
  const int tid = threadIdx.x;
  const float s = sum.s;
  const bool fine = is.live && s > 0.f && s < INFINITY && fabsf(sum.m) < INFINITY;
  const float ls = fine ? logf(s) : 0.f;
  if (tid < a.G && a.logp) {
    a.logp[row * a.G + tid] = fine && scored ? (given - sum.m) / a.temperature - ls : 0.f;
  }
  if (tid < a.top) {
    const uint64_t k = kept[tid];
    const bool is = fine && k;
    if (a.top_ids) a.top_ids[row * a.top + tid] = is ? key_index(k) : -1;
    if (a.top_logp) a.top_logp[row * a.top + tid] = is ? (key_value(k) - sum.m) / a.temperature - ls : 0.f;
  }
  if (tid == 0) {
    if (a.entropy) a.entropy[row] = fine ? fmaxf(0.f, fmaf(-kLn2, sum.t / s, ls)) : 0.f;
    if (a.norm) { a.norm[2 * row] = fine ? sum.m : 0.f; a.norm[2 * row + 1] = fine ? s : 0.f; }
    if (a.row_status) a.row_status[row] = (is.bad ? ADWIN_DEV_BAD_ID : 0) | (is.live && !fine ? ADWIN_DEV_NONFINITE : 0);
  }
}

// One pass over the row, kStep vectors to a thread at a time.  8,192 rows (7,680 of them scored) of V = 151,936 bf16 with 20
// alternatives: 368 to 390 us over machines, 6.0 to 6.3 TB/s, without alternatives 367 us.  What bounds it is the read of the logits (a plain read of them 330 to 375 us) and, at
// the clock of 2.1 GHz that it gets, the vector unit: 7.5 instructions an entry, 10 with what the alternatives take, busy
// all the time; without the entropy's two of them it takes 377 us where it took 416.
// The alternatives ride on the softmax's own maxima: the `top`-th largest of the threads' largest entries is a lower bound of the
// `top`-th largest entry.  The first kStep vectors give one, what reaches it is listed (the bound is taken anew when twice as much
// has been read), and at the end the threads' largest of all leave little more than `top` of these to rank.
constexpr int kStep = 4;

template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads, 6) void token_logp_kernel(LogpArgs a) {
  constexpr int N = Entry<T>::kPerVec;
  __shared__ Select l;
  __shared__ float part[kWaves][4];
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x / (uint32_t)a.pieces;
  const int piece = (int)(blockIdx.x - (uint32_t)r * (uint32_t)a.pieces);
  const Piece<T> p((const T*)a.z + r * a.ld, a.V, piece, a.pieces);
  const int last = p.v1 - tid;                      // a thread's vectors: p.v0 + tid + 256 k below p.v1
  // whole steps, whose loads stand in no branch: the wait for a vector then leaves the younger ones in flight
  const int whole = (p.v1 - p.v0) / (kStep * kThreads);
  int i0 = p.v0;
  uint4 v[kStep];
  auto load = [&](int u) { v[u] = p.row.template vec<PAST>(i0 + tid + kThreads * u); };
  auto load_any = [&](int u) {
    v[u] = Entry<T>::none();
    if (i0 + kThreads * u < last) load(u);
  };
  // the first vectors are under way before the ids say whether the row is computed
  if (whole > 0) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) load(u);
  } else {
#pragma unroll
    for (int u = 0; u < kStep; ++u) load_any(u);
  }
  const RowIds is = row_ids(a.ids, a.G, a.V, r);
  Sums sum = no_sums();
  float given = 0.f;
  bool scored = false;
  if (is.live) {
    float bound = INFINITY;
    int listed = 0;                                 // keys of this wave
    float edge[1] = {-INFINITY};
    if (tid < p.edge) edge[0] = Entry<T>::one(p.row.p + p.row.edge_index(tid));
    if (a.pieces == 1) given = given_logit<T>(a, r, &scored);
    auto add = [&](int u) {
      float x[N];
      Entry<T>::unpack(v[u], x);
      return add_entries(sum, x, a.c);
    };
    if (tid < p.edge) add_entries(sum, edge, a.c);
    // the first vectors, which give the first bound and are then gone through again
#pragma unroll
    for (int u = 0; u < kStep; ++u) add(u);
    const int quarter = (a.top + kWaves - 1) / kWaves;
    auto take_bound = [&](bool all) {               // a thread without entries: -inf; `all`: for the exact bound too
      const uint32_t most = order_bits(sum.m) >> 16, at = lanes_bound(most, quarter);
      if (all) l.most[tid] = most;
      if ((tid & 63) == 0) *(volatile uint32_t*)&l.bounds[tid >> 6] = at;
    };
    if (a.top > 0) {
      take_bound(true);
      __syncthreads();
      bound = bound_value(some_bound(l, a.top));
      list_entry(l, listed, tid < p.edge && edge[0] >= bound, edge[0], p.row.edge_index(tid));
#pragma unroll
      for (int u = 0; u < kStep; ++u)
        list_entries<T>(l, listed, i0 + kThreads * u < last, v[u], p.row.index(i0 + tid + kThreads * u), bound);
    }
    i0 += kStep * kThreads;
    if (whole > 1) {
#pragma unroll
      for (int u = 0; u < kStep; ++u) load(u);
    }
    for (int step = 1; step < whole; ++step) {
      if (a.top > 0 && (step & (step - 1)) == 0) {
        // A new bound at steps 1, 2, 4, 8, ....  An older one of another wave is a bound as well: nobody waits.
        take_bound(false);
        bound = fmaxf(bound, bound_value(least_bound(l.bounds)));
      }
      const int first = p.row.index(i0 + tid);
      i0 += kStep * kThreads;
      if (step + 1 < whole) {
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
          if (__any(add(u) >= bound)) list_entries<T>(l, listed, true, v[u], first + kThreads * N * u, bound);
          load(u);
        }
      } else {
#pragma unroll
        for (int u = 0; u < kStep; ++u)
          if (__any(add(u) >= bound)) list_entries<T>(l, listed, true, v[u], first + kThreads * N * u, bound);
      }
    }
    if (whole > 0) {
#pragma unroll
      for (int u = 0; u < kStep; ++u) load_any(u);
#pragma unroll
      for (int u = 0; u < kStep; ++u) {
        if (__any(i0 + kThreads * u < last) && __any(add(u) >= bound))
          list_entries<T>(l, listed, i0 + kThreads * u < last, v[u], p.row.index(i0 + tid + kThreads * u), bound);
      }
    }
    if (a.top > 0) {
      if (whole > 0) take_bound(true);
      if (!select_found(l, listed, a.top, p.edge + (p.v1 - p.v0) * N, whole > 0)) select_slowly(p, a.top, l);
    }
    sum = piece_sums(p, sum, a.c, part);
  }
  if (a.pieces == 1) {
    finish_row(a, r, sum, l.kept, is, given, scored);
    return;
  }
  if (!is.live) return;                                // the join sees that by itself
  if (tid == 0) {
    float* q = a.part + 4 * (int64_t)blockIdx.x;
    q[0] = sum.m; q[1] = sum.s; q[2] = sum.t; q[3] = 0.f;
  }
  if (tid < a.top) a.keys[(int64_t)blockIdx.x * a.top + tid] = l.kept[tid];
}

// The pieces of a row, joined in their order.
constexpr int kMaxPieces = 64;
template <typename T>
__global__ __launch_bounds__(kThreads) void join_logp_kernel(LogpArgs a) {
  __shared__ Select l;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const RowIds is = row_ids(a.ids, a.G, a.V, r);
  Sums sum = no_sums();
  float given = 0.f;
  bool scored = false;
  if (is.live) {
    given = given_logit<T>(a, r, &scored);
    const float4* part = (const float4*)a.part + r * a.pieces;
    if (a.top > 0) {
      const int n = a.pieces * a.top;
      const uint64_t* keys = a.keys + r * a.pieces * a.top;
      constexpr int kMine = kMaxPieces * ADWIN_MAX_TOP / kThreads;
      uint64_t key[kMine], most = 0;
#pragma unroll
      for (int u = 0; u < kMine; ++u)               // straight-line loads: beyond the last the last again
        if (u * kThreads < n) key[u] = keys[u * kThreads + tid < n ? u * kThreads + tid : n - 1];
#pragma unroll
      for (int u = 0; u < kMine; ++u) {
        if (u * kThreads + tid >= n) key[u] = 0;
        most = key[u] > most ? key[u] : most;
      }
      if (tid == 0) l.count = 0;
      l.most[tid] = (uint32_t)(most >> 48);
      __syncthreads();
      const uint64_t bound = (uint64_t)wave_bound(l.most, a.top) << 48;
#pragma unroll
      for (int u = 0; u < kMine; ++u)
        if (key[u] && key[u] >= bound) {
          const int q = atomicAdd(&l.count, 1);
          if (q < kFound) l.found[q] = key[u];
        }
      __syncthreads();
      if (l.count <= kFound) {
        rank_keys(l, l.found, l.count, a.top);
      } else {                                      // ties in all pieces: every key against all others
        for (int q = tid; q < n; q += kThreads) {
          const uint64_t v = keys[q];
          int rank = 0;
          for (int j = 0; j < n; ++j) rank += keys[j] > v;
          if (v && rank < a.top) l.kept[rank] = v;
        }
      }
    }
    // every wave by itself, a piece to a lane
    float4 q = part[lane < a.pieces ? lane : 0];
    if (lane >= a.pieces) q = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    sum.m = wave_max(q.x);
    const float by = (q.x - sum.m) * a.c, f = fast_exp2(by);
    sum.s = wave_sum(f * q.y);
    sum.t = wave_sum(f * fmaf(q.y, fmaxf(by, kNegBig), q.z));
    __syncthreads();
  }
  finish_row(a, r, sum, l.kept, is, given, scored);
}

// Pieces of a row.  One for calls of 256 rows or more; fewer are cut so that every compute unit has a workgroup, each with half a
// step of its threads or more.  us, target of 256 / 512 / 1,024 workgroups, bf16, V = 151,936: 64 rows 23.8 / 22.1 / 22.8, 300 rows
// 42 / 42 / 39, 500 rows 48 / 51 / 53, 1,000 rows 76 / 73 / 87; fp32, V = 32,771: 100 rows 23.4 / 21.9 / 21.7, 400 rows 26 / 31 / 31,
// 1,000 rows 35 / 35 / 49 (one piece to a row: 1 row 31 us, in pieces 20).
static int logp_pieces(int64_t T, int32_t V, int32_t dtype) {
  const int64_t step = (int64_t)kStep * kThreads * (dtype == ADWIN_DT_BF16 ? 8 : 4) / 2;
  int64_t n = (256 + T - 1) / (T > 0 ? T : 1);
  if (n > V / step) n = V / step;
  return (int)(n < 1 ? 1 : n > kMaxPieces ? kMaxPieces : n);
}

struct LogpLayout {
  int pieces;
  size_t o_keys, bytes;
  explicit LogpLayout(const adwin_opd_logp_problem* p) {
    pieces = logp_pieces(p->T, p->V, p->z_dtype);
    const size_t n = pieces > 1 ? (size_t)p->T * pieces : 0;
    o_keys = align_up(n * 4 * sizeof(float), 256);
    bytes = align_up(o_keys + n * p->top * sizeof(uint64_t), 256);
  }
};

// ---------------------------------------------------------------------------------------
// dz_j = -p_j (a + g_H (log p_j + H)) / temperature, a = sum_g g_g, and g_g / temperature more at the given tokens, whose
// entries are computed again and written once more after the row (they were read before it: dz may be z).
// ---------------------------------------------------------------------------------------
struct LogpGradArgs {
  const void* z; int64_t ld_z; void* dz; int64_t ld_dz; int64_t T;
  int32_t V, G, pieces;
  float c, per_temperature;
  const int32_t* ids; const float* norm; const float* g_logp; const float* entropy; const float* g_entropy;
};

struct GradRow {
  float m, c, per_s, log_s, a, gh, H, per_temperature;
  __device__ __forceinline__ float plain(float z) const {       // times temperature
    const float d = fmaxf((z - m) * c, -256.f);                 // p = 0 from there on; masked entries times gh stay finite
    const float p = fast_exp2(d) * per_s;
    return -p * fmaf(gh, fmaf(d, kLn2, H - log_s), a);
  }
};

// A workgroup per piece of a row.  What bounds it is the read of z and the write of dz, PAST the caches where they exceed them:
// 8,192 rows (7,168 of them scored) of V = 151,936 bf16 915 us, 5.1 TB/s; 777 x 32,771 fp32 34 us, 5.6 TB/s.  kStep of 2 or 8: 932, 918 us.
template <typename TI, typename TO, bool PAST>
__global__ __launch_bounds__(kThreads) void token_logp_grad_kernel(LogpGradArgs a) {
  constexpr int N = Entry<TI>::kPerVec;
  __shared__ float at_id[ADWIN_MAX_GIVEN], g_of[ADWIN_MAX_GIVEN];
  __shared__ int id_of[ADWIN_MAX_GIVEN];
  const int64_t r = blockIdx.x / (uint32_t)a.pieces;
  const int piece = (int)(blockIdx.x - (uint32_t)r * (uint32_t)a.pieces);
  const int tid = threadIdx.x;
  bool live = row_ids(a.ids, a.G, a.V, r).live;
  const float s = live ? a.norm[2 * r + 1] : 0.f;
  live = live && s > 0.f;
  TO* out = (TO*)a.dz + r * a.ld_dz;
  const Piece<TI> p((const TI*)a.z + r * a.ld_z, a.V, piece, a.pieces);
  constexpr int kWhole = N * sizeof(TO) < 16 ? N * (int)sizeof(TO) : 16;
  const bool whole = ((uintptr_t)(out + p.row.head) & (kWhole - 1)) == 0;
  const int steps = (p.v1 - p.v0) / (kStep * kThreads);
  if (!live) {
    float y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = 0.f;
    if (tid < p.edge) Entry<TO>::put(out + p.row.edge_index(tid), 0.f);
    for (int i = p.v0 + tid; i < p.v1; i += kThreads) put_entries<PAST>(out + p.row.index(i), y, whole);
    return;
  }
  uint4 v[kStep];
  int i0 = p.v0;
  auto load = [&](int u) { v[u] = p.row.template vec<PAST>(i0 + tid + kThreads * u); };
  if (steps > 0) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) load(u);
  }
  const float edge = tid < p.edge ? Entry<TI>::one(p.row.p + p.row.edge_index(tid)) : 0.f;
  if (tid < a.G) {
    const int id = a.ids[r * a.G + tid];
    const bool in = id >= 0 && id < a.V;
    id_of[tid] = in ? id : -1;
    g_of[tid] = in ? a.g_logp[r * a.G + tid] : 0.f;
    at_id[tid] = in ? Entry<TI>::one(p.row.p + id) : 0.f;
  }
  __syncthreads();
  GradRow g{};
  g.m = a.norm[2 * r]; g.c = a.c; g.per_s = 1.f / s; g.log_s = logf(s); g.per_temperature = a.per_temperature;
  g.gh = a.g_entropy ? a.g_entropy[r] : 0.f;
  g.H = a.g_entropy ? a.entropy[r] : 0.f;
  for (int j = 0; j < a.G; ++j) g.a += g_of[j];
  auto put = [&](int u, int first) {
    float x[N];
    Entry<TI>::unpack(v[u], x);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = g.plain(x[e]) * g.per_temperature;
    put_entries<PAST>(out + first + kThreads * N * u, x, whole);
  };
  if (tid < p.edge) Entry<TO>::put(out + p.row.edge_index(tid), g.plain(edge) * g.per_temperature);
  for (int step = 1; step < steps; ++step) {
    const int first = p.row.index(i0 + tid);
    i0 += kStep * kThreads;
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      put(u, first);
      load(u);
    }
  }
  if (steps > 0) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) put(u, p.row.index(i0 + tid));
    i0 += kStep * kThreads;
  }
  for (; i0 < p.v1; i0 += kThreads)
    if (i0 + tid < p.v1) {
      load(0);
      put(0, p.row.index(i0 + tid));
    }
  __syncthreads();                               // the piece's stores come before those of the given tokens
  if (tid < a.G && id_of[tid] >= 0) {
    const int id = id_of[tid];
    const bool in_edge = id < p.row.head || id >= p.row.index(p.row.vecs);
    const bool mine = in_edge ? piece == 0 : id >= p.row.index(p.v0) && id < p.row.index(p.v1);
    bool first = mine;
    for (int j = 0; j < tid; ++j) first = first && id_of[j] != id;
    if (first) {
      float sum = 0.f;
      for (int j = tid; j < a.G; ++j) sum += id_of[j] == id ? g_of[j] : 0.f;
      Entry<TO>::put(out + id, (sum + g.plain(at_id[tid])) * g.per_temperature);
    }
  }
}

// Pieces of a row, for 4,096 workgroups in a call, each with a step of its threads or more.
static int grad_pieces(int64_t T, int32_t V, int32_t dtype) {
  const int64_t step = (int64_t)kStep * kThreads * (dtype == ADWIN_DT_BF16 ? 8 : 4);
  int64_t n = (4096 + T - 1) / T;
  if (n > V / step) n = V / step;
  return (int)(n < 1 ? 1 : n);
}

// Whether an array of T x V is read (or written) past the caches: it is beyond the last-level cache of 256 MiB, so it has left
// before anybody can find it there.  us, kept / past, bf16, V = 151,936: logp with 20 alternatives 600 rows 54.1 / 52.8 (kept, for the
// gradient that reads the same logits), 1,300 rows 95 / 91, 8,192 rows 441 / 412; gradient 900 rows 115 / 116, 1,300 rows
// 168 / 164, 2,000 rows 250 / 256, 8,192 rows 1006 / 962; from fp32 to bf16 600 rows 112 / 114, 1,300 rows 240 / 229, 4,000 rows 713 / 689; to fp32
// from bf16 900 rows 194 / 188, 4,000 rows 813 / 792, from fp32 2,000 rows 501 / 518, 4,000 rows 954 / 930.
static bool past_caches(int64_t T, int32_t V, int32_t dtype) {
  return T * V * (dtype == ADWIN_DT_BF16 ? 2 : 4) > ((int64_t)320 << 20);
}

static bool known_temperature(float t) { return t >= 1.17549435e-38f && t <= 3.0e38f; }

static int check_logp(const adwin_opd_logp_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->z_dtype) || !known_temperature(p->temperature)) return ADWIN_E_MODE;
  if (p->T < 0 || p->T >= kMaxRows || p->V < 1 || p->V > kMaxVocab || p->ld_z < p->V || p->G < 0 || p->G > ADWIN_MAX_GIVEN ||
      p->top < 0 || p->top > ADWIN_MAX_TOP)
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

static int check_logp_grad(const adwin_opd_logp_grad_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->z_dtype) || !known_dtype(p->dz_dtype) ||
      !known_temperature(p->temperature))
    return ADWIN_E_MODE;
  if (p->T < 0 || p->T >= kMaxRows || p->V < 1 || p->V > kMaxVocab || p->ld_z < p->V || p->ld_dz < p->V || p->G < 0 ||
      p->G > ADWIN_MAX_GIVEN)
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

}  // namespace adwin

using namespace adwin;

extern "C" int adwin_opd_token_logp_workspace_bytes(const adwin_opd_logp_problem* p, size_t* bytes) {
  if (!bytes) return ADWIN_E_NULL;
  const int st = check_logp(p);
  if (st != ADWIN_OK) return st;
  *bytes = LogpLayout(p).bytes;
  return ADWIN_OK;
}

extern "C" int adwin_opd_token_logp(const adwin_opd_logp_problem* p, void* workspace, size_t workspace_bytes,
                                    void* hip_stream) {
  const int st = check_logp(p);
  if (st != ADWIN_OK) return st;
  if (p->T == 0) return ADWIN_OK;
  if (!p->z || (p->G > 0 && !p->ids)) return ADWIN_E_NULL;
  if ((uintptr_t)p->z & entry_mask(p->z_dtype)) return ADWIN_E_ALIGN;
  const LogpLayout L(p);
  if (L.bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < L.bytes)) return ADWIN_E_WORKSPACE;
  LogpArgs a{};
  a.z = p->z; a.ld = p->ld_z; a.T = p->T; a.V = p->V; a.G = p->G; a.top = p->top;
  a.temperature = p->temperature; a.c = (float)(1.4426950408889634 / (double)p->temperature);
  a.ids = p->ids; a.logp = p->logp; a.entropy = p->entropy; a.norm = p->norm; a.top_ids = p->top_ids;
  a.top_logp = p->top_logp; a.row_status = p->row_status;
  if (!a.top_ids && !a.top_logp) a.top = 0;
  a.pieces = L.pieces; a.part = (float*)workspace; a.keys = (uint64_t*)((unsigned char*)workspace + L.o_keys);
  hipStream_t stream = (hipStream_t)hip_stream;
  const unsigned blocks = (unsigned)(p->T * L.pieces);
  const bool past = past_caches(p->T, p->V, p->z_dtype);
  if (p->z_dtype == ADWIN_DT_BF16) {
    if (past) token_logp_kernel<uint16_t, true><<<blocks, kThreads, 0, stream>>>(a);
    else token_logp_kernel<uint16_t, false><<<blocks, kThreads, 0, stream>>>(a);
  } else {
    if (past) token_logp_kernel<float, true><<<blocks, kThreads, 0, stream>>>(a);
    else token_logp_kernel<float, false><<<blocks, kThreads, 0, stream>>>(a);
  }
  ADWIN_HIP_TRY(hipGetLastError());
  if (L.pieces > 1) {
    if (p->z_dtype == ADWIN_DT_BF16) join_logp_kernel<uint16_t><<<(unsigned)p->T, kThreads, 0, stream>>>(a);
    else join_logp_kernel<float><<<(unsigned)p->T, kThreads, 0, stream>>>(a);
    ADWIN_HIP_TRY(hipGetLastError());
  }
  return ADWIN_OK;
}

extern "C" int adwin_opd_token_logp_grad(const adwin_opd_logp_grad_problem* p, void* hip_stream) {
  const int st = check_logp_grad(p);
  if (st != ADWIN_OK) return st;
  if (p->T == 0) return ADWIN_OK;
  if (!p->z || !p->dz || !p->norm || (p->G > 0 && (!p->ids || !p->g_logp)) || (p->g_entropy && !p->entropy))
    return ADWIN_E_NULL;
  if (((uintptr_t)p->z & entry_mask(p->z_dtype)) || ((uintptr_t)p->dz & entry_mask(p->dz_dtype))) return ADWIN_E_ALIGN;
  LogpGradArgs a{};
  a.z = p->z; a.ld_z = p->ld_z; a.dz = p->dz; a.ld_dz = p->ld_dz; a.T = p->T; a.V = p->V; a.G = p->G;
  a.c = (float)(1.4426950408889634 / (double)p->temperature); a.per_temperature = 1.f / p->temperature;
  a.ids = p->ids; a.norm = p->norm; a.g_logp = p->g_logp; a.entropy = p->entropy; a.g_entropy = p->g_entropy;
  hipStream_t stream = (hipStream_t)hip_stream;
  a.pieces = grad_pieces(p->T, p->V, p->z_dtype);
  const bool in16 = p->z_dtype == ADWIN_DT_BF16, out16 = p->dz_dtype == ADWIN_DT_BF16;
  const bool past = past_caches(p->T, p->V, p->z_dtype) || past_caches(p->T, p->V, p->dz_dtype);
  const unsigned blocks = (unsigned)(p->T * a.pieces);
#define ADWIN_LAUNCH(...) token_logp_grad_kernel<__VA_ARGS__><<<blocks, kThreads, 0, stream>>>(a)
#define ADWIN_LAUNCH_TYPES(PAST)                              \
  if (in16 && out16) ADWIN_LAUNCH(uint16_t, uint16_t, PAST);  \
  else if (in16) ADWIN_LAUNCH(uint16_t, float, PAST);         \
  else if (out16) ADWIN_LAUNCH(float, uint16_t, PAST);        \
  else ADWIN_LAUNCH(float, float, PAST);
  if (past) { ADWIN_LAUNCH_TYPES(true) } else { ADWIN_LAUNCH_TYPES(false) }
#undef ADWIN_LAUNCH_TYPES
#undef ADWIN_LAUNCH
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}
