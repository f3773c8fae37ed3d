// Decoding by beams: the best continuations of every sequence, and what beams carry with them moved to where these are.
#include <math.h>

#include "select_shared.h"

namespace adwin {

// ---------------------------------------------------------------------------------------
// Selection.  A beam's candidate j has the total  score + (z_j - m) / temperature - log s,  s = sum_i e^((z_i - m) / temperature).
// Which of two beams' candidates is better may hang on any digit, so s is held in fp64: exponentials are fp32, relative to a
// thread's own whole-number reference r, 2^(z c - r) with c = log2(e) / temperature in two parts (a rounded c alone puts 6e-7 into the log s
// of flat rows), the terms of 16 bytes are summed in fp32 and these sums in fp64.
// ---------------------------------------------------------------------------------------
struct BeamPart { double s, base, m; };    // sum of the piece's exponentials relative to e^base, its largest logit
struct BeamArgs {
  const void* z; int64_t ld; int64_t rows, B;
  int32_t K, keep, V, pieces, end;
  float c, c_low;                          // c_low > 0: a masked entry stays -inf in both parts
  double per_temperature, power;
  const float* score; const int32_t* finished; const int32_t* length;
  BeamPart* part;                          // [rows][pieces]
  uint64_t* keys;                          // [rows][pieces][keep]
  int32_t* parent; int32_t* token; float* new_score; int32_t* new_finished; int32_t* new_length; int32_t* row_status;
};

// whether a beam goes on, so that its logits are read
__device__ __forceinline__ bool goes_on(const BeamArgs& a, int64_t row) {
  return fabsf(a.score[row]) < INFINITY && !(a.finished && a.finished[row]);
}

// A product that no sum takes in unrounded.
__device__ __forceinline__ double rounded(double x, double y) {
  double p = x * y;
  asm volatile("" : "+v"(p));
  return p;
}

// A row in vectors from its first entry on, and up to a vector's entries behind them.  Which entries are added to one another follows from
// their indices alone, never from where the row begins: beams of the same logits have the same log s, to the last bit, and rank by rising
// beam.  A vector may begin at any address that suits its entries.  Against vectors from the first multiple of 16 bytes on, whose sums went by
// the address, us: rows at multiples of 4 bytes the same (1,536 x 151,934 bf16 91 / 91, 768 x 151,935 fp32 85 / 85); bf16 rows at odd entries
// 54 / 52 where the caches hold them (768 x 151,935), 108 / 90 where they do not (1,536 rows).
template <typename T> struct Loose;
template <> struct Loose<uint16_t> { typedef u32x4 Vec __attribute__((aligned(2))); };
template <> struct Loose<float> { typedef u32x4 Vec __attribute__((aligned(4))); };
template <typename T>
struct BeamRow {
  static constexpr int kPer = Entry<T>::kPerVec;
  const T* p;
  int vecs, edge;
  __device__ __forceinline__ BeamRow(const T* row, int entries) : p(row), vecs(entries / kPer), edge(entries % kPer) {}
  __device__ __forceinline__ int edge_index(int e) const { return vecs * kPer + e; }
  template <bool PAST = false>
  __device__ __forceinline__ uint4 vec(int i) const {
    const typename Loose<T>::Vec* q = (const typename Loose<T>::Vec*)(p + (int64_t)i * kPer);
    u32x4 v;
    if constexpr (PAST) v = __builtin_nontemporal_load(q);
    else v = *q;
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ int index(int i) const { return i * kPer; }
};
template <typename T> using BeamSpan = Piece<T, BeamRow<T>>;

struct BeamSums { float r, m; double s; };
constexpr float kFarRef = -16777216.f;     // the least reference: whole numbers next to some z c are good to a half up to here
constexpr float kLeast = 1e-22f;            // the least c whose second part is a normal number
constexpr float kRise = 4.f;               // z c - r may reach this before the reference moves

__device__ __forceinline__ void beam_move(BeamSums& a, float r) {
  a.s *= (double)fast_exp2(a.r - r);       // a power of two
  a.r = r;
}
template <int N>
__device__ __forceinline__ float beam_add(BeamSums& a, const float (&x)[N], float c, float c_low) {
  float m = x[0];
  if constexpr (N > 1) m = max3(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i + 1 < N; i += 2) m = max3(m, x[i], x[i + 1]);
  if constexpr (N > 1) m = max3(m, x[N - 1], x[N - 1]);
  a.m = max3(a.m, m, m);
  if (__builtin_expect(__any(m * c > a.r + kRise), 0)) {      // a branch of the wave, or its exponential and product in 64 bits come with every vector
    if (m * c > a.r + kRise) beam_move(a, ceilf(m * c));
  }
  float e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = fast_exp2(fmaf(x[i], c_low, fmaf(x[i], c, -a.r)));
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) e[i] += e[i + n];
  a.s += (double)e[0];
  return m;
}

// The workgroup's sum, relative to e^base.  Where references do not hold (logits or 1 / temperature of millions, rows at a
// mask's finite value), or c has no second part (its digits there would lie below 2^-126), the piece is read again, differences first.
template <typename T>
__device__ __forceinline__ BeamPart beam_piece(const BeamSpan<T>& p, BeamSums a, const BeamArgs& g, float (*top)[2], double* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float r = wave_max(a.r), m = wave_max(a.m);
  if (lane == 0) { top[wave][0] = r; top[wave][1] = m; }
  __syncthreads();
  float R = top[0][0], M = top[0][1];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) { R = fmaxf(R, top[w][0]); M = fmaxf(M, top[w][1]); }
  const bool far = (fabsf(M * g.c) > -kFarRef || g.c < kLeast) && fabsf(M) < INFINITY;
  double s = 0, base = (double)R * 0.69314718055994530942;
  if (!far) {
    beam_move(a, R);
    s = a.s;
  } else {
    base = rounded((double)M, g.per_temperature);        // the join takes the same product from it
    auto add = [&](float z) { s += (double)fast_exp2((float)(((double)z - (double)M) * g.per_temperature * 1.4426950408889634)); };
    if ((int)threadIdx.x < p.edge) add(Entry<T>::one(p.row.p + p.row.edge_index(threadIdx.x)));
    for (int i = p.v0 + threadIdx.x; i < p.v1; i += kThreads) {
      float x[Entry<T>::kPerVec];
      Entry<T>::unpack(p.row.vec(i), x);
#pragma unroll
      for (int e = 0; e < Entry<T>::kPerVec; ++e) add(x[e]);
    }
  }
  s = wave_sum(s);
  if (lane == 0) sums[wave] = s;
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += sums[w];
  return {s, base, (double)M};
}

// One pass over a piece of a row, kBeamStep vectors to a thread at a time; the `keep` largest logits ride on the maxima of the threads,
// as in the log-probabilities of given tokens.
constexpr int kBeamStep = 4;
template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads, 6) void beam_rows_kernel(BeamArgs a) {
  constexpr int N = Entry<T>::kPerVec;
  __shared__ Select l;
  __shared__ float top[kWaves][2];
  __shared__ double sums[kWaves];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x / (uint32_t)a.pieces;
  const int piece = (int)(blockIdx.x - (uint32_t)row * (uint32_t)a.pieces);
  if (!goes_on(a, row)) return;                      // the join sees that by itself
  const BeamSpan<T> p((const T*)a.z + row * a.ld, a.V, piece, a.pieces);
  const int last = p.v1 - tid;                       // a thread's vectors: p.v0 + tid + 256 k below p.v1
  // whole steps, whose loads stand in no branch: the wait for a vector then leaves the younger ones in flight
  const int whole = (p.v1 - p.v0) / (kBeamStep * kThreads);
  int i0 = p.v0;
  uint4 v[kBeamStep];
  auto load = [&](int u) { v[u] = p.row.template vec<PAST>(i0 + tid + kThreads * u); };
  auto load_any = [&](int u) {
    v[u] = Entry<T>::none();
    if (i0 + kThreads * u < last) load(u);
  };
  if (whole > 0) {
#pragma unroll
    for (int u = 0; u < kBeamStep; ++u) load(u);
  } else {
#pragma unroll
    for (int u = 0; u < kBeamStep; ++u) load_any(u);
  }
  BeamSums sum = {kFarRef, -INFINITY, 0.0};
  int listed = 0;                                    // keys of this wave
  float edge[1] = {-INFINITY};
  if (tid < p.edge) edge[0] = Entry<T>::one(p.row.p + p.row.edge_index(tid));
  auto add = [&](int u) {
    float x[N];
    Entry<T>::unpack(v[u], x);
    return beam_add(sum, x, a.c, a.c_low);
  };
  if (tid < p.edge) beam_add(sum, edge, a.c, a.c_low);
  // the first vectors, which give the first bound and are then gone through again
#pragma unroll
  for (int u = 0; u < kBeamStep; ++u) add(u);
  const int quarter = (a.keep + kWaves - 1) / kWaves;
  auto take_bound = [&](bool all) {                  // a thread without entries: -inf; `all`: for the exact bound too
    const uint32_t most = order_bits(sum.m) >> 16, at = lanes_bound(most, quarter);
    if (all) l.most[tid] = most;
    if ((tid & 63) == 0) *(volatile uint32_t*)&l.bounds[tid >> 6] = at;
  };
  take_bound(true);
  __syncthreads();
  float bound = bound_value(some_bound(l, a.keep));
  list_entry(l, listed, tid < p.edge && edge[0] >= bound, edge[0], tid < p.edge ? p.row.edge_index(tid) : 0);
#pragma unroll
  for (int u = 0; u < kBeamStep; ++u)
    list_entries<T>(l, listed, i0 + kThreads * u < last, v[u], p.row.index(i0 + tid + kThreads * u), bound);
  i0 += kBeamStep * kThreads;
  if (whole > 1) {
#pragma unroll
    for (int u = 0; u < kBeamStep; ++u) load(u);
  }
  for (int step = 1; step < whole; ++step) {
    if ((step & (step - 1)) == 0) {                  // an older bound of another wave is a bound as well: nobody waits
      take_bound(false);
      bound = fmaxf(bound, bound_value(least_bound(l.bounds)));
    }
    const int first = p.row.index(i0 + tid);
    i0 += kBeamStep * kThreads;
    if (step + 1 < whole) {
#pragma unroll
      for (int u = 0; u < kBeamStep; ++u) {
        if (__any(add(u) >= bound)) list_entries<T>(l, listed, true, v[u], first + kThreads * N * u, bound);
        load(u);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kBeamStep; ++u)
        if (__any(add(u) >= bound)) list_entries<T>(l, listed, true, v[u], first + kThreads * N * u, bound);
    }
  }
  if (whole > 0) {
#pragma unroll
    for (int u = 0; u < kBeamStep; ++u) load_any(u);
#pragma unroll
    for (int u = 0; u < kBeamStep; ++u) {
      if (__any(i0 + kThreads * u < last) && __any(add(u) >= bound))
        list_entries<T>(l, listed, i0 + kThreads * u < last, v[u], p.row.index(i0 + tid + kThreads * u), bound);
    }
    take_bound(true);
  }
  if (!select_found(l, listed, a.keep, p.edge + (p.v1 - p.v0) * N, whole > 0)) select_slowly(p, a.keep, l);
  const BeamPart part = beam_piece(p, sum, a, top, sums);
  if (tid == 0) a.part[blockIdx.x] = part;
  if (tid < a.keep) a.keys[(int64_t)blockIdx.x * a.keep + tid] = l.kept[tid];
}

// One 64-bit word per rank, in the order of the numbers; 0 is none.
__device__ __forceinline__ uint64_t rank_bits(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}

// A sequence's candidates, of all its beams and pieces: the `keep` best.  A lower bound of the keep-th best is the keep-th largest of the
// threads' own best ones; what reaches it is listed and ranked by counting.  Where more does than can be listed (ties), the best
// is looked for `keep` times.
struct Candidate { uint64_t rank, key; int32_t beam; };
__device__ __forceinline__ bool better(uint64_t rank, uint64_t key, int beam, const Candidate& b) {
  return rank > b.rank || (rank == b.rank && (beam < b.beam || (beam == b.beam && key > b.key)));
}
constexpr int kListed = 512;
constexpr int kMine = 8;                             // keys of a thread that are kept
constexpr uint64_t kStands = ~0ull;                  // the key of a beam that stands as it is

__global__ __launch_bounds__(kThreads) void beam_join_kernel(BeamArgs a) {
  __shared__ Candidate list[kListed];
  __shared__ Candidate won[ADWIN_MAX_BEAMS];
  __shared__ Candidate of_wave[kWaves];
  __shared__ double base[ADWIN_MAX_BEAMS], top[ADWIN_MAX_BEAMS];    // score - log sum_i e^((z_i - top) / temperature), the largest logit
  __shared__ double per[ADWIN_MAX_BEAMS];                           // the length's power
  __shared__ int state[ADWIN_MAX_BEAMS], steps[ADWIN_MAX_BEAMS];    // 0: no candidates, 1: goes on, 2: stands
  __shared__ uint32_t most[kThreads];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.x, row0 = b * a.K;
  const int per_beam = a.pieces * a.keep, n = a.K * per_beam;
  const uint64_t* keys = a.keys + row0 * per_beam;
  // A thread's first keys and a wave's first sums are asked for at once, before anything says which of them count.
  uint64_t mine[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u)
    if (kThreads * u < n) mine[u] = keys[kThreads * u + tid < n ? kThreads * u + tid : n - 1];
  const int64_t row = row0 + (tid < a.K ? tid : 0);
  const float score = a.score[row];
  const bool stands = a.finished && a.finished[row];
  const int length = a.length ? a.length[row] : 0;
  // sums of the beams' pieces relative to the largest logit (totals of the likeliest candidates then have no terms larger than need be):
  // every wave the beams in turn, a piece to a lane (those of beams that do not go on are anything)
  for (int k = wave; k < a.K; k += kWaves) {
    const BeamPart q = a.part[(row0 + k) * a.pieces + (lane < a.pieces ? lane : 0)];
    double m = lane < a.pieces ? q.m : -INFINITY;
    if (a.pieces > 1) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
    }
    double s = lane < a.pieces && q.s != 0 ? q.s * exp(q.base - rounded(m, a.per_temperature)) : 0;     // a NaN stays one
    if (a.pieces > 1) s = wave_sum(s);
    if (lane == 0) { top[k] = m; per[k] = s; }
  }
  __syncthreads();
  if (tid < a.K) {                                   // a beam to a thread
    const bool on = fabsf(score) < INFINITY && !stands;
    const double s = per[tid];
    const bool fine = fabsf(score) < INFINITY && (!on || (s > 0 && s < INFINITY));
    const int len = on ? length + 1 : length, divisor = len > 1 ? len : 1;
    base[tid] = on ? (double)score - log(s) : (double)score;
    per[tid] = a.power == 0 ? 1.0 : a.power == 1 ? (double)divisor : pow((double)divisor, a.power);
    steps[tid] = len;
    state[tid] = !fine ? 0 : stands ? 2 : 1;
    if (a.row_status) a.row_status[row] = fine || score == -INFINITY ? 0 : (int)ADWIN_DEV_NONFINITE;
  }
  if (tid == 0) count = 0;
  __syncthreads();
  // candidate i: its rank, 0 for none
  auto rank_of = [&](int i, int* beam, uint64_t* key) __attribute__((always_inline)) -> uint64_t {
    const int k = i / per_beam;
    *beam = k;
    double total;
    if (state[k] == 1) {
      const float z = key_value(*key);
      if (*key == 0 || z == -INFINITY) return 0;
      total = fma((double)z - top[k], a.per_temperature, base[k]);
    } else {
      *key = kStands;
      if (state[k] == 0 || i != k * per_beam) return 0;
      total = base[k];
    }
    return rank_bits(a.power == 0 ? total : total / per[k]);
  };
  auto candidate = [&](int i, int* beam, uint64_t* key) __attribute__((always_inline)) -> uint64_t {
    *key = keys[i];
    return rank_of(i, beam, key);
  };
  uint64_t rank[kMine], best_here = 0;
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    rank[u] = 0;
    const int i = kThreads * u + tid;
    if (kThreads * u < n && i < n) {
      int beam;
      rank[u] = rank_of(i, &beam, &mine[u]);
      best_here = rank[u] > best_here ? rank[u] : best_here;
    }
  }
  for (int i = kThreads * kMine + tid; i < n; i += kThreads) {
    int beam; uint64_t key;
    const uint64_t r = candidate(i, &beam, &key);
    best_here = r > best_here ? r : best_here;
  }
  most[tid] = (uint32_t)(best_here >> 32);
  __syncthreads();
  uint32_t at = 0;                                   // every wave by itself: the keep-th largest of the 256, or less where that says as much
  {
    uint32_t v[kWaves], all = 0, any = ~0u;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v[w] = most[64 * w + lane];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { all |= v[w]; any &= v[w]; }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { all |= __shfl_xor(all, o, 64); any &= __shfl_xor(any, o, 64); }
    const int first = all == any ? -1 : 31 - __clz(all ^ any);        // bits above are the same in all
    at = first < 0 ? any : first == 31 ? 0 : any >> (first + 1) << (first + 1);
    for (int bit = first; bit >= 0; --bit) {
      const uint32_t t = at | (1u << bit);
      int reach = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) reach += __popcll(__ballot(v[w] >= t));
      if (reach >= a.keep) at = t;
      if (reach == a.keep) break;
    }
  }
  auto enter = [&](uint64_t r, uint64_t key, int beam) __attribute__((always_inline)) {
    if (r && (uint32_t)(r >> 32) >= at) {
      const int q = atomicAdd(&count, 1);
      if (q < kListed) list[q] = {r, key, beam};
    }
  };
#pragma unroll
  for (int u = 0; u < kMine; ++u)
    if (kThreads * u < n) enter(rank[u], mine[u], (kThreads * u + tid) / per_beam);
  for (int i = kThreads * kMine + tid; i < n; i += kThreads) {
    int beam; uint64_t key;
    const uint64_t r = candidate(i, &beam, &key);
    enter(r, key, beam);
  }
  __syncthreads();
  int have = count;
  if (have <= kListed) {
    for (int q = tid; q < have; q += kThreads) {
      const Candidate mine = list[q];
      int r = 0;
      for (int j = 0; j < have; ++j) r += better(list[j].rank, list[j].key, list[j].beam, mine);
      if (r < a.keep) won[r] = mine;
    }
    have = have < a.keep ? have : a.keep;
    __syncthreads();
  } else {
    Candidate before = {~0ull, ~0ull, -1};
    have = 0;
    for (int r = 0; r < a.keep; ++r) {
      Candidate best = {0, 0, 0};
      for (int i = tid; i < n; i += kThreads) {
        int beam; uint64_t key;
        const uint64_t rank = candidate(i, &beam, &key);
        if (rank && better(before.rank, before.key, before.beam, {rank, key, beam}) &&
            (best.rank == 0 || better(rank, key, beam, best)))
          best = {rank, key, beam};
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const Candidate q = {(uint64_t)__shfl_xor((unsigned long long)best.rank, o, 64), (uint64_t)__shfl_xor((unsigned long long)best.key, o, 64),
                             __shfl_xor(best.beam, o, 64)};
        if (q.rank && (best.rank == 0 || better(q.rank, q.key, q.beam, best))) best = q;
      }
      if (lane == 0) of_wave[wave] = best;
      __syncthreads();
      best = of_wave[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        const Candidate q = of_wave[w];
        if (q.rank && (best.rank == 0 || better(q.rank, q.key, q.beam, best))) best = q;
      }
      __syncthreads();
      if (best.rank == 0) break;
      if (tid == 0) won[r] = best;
      before = best;
      ++have;
    }
    __syncthreads();
  }
  if (tid < a.keep) {
    const int64_t out = b * a.keep + tid;
    int parent = -1, token = -1, done = 0, len = 0;
    float score = -INFINITY;
    if (tid < have) {
      const Candidate w = won[tid];
      const int k = w.beam;
      parent = k;
      len = steps[k];
      if (state[k] == 2) {
        token = a.end; done = 1; score = (float)base[k];
      } else {
        token = key_index(w.key);
        done = a.end >= 0 && token == a.end;
        score = (float)fma((double)key_value(w.key) - top[k], a.per_temperature, base[k]);
      }
    }
    a.parent[out] = parent;
    a.token[out] = token;
    if (a.new_score) a.new_score[out] = score;
    if (a.new_finished) a.new_finished[out] = done;
    if (a.new_length) a.new_length[out] = len;
  }
}

// ---------------------------------------------------------------------------------------
// Moving states.  A thread has the same V bytes of all rows of a sequence: it loads what moves before it stores anything, which makes a
// move in place safe without a second buffer, and a parent of several beams comes from memory once.
// ---------------------------------------------------------------------------------------
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
struct MoveState { const char* from; char* to; int64_t from_row, to_row, from_plane, to_plane, positions, bytes; int32_t planes, in_place; };
constexpr int kMoved = 40;                           // arrays of a launch: what its arguments hold
struct MoveArgs {
  int64_t B;
  int32_t K, keep, n;
  const int32_t* parent; const int32_t* length;
  MoveState s[kMoved];
};

// A workgroup to 256 pieces of V bytes of a plane, an array and a sequence.  The arguments lie in host memory, microseconds away: what a
// workgroup needs of them is one array's, whose place follows from the workgroup's own, and is asked for at once.
template <typename V, int MOST, bool PAST>
__global__ __launch_bounds__(256) void beam_move_kernel(MoveArgs a) {
  const int lane = threadIdx.x & 63;
  const MoveState s = a.s[blockIdx.y];
  constexpr int64_t kChunk = 256 * (int64_t)sizeof(V);
  for (int64_t b = blockIdx.z; b < a.B; b += gridDim.z) {
    const int32_t mine = lane < a.keep ? a.parent[b * a.keep + lane] : -1;
    int64_t len = a.length ? a.length[b] : s.positions;
    len = len < 0 ? 0 : len < s.positions ? len : s.positions;
    const int64_t live = len * s.bytes, chunks = (live + kChunk - 1) / kChunk;
    for (int64_t i = blockIdx.x; i < s.planes * chunks; i += gridDim.x) {
      const int64_t plane = s.planes == 1 ? 0 : s.planes * chunks < ((int64_t)1 << 31) ? (int64_t)((uint32_t)i / (uint32_t)chunks) : i / chunks;
      const int64_t chunk = (i - plane * chunks) * kChunk;
      const int64_t at = chunk + threadIdx.x * sizeof(V);
      const char* from = s.from + b * a.K * s.from_row + plane * s.from_plane + at;
      char* to = s.to + b * a.keep * s.to_row + plane * s.to_plane + at;
      int64_t to_row = s.to_row;
      asm volatile("" : "+s"(to_row));                 // (nor do 64 rows' offsets)
      auto parent_of = [&](int j) __attribute__((always_inline)) {      // read anew each time: 64 of them do not fit the scalar registers
        int m = mine;
        asm volatile("" : "+v"(m));
        return __builtin_amdgcn_readlane(m, j);
      };
      auto moves = [&](int j, int k) __attribute__((always_inline)) { return k >= 0 && k < a.K && !(s.in_place && k == j); };
      V v[MOST];
      const bool whole = at + (int64_t)sizeof(V) <= live;
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        const int k = parent_of(j);
        if (moves(j, k) && whole) {
          if constexpr (PAST) v[j] = __builtin_nontemporal_load((const V*)(from + k * s.from_row));
          else v[j] = *(const V*)(from + k * s.from_row);
        }
      }
      int64_t row = 0;
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        const int k = parent_of(j);
        if (moves(j, k) && whole) {
          if constexpr (PAST) __builtin_nontemporal_store(v[j], (V*)(to + row));
          else *(V*)(to + row) = v[j];
        }
        row += to_row;
      }
      if constexpr (sizeof(V) > 1) {                   // bytes behind the last whole V, one to a thread
        const int64_t end = live / (int64_t)sizeof(V) * (int64_t)sizeof(V);
        if (end < live && chunk <= end && end < chunk + kChunk) {
          const bool in = threadIdx.x < live - end;
          const int64_t o = end + threadIdx.x - at;
          uint8_t w[MOST];
#pragma unroll
          for (int j = 0; j < MOST; ++j) {
            const int k = parent_of(j);
            if (moves(j, k) && in) w[j] = *(const uint8_t*)(from + k * s.from_row + o);
          }
          row = o;
#pragma unroll
          for (int j = 0; j < MOST; ++j) {
            const int k = parent_of(j);
            if (moves(j, k) && in) *(uint8_t*)(to + row) = w[j];
            row += to_row;
          }
        }
      }
    }
  }
}

// ---- host -----------------------------------------------------------------------------
// Pieces of a row, as the log-probabilities of given tokens have them: one for calls of 256 rows or more, fewer rows in as many as
// give every compute unit a workgroup with half a step of its threads.
constexpr int kBeamPieces = 64;
static int beam_pieces(int64_t rows, int32_t V, int32_t dtype) {
  const int64_t step = (int64_t)kBeamStep * kThreads * (dtype == ADWIN_DT_BF16 ? 8 : 4) / 2;
  int64_t n = (256 + rows - 1) / (rows > 0 ? rows : 1);
  if (n > V / step) n = V / step;
  return (int)(n < 1 ? 1 : n > kBeamPieces ? kBeamPieces : n);
}

static int check_select(const adwin_opd_beam_select_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->z_dtype) || !(p->temperature >= 1.17549435e-38f && p->temperature <= 3.0e38f) ||
      !(p->length_power >= 0.f && p->length_power <= 8.f))
    return ADWIN_E_MODE;
  if (p->B < 0 || p->K < 1 || p->K > ADWIN_MAX_BEAMS || p->keep < 1 || p->keep > ADWIN_MAX_BEAMS || p->B >= kMaxRows ||
      p->B * p->K >= kMaxRows || p->V < 1 || p->V > kMaxVocab || p->ld_z < p->V || p->end >= p->V)
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

// What a call writes may overlap nothing else that it reads or writes: other sequences may still be read.  With keep = K new scores, ends and
// lengths may go where the old ones are, as a sequence's are read before its own are written.
static bool selects_apart(const adwin_opd_beam_select_problem* p, const void* workspace, size_t workspace_bytes) {
  const int64_t beams = 4 * p->B * p->K, kept = 4 * p->B * p->keep, size = p->z_dtype == ADWIN_DT_BF16 ? 2 : 4;
  struct Array { const void* at; int64_t bytes; const void* in_place; };
  const Array written[] = {{p->parent, kept, nullptr}, {p->token, kept, nullptr}, {p->new_score, kept, p->score}, {p->new_finished, kept, p->finished},
                           {p->new_length, kept, p->length}, {p->row_status, beams, nullptr}, {workspace, (int64_t)workspace_bytes, nullptr}};
  const Array read[] = {{p->z, ((p->B * p->K - 1) * p->ld_z + p->V) * size, nullptr}, {p->score, beams, nullptr}, {p->finished, beams, nullptr},
                        {p->length, beams, nullptr}};
  auto meet = [](const Array& a, const Array& b) {
    return a.at && b.at && (const char*)a.at < (const char*)b.at + b.bytes && (const char*)b.at < (const char*)a.at + a.bytes;
  };
  for (const Array& w : written) {
    for (const Array& r : read)
      if (meet(w, r) && !(p->keep == p->K && w.at == r.at && w.in_place == r.at)) return false;
    for (const Array* o = written; o != &w; ++o)
      if (meet(w, *o)) return false;
  }
  return true;
}

struct BeamLayout {
  int pieces;
  size_t o_keys, bytes;
  explicit BeamLayout(const adwin_opd_beam_select_problem* p) {
    const int64_t rows = p->B * p->K;
    pieces = beam_pieces(rows, p->V, p->z_dtype);
    o_keys = align_up((size_t)rows * pieces * sizeof(BeamPart), 256);
    bytes = align_up(o_keys + (size_t)rows * pieces * p->keep * sizeof(uint64_t), 256);
  }
};

static int check_reorder(const adwin_opd_beam_reorder_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || p->reserved != 0) return ADWIN_E_MODE;
  if (p->B < 0 || p->B >= kMaxRows || p->K < 1 || p->K > ADWIN_MAX_BEAMS || p->keep < 1 || p->keep > ADWIN_MAX_BEAMS ||
      p->B * p->K >= kMaxRows || p->B * p->keep >= kMaxRows || p->n < 0 || p->n > ADWIN_MAX_STATES)
    return ADWIN_E_SHAPE;
  if (p->B == 0 || p->n == 0) return ADWIN_OK;
  if (!p->states || !p->parent) return ADWIN_E_NULL;
  const int64_t most = (int64_t)1 << 40;
  for (int i = 0; i < p->n; ++i) {
    const adwin_opd_beam_state& s = p->states[i];
    if (s.reserved != 0) return ADWIN_E_MODE;
    if (s.planes < 0 || s.planes >= 1 << 20 || s.positions < 0 || s.bytes < 0 || s.positions >= most || s.bytes >= most ||
        (s.bytes > 0 && s.positions >= most / s.bytes))
      return ADWIN_E_SHAPE;
    const int64_t plane = s.positions * s.bytes;
    if (plane == 0 || s.planes == 0) continue;
    if (!s.from || !s.to) return ADWIN_E_NULL;
    if (s.from_plane < 0 || s.to_plane < 0 || s.from_plane >= most || s.to_plane >= most || s.from_row < 0 || s.to_row < 0 ||
        s.from_row >= most || s.to_row >= most)
      return ADWIN_E_SHAPE;
    // from an array's first byte to its last: within the addresses of a device, so that what follows stays within 64 bits
    auto ends = [&](int64_t row, int64_t pl, int64_t rows) {
      return (__int128)(rows - 1) * row + (__int128)(s.planes - 1) * pl + plane < (__int128)1 << 48;
    };
    if (!ends(s.from_row, s.from_plane, p->B * p->K) || !ends(s.to_row, s.to_plane, p->B * p->keep)) return ADWIN_E_SHAPE;
    // planes inside a row, or rows inside a plane: either way they must be apart
    auto apart = [&](int64_t row, int64_t pl, int64_t rows) {
      if (s.planes > 1 && pl < plane) return false;
      if (rows <= 1) return true;
      if (row >= (s.planes - 1) * pl + plane) return true;
      return row >= plane && (s.planes == 1 || pl >= (rows - 1) * row + plane);
    };
    if (!apart(s.from_row, s.from_plane, p->B * p->K) || !apart(s.to_row, s.to_plane, p->B * p->keep)) return ADWIN_E_SHAPE;
  }
  auto in_place = [](const adwin_opd_beam_state& s) { return s.from == s.to; };
  auto span = [&](const adwin_opd_beam_state& s, bool to) {
    const int64_t rows = p->B * (to ? p->keep : p->K);
    return (rows - 1) * (to ? s.to_row : s.from_row) + (s.planes - 1) * (to ? s.to_plane : s.from_plane) + s.positions * s.bytes;
  };
  for (int i = 0; i < p->n; ++i) {
    const adwin_opd_beam_state& s = p->states[i];
    if (s.positions * s.bytes == 0 || s.planes == 0) continue;
    if (in_place(s) && (s.from_row != s.to_row || s.from_plane != s.to_plane || p->K != p->keep)) return ADWIN_E_ALIGN;
    const char* to = (const char*)s.to;
    const int64_t bytes = span(s, true);
    auto meets = [&](const void* from, int64_t n) { return from && to < (const char*)from + n && (const char*)from < to + bytes; };
    if (meets(p->parent, 4 * p->B * p->keep) || meets(p->length, 4 * p->B)) return ADWIN_E_ALIGN;
    for (int j = 0; j < p->n; ++j) {
      const adwin_opd_beam_state& o = p->states[j];
      if (o.positions * o.bytes == 0 || o.planes == 0) continue;
      if (!(i == j && in_place(s)) && to < (const char*)o.from + span(o, false) && (const char*)o.from < to + bytes) return ADWIN_E_ALIGN;
      if (i != j && to < (const char*)o.to + span(o, true) && (const char*)o.to < to + bytes) return ADWIN_E_ALIGN;
    }
  }
  return ADWIN_OK;
}

// Past the caches from 320 MiB on, which the last-level cache of 256 MiB does not hold anyway.  28 caches of 32 rows, 1.1 GB in all: kept / past
// 214 / 198 us (5.6 TB/s), with two pieces to a thread and row 217 / 221, with four 226 / 254.
template <typename V, int MOST>
static hipError_t launch_move_n(const MoveArgs& a, hipStream_t st) {
  int64_t most = 0, bytes = 0;
  for (int i = 0; i < a.n; ++i) {
    const int64_t per = 256 * (int64_t)sizeof(V), n = (a.s[i].positions * a.s[i].bytes + per - 1) / per;
    const int64_t all = n < (1 << 20) ? n * a.s[i].planes : 1 << 20;
    most = all > most ? all : most;
    bytes += a.s[i].positions * a.s[i].bytes * a.s[i].planes;
  }
  const dim3 grid((unsigned)(most < (1 << 20) ? most : 1 << 20), (unsigned)a.n, (unsigned)(a.B < 65535 ? a.B : 65535));
  if constexpr (sizeof(V) >= 8)
    if ((double)bytes * (double)(a.B * a.keep) > 320.0 * (1 << 20)) {
      beam_move_kernel<V, MOST, true><<<grid, 256, 0, st>>>(a);
      return hipGetLastError();
    }
  beam_move_kernel<V, MOST, false><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}
// `width`: bytes of a load
static hipError_t launch_move(const MoveArgs& a, int width, hipStream_t st) {
  if (width == 16) {
    if (a.keep <= 4) return launch_move_n<u32x4, 4>(a, st);
    if (a.keep <= 8) return launch_move_n<u32x4, 8>(a, st);
    if (a.keep <= 16) return launch_move_n<u32x4, 16>(a, st);
    if (a.keep <= 32) return launch_move_n<u32x4, 32>(a, st);
    return launch_move_n<u32x2, 64>(a, st);
  }
  if (width == 4) return a.keep <= 8 ? launch_move_n<uint32_t, 8>(a, st) : launch_move_n<uint32_t, 64>(a, st);
  if (width == 2) return launch_move_n<uint16_t, 64>(a, st);
  return launch_move_n<uint8_t, 64>(a, st);
}

}  // namespace adwin

using namespace adwin;

extern "C" int adwin_opd_beam_select_workspace_bytes(const adwin_opd_beam_select_problem* p, size_t* bytes) {
  if (!bytes) return ADWIN_E_NULL;
  const int st = check_select(p);
  if (st != ADWIN_OK) return st;
  *bytes = BeamLayout(p).bytes;
  return ADWIN_OK;
}

extern "C" int adwin_opd_beam_select(const adwin_opd_beam_select_problem* p, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int st = check_select(p);
  if (st != ADWIN_OK) return st;
  if (p->B == 0) return ADWIN_OK;
  if (!p->z || !p->score || !p->parent || !p->token) return ADWIN_E_NULL;
  if ((uintptr_t)p->z & entry_mask(p->z_dtype)) return ADWIN_E_ALIGN;
  const BeamLayout L(p);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < L.bytes) return ADWIN_E_WORKSPACE;
  if (!selects_apart(p, workspace, L.bytes)) return ADWIN_E_ALIGN;
  BeamArgs a{};
  a.z = p->z; a.ld = p->ld_z; a.B = p->B; a.rows = p->B * p->K; a.K = p->K; a.keep = p->keep; a.V = p->V; a.pieces = L.pieces;
  a.end = p->end < 0 ? -1 : p->end;
  const double c = 1.4426950408889634 / (double)p->temperature;
  a.c = (float)c;
  if ((double)a.c >= c) a.c = nextafterf(a.c, 0.f);
  a.c_low = fmaxf((float)(c - (double)a.c), 1.17549435e-38f);      // not 0 at the largest temperatures either: -inf times 0
  a.per_temperature = 1.0 / (double)p->temperature; a.power = p->length_power;
  a.score = p->score; a.finished = p->finished; a.length = p->length;
  a.part = (BeamPart*)workspace; a.keys = (uint64_t*)((unsigned char*)workspace + L.o_keys);
  a.parent = p->parent; a.token = p->token; a.new_score = p->new_score; a.new_finished = p->new_finished; a.new_length = p->new_length;
  a.row_status = p->row_status;
  hipStream_t stream = (hipStream_t)hip_stream;
  const unsigned blocks = (unsigned)(a.rows * L.pieces);
  // read past the last-level cache of 256 MiB where the logits exceed it: they have left before anybody can find them there
  const bool past = a.rows * p->V * (p->z_dtype == ADWIN_DT_BF16 ? 2 : 4) > ((int64_t)320 << 20);
  if (p->z_dtype == ADWIN_DT_BF16) {
    if (past) beam_rows_kernel<uint16_t, true><<<blocks, kThreads, 0, stream>>>(a);
    else beam_rows_kernel<uint16_t, false><<<blocks, kThreads, 0, stream>>>(a);
  } else {
    if (past) beam_rows_kernel<float, true><<<blocks, kThreads, 0, stream>>>(a);
    else beam_rows_kernel<float, false><<<blocks, kThreads, 0, stream>>>(a);
  }
  ADWIN_HIP_TRY(hipGetLastError());
  beam_join_kernel<<<(unsigned)a.B, kThreads, 0, stream>>>(a);
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}

extern "C" int adwin_opd_beam_reorder(const adwin_opd_beam_reorder_problem* p, void* hip_stream) {
  const int st = check_reorder(p);
  if (st != ADWIN_OK) return st;
  if (p->B == 0) return ADWIN_OK;
  // arrays that are moved in pieces of the same width go together
  for (const int width : {16, 4, 2, 1}) {
    MoveArgs a{};
    a.B = p->B; a.K = p->K; a.keep = p->keep; a.parent = p->parent; a.length = p->length;
    for (int i = 0; i <= p->n; ++i) {
      if (i == p->n || a.n == kMoved) {
        if (a.n > 0) ADWIN_HIP_TRY(launch_move(a, width, (hipStream_t)hip_stream));
        a.n = 0;
        if (i == p->n) break;
      }
      const adwin_opd_beam_state& s = p->states[i];
      if (s.positions * s.bytes == 0 || s.planes == 0) continue;
      const uintptr_t all = (uintptr_t)s.from | (uintptr_t)s.to | (uintptr_t)s.from_row | (uintptr_t)s.to_row |
                            (uintptr_t)(s.planes > 1 ? s.from_plane | s.to_plane : 0);
      const int wide = (all & 15) == 0 ? 16 : (all & 3) == 0 ? 4 : (all & 1) == 0 ? 2 : 1;
      if (wide != width) continue;
      a.s[a.n++] = {(const char*)s.from, (char*)s.to, s.from_row, s.to_row, s.from_plane, s.to_plane, s.positions, s.bytes, s.planes,
                    s.from == s.to};
    }
  }
  return ADWIN_OK;
}
