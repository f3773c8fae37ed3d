// Rows to 8-bit integers, and the product of two arrays of such rows.
#include "fused_shared.h"
#include "product_rule.h"
#include "product_shared.h"

namespace adwin {

typedef int i32x16 __attribute__((ext_vector_type(16)));

struct QuantArgs {
  const void* x; int64_t ld; int64_t N;
  int32_t H, pitch;
  int8_t* q; float* scale; int32_t* row_status;
};

// Integers of eight entries: 127 x / a to the nearest, ties to even, as in exact arithmetic.  t = x (127 / a) in fp32 is off
// by up to 127 * 2^-23 = 1.5e-5; where one lies within twice that of a half, quotients in 64 bits decide (127 x is exact there,
// and one that is no tie is at least 2^-41 away from it, relative, while the division rounds by 2^-53).  Adding
// 1.5 * 2^23 rounds t to a whole number, whose low byte is the sum's.
template <typename T>
__device__ __forceinline__ uint2 quantised(const Eight<T>& x, float per_a, float a, bool tiny) {
  constexpr float kWhole = 12582912.f;
  uint32_t b[8];
  float worst = tiny ? 1.f : 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float off[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float t = x.entry(e + i) * per_a, r = t + kWhole;
      b[e + i] = __float_as_uint(r);
      off[i] = t - (r - kWhole);
    }
    asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(worst) : "v"(off[0]), "v"(off[1]));
  }
  if (worst > 0.5f - 3.0e-5f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (uint32_t)(int)rint((double)x.entry(e) * 127.0 / (double)a);
  }
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u), 0x05040100u);
  return make_uint2(w[0], w[1]);
}

// One wave per row, eight entries to a lane and group.  Up to 4096 entries the row stays in registers between the search for
// its largest magnitude and the integers; a longer one is read twice.  WHOLE: rows of whole groups that begin at multiples of
// 16 bytes.  PAST: past the caches, for arrays that they do not hold anyway.  What bounds it is the memory, and the vector unit
// close behind: 151,936 rows of 4096 bf16 305 us (6.1 TB/s), of 2048 180 us (5.2 TB/s); with the magnitudes one at a time and three
// instructions more for an integer 343 and 193 us.
constexpr int kHeld = 8;                       // groups of a lane that are held
template <typename T, bool WHOLE, bool PAST>
__device__ __forceinline__ void quant_row(const QuantArgs& p, int64_t n) {
  const int lane = threadIdx.x & 63;
  const T* x = (const T*)p.x + n * p.ld;
  const int groups = (p.H + 7) / 8;
  auto load = [&](Eight<T>& v, int g) __attribute__((always_inline)) {
    if constexpr (WHOLE) {
      v.template load<PAST>(x + 8 * (g < groups ? g : groups - 1));   // straight-line loads: beyond the row its last group again
      if (g >= groups) v.clear();
    } else {
      v.load_some(x + 8 * g, p.H - 8 * g);
    }
  };
  Eight<T> v[kHeld];
  uint32_t top = 0;
  const bool held = groups <= 64 * kHeld;
  for (int g0 = 0; g0 < groups; g0 += 64 * kHeld) {
    if (held && groups <= 64 * kHeld / 2) {
#pragma unroll
      for (int i = 0; i < kHeld / 2; ++i) load(v[i], lane + 64 * i);
#pragma unroll
      for (int i = kHeld / 2; i < kHeld; ++i) v[i].clear();
    } else {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) load(v[i], g0 + lane + 64 * i);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top = v[i].largest(top);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t b = __shfl_xor(top, o, 64);
    top = b > top ? b : top;
  }
  const bool fine = top < 0x7f800000u;
  const float a = fine ? __uint_as_float(top) : 0.f;
  if (lane == 0) {
    p.scale[n] = a / 127.f;
    if (p.row_status) p.row_status[n] = fine ? 0 : (int)ADWIN_DEV_NONFINITE;
  }
  const bool tiny = a < 1.0e-35f;                // 127 / a may overflow
  const float per_a = a > 0.f && !tiny ? 127.f / a : 0.f;
  uint2* q = (uint2*)(p.q + n * p.pitch);
  const int out = p.pitch / 8;
  for (int g0 = 0; g0 < out; g0 += 64 * kHeld) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int g = g0 + lane + 64 * i;
      if (g < out) {
        if (!held) load(v[i], g);
        const uint2 o = a > 0.f ? quantised(v[i], per_a, a, tiny) : make_uint2(0, 0);
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        if constexpr (PAST) __builtin_nontemporal_store(u32x2{o.x, o.y}, (u32x2*)(q + g));
        else q[g] = o;
      }
    }
  }
}

template <typename T, bool WHOLE, bool PAST>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs p) {
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n < p.N) quant_row<T, WHOLE, PAST>(p, n);
}

struct ProductArgs {
  const int8_t* h; const float* h_scale; const int8_t* W; const float* W_scale;
  void* z; int64_t ld_z; int64_t T;
  int32_t V, pitch;
  int32_t token_tiles, vocab_tiles, strips, group;
  int32_t whole;                   // rows of z lie and begin at multiples of 16 bytes
};

// ---------------------------------------------------------------------------------------
// The product, many tokens.  v_mfma_i32_32x32x32_i8: lane l supplies row l % 32 of either operand, 16 bytes of k of half
// l / 32 (the sum does not depend on which bytes these are, as long as both operands agree); result e of lane l is row
// 8 (e / 4) + 4 (l / 32) + e % 4 of A and row l % 32 of B.  A = entries of the head, B = tokens.
//
// Tile of 256 entries x 256 tokens, 2 x 2 waves of 128 x 128 (256 accumulators), k-steps of 128 bytes a row, staged by direct
// global->LDS loads: a ring of three 32 KiB blocks for W, whose lines come from memory, and one of two for the tokens,
// which the L2 holds.  Row r's 16-byte chunk c lies at chunk position c ^ (r / 2 % 8), so that the 16 lanes that read at a time
// fall on different banks; tile row 8 q + 4 h + r of 32 holds entry 16 h + 4 q + r, which makes a lane's 16
// results of a block 16 consecutive entries of z.
// A workgroup keeps its tokens and walks a strip of vocabulary tiles; the k-steps of all of them form one pipeline: in step s
// the blocks of step s + 2 are loaded, W behind the MFMAs of sub-steps 1 and 2 into the buffer that nobody reads any
// more, the tokens behind those of sub-step 3 into the one that this step has finished.  The one barrier of a step stands before
// its last sub-step, when every fragment of the step is in registers, and that sub-step's MFMAs cover the reads of the
// next step's first fragments.  The order of the instructions is pinned, a read, a load or a piece of bookkeeping behind each MFMA.
// 4,096 tokens, V = 151,936, H = 4096, bf16 logits: 2.11 to 2.28 ms over machines, 2.2 to 2.4 POP/s, where the library's 8-bit product
// reaches 1.85 and its bf16 one 1.3.  The matrix pipe is busy 66 % of the cycles at 1.57 to 1.67 GHz (power); the epilogue, which
// nothing overlaps with one wave to a SIMD, takes 15 % (half of it the arithmetic, half the stores, which all compute units issue at about the
// same time; workgroups begun at different times: 2 % slower), the k-steps wait 14 % for loads.  How token tiles and strips are
// grouped over the XCDs makes no difference (1, 2, 4 and 8 token tiles within 0.6 %).
// ---------------------------------------------------------------------------------------
constexpr int kQTile = 256;
constexpr int kQBlock = kQTile * 128;                 // 32 KiB
constexpr int kQRingB = 3 * kQBlock;                  // where the tokens' ring begins
constexpr int kQLds = 5 * kQBlock;                    // 160 KiB

// Where the loads of the step after next come from: tile `tile` of the strip, k-step kt.
struct QLoads {
  const char* a; const char* b;                        // of that step
  const char* a0; const char* b0;                      // of k-step 0 of its tile
  int kt, tile;
};

// One k-step.  r_a, r_b: LDS address of the blocks that it reads plus the wave's KiB, on return those of the next step.
template <bool FRESH>
__device__ __forceinline__ void q_kstep(i32x16 (&acc)[4][4], i32x4 (&fa)[2][4], i32x4 (&fb)[2][4], uint32_t& r_a, uint32_t& r_b,
                                        uint32_t a_begin, uint32_t b_begin, const uint32_t (&swA)[4], const uint32_t (&swB)[4],
                                        const uint32_t (&voffa)[8], const uint32_t (&voffb)[8], QLoads& ld, int nk, int tiles,
                                        int64_t tile_bytes, bool relaxed, int stores) {
  const i32x16 zero = {};
  uint32_t r_a_nx = 0, r_a_wr = 0, r_b_nx = 0, xa = 0, xb = 0;
#define Q_FENCE __builtin_amdgcn_sched_barrier(0);
#define Q_MM(KK, I, J)                                                                                           \
  acc[I][J] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[(KK) & 1][I], fb[(KK) & 1][J],                            \
                                                    FRESH && (KK) == 0 ? zero : acc[I][J], 0, 0, 0);             \
  Q_FENCE
  // behind MFMA M of sub-step KK
#define Q_SIDE(KK, M)                                                                                            \
  if constexpr ((M) < 8) {                                                                                       \
    constexpr int nx = ((KK) + 1) & 3, f = (M) >> 1;                                                             \
    if constexpr ((M) == 0) {                                                                                    \
      xa = ((KK) < 3 ? r_a : r_a_nx) + swA[nx];                                                                  \
      xb = ((KK) < 3 ? r_b : r_b_nx) + swB[nx];                                                                  \
      asm volatile("" : "+v"(xa), "+v"(xb));                                                                     \
    }                                                                                                            \
    if constexpr (((M) & 1) == 0) fa[nx & 1][f] = q_frag(xa, 32 * f);                                            \
    else fb[nx & 1][f] = q_frag(xb, 32 * f);                                                                     \
    if constexpr ((KK) == 0 && (M) == 0) r_a_nx = ring_next<kQBlock>(r_a, a_begin, a_begin + 3 * kQBlock);       \
    if constexpr ((KK) == 0 && (M) == 1) r_b_nx = ring_next<kQBlock>(r_b, b_begin, b_begin + 2 * kQBlock);       \
    if constexpr ((KK) == 0 && (M) == 2) r_a_wr = ring_next<kQBlock>(r_a_nx, a_begin, a_begin + 3 * kQBlock);    \
    Q_FENCE                                                                                                      \
  } else if constexpr ((KK) == 0 && (M) == 8) {                                                                  \
    const bool wrap = ld.kt + 1 == nk, on = wrap && ld.tile + 1 < tiles;                                         \
    ld.kt = wrap ? 0 : ld.kt + 1;                                                                                \
    ld.tile += on;                                                                                               \
    ld.a0 += on ? tile_bytes : 0;                                                                                \
    ld.a = wrap ? ld.a0 : ld.a + 128;                                                                            \
    ld.b = wrap ? ld.b0 : ld.b + 128;                                                                            \
    Q_FENCE                                                                                                      \
  } else if constexpr (((KK) == 1 || (KK) == 2) && (M) >= 12) {                                                  \
    dma16_at<(((KK) - 1) * 4 + (M) - 12) * 4096>(r_a_wr, voffa[(((KK) - 1) * 4 + (M) - 12) & 7], ld.a);          \
    Q_FENCE                                                                                                      \
  } else if constexpr ((KK) == 3 && (M) >= 8) {                                                                  \
    dma16_at<((M) - 8) * 4096>(r_b, voffb[((M) - 8) & 7], ld.b);                                                 \
    Q_FENCE                                                                                                      \
  }
#define Q_ROW(KK, I, M0)                                                                            \
  Q_MM(KK, I, 0) Q_SIDE(KK, (M0) + 0) Q_MM(KK, I, 1) Q_SIDE(KK, (M0) + 1)                           \
  Q_MM(KK, I, 2) Q_SIDE(KK, (M0) + 2) Q_MM(KK, I, 3) Q_SIDE(KK, (M0) + 3)
#define Q_SUB(KK) Q_ROW(KK, 0, 0) Q_ROW(KK, 1, 4) Q_ROW(KK, 2, 8) Q_ROW(KK, 3, 12)
  Q_FENCE
  Q_SUB(0)
  Q_SUB(1)
  Q_SUB(2)
  // The next step's blocks have landed, and every wave has this step's fragments.  Loads return in order: the eight youngest,
  // this step's of W, stay in flight, and in the first step of a tile the stores of the tile before, which came
  // behind the loads that are waited for.
  if (FRESH && relaxed) {
    if (stores > 32) asm volatile("s_waitcnt vmcnt(63) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(40) lgkmcnt(0)" ::: "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
  }
  __syncthreads();
  Q_FENCE
  Q_SUB(3)
  r_a = r_a_nx;
  r_b = r_b_nx;
#undef Q_SUB
#undef Q_ROW
#undef Q_SIDE
#undef Q_MM
#undef Q_FENCE
}

// An accumulator as a number.  The constraint keeps it in its accumulator register until here.
__device__ __forceinline__ float acc_read(int a) {
  int v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return (float)v;
}

// A logit is its integer sum times the token's scale, then the entry's (the product of the scales can leave fp32 where the logit does
// not).  The first product stays within fp32, as a sum is below 2^30, but for tokens of entries beyond 1e31: their logits are
// formed and stored 2^-64 times as large, which takes nothing from either type, and a wave that has such tokens raises them at its end.
constexpr float kHugeScale = 0x1p96f;
__device__ __forceinline__ float small_scale(float token) { return token >= kHugeScale ? token * 0x1p-64f : token; }
// z: the wave's first token and first entry; `scale`: from that token on; `rows` of them, `left` entries up to V in pieces of
// `piece`, `step` apart and `pieces` in number.  The wave's stores have been waited for.
template <typename T>
__device__ __forceinline__ void raise_rows(T* z, int64_t ld, const float* scale, int rows, int64_t left, int piece, int step, int pieces) {
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    if (scale[r] < kHugeScale) continue;
#pragma unroll 1
    for (int i = 0; i < pieces; ++i)
#pragma unroll 1
      for (int q = lane; q < piece; q += 64) {
        const int64_t v = (int64_t)i * step + q;
        if (v < left) Entry<T>::put(z + r * ld + v, Entry<T>::one(z + r * ld + v) * 0x1p64f);
      }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void quant_tile_kernel(ProductArgs p) {
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1, half = lane >> 5;
  int strip, tt;
  strip_and_tile(xcd_contiguous_id(blockIdx.x, gridDim.x), p.group, p.strips, p.token_tiles, &strip, &tt);
  const int vt0 = (int)((int64_t)p.vocab_tiles * strip / p.strips), vt1 = (int)((int64_t)p.vocab_tiles * (strip + 1) / p.strips);
  if (vt0 >= vt1) return;
  const int64_t t0 = (int64_t)tt * kQTile;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const uint32_t a_begin = lds0 + wave * 1024u, b_begin = a_begin + kQRingB;
  const int nk = p.pitch / 128;
  const int64_t tile_bytes = (int64_t)kQTile * p.pitch;

  // lane offsets of the wave's eight loads of a block: tile rows 32 d + 8 wave + lane / 8
  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16u;
  const int e0 = 16 * half + 4 * wave + ((lane >> 3) & 3);
  uint32_t voffa[8], voffb[8];
  auto rows_of_w = [&](int tile) {                       // rows beyond V repeat the last one
    const int left = p.V - tile * kQTile - 1;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int v = 32 * d + e0;
      voffa[d] = (uint32_t)(v < left ? v : left) * (uint32_t)p.pitch + chunk;
      asm volatile("" : "+v"(voffa[d]));
    }
  };
  rows_of_w(vt0);
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    const int64_t t = 32 * d + 8 * wave + (lane >> 3), left = p.T - t0 - 1;
    voffb[d] = (uint32_t)(t < left ? t : left) * (uint32_t)p.pitch + chunk;
    asm volatile("" : "+v"(voffb[d]));
  }
  uint32_t swA[4], swB[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const uint32_t at = (lane & 31) * 128u + (uint32_t)(((2 * kk + half) ^ (lane >> 1)) & 7) * 16u - wave * 1024u;
    swA[kk] = at + wa * (kQBlock / 2);
    swB[kk] = at + wb * (kQBlock / 2);
  }
  float sh[4];                                           // scales of the lane's tokens
  bool huge = false;                                     // some scale of the wave's tokens is
#pragma unroll
  for (int fn = 0; fn < 4; ++fn) {
    const int64_t t = t0 + 128 * wb + 32 * fn + (lane & 31);
    sh[fn] = p.h_scale[t < p.T ? t : p.T - 1];
    huge = huge || __any(sh[fn] >= kHugeScale);
    sh[fn] = small_scale(sh[fn]);
    asm volatile("" : "+v"(sh[fn]));                     // waited for here, not behind the loads that follow
  }
  // where the lane stores first: token lane / 16 of the wave's, the entries of its chunk; and the tokens from there on
  T* const z = (T*)p.z + (t0 + 128 * wb + (lane >> 4)) * p.ld_z + (lane & 15) * (int)(16 / sizeof(T));
  const int64_t row_step = 4 * p.ld_z, rows_here = p.T - t0 - 128 * wb - (lane >> 4);
  const int rows_left = (int)(rows_here < 128 ? rows_here : 128);

  QLoads ld;
  ld.a0 = ld.a = (const char*)p.W + vt0 * tile_bytes;
  ld.b0 = ld.b = (const char*)p.h + t0 * p.pitch;
  ld.kt = 0; ld.tile = 0;
  const int tiles = vt1 - vt0;
  int partial = p.V - vt1 * kQTile < 0 ? tiles - 1 : -1;      // the strip's tile that V ends in
  auto load_step = [&](uint32_t ra, uint32_t rb) {
#define Q_LOAD(D) dma16_at<(D) * 4096>(ra, voffa[D], ld.a);
    Q_LOAD(0) Q_LOAD(1) Q_LOAD(2) Q_LOAD(3) Q_LOAD(4) Q_LOAD(5) Q_LOAD(6) Q_LOAD(7)
#undef Q_LOAD
#define Q_LOAD(D) dma16_at<(D) * 4096>(rb, voffb[D], ld.b);
    Q_LOAD(0) Q_LOAD(1) Q_LOAD(2) Q_LOAD(3) Q_LOAD(4) Q_LOAD(5) Q_LOAD(6) Q_LOAD(7)
#undef Q_LOAD
  };
  // steps 0 and 1
  load_step(a_begin, b_begin);
  if (nk > 1) { ld.kt = 1; ld.a += 128; ld.b += 128; }
  else if (tiles > 1) { ld.tile = 1; ld.a0 += tile_bytes; ld.a = ld.a0; if (partial == 1) rows_of_w(vt0 + 1); }
  load_step(a_begin + kQBlock, b_begin + kQBlock);
  asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  __syncthreads();
  i32x16 acc[4][4];
  i32x4 fa[2][4], fb[2][4];
  uint32_t r_a = a_begin, r_b = b_begin;
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    fa[0][f] = q_frag(r_a + swA[0], 32 * f);
    fb[0][f] = q_frag(r_b + swB[0], 32 * f);
  }
  bool relaxed = false;
  const int stores = sizeof(T) == 2 ? 32 : 64;
  for (int i = 0; i < tiles; ++i) {
    // the loads of a step go into the tile that V ends in
    auto into_last = [&]() __attribute__((always_inline)) {
      if (ld.kt + 1 == nk && ld.tile + 1 == partial) rows_of_w(vt0 + partial);
    };
    into_last();
    q_kstep<true>(acc, fa, fb, r_a, r_b, a_begin, b_begin, swA, swB, voffa, voffb, ld, nk, tiles, tile_bytes, relaxed, stores);
    for (int kt = 1; kt < nk; ++kt) {
      into_last();
      q_kstep<false>(acc, fa, fb, r_a, r_b, a_begin, b_begin, swA, swB, voffa, voffb, ld, nk, tiles, tile_bytes, false, 0);
    }
    // z.  A lane has 16 entries of a token, which as they are would go out as 16-byte pieces of 64 different rows.  A wave
    // lays 32 tokens x 256 bytes into the LDS first and stores whole lines: into the KiBs that its own loads will fill of the
    // block that the last step has read (row r's chunk c at chunk position c ^ (r % 16): 16 lanes on different banks either way).
    const int64_t v0 = (int64_t)(vt0 + i) * kQTile + 128 * wa;
    const int left = (int)(p.V - v0);                    // may be 0 or less
    relaxed = p.whole && left >= 128 && t0 + kQTile <= p.T;
    if (left <= 0) continue;
    float sv[4][16];
    if (left >= 128) {
      // the scales of the wave's entries through the scalar cache, which the vector loads in flight do not hold up
      typedef const __attribute__((address_space(4))) float* Scales;
      uint64_t at = (uint64_t)(uintptr_t)(p.W_scale + v0);
#pragma unroll
      for (int fm = 0; fm < 4; ++fm) {
        asm volatile("" : "+s"(at));                     // 32 at a time
        const Scales s = (Scales)(uintptr_t)at + 32 * fm;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float lo = s[e], hi = s[16 + e];
          asm volatile("" : "+s"(lo), "+s"(hi));         // and not one load from an address that differs from lane to lane
          sv[fm][e] = half ? hi : lo;
          asm volatile("" : "+v"(sv[fm][e]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int fm = 0; fm < 4; ++fm)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 32 * fm + 16 * half + e;
          sv[fm][e] = p.W_scale[v0 + (j < left ? j : left - 1)];
        }
#pragma unroll
      for (int fm = 0; fm < 4; ++fm)
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(sv[fm][e]));    // waited for here: whole tiles wait for no store
    }
    typedef __attribute__((address_space(3))) u32x4* LdsVec;
    const uint32_t free = r_a == a_begin ? a_begin + 2 * kQBlock : r_a - kQBlock;
    const uint32_t mine = free + (uint32_t)((lane & 31) >> 2) * 4096u + (lane & 3) * 256u;      // the lane's token
    constexpr int kFms = sizeof(T) == 2 ? 4 : 2, kPer = 16 / sizeof(T);      // blocks of 32 entries to a row in the LDS
    const int c = lane & 15;                             // reading, a lane has chunk c of rows 4 k + lane / 16
    // formed anew for every tile: as invariants of the loop the 32 rows' addresses and masks do not fit the registers
    T* at = z + v0;
    int rows = rows_left;
    asm volatile("" : "+v"(at), "+v"(rows));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int fn = 0; fn < 4; ++fn)
#pragma unroll
      for (int f0 = 0; f0 < 4; f0 += kFms) {
#pragma unroll
        for (int f = 0; f < kFms; ++f) {
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = acc_read(acc[f0 + f][fn][e]) * sh[fn] * sv[f0 + f][e];
#pragma unroll
          for (int k = 0; k < 16 / kPer; ++k) {
            const int at = (f * 32 + 16 * half) / kPer + k;
            *(LdsVec)(uintptr_t)(mine + (uint32_t)((at ^ (lane & 15)) * 16)) = pack16(y + k * kPer, T{});
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 row[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = 4 * k + (lane >> 4);
          row[k] = *(LdsVec)(uintptr_t)(free + k * 4096u + (uint32_t)(lane >> 4) * 256u + (uint32_t)((c ^ (r & 15)) * 16));
        }
        __builtin_amdgcn_sched_barrier(0);
        const int n = left - 32 * f0 - c * kPer;         // of the lane's entries
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (rows > 32 * fn + 4 * k) {
            if (p.whole && n >= kPer) *(u32x4*)(at + 32 * f0) = row[k];
            else {
#pragma unroll
              for (int e = 0; e < kPer; ++e)
                if (e < n) at[32 * f0 + e] = entry_of<T>(row[k], e);
            }
          }
          if (f0 + kFms == 4) at += row_step;
          else if (k < 7) at += row_step;
          else at -= 7 * row_step;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // loads that nobody reads may still be writing the LDS
  if (huge) {
    const int64_t first = t0 + 128 * wb, v0 = (int64_t)vt0 * kQTile + 128 * wa;
    raise_rows((T*)p.z + first * p.ld_z + v0, p.ld_z, p.h_scale + first, (int)(p.T - first < 128 ? p.T - first : 128), p.V - v0, 128,
               kQTile, tiles);
  }
}

// ---------------------------------------------------------------------------------------
// The product, few tokens: every line of W is read once, and what bounds it is that read.
// A workgroup to a compute unit has the tokens' integers in its LDS, in the order of the fragments of
// v_mfma_i32_16x16x64_i8 (lane l: row l % 16 of either operand, 16 bytes of k of quarter l / 16; result e of lane l is row
// 4 (l / 16) + e of A and row l % 16 of B), and its 16 waves walk groups of 16 entries of the head, whose
// rows come straight from memory into the registers: a line (128 bytes of k) of 16 rows is two loads of a lane, and kAhead lines
// are under way, over the ends of groups as well.  Waves of a workgroup take its groups in turn, so that the lines of z are
// completed at about the same time, and begin at different lines of k, so that rows a power of two apart do not ask the same
// channels at once (127.6 -> 121.3 us).  1 token, V = 151,936: H = 4096 110 us (5.7 TB/s), 48 tokens, H = 2048 73 us: 4 us
// for each 16 tokens that every compute unit lays into its LDS.  Loads of W past the caches: 118 -> 121 us.
// ---------------------------------------------------------------------------------------
constexpr int kFewThreads = 1024, kFewWaves = kFewThreads / 64;
constexpr int kAhead = 4;
constexpr int kFewGroups = 128;                        // most groups of a workgroup: their scales are in the LDS too
__host__ __device__ constexpr int few_lds(int n, int pitch) { return n * 16 * pitch + kFewGroups * 16 * 4; }

template <typename T, int NT>
__global__ __launch_bounds__(kFewThreads) void quant_few_kernel(ProductArgs p) {
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (p.V + 15) / 16;
  const int g0 = (int)((int64_t)groups * blockIdx.x / gridDim.x), g1 = (int)((int64_t)groups * (blockIdx.x + 1) / gridDim.x);
  const int nk = p.pitch / 128;
  const int mine = (g1 - g0 - wave + kFewWaves - 1) / kFewWaves;      // groups of this wave
  const int total = mine > 0 ? mine * nk : 0;                        // lines

  // W: the lane's bytes of line k of group g
  const int turn = (int)((blockIdx.x * kFewWaves + wave) % (uint32_t)nk);    // the line that the wave begins with
  int ahead_g = g0 + wave, ahead_k = 0, asked = 0;
  const char* src = nullptr;
  auto begin_group = [&](int g) {
    const int64_t v = (int64_t)g * 16 + (lane & 15);
    src = (const char*)p.W + (v < p.V ? v : p.V - 1) * p.pitch + turn * 128 + (lane >> 4) * 16;   // rows beyond V repeat the last one
  };
  i32x4 w[kAhead][2];
  auto ask = [&](int j) __attribute__((always_inline)) {
    const i32x4* q = (const i32x4*)src;
    w[j][0] = q[0];
    w[j][1] = q[4];
    // the wave's last line is asked for again instead of one beyond it
    if (++asked < total) {
      src += 128;
      if (++ahead_k == nk - turn) src -= p.pitch;
      if (ahead_k == nk) {
        ahead_k = 0;
        ahead_g += kFewWaves;
        begin_group(ahead_g);
      }
    }
  };
  float* scales = (float*)(lds + NT * 16 * p.pitch);
  float sh[NT], sw[kFewGroups * 16 / kFewThreads];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = n * 16 + (lane & 15);
    sh[n] = p.h_scale[t < p.T ? t : p.T - 1];
  }
#pragma unroll
  for (int i = 0; i < kFewGroups * 16 / kFewThreads; ++i) {
    const int q = i * kFewThreads + threadIdx.x;
    const int64_t v = (int64_t)g0 * 16 + (q < (g1 - g0) * 16 ? q : 0);
    sw[i] = p.W_scale[v < p.V ? v : p.V - 1];
  }
  // the tokens: fragment (k64, n) at 1024 (k64 NT + n), by direct loads.  Rows beyond T repeat the last one; they enter
  // results that are not stored.
  uint32_t from[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = n * 16 + (lane & 15);
    from[n] = (uint32_t)(t < p.T ? t : p.T - 1) * (uint32_t)p.pitch + (lane >> 4) * 16u;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  for (int k = wave; k < 2 * nk; k += kFewWaves)
#pragma unroll
    for (int n = 0; n < NT; ++n) dma16_at<0>(lds0 + (uint32_t)(k * NT + n) * 1024u, from[n], (const char*)p.h + k * 64);
  if (total > 0) {
    begin_group(ahead_g);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ask(j);
  }
#pragma unroll
  for (int i = 0; i < kFewGroups * 16 / kFewThreads; ++i) scales[i * kFewThreads + threadIdx.x] = sw[i];
  // loads return in order: the tokens are there when no more than the lines that were asked for behind them are under way
  if (total > 0) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * kAhead) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (total == 0) return;

  i32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = i32x4{0, 0, 0, 0};
  bool huge = false;                                     // some scale of the tokens is
#pragma unroll
  for (int n = 0; n < NT; ++n) huge = huge || __any(sh[n] >= kHugeScale);
  int k = 0, g = g0 + wave;
  const char* frag = lds + lane * 16 + turn * (2 * NT * 1024);
  for (int at = 0; at < total; at += kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (at + j < total) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const i32x4 h0 = *(const i32x4*)(frag + n * 1024), h1 = *(const i32x4*)(frag + (NT + n) * 1024);
          acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j][0], h0, acc[n], 0, 0, 0);
          acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j][1], h1, acc[n], 0, 0, 0);
        }
        frag += 2 * NT * 1024;
      }
      ask(j);
      if (at + j < total && ++k == nk - turn) frag = lds + lane * 16;
      if (at + j < total && k == nk) {
        const int v = g * 16 + (lane >> 4) * 4;
        const float4 sv = *(const float4*)(scales + (g - g0) * 16 + (lane >> 4) * 4);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int64_t t = n * 16 + (lane & 15);
          float first = sh[n];
          if (huge) first = small_scale(sh[n]);
          float y[4] = {(float)acc[n][0] * first * sv.x, (float)acc[n][1] * first * sv.y,
                        (float)acc[n][2] * first * sv.z, (float)acc[n][3] * first * sv.w};
          if (huge && sh[n] >= kHugeScale) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] *= 0x1p64f;
          }
          if (t < p.T) {
            T* z = (T*)p.z + t * p.ld_z + v;
            if (p.whole && v + 4 <= p.V) put_entries<false>(z, y, true);
            else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (v + e < p.V) Entry<T>::put(z + e, y[e]);
            }
          }
          acc[n] = i32x4{0, 0, 0, 0};
        }
        k = 0;
        g += kFewWaves;
        frag = lds + lane * 16 + turn * (2 * NT * 1024);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------
// The product in smaller tiles, 64 FN tokens x 128 entries: for one token tile, so that W is read once and its tiles spread evenly
// over the compute units, and for products that large tiles would not spread over them at all.  What bounds it is the read of W, or
// latency, and what counts is how much is under way: a ring of kStages
// k-steps (128 bytes of 128 rows of W and of the tokens), all but one of them loading.  2 x 2 waves of 64 x 32 FN; operands,
// fragments and their places in the LDS as in the kernel of many tokens.  V = 151,936, H = 4096: 64 tokens 145 us with the rows'
// integers (4.4 TB/s), 128 tokens 168 to 179 us; 1,187 tiles are 4.6 rounds of 256 compute units and run as 5.
// ---------------------------------------------------------------------------------------
template <int FN>
struct MidTile {
  static constexpr int kEntries = 128, kTokens = 64 * FN;
  static constexpr int kBlockA = kEntries * 128, kStage = kBlockA + kTokens * 128;
  static constexpr int kScratch = 4 * 4096;            // 32 tokens x 128 bytes of z for each wave
  static constexpr int kStages = (160 * 1024 - kScratch) / kStage;
  static constexpr int kLds = kStages * kStage + kScratch;
  static constexpr int kLoads = 4 + 2 * FN;            // of a wave and stage
};

template <typename T, int FN>
__global__ __launch_bounds__(256) void quant_mid_kernel(ProductArgs p) {
  typedef MidTile<FN> Tile;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1, half = lane >> 5;
  int strip, tt;
  strip_and_tile(xcd_contiguous_id(blockIdx.x, gridDim.x), p.group, p.strips, p.token_tiles, &strip, &tt);
  const int vt0 = (int)((int64_t)p.vocab_tiles * strip / p.strips), vt1 = (int)((int64_t)p.vocab_tiles * (strip + 1) / p.strips);
  const int64_t t0 = (int64_t)tt * Tile::kTokens, T_left = p.T - t0;       // tokens from this tile on
  const char* const h = (const char*)p.h + t0 * p.pitch;
  const int tiles = vt1 - vt0, nk = p.pitch / 128;
  if (tiles <= 0) return;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16u;
  const int e0 = 16 * half + 4 * wave + ((lane >> 3) & 3);
  uint32_t voffa[4], voffb[2 * FN];
  auto rows_of_w = [&](int tile) {                       // rows beyond V repeat the last one
    const int64_t left = p.V - (int64_t)tile * Tile::kEntries - 1;
#pragma unroll
    for (int d = 0; d < 4; ++d) voffa[d] = (uint32_t)(32 * d + e0 < left ? 32 * d + e0 : left) * (uint32_t)p.pitch + chunk;
  };
#pragma unroll
  for (int d = 0; d < 2 * FN; ++d) {
    const int64_t t = 32 * d + 8 * wave + (lane >> 3);
    voffb[d] = (uint32_t)(t < T_left ? t : T_left - 1) * (uint32_t)p.pitch + chunk;
  }
  uint32_t swA[4], swB[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const uint32_t at = (lane & 31) * 128u + (uint32_t)(((2 * kk + half) ^ (lane >> 1)) & 7) * 16u;
    swA[kk] = at + wa * (64 * 128);
    swB[kk] = at + Tile::kBlockA + wb * (32 * FN * 128);
  }
  float sh[FN];
  bool huge = false;                                     // some scale of the wave's tokens is
#pragma unroll
  for (int fn = 0; fn < FN; ++fn) {
    const int64_t t = 32 * FN * wb + 32 * fn + (lane & 31);
    sh[fn] = p.h_scale[t0 + (t < T_left ? t : T_left - 1)];
    huge = huge || __any(sh[fn] >= kHugeScale);
    sh[fn] = small_scale(sh[fn]);
    asm volatile("" : "+v"(sh[fn]));                     // waited for here
  }

  // where the next stage's loads come from: k-step kt of tile `tile` of the strip
  int kt = 0, tile = 0;
  const char* tile_w = (const char*)p.W + (int64_t)vt0 * Tile::kEntries * p.pitch;
  uint32_t slot_w = lds0 + wave * 1024u;
  rows_of_w(vt0);
  auto ask = [&]() __attribute__((always_inline)) {
    const char* a = tile_w + kt * 128;
    const char* b = h + kt * 128;
#define Q_LOAD(D) dma16_at<(D) * 4096>(slot_w, voffa[D], a);
    Q_LOAD(0) Q_LOAD(1) Q_LOAD(2) Q_LOAD(3)
#undef Q_LOAD
#define Q_LOAD(D) if constexpr ((D) < 2 * FN) dma16_at<Tile::kBlockA + (D) * 4096>(slot_w, voffb[(D) < 2 * FN ? (D) : 0], b);
    Q_LOAD(0) Q_LOAD(1) Q_LOAD(2) Q_LOAD(3) Q_LOAD(4) Q_LOAD(5) Q_LOAD(6) Q_LOAD(7)
#undef Q_LOAD
    slot_w += Tile::kStage;
    if (slot_w == lds0 + wave * 1024u + Tile::kStages * Tile::kStage) slot_w = lds0 + wave * 1024u;
    if (++kt == nk) {                                    // behind the strip's last step its last tile again
      kt = 0;
      if (tile + 1 < tiles) {
        ++tile;
        tile_w += (int64_t)Tile::kEntries * p.pitch;
        if ((int64_t)(vt0 + tile + 1) * Tile::kEntries > p.V) rows_of_w(vt0 + tile);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < Tile::kStages - 1; ++s) ask();

  // where the lane stores: token lane / 8 of 32, 16 bytes
  constexpr int kPer = 16 / sizeof(T), kFms = sizeof(T) == 2 ? 2 : 1;     // blocks of 32 entries to 128 bytes
  const uint32_t scratch = lds0 + Tile::kStages * Tile::kStage + wave * 4096u;
  T* const z = (T*)p.z + (t0 + 32 * FN * wb + (lane >> 3)) * p.ld_z + (lane & 7) * kPer;
  const int rows_left = (int)(T_left < Tile::kTokens ? T_left : Tile::kTokens) - 32 * FN * wb - (lane >> 3);
  uint32_t slot = lds0;
  bool relaxed = false;
  constexpr int kYounger = (Tile::kStages - 2) * Tile::kLoads, kStores = FN * (2 / kFms) * 4;
  for (int i = 0; i < tiles; ++i) {
    i32x16 acc[2][FN];
#pragma unroll
    for (int fm = 0; fm < 2; ++fm)
#pragma unroll
      for (int fn = 0; fn < FN; ++fn) acc[fm][fn] = i32x16{};
    for (int k = 0; k < nk; ++k) {
      // this step has landed (loads return in order; the stores of the tile before came behind its own), and every
      // wave has read the step before, whose slot the next loads fill
      if (k == 0 && relaxed) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kYounger + kStores < 63 ? kYounger + kStores : 63) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kYounger) : "memory");
      __syncthreads();
      ask();
      i32x4 fa[4][2], fb[4][FN];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
        for (int f = 0; f < 2; ++f) fa[kk][f] = q_frag(slot + swA[kk], 32 * f);
#pragma unroll
        for (int f = 0; f < FN; ++f) fb[kk][f] = q_frag(slot + swB[kk], 32 * f);
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int fm = 0; fm < 2; ++fm)
#pragma unroll
          for (int fn = 0; fn < FN; ++fn)
            acc[fm][fn] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[kk][fm], fb[kk][fn], acc[fm][fn], 0, 0, 0);
      slot += Tile::kStage;
      if (slot == lds0 + Tile::kStages * Tile::kStage) slot = lds0;
    }
    const int64_t v0 = (int64_t)(vt0 + i) * Tile::kEntries + 64 * wa;
    const int64_t left = p.V - v0;                       // may be 0 or less
    relaxed = p.whole && left >= 64 && Tile::kTokens <= T_left;
    if (left <= 0) continue;
    float sv[2][16];
    typedef const __attribute__((address_space(4))) float* Scales;
#pragma unroll
    for (int fm = 0; fm < 2; ++fm) {
      if (left >= 64) {
        uint64_t at = (uint64_t)(uintptr_t)(p.W_scale + v0 + 32 * fm);
        asm volatile("" : "+s"(at));
        const Scales s = (Scales)(uintptr_t)at;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float lo = s[e], hi = s[16 + e];
          asm volatile("" : "+s"(lo), "+s"(hi));         // scalar loads: the loads in flight do not hold them up
          sv[fm][e] = half ? hi : lo;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 32 * fm + 16 * half + e;
          sv[fm][e] = p.W_scale[v0 + (j < left ? j : left - 1)];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(sv[fm][e]));
      }
    }
    typedef __attribute__((address_space(3))) u32x4* LdsVec;
#pragma unroll
    for (int fn = 0; fn < FN; ++fn) {
      if (32 * FN * wb + 32 * fn >= T_left) continue;
#pragma unroll
      for (int f0 = 0; f0 < 2; f0 += kFms) {
#pragma unroll
        for (int f = 0; f < kFms; ++f) {
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = (float)acc[f0 + f][fn][e] * sh[fn] * sv[f0 + f][e];
#pragma unroll
          for (int k = 0; k < 16 / kPer; ++k) {
            const int at = (f * 32 + 16 * half) / kPer + k;
            *(LdsVec)(uintptr_t)(scratch + (lane & 31) * 128u + (uint32_t)((at ^ (lane >> 1)) & 7) * 16u) = pack16(y + k * kPer, T{});
          }
        }
        const int64_t n = left - 32 * f0 - (lane & 7) * kPer;      // of the lane's entries
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 8 * k + (lane >> 3);
          const u32x4 row = *(LdsVec)(uintptr_t)(scratch + r * 128u + (uint32_t)(((lane & 7) ^ (r >> 1)) & 7) * 16u);
          T* at = z + (int64_t)(32 * fn + 8 * k) * p.ld_z + v0 + 32 * f0;
          if (rows_left > 32 * fn + 8 * k) {
            if (p.whole && n >= kPer) *(u32x4*)at = row;
            else {
#pragma unroll
              for (int e = 0; e < kPer; ++e)
                if (e < n) at[e] = entry_of<T>(row, e);
            }
          }
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // loads that nobody reads may still be writing the LDS
  if (huge) {
    constexpr int kRows = 32 * FN;
    const int64_t first = t0 + kRows * wb, v0 = (int64_t)vt0 * Tile::kEntries + 64 * wa;
    raise_rows((T*)p.z + first * p.ld_z + v0, p.ld_z, p.h_scale + first, (int)(p.T - first < kRows ? p.T - first : kRows), p.V - v0, 64,
               Tile::kEntries, tiles);
  }
}

static int check_quant(const adwin_opd_quant_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->x_dtype)) return ADWIN_E_MODE;
  if (p->N < 0 || p->N >= kMaxRows || p->H < 1 || p->H > ADWIN_QUANT_MAX_H || p->ld_x < p->H) return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

static int check_quant_logits(const adwin_opd_quant_logits_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->h_dtype) || !known_dtype(p->z_dtype)) return ADWIN_E_MODE;
  if (p->T < 0 || p->T >= kMaxRows || p->V < 1 || p->V > kMaxVocab || p->H < 1 || p->H > ADWIN_QUANT_MAX_H ||
      p->ld_h < p->H || p->ld_z < p->V)
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

// The tokens' integers and scales in the workspace.
struct QuantLayout {
  size_t o_scale, bytes;
  QuantLayout(int64_t T, int32_t H) {
    o_scale = align_up((size_t)T * ADWIN_QUANT_PITCH(H), 256);
    bytes = align_up(o_scale + sizeof(float) * (size_t)T, 256);
  }
};

// Groups of 16 tokens of the kernel for few tokens, 0 where tiles serve the call: as many as fit the LDS, at most 4, but for more than
// two where one or two tiles of 128 entries to a compute unit spread as well and are filled by the tokens.  us, few / tiles: 1 token,
// H = 1024, V = 1,000 7.5 / 10.2, V = 151,936 30.5 / 33.2, H = 4096, V = 4,000 11.5 / 19.3; 16 tokens, H = 4096, V = 16,000 21.4 / 21.1,
// H = 2048, V = 50,000 24.8 / 25.8; 30 tokens, H = 4096, V = 40,000 35.6 / 41.2; 40 tokens, H = 1024, V = 4,000 9.1 / 10.9,
// H = 2048, V = 16,000 14.3 / 14.7; 60 tokens, V = 30,000 22.1 / 18.1, V = 75,000 35.2 / 36.8, H = 1024, V = 60,000 21.5 / 19.7.
static int few_tokens(int64_t T, int32_t V, int pitch) {
  const int64_t n = (T + 15) / 16;
  const bool suits = n <= 2 || V <= 128 * 128 || V > 2 * 128 * 256;
  return n <= 4 && suits && few_lds((int)n, pitch) <= kQLds ? (int)n : 0;
}

template <typename T, int NT>
static hipError_t launch_few_n(const ProductArgs& a, hipStream_t st) {
  const int groups = (a.V + 15) / 16;
  int blocks = groups < 256 ? groups : 256;
  if ((groups + blocks - 1) / blocks > kFewGroups) blocks = (groups + kFewGroups - 1) / kFewGroups;
  quant_few_kernel<T, NT><<<blocks, kFewThreads, few_lds(NT, a.pitch), st>>>(a);
  return hipGetLastError();
}
template <typename T>
static hipError_t launch_few(const ProductArgs& a, int n, hipStream_t st) {
  switch (n) {
    case 1: return launch_few_n<T, 1>(a, st);
    case 2: return launch_few_n<T, 2>(a, st);
    case 3: return launch_few_n<T, 3>(a, st);
    default: return launch_few_n<T, 4>(a, st);
  }
}

template <typename T, int FN>
static hipError_t launch_mid(const ProductArgs& a, hipStream_t st) {
  ProductArgs b = a;
  b.token_tiles = (int32_t)((a.T + MidTile<FN>::kTokens - 1) / MidTile<FN>::kTokens);
  b.vocab_tiles = (a.V + 127) / 128;
  b.strips = product_strips(b.token_tiles, b.vocab_tiles);
  b.group = 4;
  quant_mid_kernel<T, FN><<<(unsigned)(b.token_tiles * b.strips), 256, MidTile<FN>::kLds, st>>>(b);
  return hipGetLastError();
}
// large dynamic LDS of the product, once per device
hipError_t quant_kernels_opt_in() {
  for (const void* k : {(const void*)quant_tile_kernel<uint16_t>, (const void*)quant_tile_kernel<float>,
                        (const void*)quant_mid_kernel<uint16_t, 1>, (const void*)quant_mid_kernel<uint16_t, 2>,
                        (const void*)quant_mid_kernel<float, 1>, (const void*)quant_mid_kernel<float, 2>,
                        (const void*)quant_few_kernel<uint16_t, 1>, (const void*)quant_few_kernel<uint16_t, 2>,
                        (const void*)quant_few_kernel<uint16_t, 3>, (const void*)quant_few_kernel<uint16_t, 4>,
                        (const void*)quant_few_kernel<float, 1>, (const void*)quant_few_kernel<float, 2>,
                        (const void*)quant_few_kernel<float, 3>, (const void*)quant_few_kernel<float, 4>}) {
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kQLds);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
static hipError_t quant_opt_in() { return once_on_device(kOnceQuant, quant_kernels_opt_in); }

static hipError_t launch_quant_rows(const QuantArgs& a, int32_t dtype, hipStream_t st) {
  const int64_t blocks = (a.N + 3) / 4;
  const int64_t size = dtype == ADWIN_DT_BF16 ? 2 : 4;
  const bool whole = ((uintptr_t)a.x & 15) == 0 && ((a.ld * size) & 15) == 0 && (a.H & 7) == 0;
  // past the caches from 96 MiB on: tokens of a product, which reads their integers, stay below.  us, kept / past, 4096 bf16 a row:
  // 16,000 rows 38.5 / 37.6, 30,000 rows 75 / 65, 151,936 rows 353 / 307
  const bool past = whole && a.N * a.H * size > ((int64_t)96 << 20);
#define ADWIN_LAUNCH(T)                                                                            \
  if (past) quant_rows_kernel<T, true, true><<<(unsigned)blocks, 256, 0, st>>>(a);                 \
  else if (whole) quant_rows_kernel<T, true, false><<<(unsigned)blocks, 256, 0, st>>>(a);          \
  else quant_rows_kernel<T, false, false><<<(unsigned)blocks, 256, 0, st>>>(a);
  if (dtype == ADWIN_DT_BF16) { ADWIN_LAUNCH(uint16_t) } else { ADWIN_LAUNCH(float) }
#undef ADWIN_LAUNCH
  return hipGetLastError();
}

}  // namespace adwin

using namespace adwin;

extern "C" int adwin_opd_quant_rows(const adwin_opd_quant_problem* p, void* hip_stream) {
  const int st = check_quant(p);
  if (st != ADWIN_OK) return st;
  if (p->N == 0) return ADWIN_OK;
  if (!p->x || !p->q || !p->scale) return ADWIN_E_NULL;
  if (((uintptr_t)p->x & entry_mask(p->x_dtype)) || ((uintptr_t)p->q & 15)) return ADWIN_E_ALIGN;
  const QuantArgs a{p->x, p->ld_x, p->N, p->H, ADWIN_QUANT_PITCH(p->H), p->q, p->scale, p->row_status};
  ADWIN_HIP_TRY(launch_quant_rows(a, p->x_dtype, (hipStream_t)hip_stream));
  return ADWIN_OK;
}

extern "C" int adwin_opd_quant_logits_workspace_bytes(const adwin_opd_quant_logits_problem* p, size_t* bytes) {
  if (!bytes) return ADWIN_E_NULL;
  const int st = check_quant_logits(p);
  if (st != ADWIN_OK) return st;
  *bytes = QuantLayout(p->T, p->H).bytes;
  return ADWIN_OK;
}

extern "C" int adwin_opd_quant_logits(const adwin_opd_quant_logits_problem* p, void* workspace, size_t workspace_bytes,
                                      void* hip_stream) {
  const int st = check_quant_logits(p);
  if (st != ADWIN_OK) return st;
  if (p->T == 0) return ADWIN_OK;
  if (!p->h || !p->W_q || !p->W_scale || !p->z) return ADWIN_E_NULL;
  if (((uintptr_t)p->h & entry_mask(p->h_dtype)) || ((uintptr_t)p->z & entry_mask(p->z_dtype)) || ((uintptr_t)p->W_q & 15))
    return ADWIN_E_ALIGN;
  const QuantLayout L(p->T, p->H);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < L.bytes) return ADWIN_E_WORKSPACE;
  hipStream_t stream = (hipStream_t)hip_stream;
  int8_t* q = (int8_t*)workspace;
  float* scale = (float*)((unsigned char*)workspace + L.o_scale);
  const QuantArgs rows{p->h, p->ld_h, p->T, p->H, ADWIN_QUANT_PITCH(p->H), q, scale, p->row_status};
  ADWIN_HIP_TRY(launch_quant_rows(rows, p->h_dtype, stream));
  ProductArgs a{};
  a.h = q; a.h_scale = scale; a.W = p->W_q; a.W_scale = p->W_scale; a.z = p->z; a.ld_z = p->ld_z; a.T = p->T; a.V = p->V;
  a.pitch = ADWIN_QUANT_PITCH(p->H);
  const int64_t size = p->z_dtype == ADWIN_DT_BF16 ? 2 : 4;
  a.whole = ((uintptr_t)p->z & 15) == 0 && (p->ld_z * size & 15) == 0;
  ADWIN_HIP_TRY(quant_opt_in());
  const int few = few_tokens(p->T, p->V, a.pitch);
  if (few > 0) {
    ADWIN_HIP_TRY(p->z_dtype == ADWIN_DT_BF16 ? launch_few<uint16_t>(a, few, stream) : launch_few<float>(a, few, stream));
    return ADWIN_OK;
  }
  if (const int way = product_tile(p->T, p->V, a.pitch, (int)size)) {
    const bool bf16 = p->z_dtype == ADWIN_DT_BF16;
    ADWIN_HIP_TRY(way == 1 ? (bf16 ? launch_mid<uint16_t, 1>(a, stream) : launch_mid<float, 1>(a, stream))
                           : (bf16 ? launch_mid<uint16_t, 2>(a, stream) : launch_mid<float, 2>(a, stream)));
    return ADWIN_OK;
  }
  const int64_t tiles = (p->T + kQTile - 1) / kQTile;
  a.token_tiles = (int32_t)tiles;
  a.vocab_tiles = (p->V + kQTile - 1) / kQTile;
  a.strips = product_strips(tiles, a.vocab_tiles);
  a.group = 4;
  const unsigned blocks = (unsigned)(tiles * a.strips);
  if (p->z_dtype == ADWIN_DT_BF16) quant_tile_kernel<uint16_t><<<blocks, 256, kQLds, stream>>>(a);
  else quant_tile_kernel<float><<<blocks, 256, kQLds, stream>>>(a);
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}
