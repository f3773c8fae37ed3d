// Rows to blocks of 8-bit floats with a power-of-two scale each, and the product of two arrays of such blocks.
#include "fused_shared.h"
#include "block_rule.h"
#include "product_shared.h"

namespace adwin {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------------------
// Rows to blocks.  Both formats' largest numbers are 1.75 * 2^k, k = 8 and 15: with a block's largest magnitude m * 2^x, 1 <= m < 2,
// the scale is 2^(x - k), or twice that where m > 1.75.
// ---------------------------------------------------------------------------------------
struct BlockRowsArgs {
  const void* x; int64_t ld; int64_t N;
  int32_t H, tile;
  int32_t along, across;
  uint8_t* q; uint8_t* scale; uint8_t* q_t; uint8_t* scale_t;
  int32_t* row_status; const int32_t* x_status;
  int64_t pitch, scales, pitch_t, scales_t;       // bytes from row to row
};

constexpr uint32_t kInfBits = 0x7f800000u;

template <int F8>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {      // most: bits of the largest magnitude, finite
  const int e = (int)(most >> 23) - (F8 == ADWIN_F8_E4M3 ? 8 : 15) + ((most & 0x7fffffu) > 0x600000u);
  return most == 0 || e < 0 ? 0 : (uint32_t)e;
}
// 1 / scale: 2^(127 - byte), byte <= 247
__device__ __forceinline__ float per_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four numbers to 8-bit floats, to nearest even; they lie within the format.
template <int F8>
__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d) {
  if constexpr (F8 == ADWIN_F8_E4M3)
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  else
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
}
template <int F8, typename T>
__device__ __forceinline__ uint2 block_entries(const Eight<T>& v, float per) {
  return make_uint2(pack_f8<F8>(v.entry(0) * per, v.entry(1) * per, v.entry(2) * per, v.entry(3) * per),
                    pack_f8<F8>(v.entry(4) * per, v.entry(5) * per, v.entry(6) * per, v.entry(7) * per));
}
// Where a magnitude (as bits) is inf, NaN or so large that its 8-bit float would stand for 2^128: 1.9375 * 2^127 and 1.875 * 2^127.
template <int F8>
constexpr uint32_t kFarBits = F8 == ADWIN_F8_E4M3 ? 0x7f780000u : 0x7f700000u;
// Rare: entries that are inf or NaN become 0, and those that are too large a number that leaves their block's scale as it is and
// rounds to the largest float that stands within fp32's range, 1.875 * 2^127 and 1.75 * 2^127.
template <int F8, typename T>
__device__ __forceinline__ void keep_within(Eight<T>& v) {
  constexpr uint32_t kCut = F8 == ADWIN_F8_E4M3 ? 0x7f700000u : 0x7f610000u;
#pragma unroll
  for (int i = 0; i < 4 * Eight<T>::kVecs; ++i) {
    uint32_t w = v.v[i >> 2][i & 3];
    if constexpr (sizeof(T) == 2) {
      const uint32_t lo = (w & 0x7fffu) << 16, hi = w & 0x7fff0000u;
      if (lo >= kFarBits<F8>) w = (w & 0xffff8000u) | (lo >= kInfBits ? 0u : kCut >> 16);
      if (hi >= kFarBits<F8>) w = (w & 0x8000ffffu) | (hi >= kInfBits ? 0u : kCut);
    } else {
      const uint32_t b = w & 0x7fffffffu;
      if (b >= kFarBits<F8>) w = (w & 0x80000000u) | (b >= kInfBits ? 0u : kCut);
    }
    v.v[i >> 2][i & 3] = w;
  }
}
// words of excluded rows, else zeros
__global__ __launch_bounds__(256) void begin_status_kernel(int32_t* status, const int32_t* excluded, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) status[i] = excluded ? excluded[i] : 0;
}

// The largest of the 16 lanes of a block, in all of them, by rotations within them, which take no turn of the LDS.
template <int BY>
__device__ __forceinline__ uint32_t max_rotated(uint32_t m) {
  const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x120 + BY, 0xf, 0xf, false);
  return b > m ? b : m;
}
__device__ __forceinline__ uint32_t max16(uint32_t m) { return max_rotated<1>(max_rotated<2>(max_rotated<4>(max_rotated<8>(m)))); }

template <bool PAST>
__device__ __forceinline__ void put8(uint8_t* p, uint2 q) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (PAST) __builtin_nontemporal_store(u32x2{q.x, q.y}, (u32x2*)p);
  else *(uint2*)p = q;
}

// Along the rows, a scale to each row's block: a wave takes four blocks of a row at a time, sixteen lanes to a block, kUnits times.  What
// bounds it is the memory: 30,000 x 4096 bf16 72 us (5.2 TB/s); 64 x 4096 3.6 us, a launch.
constexpr int kUnits = 4;
template <typename T, int F8, bool WHOLE, bool PAST>
__global__ __launch_bounds__(256) void block_rows_kernel(BlockRowsArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= p.N) return;
  const T* x = (const T*)p.x + n * p.ld;
  const int H = p.x_status && p.x_status[n] != 0 ? 0 : p.H;      // entries that are read
  const int c0 = (int)blockIdx.y * (512 * kUnits) + 8 * lane;
  Eight<T> v[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int c = c0 + 512 * u;
    v[u].clear();
    if constexpr (WHOLE) {
      if (c < H) v[u].template load<PAST>(x + c);
    } else if (c < H) {
      v[u].load_some(x + c, H - c);
    }
  }
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int c = c0 + 512 * u;
    uint32_t top = v[u].largest(0);
    if (top >= kFarBits<F8>) {
      bad = bad || top >= kInfBits;
      keep_within<F8>(v[u]);
      top = v[u].largest(0);
    }
    const uint32_t byte = scale_byte<F8>(max16(top));
    const uint2 q = block_entries<F8>(v[u], per_scale(byte));
    if (c < p.pitch) put8<PAST>(p.q + n * p.pitch + c, q);
    if ((lane & 15) == 0 && (c >> 7) < p.scales) p.scale[n * p.scales + (c >> 7)] = (uint8_t)byte;
  }
  if (p.row_status && __any(bad) && lane == 0) atomicOr(p.row_status + n, (int)ADWIN_DEV_NONFINITE);
}

// Tiles of 128 x 128: scales of tiles, and blocks across the rows.  A thread has eight entries of each of eight rows; what goes across
// is transposed in the LDS, whose rows (of eight-byte words) are shifted against each other.  A tile's lines of x, q and q_t are whole ones.
// What bounds it is the memory, and with a scale to each row and column the stores of single bytes, each a transaction: both ways 1,024 x 151,936
// bf16 124 us (5.0 TB/s), a head of 151,936 x 4096 in tiles 461 us (5.4 TB/s).
constexpr int kTransposed = 128 + 8;
template <typename T, int F8, bool WHOLE, bool PAST>
__global__ __launch_bounds__(256) void block_tile_kernel(BlockRowsArgs p) {
  __shared__ __align__(16) uint8_t turned[128 * kTransposed];
  __shared__ uint32_t most[4][128];
  const int tid = threadIdx.x, l = tid & 15, g = tid >> 4, lane = tid & 63, wave = tid >> 6;
  const uint32_t tiles = (uint32_t)(p.pitch / 128), down = blockIdx.x / tiles, right = blockIdx.x - down * tiles;
  const int64_t n0 = (int64_t)down * 128;
  const int c0 = (int)right * 128, c = c0 + 8 * l;
  uint32_t excluded = 0;                               // bits of the thread's rows
  if (p.x_status) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int64_t n = n0 + 8 * g + r;
      if (n < p.N && p.x_status[n] != 0) excluded |= 1u << r;
    }
  }
  Eight<T> v[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int64_t n = n0 + 8 * g + r;
    const T* x = (const T*)p.x + n * p.ld + c;
    v[r].clear();
    if (n < p.N && c < p.H && !(excluded >> r & 1)) {
      if constexpr (WHOLE) v[r].template load<PAST>(x);
      else v[r].load_some(x, p.H - c);
    }
  }
  uint32_t top[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    top[r] = v[r].largest(0);
    if (top[r] >= kFarBits<F8>) {
      const bool bad = top[r] >= kInfBits;
      keep_within<F8>(v[r]);
      top[r] = v[r].largest(0);
      if (bad && p.row_status) atomicOr(p.row_status + n0 + 8 * g + r, (int)ADWIN_DEV_NONFINITE);
    }
  }
  uint32_t byte[8];                                    // of the thread's rows
  if (p.tile == 1) {
    if (p.along) {
#pragma unroll
      for (int r = 0; r < 8; ++r) byte[r] = scale_byte<F8>(max16(top[r]));
    }
  } else {
    uint32_t m = top[0];
#pragma unroll
    for (int r = 1; r < 8; ++r) m = top[r] > m ? top[r] : m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint32_t b = __shfl_xor(m, o, 64);
      m = b > m ? b : m;
    }
    if (lane == 0) most[wave][0] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = most[w][0] > m ? most[w][0] : m;
    const uint32_t b = scale_byte<F8>(m);
#pragma unroll
    for (int r = 0; r < 8; ++r) byte[r] = b;
  }
  if (p.along) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int64_t n = n0 + 8 * g + r;
      if (n < p.N) {
        put8<PAST>(p.q + n * p.pitch + c, block_entries<F8>(v[r], per_scale(byte[r])));
        if (p.tile == 1 && l == 0) p.scale[n * p.scales + right] = (uint8_t)byte[r];
      }
    }
    // the scales' own bytes of a tile, and behind the last ones zeros
    const bool last = right + 1 == tiles;
    if (p.tile == 1) {
      if (last && tid < 128 && n0 + tid < p.N)
        for (int64_t k = (int64_t)right + 1; k < p.scales; ++k) p.scale[(n0 + tid) * p.scales + k] = 0;
    } else if (tid == 0) {
      p.scale[down * p.scales + right] = (uint8_t)byte[0];
      if (last)
        for (int64_t k = (int64_t)right + 1; k < p.scales; ++k) p.scale[down * p.scales + k] = 0;
    }
  }
  if (!p.across) return;
  uint32_t of[8];                                      // scales of the thread's columns
  if (p.tile == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t m = 0;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const uint32_t b = __float_as_uint(v[r].entry(e)) & 0x7fffffffu;
        m = b > m ? b : m;
      }
#pragma unroll
      for (int o = 16; o < 64; o <<= 1) {
        const uint32_t b = __shfl_xor(m, o, 64);
        m = b > m ? b : m;
      }
      if (lane < 16) most[wave][8 * l + e] = m;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t m = most[0][8 * l + e];
#pragma unroll
      for (int w = 1; w < 4; ++w) { const uint32_t b = most[w][8 * l + e]; m = b > m ? b : m; }
      of[e] = scale_byte<F8>(m);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) of[e] = byte[0];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float per = per_scale(of[e]);
    const uint32_t lo = pack_f8<F8>(v[0].entry(e) * per, v[1].entry(e) * per, v[2].entry(e) * per, v[3].entry(e) * per);
    const uint32_t hi = pack_f8<F8>(v[4].entry(e) * per, v[5].entry(e) * per, v[6].entry(e) * per, v[7].entry(e) * per);
    *(uint2*)(turned + (8 * l + e) * kTransposed + 8 * g) = make_uint2(lo, hi);
  }
  const bool last = n0 + 128 >= p.N;
  if (p.tile == 1) {
    if (g == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < p.H) {
          uint8_t* s = p.scale_t + (int64_t)(c + e) * p.scales_t;
          s[down] = (uint8_t)of[e];
          if (last)
            for (int64_t k = (int64_t)down + 1; k < p.scales_t; ++k) s[k] = 0;
        }
    }
  } else if (tid == 0) {
    uint8_t* s = p.scale_t + right * p.scales_t;
    s[down] = (uint8_t)of[0];
    if (last)
      for (int64_t k = (int64_t)down + 1; k < p.scales_t; ++k) s[k] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int col = 32 * k + (tid >> 3), at = 16 * (tid & 7);
    if (c0 + col < p.H) {
      const uint2 a = *(const uint2*)(turned + col * kTransposed + at), b = *(const uint2*)(turned + col * kTransposed + at + 8);
      const u32x4 o = {a.x, a.y, b.x, b.y};
      u32x4* to = (u32x4*)(p.q_t + (int64_t)(c0 + col) * p.pitch_t + n0 + at);
      if constexpr (PAST) __builtin_nontemporal_store(o, to);
      else *to = o;
    }
  }
}

// ---------------------------------------------------------------------------------------
// The product.  Rows of b are called entries and rows of a tokens: c is [tokens, entries].  For bf16 results, and the parts that are joined to
// such, the 8-bit instructions, at twice the rate: they cut each of eight products at 2^-13 of the largest's power of two before they add
// them to fp32, 1.4e-5 of c's norm for normal entries where rounding to bf16 takes 1.7e-3.  For fp32 results (EXACT) bf16's, which cut nothing.
// ---------------------------------------------------------------------------------------
struct BlockArgs {
  const uint8_t* a; const uint8_t* a_scale; const uint8_t* b; const uint8_t* b_scale;
  void* c; int64_t ld_c; int64_t M;
  const int32_t* a_status;
  int32_t N, pitch, scales;
  int32_t a_shift, b_shift;        // log2 of the rows of a block
  int32_t token_tiles, entry_tiles, strips, group;
  int32_t by_tokens;               // large tiles: a workgroup keeps its entries and walks a strip of token tiles
  int32_t splits;                  // parts of the contraction, each to its own [M][ld_c] of c
  int32_t whole;                   // rows of c lie and begin at multiples of 16 bytes
};

// Four bytes a lane: lane l moves the word at sbase + voff(l) to LDS address lds_base + 4 l.
__device__ __forceinline__ void dma4(uint32_t lds_base, uint32_t voff, const char* sbase) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :: "s"(lds_base), "v"(voff), "s"(sbase) : "memory");
}

// Sixteen 8-bit floats times a power of two, exactly, as bf16.
template <int F8>
__device__ __forceinline__ void widen(const i32x4& q, float scale, bf16x8 (&w)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2 lo, hi;
    if constexpr (F8 == ADWIN_F8_E4M3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)q[i], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)q[i], scale, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)q[i], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)q[i], scale, true);
    }
    w[i >> 1][4 * (i & 1) + 0] = lo[0]; w[i >> 1][4 * (i & 1) + 1] = lo[1];
    w[i >> 1][4 * (i & 1) + 2] = hi[0]; w[i >> 1][4 * (i & 1) + 3] = hi[1];
  }
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// 64 FN tokens x 128 entries, 2 x 2 waves of 64 x 32 FN.  A k-step is a block of 128 of either operand; kStages of them are in a ring in the
// LDS, all but one loading, each with a word of the scales of every row (the four blocks that the step's is one of).
// What bounds it is the read of b, or latency.  Strips begin at different blocks, so that rows a power of two apart do not ask the same channels at
// once: against 151,936 entries, K = 4096, bf16, 64 tokens 157 -> 129 us (4.8 TB/s), 128 tokens 175 -> 154, 1 token 137 -> 111.
// (us at other sizes stand with the rule that chooses it.)
// Chunk c of 16 bytes of row r lies at chunk position c ^ (r / 2 % 8), and tile row 8 q + 4 h + r of 32 holds entry 16 h + 4 q + r, which makes a lane's 16
// results of a block 16 consecutive entries of c.
template <int FN>
struct BlockTile {
  static constexpr int kEntries = 128, kTokens = 64 * FN;
  static constexpr int kBlockB = kEntries * 128, kScales = kBlockB + kTokens * 128, kStage = kScales + 4 * 256;
  static constexpr int kScratch = 4 * 4096;            // 32 tokens x 128 bytes of c for each wave
  static constexpr int kStages = (160 * 1024 - kScratch) / kStage;
  static constexpr int kLds = kStages * kStage + kScratch;
  static constexpr int kLoads = 5 + 2 * FN;            // of a wave and stage
};

template <typename T, int FN, int F8, bool EXACT>
__global__ __launch_bounds__(256) void block_mid_kernel(BlockArgs p) {
  typedef BlockTile<FN> Tile;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1, half = lane >> 5;
  int strip, tt;
  const int vid = xcd_contiguous_id(blockIdx.x, gridDim.x), per = p.token_tiles * p.strips, split = vid / per;
  strip_and_tile(vid - split * per, p.group, p.strips, p.token_tiles, &strip, &tt);
  const int vt0 = (int)((int64_t)p.entry_tiles * strip / p.strips), vt1 = (int)((int64_t)p.entry_tiles * (strip + 1) / p.strips);
  const int64_t t0 = (int64_t)tt * Tile::kTokens, T_left = p.M - t0;       // tokens from this tile on
  const int steps = p.pitch / 128, k0 = (int)((int64_t)steps * split / p.splits), k1 = (int)((int64_t)steps * (split + 1) / p.splits);
  const int tiles = vt1 - vt0, nk = k1 - k0;
  if (tiles <= 0 || nk <= 0) return;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16u;
  const int e0 = 16 * half + 4 * wave + ((lane >> 3) & 3);
  uint32_t voffb[4], voffa[2 * FN], voffs;
  const char* const a = (const char*)p.a + t0 * p.pitch;
  // Words of scales: waves 0 and 1 those of the tile's entries, in the order of its rows, 2 and 3 those of the tokens (wave 3 of 64
  // tokens the same ones as wave 2).
  const char* const sb = wave < 2 ? (const char*)p.b_scale : (const char*)p.a_scale;
  auto rows_of_b = [&](int tile) {                       // rows beyond N repeat the last one
    const int64_t first = (int64_t)tile * Tile::kEntries, left = p.N - first - 1;
#pragma unroll
    for (int d = 0; d < 4; ++d) voffb[d] = (uint32_t)(32 * d + e0 < left ? 32 * d + e0 : left) * (uint32_t)p.pitch + chunk;
    if (wave < 2) {
      const int i = lane & 31, e = 64 * wave + 32 * half + 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
      voffs = (uint32_t)((first + (e < left ? e : left)) >> p.b_shift) * (uint32_t)p.scales;
    }
  };
#pragma unroll
  for (int d = 0; d < 2 * FN; ++d) {
    const int64_t t = 32 * d + 8 * wave + (lane >> 3);
    voffa[d] = (uint32_t)(t < T_left ? t : T_left - 1) * (uint32_t)p.pitch + chunk;
  }
  if (wave >= 2) {
    const int64_t t = FN == 2 ? 64 * (wave - 2) + lane : lane;
    voffs = (uint32_t)((t0 + (t < T_left ? t : T_left - 1)) >> p.a_shift) * (uint32_t)p.scales;
  }
  uint32_t swB[4], swA[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const uint32_t at = (lane & 31) * 128u + (uint32_t)(((2 * kk + half) ^ (lane >> 1)) & 7) * 16u;
    swB[kk] = at + wa * (64 * 128);
    swA[kk] = at + Tile::kBlockB + wb * (32 * FN * 128);
  }
  bool dead[FN];                                         // tokens that are excluded
#pragma unroll
  for (int fn = 0; fn < FN; ++fn) {
    const int64_t t = 32 * FN * wb + 32 * fn + (lane & 31);
    int s = p.a_status ? p.a_status[t0 + (t < T_left ? t : T_left - 1)] : 0;
    asm volatile("" : "+v"(s));                          // waited for here
    dead[fn] = s != 0;
  }

  // where the next stage's loads come from: k-step kt of tile `tile` of the strip
  const int begin = k0 + strip % nk;                     // strips begin at different blocks: rows a power of two apart share channels
  int kt = begin, tile = 0;
  const char* tile_b = (const char*)p.b + (int64_t)vt0 * Tile::kEntries * p.pitch;
  uint32_t slot_w = lds0;
  rows_of_b(vt0);
  auto ask = [&]() __attribute__((always_inline)) {
    const char* from_b = tile_b + kt * 128;
    const char* from_a = a + kt * 128;
    const uint32_t to = slot_w + wave * 1024u;
#define B_LOAD(D) dma16_at<(D) * 4096>(to, voffb[D], from_b);
    B_LOAD(0) B_LOAD(1) B_LOAD(2) B_LOAD(3)
#undef B_LOAD
#define B_LOAD(D) if constexpr ((D) < 2 * FN) dma16_at<Tile::kBlockB + (D) * 4096>(to, voffa[(D) < 2 * FN ? (D) : 0], from_a);
    B_LOAD(0) B_LOAD(1) B_LOAD(2) B_LOAD(3)
#undef B_LOAD
    dma4(slot_w + Tile::kScales + wave * 256u, voffs, sb + (kt & ~3));
    slot_w += Tile::kStage;
    if (slot_w == lds0 + Tile::kStages * Tile::kStage) slot_w = lds0;
    if (++kt == k1) kt = k0;
    if (kt == begin) {                                   // behind the strip's last step its last tile again
      if (tile + 1 < tiles) {
        ++tile;
        tile_b += (int64_t)Tile::kEntries * p.pitch;
        rows_of_b(vt0 + tile);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < Tile::kStages - 1; ++s) ask();

  // where the lane stores: token lane / 8 of 32, 16 bytes
  constexpr int kPer = 16 / sizeof(T), kFms = sizeof(T) == 2 ? 2 : 1;     // blocks of 32 entries to 128 bytes
  const uint32_t scratch = lds0 + Tile::kStages * Tile::kStage + wave * 4096u;
  T* const c = (T*)p.c + ((int64_t)split * p.M + t0 + 32 * FN * wb + (lane >> 3)) * p.ld_c + (lane & 7) * kPer;
  const int rows_left = (int)(T_left < Tile::kTokens ? T_left : Tile::kTokens) - 32 * FN * wb - (lane >> 3);
  uint32_t slot = lds0;
  typedef const __attribute__((address_space(3))) uint32_t* LdsWord;
  constexpr int kYounger = (Tile::kStages - 2) * Tile::kLoads;
  static_assert(kYounger <= 63, "the wait counts to 63");
  for (int i = 0; i < tiles; ++i) {
    f32x16 acc[2][FN];
#pragma unroll
    for (int fm = 0; fm < 2; ++fm)
#pragma unroll
      for (int fn = 0; fn < FN; ++fn) acc[fm][fn] = f32x16{};
    for (int n = 0, k = begin; n < nk; ++n, k = k + 1 < k1 ? k + 1 : k0) {
      // this step has landed (loads return in order; stores of the tile before count as younger at worst), and every
      // wave has read the step before, whose slot the next loads fill
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kYounger) : "memory");
      __syncthreads();
      ask();
      i32x4 fb[4][2], fa[4][FN];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
        for (int f = 0; f < 2; ++f) fb[kk][f] = q_frag(slot + swB[kk], 32 * f);
#pragma unroll
        for (int f = 0; f < FN; ++f) fa[kk][f] = q_frag(slot + swA[kk], 32 * f);
      }
      uint32_t wb_[2], wa_[FN];                          // bytes of the scales
      const int shift = 8 * (k & 3);
#pragma unroll
      for (int f = 0; f < 2; ++f)
        wb_[f] = (((LdsWord)(uintptr_t)(slot + Tile::kScales))[64 * wa + 32 * f + (lane & 31)] >> shift) & 255u;
#pragma unroll
      for (int f = 0; f < FN; ++f)
        wa_[f] = (((LdsWord)(uintptr_t)(slot + Tile::kScales + 512))[32 * FN * wb + 32 * f + (lane & 31)] >> shift) & 255u;
      if constexpr (EXACT) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          bf16x8 b[2][2], t[FN][2];
#pragma unroll
          for (int f = 0; f < 2; ++f) widen<ADWIN_F8_E4M3>(fb[kk][f], scale_of(wb_[f]), b[f]);
#pragma unroll
          for (int f = 0; f < FN; ++f) widen<F8>(fa[kk][f], scale_of(wa_[f]), t[f]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int fm = 0; fm < 2; ++fm)
#pragma unroll
              for (int fn = 0; fn < FN; ++fn)
                acc[fm][fn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[fm][h], t[fn][h], acc[fm][fn], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < 4; kk += 2)
#pragma unroll
          for (int fm = 0; fm < 2; ++fm)
#pragma unroll
            for (int fn = 0; fn < FN; ++fn)
              acc[fm][fn] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                  __builtin_shufflevector(fb[kk][fm], fb[kk + 1][fm], 0, 1, 2, 3, 4, 5, 6, 7),
                  __builtin_shufflevector(fa[kk][fn], fa[kk + 1][fn], 0, 1, 2, 3, 4, 5, 6, 7), acc[fm][fn], 0, F8, 0, (int)wb_[fm], 0,
                  (int)wa_[fn]);
      }
      slot += Tile::kStage;
      if (slot == lds0 + Tile::kStages * Tile::kStage) slot = lds0;
    }
    const int64_t v0 = (int64_t)(vt0 + i) * Tile::kEntries + 64 * wa;
    const int64_t left = p.N - v0;                       // may be 0 or less
    if (left <= 0) continue;
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
          for (int e = 0; e < 16; ++e) y[e] = dead[fn] ? 0.f : acc[f0 + f][fn][e];
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
          T* at = c + (int64_t)(32 * fn + 8 * k) * p.ld_c + v0 + 32 * f0;
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
}

// ---------------------------------------------------------------------------------------
// Many tokens.  Tile of 256 entries x 256 tokens, 2 x 2 waves of 128 x 128 (256 accumulators).  A block of k (128 bytes of 256 rows of
// either operand, 64 KiB) is a stage of two in the LDS, laid out as in the smaller tiles.  A wave holds the fragments of half a block and
// reads those of the other half meanwhile; when every wave has all of block s, in the middle of its first half, its stage takes the loads of
// block s + 2, which have three quarters of a block (24 MFMAs, 1536 cycles) and more to land.  (Stages of half a block, four of them, ask for
// each line of memory twice, while it is still under way: 2.89 ms where this takes 2.42.)  A word of scales of every row, those of four
// blocks, comes when the first of these is loaded, in a ring of two of its own: a word for each block took 3.23 ms, as each of its lines holds
// one row's.
// A workgroup keeps its tokens and walks a strip of entry tiles; the blocks of all of them form one pipeline.  The order of the
// instructions is pinned, a read, a load or a piece of bookkeeping behind each MFMA; two loads behind one MFMA hold up the next, as the four waves
// then ask for more than a compute unit's 64 bytes a cycle (2.36 against 2.23 ms).
// 4,096 tokens, 151,936 entries, K = 4096, bf16: 2.00 to 2.12 ms over machines, 2.4 to 2.55 PFLOP/s; the matrix pipe is busy 60 % of the cycles
// at 1.84 GHz (power: with operands from registers alone it gives 3.7).  Where the barrier stands (8 to 13 of the 16 MFMAs) makes no difference.
// By the hidden states of 512 tokens, K = 151,936 in 16 parts: 148 us and 11 for their join.
// ---------------------------------------------------------------------------------------
constexpr int kBTile = 256;
constexpr uint32_t kBStage = 2 * kBTile * 128;         // entries, then tokens
constexpr uint32_t kBTokens = kBTile * 128;
constexpr uint32_t kBScales = 2 * kBStage;             // two of 2 KiB: words of entries, then of tokens
constexpr uint32_t kBScratch = kBScales + 2 * 2048;
constexpr int kBLds = (int)kBScratch + 4 * 4096;

// Where the loads of the block after next come from: block kt of tile `tile` of the strip.
struct BLoads {
  const char* b; const char* a;                        // of that block
  const char* b0; const char* a0;                      // of the first block of its tile
  const char* sb; const char* sa;                      // scales of the tile
  int kt, tile;
  uint32_t slot;                                       // of its scales
};
// From one tile of the strip to the next; 0 for the operand that the workgroup keeps.
struct BStride { int64_t b, a, sb, sa; };
// whether block kt begins a word of scales
__device__ __forceinline__ bool new_word(int kt, int k0) { return kt == k0 || (kt & 3) == 0; }

__device__ __forceinline__ uint32_t lds_byte(uint32_t addr) {
  return *(const __attribute__((address_space(3))) uint8_t*)(uintptr_t)addr;
}

struct BWave {                                         // what stays the same for a wave
  uint32_t swB[4], swA[4];                             // the lane's chunks of a stage
  uint32_t voffb[8], voffa[8], voffsb, voffsa;
  uint32_t word_b, word_a;                             // the lane's words of a block's scales
};

// One block.  r: its stage, of which the fragments of the first half are in registers; s: slot of its scales; next: the block after it;
// stores: of the tile before, which came behind the loads that the first block of a tile waits for and stay in flight.
template <int F8, bool FRESH>
__device__ __forceinline__ void b_step(f32x16 (&acc)[4][4], i32x4 (&fb)[2][4][2], i32x4 (&fa)[2][4][2], uint32_t (&eb)[4], uint32_t (&ea)[4],
                                       uint32_t& r, uint32_t& s, uint32_t lds0, uint32_t wave_kib, uint32_t wave_word, const BWave& w,
                                       BLoads& ld, int k0, int k1, int tiles, const BStride& to_next, int next, int stores) {
  const f32x16 zero = {};
  uint32_t at = 0, x[4], nb[4], na[4];
  const uint32_t nx = 2 * lds0 + kBStage - r, to = r + wave_kib;
  const uint32_t both = lds0 + kBScales + (lds0 + kBScales + 2048);      // the two slots' sum
  const uint32_t sn = new_word(next, k0) ? both - s : s;
#define B_FENCE __builtin_amdgcn_sched_barrier(0);
#define B_PAIR(F) __builtin_shufflevector(F[0], F[1], 0, 1, 2, 3, 4, 5, 6, 7)
#define B_MM(HH, I, J)                                                                                                     \
  acc[I][J] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(B_PAIR(fb[HH][I]), B_PAIR(fa[HH][J]),                        \
                                                              FRESH && (HH) == 0 ? zero : acc[I][J], 0, F8, 0, (int)eb[I], 0, (int)ea[J]); \
  B_FENCE
  // read R of the 16 of the other half: of entries and tokens in turn
#define B_READ(HH, R)                                                                                                      \
  {                                                                                                                        \
    constexpr int f = ((R) >> 2) & 3, j = (R) & 1;                                                                         \
    if constexpr (((R) & 2) == 0) fb[1 - (HH)][f][j] = q_frag(x[j], 32 * f);                                               \
    else fa[1 - (HH)][f][j] = q_frag(x[2 + j], 32 * f);                                                                    \
  }
  // load L of 16: the entries first, whose lines come from further away
#define B_LOAD(L)                                                                                                          \
  if constexpr ((L) >= 0 && (L) < 8) dma16_at<((L) & 7) * 4096>(to, w.voffb[(L) & 7], ld.b);                               \
  else if constexpr ((L) >= 8 && (L) < 16) dma16_at<(int)kBTokens + ((L) & 7) * 4096>(to, w.voffa[(L) & 7], ld.a);
  // behind MFMA M of half HH
#define B_SIDE(HH, M)                                                                                                      \
  if constexpr ((M) == 0) {                                                                                                \
    at = (HH) == 0 ? r : nx;                                                                                               \
    x[0] = at + w.swB[2 - 2 * (HH)]; x[1] = at + w.swB[3 - 2 * (HH)];                                                      \
    x[2] = at + w.swA[2 - 2 * (HH)]; x[3] = at + w.swA[3 - 2 * (HH)];                                                      \
    asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));                                                     \
  }                                                                                                                        \
  if constexpr ((HH) == 0 && (M) < 8) { B_READ(0, 2 * (M)) B_READ(0, 2 * (M) + 1) }                                        \
  if constexpr ((HH) == 1) { B_READ(1, M) }                                                                                \
  if constexpr ((HH) == 0 && (M) == 8) {                                                                                   \
    const bool wrap = ld.kt + 1 == k1, on = wrap && ld.tile + 1 < tiles;                                                   \
    ld.kt = wrap ? k0 : ld.kt + 1;                                                                                         \
    ld.tile += on;                                                                                                         \
    ld.b0 += on ? to_next.b : 0;                                                                                           \
    ld.a0 += on ? to_next.a : 0;                                                                                           \
    ld.sb += on ? to_next.sb : 0;                                                                                          \
    ld.sa += on ? to_next.sa : 0;                                                                                          \
    ld.b = wrap ? ld.b0 : ld.b + 128;                                                                                      \
    ld.a = wrap ? ld.a0 : ld.a + 128;                                                                                      \
  }                                                                                                                        \
  /* the next block has landed, and every wave has this one's fragments */                                                 \
  if constexpr ((HH) == 0 && (M) == 9) {                                                                                   \
    if (FRESH && stores == 32) asm volatile("s_waitcnt vmcnt(32) lgkmcnt(0)" ::: "memory");                                \
    else if (FRESH && stores == 64) asm volatile("s_waitcnt vmcnt(63) lgkmcnt(0)" ::: "memory");                           \
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");                                                       \
    __syncthreads();                                                                                                       \
  }                                                                                                                        \
  if constexpr ((HH) == 0 && (M) >= 10) { B_LOAD((M) - 10) }                                                               \
  if constexpr ((HH) == 1 && (M) < 10) { B_LOAD(6 + (M)) }                                                                 \
  if constexpr ((HH) == 1 && (M) == 10)                                                                                     \
    if (new_word(ld.kt, k0)) {                                                                                             \
      ld.slot = both - ld.slot;                                                                                            \
      dma4(ld.slot + wave_word, w.voffsb, ld.sb + (ld.kt & ~3));                                                           \
      dma4(ld.slot + 1024 + wave_word, w.voffsa, ld.sa + (ld.kt & ~3));                                                    \
    }                                                                                                                      \
  if constexpr ((HH) == 1 && (M) >= 12) {                                                                                  \
    constexpr int f = (M) & 3;                                                                                             \
    nb[f] = lds_byte(sn + w.word_b + 128 * f + (next & 3));                                                                \
    na[f] = lds_byte(sn + w.word_a + 128 * f + (next & 3));                                                                \
  }                                                                                                                        \
  B_FENCE
#define B_ROW(HH, I, M0)                                                                            \
  B_MM(HH, I, 0) B_SIDE(HH, (M0) + 0) B_MM(HH, I, 1) B_SIDE(HH, (M0) + 1)                           \
  B_MM(HH, I, 2) B_SIDE(HH, (M0) + 2) B_MM(HH, I, 3) B_SIDE(HH, (M0) + 3)
#define B_HALF(HH) B_ROW(HH, 0, 0) B_ROW(HH, 1, 4) B_ROW(HH, 2, 8) B_ROW(HH, 3, 12)
  B_FENCE
  B_HALF(0)
  B_HALF(1)
  r = nx;
  s = sn;
#pragma unroll
  for (int f = 0; f < 4; ++f) { eb[f] = nb[f]; ea[f] = na[f]; }
#undef B_HALF
#undef B_ROW
#undef B_SIDE
#undef B_LOAD
#undef B_READ
#undef B_MM
#undef B_PAIR
#undef B_FENCE
}

// The same for fp32 results: every eight-bit float goes through bf16, which holds it with its scale, and 32x32x16 instructions, whose products
// and sums are fp32's.  A quarter of a block (16 bytes a lane and fragment) is 32 MFMAs of 32 cycles: rows I of four fragments of tokens,
// lower and upper half.  Behind row I the entries' fragment of the next row is widened, behind rows 2 and 3 the tokens' of the next
// quarter; what is read from the LDS goes where the raw fragment before it has just been widened.  The loads of block s + 2 begin when all waves have
// read block s, behind the first MFMAs of its last quarter: those of the entries in that quarter, those of the tokens in the next.
// Gradient of a head of 151,936 x 2048 from 2,048 tokens: 0.98 to 1.08 ms, 1.2 to 1.3 PFLOP/s with 1.2 GB of results, where bf16 operands from
// registers alone give 1.7; the smaller tiles take 1.48.
struct XWave {
  i32x4 ra[4], rb[4];                                  // raw fragments
  i32x4 ca[2][4][2], cb[2][2];                         // widened ones
  float ea[4], eb[4];                                  // scales of the block
};

template <int F8, int SEL>
__device__ __forceinline__ int widen_pair(int word, float scale) {
  if constexpr (F8 == ADWIN_F8_E4M3) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)word, scale, SEL));
  else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)word, scale, SEL));
}

// As an instruction, which leaves the sum in its registers: of 256 of the builtin in one loop the compiler copied sums to and fro and
// spilled 580 registers.  Operands are written four instructions or more ahead.
__device__ __forceinline__ void mfma_bf16(f32x16& c, const i32x4& b, const i32x4& a) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}

template <int F8, typename Last>
__device__ __forceinline__ void x_step(f32x16 (&acc)[4][4], XWave& f, uint32_t& r, uint32_t& s, uint32_t lds0, uint32_t wave_kib,
                                       uint32_t wave_word, const BWave& w, BLoads& ld, int k0, int k1, int tiles, const BStride& to_next,
                                       int next, Last into_last) {
  uint32_t xb = 0, xa = 0, nb[4], na[4];
  float eb[4], ea[4];                                  // of the next block
  const uint32_t nx = 2 * lds0 + kBStage - r;
  const uint32_t both = lds0 + kBScales + (lds0 + kBScales + 2048);
  const uint32_t sn = new_word(next, k0) ? both - s : s;
#define X_FENCE __builtin_amdgcn_sched_barrier(0);
#define X_MM(KK, I, T)                                                                                                     \
  mfma_bf16(acc[I][(T) & 3], f.cb[(I) & 1][(T) >> 2], f.ca[(KK) & 1][(T) & 3][(T) >> 2]);   \
  X_FENCE
  // behind MFMA T of row I of quarter KK
#define X_SIDE(KK, I, T)                                                                                                   \
  {                                                                                                                        \
    constexpr int nk = ((KK) + 1) & 3, row = ((I) + 1) & 3, word = (T) >> 1;                                               \
    f.cb[row & 1][word >> 1][2 * (word & 1) + ((T) & 1)] =                                                                 \
        widen_pair<ADWIN_F8_E4M3, (T) & 1>(f.rb[row][word], (KK) == 3 && (I) == 3 ? eb[0] : f.eb[row]);                    \
    if constexpr ((I) >= 2) {                                                                                              \
      constexpr int g = 2 * ((I) & 1) + ((T) >> 2), q = (T) & 3;                                                           \
      const float e = (KK) == 3 ? ea[g] : f.ea[g];                                                                         \
      f.ca[nk & 1][g][q >> 1][2 * (q & 1)] = widen_pair<F8, 0>(f.ra[g][q], e);                                             \
      f.ca[nk & 1][g][q >> 1][2 * (q & 1) + 1] = widen_pair<F8, 1>(f.ra[g][q], e);                                         \
    }                                                                                                                      \
    if constexpr ((I) == 0 && (T) == 0) {                                                                                  \
      xb = ((KK) < 3 ? r : nx) + w.swB[nk];                                                                                \
      xa = ((KK) < 3 ? r : nx) + w.swA[nk];                                                                                \
      asm volatile("" : "+v"(xb), "+v"(xa));                                                                               \
    }                                                                                                                      \
    /* the next block has landed, and every wave has this one's fragments */                                               \
    if constexpr ((KK) == 3 && (I) == 0 && (T) == 1) {                                                                     \
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");                                                          \
      __syncthreads();                                                                                                     \
    }                                                                                                                      \
    if constexpr ((I) == 0 && (T) >= 2 && (T) < 6) f.ra[((T) - 2) & 3] = q_frag(xa, 32 * (((T) - 2) & 3));                 \
    if constexpr ((T) == 6) f.rb[I] = q_frag(xb, 32 * (I));                                                                \
    if constexpr ((KK) == 3 && (I) == 1 && (T) < 4) {                                                                      \
      nb[(T) & 3] = lds_byte(sn + w.word_b + 128 * ((T) & 3) + (next & 3));                                                \
      na[(T) & 3] = lds_byte(sn + w.word_a + 128 * ((T) & 3) + (next & 3));                                                \
    }                                                                                                                      \
    if constexpr ((KK) == 3 && (I) == 1 && (T) == 7) {                                                                     \
      _Pragma("unroll") for (int j = 0; j < 4; ++j) { eb[j] = scale_of(nb[j]); ea[j] = scale_of(na[j]); }                  \
    }                                                                                                                      \
    if constexpr ((KK) == 2 && (I) == 3 && (T) == 3) {                                                                     \
      const bool wrap = ld.kt + 1 == k1, on = wrap && ld.tile + 1 < tiles;                                                 \
      ld.kt = wrap ? k0 : ld.kt + 1;                                                                                       \
      ld.tile += on;                                                                                                       \
      ld.b0 += on ? to_next.b : 0;                                                                                         \
      ld.a0 += on ? to_next.a : 0;                                                                                         \
      ld.sb += on ? to_next.sb : 0;                                                                                        \
      ld.sa += on ? to_next.sa : 0;                                                                                        \
      ld.b = wrap ? ld.b0 : ld.b + 128;                                                                                    \
      ld.a = wrap ? ld.a0 : ld.a + 128;                                                                                    \
    }                                                                                                                      \
    constexpr int n = 8 * (I) + (T);                                                                                       \
    if constexpr ((KK) == 3 && n >= 4 && n < 28 && (n - 4) % 3 == 0)                                                       \
      dma16_at<(n - 4) / 3 % 8 * 4096>(r + wave_kib, w.voffb[(n - 4) / 3 % 8], ld.b);                                      \
    if constexpr ((KK) == 0 && n >= 3 && n < 27 && n % 3 == 0)                                                             \
      dma16_at<(int)kBTokens + (n - 3) / 3 % 8 * 4096>(nx + wave_kib, w.voffa[(n - 3) / 3 % 8], ld.a);                     \
    if constexpr ((KK) == 3 && n == 28)                                                                                    \
      if (new_word(ld.kt, k0)) {                                                                                           \
        ld.slot = both - ld.slot;                                                                                          \
        dma4(ld.slot + wave_word, w.voffsb, ld.sb + (ld.kt & ~3));                                                         \
        dma4(ld.slot + 1024 + wave_word, w.voffsa, ld.sa + (ld.kt & ~3));                                                  \
      }                                                                                                                    \
  }                                                                                                                        \
  X_FENCE
#define X_ROW(KK, I)                                                                                                       \
  X_MM(KK, I, 0) X_SIDE(KK, I, 0) X_MM(KK, I, 1) X_SIDE(KK, I, 1) X_MM(KK, I, 2) X_SIDE(KK, I, 2) X_MM(KK, I, 3) X_SIDE(KK, I, 3) \
  X_MM(KK, I, 4) X_SIDE(KK, I, 4) X_MM(KK, I, 5) X_SIDE(KK, I, 5) X_MM(KK, I, 6) X_SIDE(KK, I, 6) X_MM(KK, I, 7) X_SIDE(KK, I, 7)
#define X_QUARTER(KK) X_ROW(KK, 0) X_ROW(KK, 1) X_ROW(KK, 2) X_ROW(KK, 3)
  X_FENCE
  X_QUARTER(0)
  into_last();                                         // behind the loads of the block before it
  X_QUARTER(1)
  X_QUARTER(2)
  X_QUARTER(3)
  r = nx;
  s = sn;
#pragma unroll
  for (int j = 0; j < 4; ++j) { f.eb[j] = eb[j]; f.ea[j] = ea[j]; }
#undef X_QUARTER
#undef X_ROW
#undef X_SIDE
#undef X_MM
#undef X_FENCE
}

// An accumulator's number.  The constraint keeps it in its accumulator register until here.
__device__ __forceinline__ float held(float a) {
  float v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return v;
}

template <typename T, int F8, bool EXACT>
__global__ __launch_bounds__(256) void block_big_kernel(BlockArgs p) {
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave & 1, wb = wave >> 1, half = lane >> 5;
  int strip, fixed;
  const int fixed_tiles = p.by_tokens ? p.entry_tiles : p.token_tiles, walked = p.by_tokens ? p.token_tiles : p.entry_tiles;
  const int vid = xcd_contiguous_id(blockIdx.x, gridDim.x), per = fixed_tiles * p.strips, split = vid / per;
  strip_and_tile(vid - split * per, p.group, p.strips, fixed_tiles, &strip, &fixed);
  const int w0 = (int)((int64_t)walked * strip / p.strips), w1 = (int)((int64_t)walked * (strip + 1) / p.strips);
  const int vt0 = p.by_tokens ? fixed : w0, tt0 = p.by_tokens ? w0 : fixed;
  const int steps = p.pitch / 128, k0 = (int)((int64_t)steps * split / p.splits), k1 = (int)((int64_t)steps * (split + 1) / p.splits);
  const int tiles = w1 - w0;
  if (tiles <= 0 || k1 <= k0) return;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int64_t tile_bytes = (int64_t)kBTile * p.pitch, scales_b = (int64_t)(kBTile >> p.b_shift) * p.scales,
                scales_a = (int64_t)(kBTile >> p.a_shift) * p.scales;
  const BStride to_next = {p.by_tokens ? 0 : tile_bytes, p.by_tokens ? tile_bytes : 0, p.by_tokens ? 0 : scales_b, p.by_tokens ? scales_a : 0};

  BWave w;
  // a load instruction moves eight rows: those of the wave's are tile rows 32 d + 8 wave + lane / 8
  const uint32_t chunk = (uint32_t)((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16u;
  const int e0 = 16 * half + 4 * wave + ((lane >> 3) & 3);
  auto rows_of_b = [&](int tile) {                       // rows beyond N repeat the last one
    int left = p.N - tile * kBTile - 1;
    asm volatile("" : "+s"(left));                       // formed when it is needed, not kept ahead of it
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int v = 32 * d + e0;
      w.voffb[d] = (uint32_t)(v < left ? v : left) * (uint32_t)p.pitch + chunk;
      asm volatile("" : "+v"(w.voffb[d]));
    }
    const int i = lane & 31, v = 64 * wave + 32 * half + 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
    w.voffsb = (uint32_t)((v < left ? v : left) >> p.b_shift) * (uint32_t)p.scales;
    asm volatile("" : "+v"(w.voffsb));
  };
  auto rows_of_a = [&](int tile) {                       // rows beyond M repeat the last one
    int left = (int)p.M - tile * kBTile - 1;
    asm volatile("" : "+s"(left));
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int t = 32 * d + 8 * wave + (lane >> 3);
      w.voffa[d] = (uint32_t)(t < left ? t : left) * (uint32_t)p.pitch + chunk;
      asm volatile("" : "+v"(w.voffa[d]));
    }
    const int t = 64 * wave + lane;
    w.voffsa = (uint32_t)((t < left ? t : left) >> p.a_shift) * (uint32_t)p.scales;
    asm volatile("" : "+v"(w.voffsa));
  };
  rows_of_b(vt0);
  rows_of_a(tt0);
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const uint32_t at = (lane & 31) * 128u + (uint32_t)(((2 * kk + half) ^ (lane >> 1)) & 7) * 16u;
    w.swB[kk] = at + wa * (128 * 128);
    w.swA[kk] = at + kBTokens + wb * (128 * 128);
  }
  w.word_b = 4u * (128 * wa + (lane & 31));
  w.word_a = 1024u + 4u * (128 * wb + (lane & 31));

  BLoads ld;
  ld.b0 = (const char*)p.b + vt0 * tile_bytes + k0 * 128;
  ld.a0 = (const char*)p.a + tt0 * tile_bytes + k0 * 128;
  ld.sb = (const char*)p.b_scale + vt0 * scales_b;
  ld.sa = (const char*)p.a_scale + tt0 * scales_a;
  ld.b = ld.b0; ld.a = ld.a0; ld.kt = k0; ld.tile = 0; ld.slot = lds0 + kBScales;
  // the strip's tile that N, or M, ends in
  const int partial = (p.by_tokens ? (int)p.M : p.N) - w1 * kBTile < 0 ? tiles - 1 : -1;
  auto rows_of_partial = [&]() __attribute__((always_inline)) {
    if (p.by_tokens) rows_of_a(tt0 + partial);
    else rows_of_b(vt0 + partial);
  };
  const uint32_t wave_kib = wave * 1024u, wave_word = wave * 256u;
  // blocks 0 and 1
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (b == 1) {
      if (ld.kt + 1 < k1) { ++ld.kt; ld.b += 128; ld.a += 128; }
      else {
        if (tiles > 1) {
          ld.tile = 1; ld.b0 += to_next.b; ld.a0 += to_next.a; ld.sb += to_next.sb; ld.sa += to_next.sa;
          if (partial == 1) rows_of_partial();
        }
        ld.b = ld.b0; ld.a = ld.a0;
      }
    }
    const uint32_t to = lds0 + b * kBStage + wave_kib;
#define B_LOAD(D)                                          \
    dma16_at<(D) * 4096>(to, w.voffb[D], ld.b);            \
    if (!EXACT || b == 0) dma16_at<(int)kBTokens + (D) * 4096>(to, w.voffa[D], ld.a);
    B_LOAD(0) B_LOAD(1) B_LOAD(2) B_LOAD(3) B_LOAD(4) B_LOAD(5) B_LOAD(6) B_LOAD(7)
#undef B_LOAD
    if (b == 0 || new_word(ld.kt, k0)) {
      if (b == 1) ld.slot += 2048;
      dma4(ld.slot + wave_word, w.voffsb, ld.sb + (ld.kt & ~3));
      dma4(ld.slot + 1024 + wave_word, w.voffsa, ld.sa + (ld.kt & ~3));
    }
  }
  // block 0 and its scales: 16 loads or 18 are younger (8 or 10 where the first step loads the tokens of block 1)
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(EXACT ? 8 : 16) : "memory");
  __syncthreads();
  f32x16 acc[4][4];
  uint32_t r = lds0, s = lds0 + kBScales;
  [[maybe_unused]] i32x4 fb[2][4][2], fa[2][4][2];
  [[maybe_unused]] uint32_t eb[4], ea[4];
  [[maybe_unused]] XWave x;
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const uint32_t sb = lds_byte(s + w.word_b + 128 * f + (k0 & 3)), sa = lds_byte(s + w.word_a + 128 * f + (k0 & 3));
    if constexpr (EXACT) {
      x.rb[f] = q_frag(r + w.swB[0], 32 * f);
      x.ra[f] = q_frag(r + w.swA[0], 32 * f);
      x.eb[f] = scale_of(sb);
      x.ea[f] = scale_of(sa);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x.ca[0][f][q >> 1][2 * (q & 1)] = widen_pair<F8, 0>(x.ra[f][q], x.ea[f]);
        x.ca[0][f][q >> 1][2 * (q & 1) + 1] = widen_pair<F8, 1>(x.ra[f][q], x.ea[f]);
        if (f == 0) {
          x.cb[0][q >> 1][2 * (q & 1)] = widen_pair<ADWIN_F8_E4M3, 0>(x.rb[0][q], x.eb[0]);
          x.cb[0][q >> 1][2 * (q & 1) + 1] = widen_pair<ADWIN_F8_E4M3, 1>(x.rb[0][q], x.eb[0]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        fb[0][f][j] = q_frag(r + w.swB[j], 32 * f);
        fa[0][f][j] = q_frag(r + w.swA[j], 32 * f);
      }
      eb[f] = sb;
      ea[f] = sa;
    }
  }
  constexpr int kPer = 16 / sizeof(T), kFms = sizeof(T) == 2 ? 2 : 1;     // blocks of 32 entries to 128 bytes
  const uint32_t scratch = lds0 + kBScratch + wave * 4096u;
  T* const c = (T*)p.c + (int64_t)split * p.M * p.ld_c;
  const int64_t row_step = 8 * p.ld_c;
  int stores = 0;
  for (int i = 0; i < tiles; ++i) {
    // the loads of a block go into the tile that N, or M, ends in
    auto into_last = [&]() __attribute__((always_inline)) {
      if (ld.kt + 1 == k1 && ld.tile + 1 == partial) rows_of_partial();
    };
    if constexpr (EXACT) {
#pragma unroll
      for (int fm = 0; fm < 4; ++fm)
#pragma unroll
        for (int fn = 0; fn < 4; ++fn) {
          acc[fm][fn] = f32x16{};
          asm volatile("s_nop 1" : "+a"(acc[fm][fn]));   // written before an instruction that the compiler does not look into reads it
        }
      for (int kt = k0; kt < k1; ++kt)
        x_step<F8>(acc, x, r, s, lds0, wave_kib, wave_word, w, ld, k0, k1, tiles, to_next, kt + 1 < k1 ? kt + 1 : k0, into_last);
    } else {
      into_last();
      b_step<F8, true>(acc, fb, fa, eb, ea, r, s, lds0, wave_kib, wave_word, w, ld, k0, k1, tiles, to_next, k0 + 1 < k1 ? k0 + 1 : k0, stores);
      for (int kt = k0 + 1; kt < k1; ++kt) {
        into_last();
        b_step<F8, false>(acc, fb, fa, eb, ea, r, s, lds0, wave_kib, wave_word, w, ld, k0, k1, tiles, to_next, kt + 1 < k1 ? kt + 1 : k0, 0);
      }
    }
    // c, 32 tokens x 128 bytes of the wave at a time by way of the LDS, so that whole lines are stored
    const int64_t v0 = (int64_t)(vt0 + (p.by_tokens ? 0 : i)) * kBTile + 128 * wa, t0 = (int64_t)(tt0 + (p.by_tokens ? i : 0)) * kBTile + 128 * wb;
    const int64_t left = p.N - v0;                       // may be 0 or less
    const int rows_here = (int)(p.M - t0 < 128 ? p.M - t0 : 128);      // may be 0 or less
    stores = p.whole && left >= 128 && rows_here >= 128 ? 32 * (int)sizeof(T) / 2 : 0;
    if (left <= 0) continue;
    typedef __attribute__((address_space(3))) u32x4* LdsVec;
    int l = lane;
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last results are written: the compiler does not look into held()
    asm volatile("" : "+v"(l));                          // formed anew for every tile: the registers do not hold the addresses
    T* at = c + t0 * p.ld_c + v0 + (l >> 3) * p.ld_c + (l & 7) * kPer;
    const int rows = rows_here - (l >> 3);
    const uint32_t put = scratch + (l & 31) * 128u, get = scratch + (uint32_t)(l >> 3) * 128u;
#pragma unroll
    for (int fn = 0; fn < 4; ++fn)
#pragma unroll
      for (int f0 = 0; f0 < 4; f0 += kFms) {
#pragma unroll
        for (int f = 0; f < kFms; ++f) {
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = held(acc[f0 + f][fn][e]);
#pragma unroll
          for (int k = 0; k < 16 / kPer; ++k)
            *(LdsVec)(uintptr_t)(put + (uint32_t)((((f * 32 + 16 * (l >> 5)) / kPer + k) ^ (l >> 1)) & 7) * 16u) = pack16(y + k * kPer, T{});
        }
        u32x4 row[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)                      // row 8 k + l / 8
          row[k] = *(LdsVec)(uintptr_t)(get + k * 1024u + (uint32_t)(((l & 7) ^ (4 * k + (l >> 4))) & 7) * 16u);
        const int n = (int)(left < 128 ? left : 128) - 32 * f0 - (l & 7) * kPer;      // of the lane's entries
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (rows > 32 * fn + 8 * k) {
            if (p.whole && n >= kPer) *(u32x4*)(at + 32 * f0) = row[k];
            else {
#pragma unroll
              for (int e = 0; e < kPer; ++e)
                if (e < n) at[32 * f0 + e] = entry_of<T>(row[k], e);
            }
          }
          if (f0 + kFms == 4) at += row_step;
          else if (k < 3) at += row_step;
          else at -= 3 * row_step;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // loads that nobody reads may still be writing the LDS
  if (!p.a_status) return;
  uint64_t dead[2] = {0, 0};                             // of the wave's tokens: rare, their rows are written once more
#pragma unroll 1
  for (int i = 0; i < tiles; ++i) {
    const int64_t v0 = (int64_t)(vt0 + (p.by_tokens ? 0 : i)) * kBTile + 128 * wa, t0 = (int64_t)(tt0 + (p.by_tokens ? i : 0)) * kBTile + 128 * wb;
    if (i == 0 || p.by_tokens) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t t = t0 + 64 * j + lane;
        dead[j] = __ballot(t < p.M && p.a_status[t < p.M ? t : p.M - 1] != 0);
      }
      if (!p.by_tokens && (dead[0] | dead[1]) == 0) return;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll 1
      for (uint64_t left = dead[j]; left != 0; left &= left - 1) {
        T* row = c + (t0 + 64 * j + __ffsll((unsigned long long)left) - 1) * p.ld_c + v0;
        if (v0 + lane < p.N) row[lane] = T{};
        if (v0 + 64 + lane < p.N) row[64 + lane] = T{};
      }
  }
}

// ---------------------------------------------------------------------------------------
// Few tokens, fp32 results: every line of b is read once, and what bounds it is that read.  A workgroup to a compute unit has the tokens in its LDS, in the
// order of the fragments of the 16x16 instructions (lane l: row l % 16 of either operand, bytes 16 (l / 16) and 64 + 16 (l / 16) of a block;
// result e of lane l is row 4 (l / 16) + e of the first and row l % 16 of the second operand), with their scales behind them, and its 16 waves
// walk groups of 16 entries, whose rows come straight from memory into the registers, kAhead blocks under way, over the ends of groups as
// well.  Waves of a workgroup take its groups in turn and begin at different blocks of k, so that rows a power of two apart do not ask the same
// channels at once.  Where a workgroup has fewer than 16 groups, several waves share one and add up in the LDS, in their order.
// 1 token, 151,936 entries, K = 4096 113 us (5.5 TB/s).  (bf16 results, whose tiles have no bf16 to make, gain nothing: 111 us by either, 16
// tokens 120 and 116.)
// ---------------------------------------------------------------------------------------
constexpr int kFewThreads = 1024, kFewWaves = kFewThreads / 64;
constexpr int kAhead = 4;
__host__ __device__ constexpr int few_lds(int n, int pitch) {
  const int tokens = n * 16 * pitch + n * 16 * (pitch / 128), sums = kFewWaves * n * 1024;
  return tokens > sums ? tokens : sums;
}

template <int NT, int F8>
__global__ __launch_bounds__(kFewThreads) void block_few_kernel(BlockArgs p) {
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (p.N + 15) / 16;
  const int g0 = (int)((int64_t)groups * blockIdx.x / gridDim.x), g1 = (int)((int64_t)groups * (blockIdx.x + 1) / gridDim.x);
  const int nk = p.pitch / 128, here = g1 - g0;
  // waves to a group: a power of two
  int share = 1;
  while (share * 2 * here <= kFewWaves && share * 2 <= nk) share *= 2;
  const int lead = kFewWaves / share, first = wave / share, part = wave - first * share;       // groups at a time, this wave's, its part
  const int b0 = nk * part / share, b1 = nk * (part + 1) / share, blocks = b1 - b0;
  const int mine = first < here ? (here - first + lead - 1) / lead : 0;
  const int total = mine * blocks;

  // b: the lane's bytes of block k of group g
  const int turn = share == 1 ? (int)((blockIdx.x * kFewWaves + wave) % (uint32_t)nk) : 0;     // the block that the wave begins with
  int ahead_g = g0 + first, ahead_k = 0, asked = 0;
  const char* src = nullptr;
  const uint8_t* ssrc = nullptr;
  auto begin_group = [&](int g) {
    const int64_t v = (int64_t)g * 16 + (lane & 15), row = v < p.N ? v : p.N - 1;               // rows beyond N repeat the last one
    src = (const char*)p.b + row * p.pitch + (b0 + turn) * 128 + (lane >> 4) * 16;
    ssrc = p.b_scale + (row >> p.b_shift) * p.scales + b0 + turn;
  };
  i32x4 w[kAhead][2];
  uint32_t sw[kAhead];
  auto ask = [&](int j) __attribute__((always_inline)) {
    const i32x4* q = (const i32x4*)src;
    w[j][0] = q[0];
    w[j][1] = q[4];
    sw[j] = *ssrc;
    // the wave's last block is asked for again instead of one beyond it
    if (++asked < total) {
      src += 128;
      ++ssrc;
      if (++ahead_k == blocks - turn) { src -= blocks * 128; ssrc -= blocks; }
      if (ahead_k == blocks) {
        ahead_k = 0;
        ahead_g += lead;
        begin_group(ahead_g);
      }
    }
  };
  // the tokens: block k, half h of group n at 1024 ((2 k + h) NT + n), by direct loads.  Rows beyond M are not loaded: they enter
  // results that are not stored, and no others.
  uint32_t from[NT];
  bool dead[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t t = n * 16 + (lane & 15), row = t < p.M ? t : p.M - 1;
    from[n] = (uint32_t)row * (uint32_t)p.pitch + (lane >> 4) * 16u;
    dead[n] = p.a_status && p.a_status[row] != 0;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  uint8_t* const scales = (uint8_t*)lds + NT * 16 * p.pitch;     // [block][token]
  constexpr int kWords = 2 * NT;                         // of a thread, at 128 blocks
  uint32_t sa[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const int q = i * kFewThreads + threadIdx.x, k = q / (16 * NT), t = q - k * (16 * NT);
    sa[i] = 0;
    if (k < nk && t < p.M) sa[i] = p.a_scale[(int64_t)(t >> p.a_shift) * p.scales + k];
  }
  for (int k = wave; k < 2 * nk; k += kFewWaves)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (n * 16 + (lane & 15) < p.M) dma16_at<0>(lds0 + (uint32_t)(k * NT + n) * 1024u, from[n], (const char*)p.a + k * 64);
  if (total > 0) {
    begin_group(ahead_g);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ask(j);
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const int q = i * kFewThreads + threadIdx.x;
    if (q < nk * 16 * NT) scales[q] = (uint8_t)sa[i];
  }
  // loads return in order: the tokens are there when no more than what was asked for behind them is under way
  if (total > 0) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * kAhead) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{};
  auto store = [&](int g) __attribute__((always_inline)) {
    const int v = g * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t t = n * 16 + (lane & 15);
      const float y[4] = {dead[n] ? 0.f : acc[n][0], dead[n] ? 0.f : acc[n][1], dead[n] ? 0.f : acc[n][2], dead[n] ? 0.f : acc[n][3]};
      if (t < p.M) {
        float* c = (float*)p.c + t * p.ld_c + v;
        if (p.whole && v + 4 <= p.N) put_entries<false>(c, y, true);
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < p.N) c[e] = y[e];
        }
      }
      acc[n] = f32x4{};
    }
  };
  int k = 0, g = g0 + first, kb = b0 + turn;                     // kb: the block
  for (int at = 0; at < total; at += kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (at + j < total) {
        const char* frag = lds + lane * 16 + kb * (2 * NT * 1024);
        bf16x8 wide[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) widen<ADWIN_F8_E4M3>(w[j][h], scale_of(sw[j]), wide[h]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float scale = scale_of(scales[kb * 16 * NT + n * 16 + (lane & 15)]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            bf16x8 t[2];
            widen<F8>(*(const i32x4*)(frag + (h * NT + n) * 1024), scale, t);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[h][i], t[i], acc[n], 0, 0, 0);
          }
        }
        ++kb;
      }
      ask(j);
      if (at + j < total && ++k == blocks - turn) kb = b0;
      if (share == 1 && at + j < total && k == blocks) {
        store(g);
        k = 0;
        g += lead;
        kb = b0 + turn;
      }
    }
  }
  if (share == 1) return;
  // one group to a wave, or none: its parts in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  f32x4* sums = (f32x4*)lds;
#pragma unroll
  for (int n = 0; n < NT; ++n) sums[(wave * NT + n) * 64 + lane] = acc[n];
  __syncthreads();
  if (part != 0 || mine == 0) return;
#pragma unroll
  for (int n = 0; n < NT; ++n)
    for (int q = 1; q < share; ++q) acc[n] += sums[((wave + q) * NT + n) * 64 + lane];
  store(g0 + first);
}

// The parts of a contraction, added in their order.
struct JoinArgs {
  const float* part; int64_t ld_part, M;
  void* c; int64_t ld_c;
  int32_t N, splits;
};
template <typename T>
__global__ __launch_bounds__(256) void join_block_kernel(JoinArgs p) {
  const int n = 4 * ((int)blockIdx.x * 256 + (int)threadIdx.x);
  if (n >= p.N) return;
  for (int64_t m = blockIdx.y; m < p.M; m += gridDim.y) {
    const float* q = p.part + m * p.ld_part + n;
    float4 s = *(const float4*)q;
    for (int i = 1; i < p.splits; ++i) {
      q += p.M * p.ld_part;
      const float4 v = *(const float4*)q;
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float y[4] = {s.x, s.y, s.z, s.w};
    T* c = (T*)p.c + m * p.ld_c + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < p.N) Entry<T>::put(c + e, y[e]);
  }
}

// ---- host -----------------------------------------------------------------------------
static bool known_f8(int32_t f) { return f == ADWIN_F8_E4M3 || f == ADWIN_F8_E5M2; }
static bool known_tile(int32_t t) { return t == 1 || t == 128; }

static int check_rows(const adwin_opd_block_rows_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_dtype(p->x_dtype) || !known_f8(p->f8) || !known_tile(p->tile)) return ADWIN_E_MODE;
  if (p->N < 0 || p->N >= kMaxRows || p->H < 1 || p->H > ADWIN_BLOCK_MAX_K || p->ld_x < p->H ||
      (p->q_t && p->N > ADWIN_BLOCK_MAX_K))
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}
static int check_product(const adwin_opd_block_product_problem* p) {
  if (!p) return ADWIN_E_NULL;
  if (p->struct_bytes != sizeof(*p) || !known_f8(p->a_f8) || p->b_f8 != ADWIN_F8_E4M3 || !known_tile(p->a_tile) ||
      !known_tile(p->b_tile) || !known_dtype(p->c_dtype))
    return ADWIN_E_MODE;
  if (p->M < 0 || p->M >= kMaxRows || p->N < 0 || p->N >= kMaxRows || p->K < 1 || p->K > ADWIN_BLOCK_MAX_K || p->ld_c < p->N)
    return ADWIN_E_SHAPE;
  return ADWIN_OK;
}

// Groups of 16 tokens of the kernel for few tokens, 0 where tiles serve the call: fp32 results of up to 32 tokens as far as they fit the LDS,
// where b is large or the sums are short.  us, few / tiles, fp32, 1 token: K = 4096, V = 16,000 17.5 / 17.1, 30,000 24.6 / 25.0,
// 35,000 24.8 / 36, 45,000 31 / 39, 75,000 50 / 69, 151,936 113 / 133; K = 2048, V = 60,000 25.2 / 25.6, 80,000 30 / 36, 151,936 53 / 64;
// K = 10,000, V = 14,000 30.4 / 30.1, 18,000 34 / 46; K = 1280, V = 100,000 24.5 / 31.3; K = 1024, V = 4,000 6.9 / 8.6, 50,000 14.3 / 15.6.  32 tokens:
// K = 4096, V = 16,000 21 / 19, 30,000 28.5 / 24.3, 35,000 29 / 39, 45,000 35 / 42, 151,936 133 / 133; K = 2048, V = 60,000 27.3 / 26.5,
// 80,000 32 / 37, 151,936 66 / 72.  16 tokens, K = 10,000, V = 14,000 33 / 31.
static int few_tokens(const adwin_opd_block_product_problem* p) {
  const int64_t n = (p->M + 15) / 16;
  const int pitch = ADWIN_BLOCK_PITCH(p->K);
  if (p->c_dtype != ADWIN_DT_F32 || n < 1 || n > 2 || p->N < 1 || pitch > 16384 || few_lds((int)n, pitch) > 160 * 1024) return 0;
  return p->N * pitch >= (int64_t)128 << 20 || pitch <= 1024 ? (int)n : 0;
}

// How a product is served: by the kernel for few tokens (fn < 0), or by tiles of 64 fn tokens, its contraction in `splits` parts.
struct BlockWay {
  int fn, splits;
  size_t bytes;                    // of the parts
  explicit BlockWay(const adwin_opd_block_product_problem* p) {
    fn = -few_tokens(p);
    splits = 1;
    if (fn == 0 && p->M > 0 && p->N > 0) {
      const BlockChoice c = block_choice(p->M, p->N, ADWIN_BLOCK_PITCH(p->K), p->c_dtype == ADWIN_DT_F32);
      fn = c.fn;
      splits = c.splits;
    }
    bytes = splits > 1 ? align_up((size_t)splits * p->M * align_up((size_t)p->N, 4) * sizeof(float), 256) : 0;
  }
};

template <typename T, int FN, int F8, bool EXACT>
static hipError_t launch_block_mid(const BlockArgs& a, hipStream_t st) {
  BlockArgs b = a;
  b.token_tiles = (int32_t)((a.M + BlockTile<FN>::kTokens - 1) / BlockTile<FN>::kTokens);
  b.entry_tiles = (a.N + 127) / 128;
  b.strips = product_strips((int64_t)b.token_tiles * a.splits, b.entry_tiles);
  b.group = 4;
  block_mid_kernel<T, FN, F8, EXACT><<<(unsigned)((int64_t)b.token_tiles * b.strips * a.splits), 256, BlockTile<FN>::kLds, st>>>(b);
  return hipGetLastError();
}
template <typename T, int F8, bool EXACT>
static hipError_t launch_block_big(const BlockArgs& a, hipStream_t st) {
  BlockArgs b = a;
  b.token_tiles = (int32_t)((a.M + kBTile - 1) / kBTile);
  b.entry_tiles = (a.N + kBTile - 1) / kBTile;
  // What is walked: the strips that give the busiest compute unit the fewest tiles, and of as good ones the fewest workgroups, each of which
  // fills its pipeline anew.  594 x 8 tiles of 16 blocks, fp32: 8 strips of single entry tiles 1,112 us, 32 strips of 18 or 19 token tiles 1,065.
  int64_t turns_e, turns_t;
  const int strips_e = product_strips((int64_t)b.token_tiles * a.splits, b.entry_tiles, &turns_e);
  const int strips_t = product_strips((int64_t)b.entry_tiles * a.splits, b.token_tiles, &turns_t);
  const int64_t all_e = (int64_t)b.token_tiles * a.splits * strips_e, all_t = (int64_t)b.entry_tiles * a.splits * strips_t;
  b.by_tokens = turns_t < turns_e || (turns_t == turns_e && (all_t + 255) / 256 < (all_e + 255) / 256);
  b.strips = b.by_tokens ? strips_t : strips_e;
  b.group = 4;
  block_big_kernel<T, F8, EXACT><<<(unsigned)(b.by_tokens ? all_t : all_e), 256, kBLds, st>>>(b);
  return hipGetLastError();
}
template <int NT>
static hipError_t launch_block_few(const BlockArgs& a, int f8, hipStream_t st) {
  const int groups = (a.N + 15) / 16, blocks = groups < 256 ? groups : 256;
  if (f8 == ADWIN_F8_E4M3) block_few_kernel<NT, ADWIN_F8_E4M3><<<blocks, kFewThreads, few_lds(NT, a.pitch), st>>>(a);
  else block_few_kernel<NT, ADWIN_F8_E5M2><<<blocks, kFewThreads, few_lds(NT, a.pitch), st>>>(a);
  return hipGetLastError();
}
template <typename T, bool EXACT>
static hipError_t launch_block(const BlockArgs& a, int fn, int f8, hipStream_t st) {
  if constexpr (EXACT)
    if (fn < 0) return fn == -1 ? launch_block_few<1>(a, f8, st) : launch_block_few<2>(a, f8, st);      // never cut
  if (fn == 4) return f8 == ADWIN_F8_E4M3 ? launch_block_big<T, ADWIN_F8_E4M3, EXACT>(a, st) : launch_block_big<T, ADWIN_F8_E5M2, EXACT>(a, st);
  if (f8 == ADWIN_F8_E4M3)
    return fn == 1 ? launch_block_mid<T, 1, ADWIN_F8_E4M3, EXACT>(a, st) : launch_block_mid<T, 2, ADWIN_F8_E4M3, EXACT>(a, st);
  return fn == 1 ? launch_block_mid<T, 1, ADWIN_F8_E5M2, EXACT>(a, st) : launch_block_mid<T, 2, ADWIN_F8_E5M2, EXACT>(a, st);
}

// large dynamic LDS, once per device
template <typename T, bool EXACT>
static hipError_t opt_in_types() {
  if constexpr (EXACT)
    for (const void* k : {(const void*)block_few_kernel<1, 0>, (const void*)block_few_kernel<2, 0>, (const void*)block_few_kernel<1, 1>,
                          (const void*)block_few_kernel<2, 1>}) {
      const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
      if (e != hipSuccess) return e;
    }
  for (const void* k : {(const void*)block_mid_kernel<T, 1, 0, EXACT>, (const void*)block_mid_kernel<T, 2, 0, EXACT>,
                        (const void*)block_mid_kernel<T, 1, 1, EXACT>, (const void*)block_mid_kernel<T, 2, 1, EXACT>,
                        (const void*)block_big_kernel<T, 0, EXACT>, (const void*)block_big_kernel<T, 1, EXACT>}) {
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
hipError_t block_kernels_opt_in() {
  hipError_t e = opt_in_types<uint16_t, false>();
  if (e == hipSuccess) e = opt_in_types<float, false>();
  if (e == hipSuccess) e = opt_in_types<float, true>();
  return e;
}

}  // namespace adwin

using namespace adwin;

extern "C" int adwin_opd_block_rows(const adwin_opd_block_rows_problem* p, void* hip_stream) {
  const int st = check_rows(p);
  if (st != ADWIN_OK) return st;
  if (p->N == 0) return ADWIN_OK;
  if ((ADWIN_BLOCK_PITCH((int64_t)p->H) / 128) * ((p->N + 127) / 128) >= (int64_t)1 << 24) return ADWIN_E_SHAPE;    // a launch holds no more
  if (!p->x || !p->q != !p->scale || !p->q_t != !p->scale_t || (!p->q && !p->q_t)) return ADWIN_E_NULL;
  if (((uintptr_t)p->x & entry_mask(p->x_dtype)) || (((uintptr_t)p->q | (uintptr_t)p->q_t | (uintptr_t)p->scale | (uintptr_t)p->scale_t) & 15))
    return ADWIN_E_ALIGN;
  // words of row_status are set while others are still asked for whether their row is excluded
  if (p->row_status && p->x_status && p->row_status < p->x_status + p->N && p->x_status < p->row_status + p->N) return ADWIN_E_ALIGN;
  hipStream_t stream = (hipStream_t)hip_stream;
  BlockRowsArgs a{};
  a.x = p->x; a.ld = p->ld_x; a.N = p->N; a.H = p->H; a.tile = p->tile;
  a.along = p->q != nullptr; a.across = p->q_t != nullptr;
  a.q = p->q; a.scale = p->scale; a.q_t = p->q_t; a.scale_t = p->scale_t; a.row_status = p->row_status; a.x_status = p->x_status;
  a.pitch = ADWIN_BLOCK_PITCH((int64_t)p->H); a.scales = ADWIN_BLOCK_SCALES((int64_t)p->H);
  a.pitch_t = ADWIN_BLOCK_PITCH(p->N); a.scales_t = ADWIN_BLOCK_SCALES(p->N);
  const int64_t size = p->x_dtype == ADWIN_DT_BF16 ? 2 : 4;
  const bool whole = ((uintptr_t)a.x & 15) == 0 && ((a.ld * size) & 15) == 0 && (a.H & 7) == 0;
  // past the caches from 96 MiB of bf16 on, and from 256 of fp32 along the rows.  us, past / kept: bf16 30,000 x 4096 72 / 75, both ways
  // 1,024 x 151,936 124 / 134, 151,936 x 4096 in tiles 461 / 481 (along alone 318 / 344); fp32 along the rows 15,000 x 4096 58 / 50,
  // 18,000 69 / 75, 30,000 114 / 132, 151,936 x 2048 269 / 289, both ways 30,000 x 4096 145 / 142, in tiles 137 / 141
  const bool alone = a.tile == 1 && !a.across;
  const bool past = whole && (size == 2 || alone) && a.N * a.H * size > ((int64_t)(size == 2 ? 96 : 256) << 20);
  if (a.row_status) {
    begin_status_kernel<<<(unsigned)((a.N + 255) / 256), 256, 0, stream>>>(a.row_status, a.x_status, a.N);
    ADWIN_HIP_TRY(hipGetLastError());
  }
  // PAST: whether `past` occurs
#define ADWIN_LAUNCH_T(KERNEL, GRID, T, F8, PAST)                               \
  if (PAST && past) KERNEL<T, F8, true, PAST><<<GRID, 256, 0, stream>>>(a);     \
  else if (whole) KERNEL<T, F8, true, false><<<GRID, 256, 0, stream>>>(a);      \
  else KERNEL<T, F8, false, false><<<GRID, 256, 0, stream>>>(a);
#define ADWIN_LAUNCH(KERNEL, GRID, PAST_F32)                                            \
  if (p->x_dtype == ADWIN_DT_BF16) {                                                    \
    if (p->f8 == ADWIN_F8_E4M3) { ADWIN_LAUNCH_T(KERNEL, GRID, uint16_t, 0, true) }     \
    else { ADWIN_LAUNCH_T(KERNEL, GRID, uint16_t, 1, true) }                            \
  } else {                                                                              \
    if (p->f8 == ADWIN_F8_E4M3) { ADWIN_LAUNCH_T(KERNEL, GRID, float, 0, PAST_F32) }    \
    else { ADWIN_LAUNCH_T(KERNEL, GRID, float, 1, PAST_F32) }                           \
  }
  if (alone) {
    const dim3 grid((unsigned)((a.N + 3) / 4), (unsigned)((a.pitch + 512 * kUnits - 1) / (512 * kUnits)));
    ADWIN_LAUNCH(block_rows_kernel, grid, true)
  } else {
    const dim3 grid((unsigned)(a.pitch / 128 * ((a.N + 127) / 128)));
    ADWIN_LAUNCH(block_tile_kernel, grid, false)
  }
#undef ADWIN_LAUNCH
#undef ADWIN_LAUNCH_T
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}

extern "C" int adwin_opd_block_product_workspace_bytes(const adwin_opd_block_product_problem* p, size_t* bytes) {
  if (!bytes) return ADWIN_E_NULL;
  const int st = check_product(p);
  if (st != ADWIN_OK) return st;
  *bytes = BlockWay(p).bytes;
  return ADWIN_OK;
}

extern "C" int adwin_opd_block_product(const adwin_opd_block_product_problem* p, void* workspace, size_t workspace_bytes,
                                       void* hip_stream) {
  const int st = check_product(p);
  if (st != ADWIN_OK) return st;
  if (p->M == 0 || p->N == 0) return ADWIN_OK;
  if (!p->a || !p->a_scale || !p->b || !p->b_scale || !p->c) return ADWIN_E_NULL;
  if ((((uintptr_t)p->a | (uintptr_t)p->a_scale | (uintptr_t)p->b | (uintptr_t)p->b_scale) & 15) ||
      ((uintptr_t)p->c & entry_mask(p->c_dtype)))
    return ADWIN_E_ALIGN;
  const BlockWay way(p);
  if (way.bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < way.bytes)) return ADWIN_E_WORKSPACE;
  hipStream_t stream = (hipStream_t)hip_stream;
  ADWIN_HIP_TRY(once_on_device(kOnceBlocks, block_kernels_opt_in));
  BlockArgs a{};
  a.a = p->a; a.a_scale = p->a_scale; a.b = p->b; a.b_scale = p->b_scale; a.a_status = p->a_status;
  a.M = p->M; a.N = (int32_t)p->N; a.pitch = ADWIN_BLOCK_PITCH(p->K); a.scales = ADWIN_BLOCK_SCALES(p->K);
  a.a_shift = p->a_tile == 1 ? 0 : 7; a.b_shift = p->b_tile == 1 ? 0 : 7; a.splits = way.splits;
  const int64_t size = p->c_dtype == ADWIN_DT_BF16 ? 2 : 4;
  const bool bf16 = p->c_dtype == ADWIN_DT_BF16;
  if (way.splits == 1) {
    a.c = p->c; a.ld_c = p->ld_c;
    a.whole = ((uintptr_t)p->c & 15) == 0 && (p->ld_c * size & 15) == 0;
    ADWIN_HIP_TRY((bf16 ? launch_block<uint16_t, false>(a, way.fn, p->a_f8, stream) : launch_block<float, true>(a, way.fn, p->a_f8, stream)));
    return ADWIN_OK;
  }
  a.c = workspace; a.ld_c = (int64_t)align_up((size_t)p->N, 4); a.whole = 1;
  ADWIN_HIP_TRY((bf16 ? launch_block<float, false>(a, way.fn, p->a_f8, stream) : launch_block<float, true>(a, way.fn, p->a_f8, stream)));
  const JoinArgs j{(const float*)workspace, a.ld_c, p->M, p->c, p->ld_c, (int32_t)p->N, way.splits};
  const dim3 grid((unsigned)((p->N + 1023) / 1024), (unsigned)(p->M < 32768 ? p->M : 32768));
  if (bf16) join_block_kernel<uint16_t><<<grid, 256, 0, stream>>>(j);
  else join_block_kernel<float><<<grid, 256, 0, stream>>>(j);
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}
