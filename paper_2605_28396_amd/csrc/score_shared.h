// What the token-scoring kernels share: entries of bf16 or fp32, rows at any address.
#pragma once
#include "common.h"
#include "device_utils.h"

namespace adwin {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row: 8 entries of bf16, 4 of fp32.
template <typename T> struct Entry;
template <> struct Entry<uint16_t> {               // bf16
  static constexpr int kPerVec = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }   // -inf
  static __device__ __forceinline__ float one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
  static __device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16(x, 0.f); }
};
template <> struct Entry<float> {
  static constexpr int kPerVec = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
};

// y[0, N) to p: whole when p is a multiple of the bytes that they take (at most 16).  PAST: past the caches, but for 32 bytes, whose two
// halves are whole lines only when a cache has joined them (4,000 x 151,936 from bf16 to fp32 1213 us, so 792).
template <bool PAST, int N>
__device__ __forceinline__ void put_entries(float* p, const float (&y)[N], bool whole) {
  if (whole) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      u32x4 v = {__float_as_uint(y[i]), __float_as_uint(y[i + 1]), __float_as_uint(y[i + 2]), __float_as_uint(y[i + 3])};
      if constexpr (PAST && N == 4) __builtin_nontemporal_store(v, (u32x4*)(p + i));
      else *(u32x4*)(p + i) = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = y[i];
  }
}
template <bool PAST, int N>
__device__ __forceinline__ void put_entries(uint16_t* p, const float (&y)[N], bool whole) {
  typedef uint32_t Words __attribute__((ext_vector_type(N / 2)));
  Words v;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) v[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
  if (whole) {
    if constexpr (PAST) __builtin_nontemporal_store(v, (Words*)p);
    else *(Words*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
  }
}

// A row of n entries at any address that suits its entries: `head` entries up to the first multiple of 16 bytes,
// `vecs` whole vectors behind them, and `edge` entries outside the vectors (the head's and those after the last vector).
template <typename T>
struct RowSpan {
  static constexpr int kPer = Entry<T>::kPerVec;
  const T* p;
  int n, head, vecs, edge;
  __device__ __forceinline__ RowSpan(const T* row, int entries) : p(row), n(entries) {
    const int over = (int)((uintptr_t)row & 15) / (int)sizeof(T);
    head = over ? kPer - over : 0;
    if (head > n) head = n;
    vecs = (n - head) / kPer;
    edge = n - vecs * kPer;
  }
  __device__ __forceinline__ int edge_index(int e) const { return e < head ? e : e + vecs * kPer; }
  // PAST: lines that nobody reads again
  template <bool PAST = false>
  __device__ __forceinline__ uint4 vec(int i) const {
    const u32x4* q = (const u32x4*)(p + head) + i;
    u32x4 v;
    if constexpr (PAST) v = __builtin_nontemporal_load(q);
    else v = *q;
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ int index(int i) const { return head + i * kPer; }
};

inline bool known_dtype(int32_t d) { return d == ADWIN_DT_BF16 || d == ADWIN_DT_F32; }
inline uintptr_t entry_mask(int32_t d) { return d == ADWIN_DT_BF16 ? 1 : 3; }
constexpr int64_t kMaxRows = (int64_t)1 << 24;      // rows of a call: fewer than this (a launch has fewer than 2^32 threads)
constexpr int32_t kMaxVocab = 1 << 28;

}  // namespace adwin
