// Rows to 8-bit integers, and the product of two arrays of such rows.
#include "score_shared.h"

namespace adwin {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct QuantArgs {
  const void* x; int64_t ld; int64_t N;
  int32_t H, pitch;
  int8_t* q; float* scale; int32_t* row_status;
};

// 127 x / a to the nearest integer, ties to even, as in exact arithmetic.  per_a = 127 / a rounded: the fp32 quotient is
// off by up to 127 * 2^-23 = 1.5e-5; within twice that of a half, the quotient in 64 bits decides (127 x is exact there, and a quotient
// that is no tie is at least 2^-41 away from one, relative, while the division rounds by 2^-53).
__device__ __forceinline__ int quantised(float x, float per_a, float a) {
  const float t = x * per_a, r = rintf(t);
  if (fabsf(fabsf(t - r) - 0.5f) > 3.0e-5f) return (int)r;
  return (int)rint((double)x * 127.0 / (double)a);
}

// One wave per row, twice over it: largest magnitude (as bits, so that a NaN counts as larger than inf), then the integers,
// 8 to a lane and step.
template <typename T>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= p.N) return;
  const T* x = (const T*)p.x + n * p.ld;
  uint32_t top = 0;
  for (int j = lane; j < p.H; j += 64) {
    const uint32_t b = __float_as_uint(Entry<T>::one(x + j)) & 0x7fffffffu;
    top = b > top ? b : top;
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
  for (int g = lane; g < p.pitch / 8; g += 64) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = 8 * g + e;
      int v = 0;
      if (j < p.H && a > 0.f) {
        const float xj = Entry<T>::one(x + j);
        v = tiny ? (int)rint((double)xj * 127.0 / (double)a) : quantised(xj, per_a, a);
      }
      w[e >> 2] |= (uint32_t)(v & 255) << (8 * (e & 3));
    }
    q[g] = make_uint2(w[0], w[1]);
  }
}

struct ProductArgs {
  const int8_t* h; const float* h_scale; const int8_t* W; const float* W_scale;
  void* z; int64_t ld_z; int64_t T;
  int32_t V, pitch, token_tiles;
};

// v_mfma_i32_32x32x32_i8: lane l supplies row l % 32 of either operand, 16 bytes of k at half l / 32 (the sum does not depend
// on which bytes these are, as long as both operands agree); result e of lane l is row 8 (e / 4) + 4 (l / 32) + e % 4 of A and row l % 32 of B.
// A = entries of the head, B = tokens.  One wave per 32 x 32 block, straight from memory.
template <typename T>
__global__ __launch_bounds__(256) void quant_product_kernel(ProductArgs p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t0 = (int64_t)(blockIdx.x % p.token_tiles) * 32;
  const int64_t v0 = ((int64_t)(blockIdx.x / p.token_tiles) * 4 + wave) * 32;
  if (v0 >= p.V) return;
  const int64_t t = t0 + (lane & 31), v = v0 + (lane & 31);
  const i32x4* W = (const i32x4*)(p.W + (v < p.V ? v : p.V - 1) * p.pitch) + (lane >> 5);   // rows beyond the last repeat it
  const i32x4* h = (const i32x4*)(p.h + (t < p.T ? t : p.T - 1) * p.pitch) + (lane >> 5);
  i32x16 acc = {};
  for (int k = 0; k < p.pitch / 32; ++k) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(W[2 * k], h[2 * k], acc, 0, 0, 0);
  if (t >= p.T) return;
  const float s = p.h_scale[t];
  T* z = (T*)p.z + t * p.ld_z;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int64_t j = v0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
    if (j < p.V) Entry<T>::put(z + j, (float)acc[e] * (s * p.W_scale[j]));
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

static hipError_t launch_quant_rows(const QuantArgs& a, int32_t dtype, hipStream_t st) {
  const unsigned blocks = (unsigned)((a.N + 3) / 4);
  if (dtype == ADWIN_DT_BF16) quant_rows_kernel<uint16_t><<<blocks, 256, 0, st>>>(a);
  else quant_rows_kernel<float><<<blocks, 256, 0, st>>>(a);
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
  ProductArgs a{q, scale, p->W_q, p->W_scale, p->z, p->ld_z, p->T, p->V, ADWIN_QUANT_PITCH(p->H), 0};
  a.token_tiles = (int32_t)((p->T + 31) / 32);
  const int64_t blocks = (int64_t)a.token_tiles * ((p->V + 127) / 128);
  if (blocks >= kMaxRows) return ADWIN_E_SHAPE;
  if (p->z_dtype == ADWIN_DT_BF16) quant_product_kernel<uint16_t><<<(unsigned)blocks, 256, 0, stream>>>(a);
  else quant_product_kernel<float><<<(unsigned)blocks, 256, 0, stream>>>(a);
  ADWIN_HIP_TRY(hipGetLastError());
  return ADWIN_OK;
}
