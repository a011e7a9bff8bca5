// What the kernels over the 8-bit cache share: the cache, codes as matrix operands, loads of pages.
#pragma once
#include "common.h"

namespace {

struct Q8Cache {
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  const float* k_scale;
  const float* v_scale;
  int n_pages, hkv;
};

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) float f32x8;
// Eight codes, times a power of two, as bf16 (exact: e4m3 has four significant bits).
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi, float power = 1.f) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true));
  return __builtin_bit_cast(bf16x8, x);
}

// Value scales z go into the exponent, and the sum of the probabilities takes them out again.  The exponential's results end at 2^-126, so under
// z = 2^-100, the scale of a page of zeros, a key 2^-27 of the largest would be missing from the sum (2^20 of them: 1 % of it).  So the exponent
// gets no less than 2^LEAST_VALUE, and a key is missing from 2^-66 of the largest on; the power of two that is left over goes into the values as
// they become bf16.
constexpr float LEAST_VALUE = -60.f;
__device__ __forceinline__ float value_log2(float z) {
  const float lv = __builtin_amdgcn_logf(z);
  return lv < -149.f ? -149.f : lv;  // (not minus infinity; no number stays none)
}
// What the exponent gets of value_log2's result; *left: the power of two for the values.
__device__ __forceinline__ float value_exponent(float lv, float* left) {
  const float t = fminf(floorf(lv) - LEAST_VALUE, 0.f);
  *left = __builtin_amdgcn_exp2f(t);
  return lv - t;
}

__device__ __forceinline__ float other_half(float x) { return __uint_as_float(dag_other_group<32>(__float_as_uint(x))); }  // of lane ^ 32

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const uint8_t* p) {  // ONCE: passes the caches by
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}

// Query operands of the lane's row: step 2 s + u has dims 16 (2 s + H) + 8 u .., with the sign of the softmax scale.
template <int D>
__device__ __forceinline__ void fetch_q(bf16x8 (&q)[D / 16], const uint16_t* row, int lane) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) q[s] = *(const bf16x8*)(row + 16 * (lane >> 5) + 32 * (s >> 1) + 8 * (s & 1));
}
template <int D>
__device__ __forceinline__ void sign_q(bf16x8 (&q)[D / 16], float sc) {
  const uint32_t sign = sc < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    u32x4 x = __builtin_bit_cast(u32x4, q[s]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] ^= sign;
    q[s] = __builtin_bit_cast(bf16x8, x);
  }
}

}  // namespace
