// dag_kv_append_rope_q8: new keys (rotated at their positions) and values into a paged cache held in 8 bits.
//
// A page and KV head have one scale for K and one for V, a code c stands for scale * c.  With A the largest magnitude among the new
// values of a page and head, scale = max(scale so far, 2^k), k the smallest integer with A <= 448 2^k (at least -100), and
// codes = e4m3(x / scale), to nearest even.  x / 2^k is exact, so a code is one rounding of a value; and because a page gets its tokens
// one by one its scale has to grow: by a power of two that is exact again for all but the codes that fall under the format's smallest
// normal, 2^-15 of the page's largest value.
//
// The tokens of a page stand together in the list (a run), and a wave takes a run and a head, so nothing is shared and no
// atomics are needed.  Keys: lane (slot, 16 dims and their partners), whose 2 x 16 codes are two pieces of the pool as they are.
// Values: lane (two dims), all 16 slots, 32 bytes of the pool.
#include "common.h"

namespace {

constexpr int PAGE = DAG_PAGE_SIZE;

struct AppendArgs {
  const int32_t* slots;
  const int32_t* pos;
  const void* k_new;
  const void* v_new;
  uint8_t* k_pool;
  uint8_t* v_pool;
  float* k_scale;
  float* v_scale;
  int64_t n_tokens;
  int64_t n_slots;
  int hkv;
  RopeTheta theta;
};

// 2^k with the smallest k of at least -100 that brings `most` (finite, not negative) within 448 = 0.875 * 2^9.
__device__ __forceinline__ float q8_scale(float most) {
  const uint32_t u = __float_as_uint(most);
  const int k = (int)(u >> 23) - 126 - 9 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(k, -100) + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float y = fabsf(x);
  return y < INFINITY ? y : 0.f;
}
// Four values, times the inverse of the scale, as codes (what is no number, or infinite, becomes the code of no number).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}
__device__ __forceinline__ u32x4 rescaled(u32x4 x, float f) {
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = rescaled(x[i], f);
  return y;
}

template <bool BF16>
__device__ __forceinline__ void load16(const void* base, size_t at, float (&x)[16]) {
  if constexpr (BF16) {
    const u32x4* const p = (const u32x4*)((const uint16_t*)base + at);
    const u32x4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = dag_bf_lo(a[i]);
      x[2 * i + 1] = dag_bf_hi(a[i]);
      x[8 + 2 * i] = dag_bf_lo(b[i]);
      x[9 + 2 * i] = dag_bf_hi(b[i]);
    }
  } else {
    const f32x4* const p = (const f32x4*)((const float*)base + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 a = p[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = a[e];
    }
  }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(64) k_kv_append_q8(AppendArgs a) {
  const int64_t t0 = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x;
  const int64_t s0 = a.slots[t0];
  if (s0 < 0 || s0 >= a.n_slots) return;
  const int i0 = (int)(s0 % PAGE);
  if (i0 > 0 && t0 > 0 && a.slots[t0 - 1] == s0 - 1) return;  // not the first of its run
  int n = 1;
  while (i0 + n < PAGE && t0 + n < a.n_tokens && a.slots[t0 + n] == s0 + n) ++n;
  const bool begins = i0 == 0;
  const size_t ph = (size_t)(s0 / PAGE) * a.hkv + h;

  {  // keys
    constexpr int HALF = D / 2;
    const int slot = lane & 15, g = lane >> 4, j = slot - i0;
    const bool active = g < HALF / 16, mine = active && j >= 0 && j < n;
    float lo[16], hi[16], most = 0.f;
    if (mine) {
      const size_t at = ((size_t)(t0 + j) * a.hkv + h) * D + 16 * g;
      load16<BF16>(a.k_new, at, lo);
      load16<BF16>(a.k_new, at + HALF, hi);
      const double p = (double)a.pos[t0 + j];
      for (int e = 0; e < 16; ++e) {
        double sn, cs;
        sincos(p * dag_rope_freq(a.theta, 16 * g + e, D), &sn, &cs);
        const float c = (float)cs, s = (float)sn, x = lo[e], y = hi[e];
        lo[e] = fmaf(x, c, -(y * s));  // (as dag_kv_append_rope rotates)
        hi[e] = fmaf(x, s, y * c);
        most = fmaxf(most, fmaxf(finite_abs(lo[e]), finite_abs(hi[e])));
      }
    }
    most = dag_wave_max(most);
    const float before = begins ? 0.f : a.k_scale[ph], scale = fmaxf(before, q8_scale(most)), inv = 1.f / scale;
    const bool grows = !begins && scale != before;
    if (active) {
      u32x4* const p = (u32x4*)(a.k_pool + ph * (D * PAGE) + g * 256 + slot * 16);
      u32x4* const q = p + HALF;  // 16 dims = 16 16-byte pieces
      if (mine) {
        u32x4 x, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = codes4(lo[4 * i] * inv, lo[4 * i + 1] * inv, lo[4 * i + 2] * inv, lo[4 * i + 3] * inv);
          y[i] = codes4(hi[4 * i] * inv, hi[4 * i + 1] * inv, hi[4 * i + 2] * inv, hi[4 * i + 3] * inv);
        }
        *p = x;
        *q = y;
      } else if (begins) {
        *p = u32x4{0, 0, 0, 0};
        *q = u32x4{0, 0, 0, 0};
      } else if (grows) {
        const float f = before * inv;
        *p = rescaled(*p, f);
        *q = rescaled(*q, f);
      }
    }
    if (lane == 0) a.k_scale[ph] = scale;
  }
  {  // values
    const bool active = lane < D / 2;
    float x[PAGE][2], most = 0.f;
#pragma unroll
    for (int i = 0; i < PAGE; ++i) {
      x[i][0] = x[i][1] = 0.f;
      const int j = i - i0;
      if (active && j >= 0 && j < n) {
        const size_t at = ((size_t)(t0 + j) * a.hkv + h) * D + 2 * lane;
        if constexpr (BF16) {
          const uint32_t w = *(const uint32_t*)((const uint16_t*)a.v_new + at);
          x[i][0] = dag_bf_lo(w);
          x[i][1] = dag_bf_hi(w);
        } else {
          const float2 w = *(const float2*)((const float*)a.v_new + at);
          x[i][0] = w.x;
          x[i][1] = w.y;
        }
        most = fmaxf(most, fmaxf(finite_abs(x[i][0]), finite_abs(x[i][1])));
      }
    }
    most = dag_wave_max(most);
    const float before = begins ? 0.f : a.v_scale[ph], scale = fmaxf(before, q8_scale(most)), inv = 1.f / scale;
    if (active) {
      u32x4* const p = (u32x4*)(a.v_pool + ph * (D * PAGE) + lane * 32);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 c;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = codes4(x[4 * i][e] * inv, x[4 * i + 1][e] * inv, x[4 * i + 2][e] * inv, x[4 * i + 3][e] * inv);
        if (!begins) {
          u32x4 old = p[e];
          if (scale != before) old = rescaled(old, before * inv);
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // bytes i0 .. i0 + n - 1 are new
            const int first = max(i0 - 4 * i, 0), end = min(i0 + n - 4 * i, 4);
            const uint32_t mask = end <= first ? 0u : (uint32_t)((1ull << 8 * end) - (1ull << 8 * first));
            c[i] = (c[i] & mask) | (old[i] & ~mask);
          }
        }
        p[e] = c;
      }
    }
    if (lane == 0) a.v_scale[ph] = scale;
  }
}

}  // namespace

extern "C" int dag_kv_append_rope_q8(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new,
                                     const void* v_new, float theta, dag_dtype_t dtype, void* stream_) {
  if (!kv) return DAG_ERR_NULL;
  if (n_tokens < 0 || n_tokens > INT32_MAX || kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  const int D = kv->head_dim;
  if (dtype != DAG_F32 && dtype != DAG_BF16) return DAG_ERR_UNSUPPORTED;
  if (kv->hkv < 1 || kv->hkv > 65535 || (D != 64 && D != 128) || !(theta > 0.f)) return DAG_ERR_UNSUPPORTED;
  if (n_tokens == 0) return DAG_OK;
  if (!slots || !pos || !k_new || !v_new || !kv->k_pool || !kv->v_pool || !kv->k_scale || !kv->v_scale) return DAG_ERR_NULL;
  if (!dag_aligned16(k_new) || !dag_aligned16(v_new) || !dag_aligned16(kv->k_pool) || !dag_aligned16(kv->v_pool) ||
      ((uintptr_t)kv->k_scale & 3) || ((uintptr_t)kv->v_scale & 3))
    return DAG_ERR_ALIGN;
  const AppendArgs a = {slots, pos, k_new, v_new, (uint8_t*)kv->k_pool, (uint8_t*)kv->v_pool, kv->k_scale, kv->v_scale, n_tokens,
                        (int64_t)kv->n_pages * PAGE, kv->hkv, dag_rope_theta(theta)};
  auto* const kernel = dtype == DAG_BF16 ? (D == 128 ? k_kv_append_q8<128, true> : k_kv_append_q8<64, true>)
                                         : (D == 128 ? k_kv_append_q8<128, false> : k_kv_append_q8<64, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)n_tokens, (unsigned)kv->hkv), dim3(64), 0, (hipStream_t)stream_, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}
