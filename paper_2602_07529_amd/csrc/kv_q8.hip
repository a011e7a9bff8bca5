// dag_kv_append_rope_q8: new keys (rotated at their positions) and values into a paged cache held in 8 bits.
//
// A page and KV head have one scale for K and one for V, a code c stands for scale * c.  With A the largest magnitude among the new
// values of a page and head, scale = max(scale so far, 2^k), k the smallest integer with A <= 448 2^k (at least -100), and
// codes = e4m3(x / scale), to nearest even.  x / 2^k is exact, so a code is one rounding of a value; and because a page gets its tokens
// one by one its scale has to grow: by a power of two that is exact again for all but the codes that fall under the format's smallest
// normal, 2^-15 of the page's largest value.
//
// The tokens of a page stand together in the list (a run), and a wave takes a run and a head, so nothing is shared and no
// atomics are needed.  A workgroup takes the runs that start in its `span` tokens: it turns the angles of their tokens into cosines and
// sines once for all heads (in LDS) and its waves share out (run, head).  Long runs: keys by lane (slot, 16 dims and their partners), whose
// 2 x 16 codes are two pieces of the pool as they are; values by lane (two dims), all 16 slots, 32 bytes of the pool.
// Single tokens (a decode step): a lane has a pair of the key's dims and two of the value's.
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

// Sixteen values as they lie in memory (half the registers of 32-bit values while they are on their way).
template <bool BF16>
struct Raw16 {
  u32x4 x[BF16 ? 2 : 4];
  __device__ __forceinline__ void load(const void* base, size_t at) {
    const u32x4* const p = (const u32x4*)((const char*)base + at * (BF16 ? 2 : 4));
#pragma unroll
    for (int i = 0; i < (BF16 ? 2 : 4); ++i) x[i] = p[i];
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (BF16) return e & 1 ? dag_bf_hi(x[e >> 3][(e & 7) >> 1]) : dag_bf_lo(x[e >> 3][(e & 7) >> 1]);
    else return __uint_as_float(x[e >> 2][e & 3]);
  }
};
template <bool BF16>
struct Raw2 {
  uint32_t x[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* base, size_t at) {
    if constexpr (BF16) x[0] = *(const uint32_t*)((const uint16_t*)base + at);
    else {
      const u32x2 w = *(const u32x2*)((const float*)base + at);
      x[0] = w[0];
      x[1] = w[1];
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (BF16) return e ? dag_bf_hi(x[0]) : dag_bf_lo(x[0]);
    else return __uint_as_float(x[e]);
  }
};

// Cosine and sine of x turns: the nearest quarter is taken off exactly, and what is left, an angle y of at most pi / 4, goes through the
// Taylor series (the terms left out are below 2e-14 there).  A library call for any angle takes three times as long.
__device__ __forceinline__ void cos_sin_of_turns(double x, float* c, float* s) {
  const double quarter = rint(4. * x), y = fma(-0.25, quarter, x) * 6.283185307179586477, z = y * y;
  double sn = 1. / 6227020800., cs = -1. / 87178291200.;
  sn = fma(sn, z, -1. / 39916800.);
  sn = fma(sn, z, 1. / 362880.);
  sn = fma(sn, z, -1. / 5040.);
  sn = fma(sn, z, 1. / 120.);
  sn = fma(sn, z, -1. / 6.);
  sn = fma(sn * z, y, y);
  cs = fma(cs, z, 1. / 479001600.);
  cs = fma(cs, z, -1. / 3628800.);
  cs = fma(cs, z, 1. / 40320.);
  cs = fma(cs, z, -1. / 720.);
  cs = fma(cs, z, 1. / 24.);
  cs = fma(cs, z, -0.5);
  cs = fma(cs, z, 1.);
  const int k = (int)((int64_t)quarter & 3);
  const float u = (float)(k & 1 ? sn : cs), v = (float)(k & 1 ? cs : sn);
  *c = k == 1 || k == 2 ? -u : u;
  *s = k >= 2 ? -v : v;
}

constexpr int SPAN = 16, THREADS = 256;
template <int D>
struct Angles {  // of the tokens from a workgroup's first one on; lines four longer: 16 slots read 16 bytes each from all banks
  float cs[SPAN + PAGE - 1][D / 2 + 4], sn[SPAN + PAGE - 1][D / 2 + 4];
};

// A run of n tokens from token t0 on, which go to the slots i0 .. of a page; ang: row of the first one's angles.
template <int D, bool BF16>
__device__ __forceinline__ void append_run(const AppendArgs& a, const Angles<D>& angles, int ang, int64_t t0, int n, int64_t page, int i0, int h,
                                           int lane) {
  const bool begins = i0 == 0;
  const size_t ph = (size_t)page * a.hkv + h;
  constexpr int HALF = D / 2;
  // keys
  const int slot = lane & 15, g = lane >> 4, j = slot - i0;
  const bool active = g < HALF / 16, mine = active && j >= 0 && j < n;
  Raw16<BF16> k_lo, k_hi;
  if (mine) {
    const size_t at = ((size_t)(t0 + j) * a.hkv + h) * D + 16 * g;
    k_lo.load(a.k_new, at);
    k_hi.load(a.k_new, at + HALF);
  }
  // values
  const bool active_v = lane < D / 2;
  Raw2<BF16> v[PAGE] = {};
#pragma unroll
  for (int i = 0; i < PAGE; ++i)
    if (active_v && i >= i0 && i < i0 + n) v[i].load(a.v_new, ((size_t)(t0 + i - i0) * a.hkv + h) * D + 2 * lane);
  const float before = begins ? 0.f : a.k_scale[ph], before_v = begins ? 0.f : a.v_scale[ph];
  float lo[16], hi[16], most = 0.f;
  if (mine) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float c = angles.cs[ang + j][16 * g + e], s = angles.sn[ang + j][16 * g + e], x = k_lo[e], y = k_hi[e];
      lo[e] = fmaf(x, c, -(y * s));  // (as dag_kv_append_rope rotates)
      hi[e] = fmaf(x, s, y * c);
      most = fmaxf(most, fmaxf(finite_abs(lo[e]), finite_abs(hi[e])));
    }
  }
  {
    most = dag_wave_max(most);
    const float scale = fmaxf(before, q8_scale(most)), inv = 1.f / scale;
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
      } else if (scale != before) {
        const float f = before * inv;
        *p = rescaled(*p, f);
        *q = rescaled(*q, f);
      }
    }
    if (lane == 0) a.k_scale[ph] = scale;
  }
  float most_v = 0.f;
#pragma unroll
  for (int i = 0; i < PAGE; ++i) most_v = fmaxf(most_v, fmaxf(finite_abs(v[i][0]), finite_abs(v[i][1])));
  most_v = dag_wave_max(most_v);
  const float scale = fmaxf(before_v, q8_scale(most_v)), inv = 1.f / scale;
  if (active_v) {
    u32x4* const p = (u32x4*)(a.v_pool + ph * (D * PAGE) + lane * 32);
    u32x4 c[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e) c[e][i] = codes4(v[4 * i][e] * inv, v[4 * i + 1][e] * inv, v[4 * i + 2][e] * inv, v[4 * i + 3][e] * inv);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (!begins) {
        u32x4 old = p[e];
        if (scale != before_v) old = rescaled(old, before_v * inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // bytes i0 .. i0 + n - 1 are new
          const int first = max(i0 - 4 * i, 0), end = min(i0 + n - 4 * i, 4);
          const uint32_t mask = end <= first ? 0u : (uint32_t)((1ull << 8 * end) - (1ull << 8 * first));
          c[e][i] = (c[e][i] & mask) | (old[i] & ~mask);
        }
      }
      p[e] = c[e];
    }
  }
  if (lane == 0) a.v_scale[ph] = scale;
}

// A single token.  Where its page begins or its scale grows the whole page is written, else the token's bytes.
template <int D, bool BF16>
__device__ __forceinline__ void append_one(const AppendArgs& a, const Angles<D>& angles, int ang, uint8_t* lds, int64_t t, int64_t page, int i0, int h,
                                           int lane) {
  constexpr int HALF = D / 2;
  const bool begins = i0 == 0, active = lane < HALF;
  const int m = active ? lane : 0;
  const size_t ph = (size_t)page * a.hkv + h, at = ((size_t)t * a.hkv + h) * D;
  float x, y;
  if constexpr (BF16) {
    x = __uint_as_float((uint32_t)((const uint16_t*)a.k_new)[at + m] << 16);
    y = __uint_as_float((uint32_t)((const uint16_t*)a.k_new)[at + m + HALF] << 16);
  } else {
    x = ((const float*)a.k_new)[at + m];
    y = ((const float*)a.k_new)[at + m + HALF];
  }
  Raw2<BF16> v;
  v.load(a.v_new, at + 2 * m);
  const float before = begins ? 0.f : a.k_scale[ph], before_v = begins ? 0.f : a.v_scale[ph];
  const float c = angles.cs[ang][m], s = angles.sn[ang][m];
  const float lo = fmaf(x, c, -(y * s)), hi = fmaf(x, s, y * c);
  const float scale = fmaxf(before, q8_scale(dag_wave_max(fmaxf(finite_abs(lo), finite_abs(hi))))), inv = 1.f / scale;
  const float scale_v = fmaxf(before_v, q8_scale(dag_wave_max(fmaxf(finite_abs(v[0]), finite_abs(v[1]))))), inv_v = 1.f / scale_v;
  const uint32_t ck = codes4(lo * inv, hi * inv, 0.f, 0.f), cv = codes4(v[0] * inv_v, v[1] * inv_v, 0.f, 0.f);
  uint8_t* const kp = a.k_pool + ph * (D * PAGE);
  uint8_t* const vp = a.v_pool + ph * (D * PAGE);
  if (begins || scale != before) {
    if (active) {
      lds[m] = (uint8_t)ck;
      lds[m + HALF] = (uint8_t)(ck >> 8);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const float f = before * inv;
#pragma unroll
    for (int i = lane; i < D; i += 64) {  // pieces of 16 dims of a slot
      u32x4* const p = (u32x4*)(kp + i * 16);
      if (i % PAGE == i0) *p = *(const u32x4*)(lds + i / PAGE * 16);
      else *p = begins ? u32x4{0, 0, 0, 0} : rescaled(*p, f);
    }
  } else if (active) {
    kp[m / 16 * 256 + i0 * 16 + m % 16] = (uint8_t)ck;
    kp[(m + HALF) / 16 * 256 + i0 * 16 + m % 16] = (uint8_t)(ck >> 8);
  }
  if (active) {
    if (begins || scale_v != before_v) {
      u32x4* const p = (u32x4*)(vp + 32 * m);
      const float f = before_v * inv_v;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 w = begins ? u32x4{0, 0, 0, 0} : rescaled(p[e], f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t mask = i0 / 4 == i ? 0xffu << 8 * (i0 % 4) : 0u;
          w[i] = (w[i] & ~mask) | ((e ? cv >> 8 : cv) & 0xffu) * 0x01010101u & mask;
        }
        p[e] = w;
      }
    } else {
      vp[2 * m * PAGE + i0] = (uint8_t)cv;
      vp[(2 * m + 1) * PAGE + i0] = (uint8_t)(cv >> 8);
    }
  }
  if (lane == 0) {
    a.k_scale[ph] = scale;
    a.v_scale[ph] = scale_v;
  }
  __builtin_amdgcn_wave_barrier();  // (the next head writes the same bytes of LDS, in the order of the instructions)
}

template <int D, bool BF16>
__global__ void __launch_bounds__(THREADS, BF16 ? 3 : 2) k_kv_append_q8(AppendArgs a, int span) {
  __shared__ Angles<D> angles;
  __shared__ __attribute__((aligned(16))) uint8_t one[THREADS / 64][D];
  constexpr int HALF = D / 2;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t first = (int64_t)blockIdx.x * span;
  // lane i: token first - 1 + i
  const int64_t t = first - 1 + lane;
  const int64_t s = lane < span + PAGE && t >= 0 && t < a.n_tokens ? a.slots[t] : -1;
  const bool there = s >= 0 && s < a.n_slots;
  const int64_t behind = __shfl_up(s, 1);
  const bool goes_on = there && lane > 0 && s % PAGE != 0 && behind == s - 1;
  const uint64_t run_on = __builtin_amdgcn_ballot_w64(goes_on);
  uint64_t lead = __builtin_amdgcn_ballot_w64(there && !goes_on && lane >= 1 && lane <= span);
  if (lead == 0) return;
  auto length = [&](int i) { return 1 + __builtin_ctzll(~(run_on >> i >> 1)); };  // of the run that lane i leads
  const int begin = __builtin_ctzll(lead), last = 63 - __builtin_clzll(lead), n_ang = last + length(last) - begin;
  {
    const int m = tid % HALF;
    const double f = dag_rope_freq(a.theta, m, D) * 0.15915494309189533577;  // turns
    for (int i = tid / HALF; i < n_ang; i += THREADS / HALF) cos_sin_of_turns((double)a.pos[first - 1 + begin + i] * f, &angles.cs[i][m], &angles.sn[i][m]);
  }
  __syncthreads();
  for (int x = w; lead; lead &= lead - 1) {
    const int i = __builtin_ctzll(lead), n = length(i);
    const int64_t s0 = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s, i);
    for (; x < a.hkv; x += THREADS / 64) {
      if (n > 1) append_run<D, BF16>(a, angles, i - begin, first - 1 + i, n, s0 / PAGE, (int)(s0 % PAGE), x, lane);
      else append_one<D, BF16>(a, angles, i - begin, one[w], first - 1 + i, s0 / PAGE, (int)(s0 % PAGE), x, lane);
    }
    x -= a.hkv;
  }
}

}  // namespace

extern "C" int dag_kv_append_rope_q8(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new,
                                     const void* v_new, float theta, dag_dtype_t dtype, void* stream_) {
  if (!kv) return DAG_ERR_NULL;
  if (n_tokens < 0 || n_tokens > INT32_MAX || kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  const int D = kv->head_dim;
  if (dtype != DAG_F32 && dtype != DAG_BF16) return DAG_ERR_UNSUPPORTED;
  if (kv->hkv < 1 || (D != 64 && D != 128) || !(theta > 0.f)) return DAG_ERR_UNSUPPORTED;
  if (n_tokens == 0) return DAG_OK;
  if (!slots || !pos || !k_new || !v_new || !kv->k_pool || !kv->v_pool || !kv->k_scale || !kv->v_scale) return DAG_ERR_NULL;
  if (!dag_aligned16(k_new) || !dag_aligned16(v_new) || !dag_aligned16(kv->k_pool) || !dag_aligned16(kv->v_pool) ||
      ((uintptr_t)kv->k_scale & 3) || ((uintptr_t)kv->v_scale & 3))
    return DAG_ERR_ALIGN;
  const AppendArgs a = {slots, pos, k_new, v_new, (uint8_t*)kv->k_pool, (uint8_t*)kv->v_pool, kv->k_scale, kv->v_scale, n_tokens,
                        (int64_t)kv->n_pages * PAGE, kv->hkv, dag_rope_theta(theta)};
  auto* const kernel = dtype == DAG_BF16 ? (D == 128 ? k_kv_append_q8<128, true> : k_kv_append_q8<64, true>)
                                         : (D == 128 ? k_kv_append_q8<128, false> : k_kv_append_q8<64, false>);
  const int span = n_tokens >= 512 * SPAN ? SPAN : n_tokens >= 2048 ? 4 : 1;
  hipLaunchKernelGGL(kernel, dim3((unsigned)dag_ceil_div(n_tokens, span)), dim3(THREADS), 0, (hipStream_t)stream_, a, span);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}
