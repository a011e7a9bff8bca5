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
#include <type_traits>

#include "common.h"
#include "turns.h"

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
// With rotary positions as a description has them.
struct RotaryAppendArgs : AppendArgs {
  const double* freq;
  double factor;
  int rotary;
  bool pairs;
  int64_t k_stride, v_stride;  // elements from a token to the next
};

// Where the element (or the piece of 16) m of the lower half of a head's pairs lies, and its partner: (m, m + half) of the rotated part in the layout
// of halves, else next to each other; those behind the rotated part, which stay as they are, next to each other too.
struct Partners {
  int lo, hi;
  bool turned, apart;
};
template <int D>
__device__ __forceinline__ Partners partners(const AppendArgs&, int m, int each) { return Partners{m, m + D / (2 * each), true, true}; }
template <int D>
__device__ __forceinline__ Partners partners(const RotaryAppendArgs& a, int m, int each) {
  const int half = a.rotary / (2 * each);
  Partners p;
  p.turned = m < half;
  p.apart = p.turned && !a.pairs;
  p.lo = p.apart ? m : 2 * m;
  p.hi = p.apart ? m + half : 2 * m + 1;
  return p;
}
// Where head h of token t begins among the new keys, the new values; what pair m turns by for a position (0 for one that does not).
template <int D>
__device__ __forceinline__ size_t key_at(const AppendArgs& a, int64_t t, int h) { return ((size_t)t * a.hkv + h) * D; }
template <int D>
__device__ __forceinline__ size_t key_at(const RotaryAppendArgs& a, int64_t t, int h) { return (size_t)t * a.k_stride + h * D; }
template <int D>
__device__ __forceinline__ size_t value_at(const AppendArgs& a, int64_t t, int h) { return ((size_t)t * a.hkv + h) * D; }
template <int D>
__device__ __forceinline__ size_t value_at(const RotaryAppendArgs& a, int64_t t, int h) { return (size_t)t * a.v_stride + h * D; }
template <int D>
__device__ __forceinline__ double frequency(const AppendArgs& a, int m) { return dag_rope_freq(a.theta, m, D); }
template <int D>
__device__ __forceinline__ double frequency(const RotaryAppendArgs& a, int m) { return m < a.rotary / 2 ? a.freq[m] : 0.; }

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

constexpr int SPAN = 16, THREADS = 256;
template <bool ROTARY>
using ArgsOf = std::conditional_t<ROTARY, RotaryAppendArgs, AppendArgs>;
template <bool ROTARY>
using Angle = std::conditional_t<ROTARY, double, float>;
// x cos - y sin and x sin + y cos (as dag_kv_append_rope rotates, in 32 bits).
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
  const float a = fmaf(x, c, -(y * s)), b = fmaf(x, s, y * c);
  x = a;
  y = b;
}
__device__ __forceinline__ void turn(float& x, float& y, double c, double s) {
  const double u = x, v = y;
  x = (float)fma(u, c, -(v * s));
  y = (float)fma(u, s, v * c);
}
// (ROTARY: in 64 bits, and the rotation too: of 20000 x 8 keys of 128 a code in 25000 is another one otherwise, for the same time)
template <int D, typename T>
struct Angles {  // of the tokens from a workgroup's first one on; lines four longer: 16 slots read 16 bytes each from all banks
  T cs[SPAN + PAGE - 1][D / 2 + 4], sn[SPAN + PAGE - 1][D / 2 + 4];
};

// A run of n tokens from token t0 on, which go to the slots i0 .. of a page; ang: row of the first one's angles.
template <int D, bool BF16, bool ROTARY>
__device__ __forceinline__ void append_run(const ArgsOf<ROTARY>& a, const Angles<D, Angle<ROTARY>>& angles, int ang, int64_t t0, int n, int64_t page, int i0, int h,
                                           int lane) {
  const bool begins = i0 == 0;
  const size_t ph = (size_t)page * a.hkv + h;
  constexpr int HALF = D / 2;
  // keys
  const int slot = lane & 15, g = lane >> 4, j = slot - i0;
  const bool active = g < HALF / 16, mine = active && j >= 0 && j < n;
  const Partners pt = partners<D>(a, g, 16);
  Raw16<BF16> k_lo, k_hi;
  if (mine) {
    const size_t at = key_at<D>(a, t0 + j, h);
    k_lo.load(a.k_new, at + 16 * pt.lo);
    k_hi.load(a.k_new, at + 16 * pt.hi);
  }
  // values
  const bool active_v = lane < D / 2;
  Raw2<BF16> v[PAGE] = {};
#pragma unroll
  for (int i = 0; i < PAGE; ++i)
    if (active_v && i >= i0 && i < i0 + n) v[i].load(a.v_new, value_at<D>(a, t0 + i - i0, h) + 2 * lane);
  const float before = begins ? 0.f : a.k_scale[ph], before_v = begins ? 0.f : a.v_scale[ph];
  float lo[16], hi[16], most = 0.f;
  if (mine) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      lo[e] = k_lo[e];
      hi[e] = k_hi[e];
    }
    if (pt.apart) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        turn(lo[e], hi[e], angles.cs[ang + j][16 * g + e], angles.sn[ang + j][16 * g + e]);
      }
    } else if (pt.turned) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float& x = e < 8 ? lo[2 * (e & 7)] : hi[2 * (e & 7)];
        float& y = e < 8 ? lo[2 * (e & 7) + 1] : hi[2 * (e & 7) + 1];
        turn(x, y, angles.cs[ang + j][16 * g + e], angles.sn[ang + j][16 * g + e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) most = fmaxf(most, fmaxf(finite_abs(lo[e]), finite_abs(hi[e])));
  }
  {
    most = dag_wave_max(most);
    const float scale = fmaxf(before, q8_scale(most)), inv = 1.f / scale;
    if (active) {
      u32x4* const p = (u32x4*)(a.k_pool + ph * (D * PAGE) + pt.lo * 256 + slot * 16);
      u32x4* const q = (u32x4*)(a.k_pool + ph * (D * PAGE) + pt.hi * 256 + slot * 16);
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
template <int D, bool BF16, bool ROTARY>
__device__ __forceinline__ void append_one(const ArgsOf<ROTARY>& a, const Angles<D, Angle<ROTARY>>& angles, int ang, uint8_t* lds, int64_t t, int64_t page, int i0, int h,
                                           int lane) {
  constexpr int HALF = D / 2;
  const bool begins = i0 == 0, active = lane < HALF;
  const int m = active ? lane : 0;
  const size_t ph = (size_t)page * a.hkv + h, at = key_at<D>(a, t, h), at_v = value_at<D>(a, t, h);
  const Partners pt = partners<D>(a, m, 1);
  float x, y;
  if constexpr (BF16) {
    x = __uint_as_float((uint32_t)((const uint16_t*)a.k_new)[at + pt.lo] << 16);
    y = __uint_as_float((uint32_t)((const uint16_t*)a.k_new)[at + pt.hi] << 16);
  } else {
    x = ((const float*)a.k_new)[at + pt.lo];
    y = ((const float*)a.k_new)[at + pt.hi];
  }
  Raw2<BF16> v;
  v.load(a.v_new, at_v + 2 * m);
  const float before = begins ? 0.f : a.k_scale[ph], before_v = begins ? 0.f : a.v_scale[ph];
  float lo = x, hi = y;
  if (pt.turned) turn(lo, hi, angles.cs[ang][m], angles.sn[ang][m]);
  const float scale = fmaxf(before, q8_scale(dag_wave_max(fmaxf(finite_abs(lo), finite_abs(hi))))), inv = 1.f / scale;
  const float scale_v = fmaxf(before_v, q8_scale(dag_wave_max(fmaxf(finite_abs(v[0]), finite_abs(v[1]))))), inv_v = 1.f / scale_v;
  const uint32_t ck = codes4(lo * inv, hi * inv, 0.f, 0.f), cv = codes4(v[0] * inv_v, v[1] * inv_v, 0.f, 0.f);
  uint8_t* const kp = a.k_pool + ph * (D * PAGE);
  uint8_t* const vp = a.v_pool + ph * (D * PAGE);
  if (begins || scale != before) {
    if (active) {
      lds[pt.lo] = (uint8_t)ck;
      lds[pt.hi] = (uint8_t)(ck >> 8);
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
    kp[pt.lo / 16 * 256 + i0 * 16 + pt.lo % 16] = (uint8_t)ck;
    kp[pt.hi / 16 * 256 + i0 * 16 + pt.hi % 16] = (uint8_t)(ck >> 8);
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

template <int D, bool BF16, bool ROTARY>
__global__ void __launch_bounds__(THREADS, BF16 ? 3 : 2) k_kv_append_q8(ArgsOf<ROTARY> a, int span) {
  __shared__ Angles<D, Angle<ROTARY>> angles;
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
    const double f = frequency<D>(a, m) * 0.15915494309189533577;  // turns
    for (int i = tid / HALF; i < n_ang; i += THREADS / HALF) {
      cos_sin_of_turns((double)a.pos[first - 1 + begin + i] * f, &angles.cs[i][m], &angles.sn[i][m]);
      if constexpr (ROTARY) {
        angles.cs[i][m] *= a.factor;
        angles.sn[i][m] *= a.factor;
      }
    }
  }
  __syncthreads();
  for (int x = w; lead; lead &= lead - 1) {
    const int i = __builtin_ctzll(lead), n = length(i);
    const int64_t s0 = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s, i);
    for (; x < a.hkv; x += THREADS / 64) {
      if (n > 1) append_run<D, BF16, ROTARY>(a, angles, i - begin, first - 1 + i, n, s0 / PAGE, (int)(s0 % PAGE), x, lane);
      else append_one<D, BF16, ROTARY>(a, angles, i - begin, one[w], first - 1 + i, s0 / PAGE, (int)(s0 % PAGE), x, lane);
    }
    x -= a.hkv;
  }
}

template <bool ROTARY>
int launch_append(const ArgsOf<ROTARY>& a, int D, dag_dtype_t dtype, hipStream_t stream) {
  auto* const kernel = dtype == DAG_BF16 ? (D == 128 ? k_kv_append_q8<128, true, ROTARY> : k_kv_append_q8<64, true, ROTARY>)
                                         : (D == 128 ? k_kv_append_q8<128, false, ROTARY> : k_kv_append_q8<64, false, ROTARY>);
  // With 1 / 2 / 4 / 8 / 16 tokens to a workgroup, general positions, 8 heads of 128 in bf16, us: 128 single tokens 5.4 / 7.8 / 13 / 23 / 42, 4096 33 / 29 / 30 / 31 / 48;
  // prompts, 2048 tokens in all 16 / 16 / 12 / 15 / 15, 20000 88 / 80 / 43 / 30 / 29.5, 65536 341 / 180 / 165 / 115 / 97.  (A list does not say which of the two it is: prompts of 1500
  // take 15 / 12 / 9.6 / 15 / 15, of 4096 30 / 22 / 21 / 17 / 16.)
  const int span = a.n_tokens >= 512 * SPAN ? SPAN : a.n_tokens >= 2048 ? 4 : 1;
  hipLaunchKernelGGL(kernel, dim3((unsigned)dag_ceil_div(a.n_tokens, span)), dim3(THREADS), 0, stream, a, span);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

// What both appends ask of the cache and the tokens (theta and rope apart).
int check_append(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new, const void* v_new, dag_dtype_t dtype) {
  const int D = kv->head_dim;
  if (dtype != DAG_F32 && dtype != DAG_BF16) return DAG_ERR_UNSUPPORTED;
  if (kv->hkv < 1 || (D != 64 && D != 128)) return DAG_ERR_UNSUPPORTED;
  if (n_tokens == 0) return DAG_OK;
  if (!slots || !pos || !k_new || !v_new || !kv->k_pool || !kv->v_pool || !kv->k_scale || !kv->v_scale) return DAG_ERR_NULL;
  if (!dag_aligned16(k_new) || !dag_aligned16(v_new) || !dag_aligned16(kv->k_pool) || !dag_aligned16(kv->v_pool) ||
      ((uintptr_t)kv->k_scale & 3) || ((uintptr_t)kv->v_scale & 3))
    return DAG_ERR_ALIGN;
  return DAG_OK;
}

template <typename A>
A append_args(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new, const void* v_new) {
  A a = {};
  a.slots = slots;
  a.pos = pos;
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_pool = (uint8_t*)kv->k_pool;
  a.v_pool = (uint8_t*)kv->v_pool;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.n_tokens = n_tokens;
  a.n_slots = (int64_t)kv->n_pages * PAGE;
  a.hkv = kv->hkv;
  return a;
}

}  // namespace

extern "C" int dag_kv_append_rope_q8(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new,
                                     const void* v_new, float theta, dag_dtype_t dtype, void* stream_) {
  if (!kv) return DAG_ERR_NULL;
  if (n_tokens < 0 || n_tokens > INT32_MAX || kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  if (!(theta > 0.f)) return DAG_ERR_UNSUPPORTED;
  const int rc = check_append(kv, slots, pos, n_tokens, k_new, v_new, dtype);
  if (rc != DAG_OK || n_tokens == 0) return rc;
  AppendArgs a = append_args<AppendArgs>(kv, slots, pos, n_tokens, k_new, v_new);
  a.theta = dag_rope_theta(theta);
  return launch_append<false>(a, kv->head_dim, dtype, (hipStream_t)stream_);
}

extern "C" int dag_kv_append_rotary_q8(const dag_kv_q8_t* kv, const int32_t* slots, const int32_t* pos, int64_t n_tokens, const void* k_new,
                                       int64_t k_stride, const void* v_new, int64_t v_stride, const dag_rope_t* rope, dag_dtype_t dtype, void* stream_) {
  if (!kv || !rope) return DAG_ERR_NULL;
  if (n_tokens < 0 || n_tokens > INT32_MAX || kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  const int rc = check_append(kv, slots, pos, n_tokens, k_new, v_new, dtype);
  if (rc != DAG_OK) return rc;
  if ((rope->layout != DAG_ROPE_HALVES && rope->layout != DAG_ROPE_PAIRS) || rope->rotary_dim < 32 || rope->rotary_dim % 32 != 0 ||
      rope->rotary_dim > kv->head_dim)
    return DAG_ERR_UNSUPPORTED;
  if (n_tokens == 0) return DAG_OK;
  const int64_t row = (int64_t)kv->hkv * kv->head_dim, each = dtype == DAG_BF16 ? 8 : 4;
  if (k_stride < row || v_stride < row) return DAG_ERR_BAD_LEN;
  if (!rope->freq) return DAG_ERR_NULL;
  if (k_stride % each != 0 || v_stride % each != 0 || ((uintptr_t)rope->freq & 7)) return DAG_ERR_ALIGN;
  RotaryAppendArgs a = append_args<RotaryAppendArgs>(kv, slots, pos, n_tokens, k_new, v_new);
  a.freq = rope->freq;
  a.factor = rope->factor;
  a.rotary = rope->rotary_dim;
  a.pairs = rope->layout == DAG_ROPE_PAIRS;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  return launch_append<true>(a, kv->head_dim, dtype, (hipStream_t)stream_);
}
