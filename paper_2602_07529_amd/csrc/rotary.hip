// dag_rope_frequencies, dag_rope_apply: rotary positions by a table of frequencies, in either layout of the pairs, for the leading part of a
// head, forward or transposed.
//
// Pair m of a head turns by pos * freq[m]: y = factor (x cos - x' sin, x' cos + x sin); transposed, which is what the gradients go through, the
// angle has the other sign.  Angles are taken in 64 bits, the rotation in 32 for
// bf16 and in 64 for 32-bit tensors, with one rounding to their type.  Everything is read and written once, which is what bounds it.  A workgroup turns the angles of its tokens into cosines and sines once for all heads (in LDS), and then
// a thread has units of two 16-byte pieces whose elements are each other's partners (or stay as they are), two on their way together.
// 18432 tokens of 40 heads of 128 in bf16: 67 us, 5.6 TB/s, with two units on their way (one 72, five 73).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "turns.h"

namespace {

constexpr int THREADS = 256, MAX_HALF = 128, AHEAD = 2;

struct RotaryArgs {
  const int32_t* pos;
  const double* freq;
  const void* in[2];  // queries, keys
  void* out[2];
  int64_t in_stride[2], out_stride[2];  // bytes from a token to the next
  int64_t n_tokens;
  int heads[2];
  int D, rotary;
  double factor, sign;
  bool pairs;
};

template <bool BF16, int TOKENS>
__global__ void __launch_bounds__(THREADS) k_rotary(RotaryArgs a) {
  using T = std::conditional_t<BF16, float, double>;
  __shared__ T s_cos[TOKENS][MAX_HALF], s_sin[TOKENS][MAX_HALF];
  constexpr int EPV = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
  const int half = a.rotary / 2;
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const int n = (int)min((int64_t)TOKENS, a.n_tokens - t0);
  for (int i = threadIdx.x; i < n * half; i += THREADS) {
    const int t = i / half, m = i % half;
    double c, s;
    cos_sin_of_turns((double)a.pos[t0 + t] * (a.freq[m] * 0.15915494309189533577), &c, &s);
    s_cos[t][m] = (T)(c * a.factor);
    s_sin[t][m] = (T)(s * a.factor * a.sign);
  }
  __syncthreads();
  const int upr = a.D / (2 * EPV), rows = a.heads[0] + a.heads[1], total = n * rows * upr, turned = half / EPV;
  for (int base = threadIdx.x; base < total; base += AHEAD * THREADS) {
    u32x4 lo[AHEAD], hi[AHEAD];
    u32x4 *to_lo[AHEAD], *to_hi[AHEAD];
    int unit[AHEAD], token[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int idx = min(base + i * THREADS, total - 1), u = idx % upr, tr = idx / upr, row = tr % rows, t = tr / rows;
      const bool key = row >= a.heads[0];
      const int head = key ? row - a.heads[0] : row;
      const bool apart = !a.pairs && u < turned;
      const int at_lo = (apart ? u : 2 * u) * 16, at_hi = (apart ? u + turned : 2 * u + 1) * 16;
      const char* const from = (const char*)a.in[key] + (t0 + t) * a.in_stride[key] + (size_t)head * a.D * SIZE;
      char* const to = (char*)a.out[key] + (t0 + t) * a.out_stride[key] + (size_t)head * a.D * SIZE;
      lo[i] = *(const u32x4*)(from + at_lo);
      hi[i] = *(const u32x4*)(from + at_hi);
      to_lo[i] = (u32x4*)(to + at_lo);
      to_hi[i] = (u32x4*)(to + at_hi);
      unit[i] = u;
      token[i] = t;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (base + i * THREADS >= total) break;
      float x[2 * EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        if constexpr (BF16) {
          x[e] = e & 1 ? dag_bf_hi(lo[i][e >> 1]) : dag_bf_lo(lo[i][e >> 1]);
          x[EPV + e] = e & 1 ? dag_bf_hi(hi[i][e >> 1]) : dag_bf_lo(hi[i][e >> 1]);
        } else {
          x[e] = __uint_as_float(lo[i][e]);
          x[EPV + e] = __uint_as_float(hi[i][e]);
        }
      }
      if (unit[i] < turned) {
        const T* const cs = &s_cos[token[i]][unit[i] * EPV];
        const T* const sn = &s_sin[token[i]][unit[i] * EPV];
        float y[2 * EPV];
        if (a.pairs) {  // elements 2 e, 2 e + 1 of the two pieces behind one another
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            y[2 * e] = (float)(x[2 * e] * cs[e] - x[2 * e + 1] * sn[e]);
            y[2 * e + 1] = (float)(x[2 * e + 1] * cs[e] + x[2 * e] * sn[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            y[e] = (float)(x[e] * cs[e] - x[EPV + e] * sn[e]);
            y[EPV + e] = (float)(x[EPV + e] * cs[e] + x[e] * sn[e]);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (BF16) {
            lo[i][e] = dag_pack_bf2(y[2 * e], y[2 * e + 1]);
            hi[i][e] = dag_pack_bf2(y[EPV + 2 * e], y[EPV + 2 * e + 1]);
          } else {
            lo[i][e] = __float_as_uint(y[e]);
            hi[i][e] = __float_as_uint(y[EPV + e]);
          }
        }
      }
      *to_lo[i] = lo[i];
      *to_hi[i] = hi[i];
    }
  }
}

template <bool BF16>
int launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  // (a workgroup's chain of frequencies, angles and rows is shared by more tokens where a token has few units: with 1 / 2 / 4 / 8 / 16 tokens, 20000 of 320
  // units in bf16 take 72 / 73 / 76 / 80 / 84 us, of 80 29 / 21 / 17.5 / 17.5 / 18, of 20 19 / 11 / 10 / 8 / 6.7, of 640 in 32 bits 140 / 147 / 155 / 162 / 164; 1024 of 320
  // 5.2 / 5.2 / 5.4 / 7.3 / 11.7, of 20 2.8 whichever; 2048 of 320 8.4 / 7.4 / 7.9 / 9.0 / 13.0, of 80 5.0 / 4.1 / 3.9 / 4.4 / 5.8)
  const int units = (a.heads[0] + a.heads[1]) * (a.D / (BF16 ? 16 : 8));
  const int tokens = a.n_tokens < 2048 ? 1 : units >= 192 ? 2 : units >= 48 ? 4 : 16;
  auto* const kernel = tokens == 1 ? k_rotary<BF16, 1> : tokens == 2 ? k_rotary<BF16, 2> : tokens == 4 ? k_rotary<BF16, 4> : k_rotary<BF16, 16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)dag_ceil_div(a.n_tokens, tokens)), dim3(THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

}  // namespace

extern "C" int dag_rope_frequencies(double* freq, int32_t rotary_dim, double theta, double stretch, double original, double low, double high) {
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > 2 * MAX_HALF) return DAG_ERR_UNSUPPORTED;
  if (!(theta > 0.) || !std::isfinite(theta) || !(stretch > 0.) || !std::isfinite(stretch) || !(original >= 0.) || !std::isfinite(original) ||
      (original > 0. && !(high > low)))
    return DAG_ERR_UNSUPPORTED;
  if (!freq) return DAG_ERR_NULL;
  double table[MAX_HALF];
  for (int m = 0; m < rotary_dim / 2; ++m) {
    const double f = std::pow(theta, -2. * m / rotary_dim);
    double keep = 0.;
    if (original > 0.) {
      keep = (original * f / 6.283185307179586477 - low) / (high - low);
      keep = keep < 0. ? 0. : keep > 1. ? 1. : keep;
    }
    table[m] = keep * f + (1. - keep) * f / stretch;
    if (!std::isfinite(table[m])) return DAG_ERR_UNSUPPORTED;  // (a bound of the parts, or a theta or stretch, past what numbers hold)
  }
  std::copy(table, table + rotary_dim / 2, freq);
  return DAG_OK;
}

extern "C" int dag_rope_apply(const dag_rope_t* rope, const int32_t* pos, int64_t n_tokens, const void* q, int64_t q_stride, void* q_out,
                              int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out, int64_t k_out_stride, int32_t hq, int32_t hkv,
                              int32_t head_dim, int32_t transposed, dag_dtype_t dtype, void* stream_) {
  if (!rope) return DAG_ERR_NULL;
  if (n_tokens < 0 || n_tokens > INT32_MAX) return DAG_ERR_BAD_LEN;
  if (dtype != DAG_F32 && dtype != DAG_BF16) return DAG_ERR_UNSUPPORTED;
  if (head_dim < 16 || head_dim > 2 * MAX_HALF || head_dim % 16 != 0 || rope->rotary_dim < 16 || rope->rotary_dim % 16 != 0 || rope->rotary_dim > head_dim ||
      (rope->layout != DAG_ROPE_HALVES && rope->layout != DAG_ROPE_PAIRS))
    return DAG_ERR_UNSUPPORTED;
  if ((q && hq < 1) || (k && hkv < 1) || (q && hq > 4096) || (k && hkv > 4096)) return DAG_ERR_UNSUPPORTED;
  if (n_tokens == 0 || (!q && !k)) return DAG_OK;
  if (!pos || !rope->freq || (q && !q_out) || (k && !k_out)) return DAG_ERR_NULL;
  const int64_t size = dtype == DAG_BF16 ? 2 : 4;
  if ((q && (q_stride < (int64_t)hq * head_dim || q_out_stride < (int64_t)hq * head_dim)) ||
      (k && (k_stride < (int64_t)hkv * head_dim || k_out_stride < (int64_t)hkv * head_dim)))
    return DAG_ERR_BAD_LEN;
  RotaryArgs a = {};
  const void* const in[2] = {q, k};
  void* const out[2] = {q_out, k_out};
  const int64_t in_stride[2] = {q_stride, k_stride}, out_stride[2] = {q_out_stride, k_out_stride};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    if (!dag_aligned16(in[i]) || !dag_aligned16(out[i]) || in_stride[i] * size % 16 != 0 || out_stride[i] * size % 16 != 0) return DAG_ERR_ALIGN;
    a.in[i] = in[i];
    a.out[i] = out[i];
    a.in_stride[i] = in_stride[i] * size;
    a.out_stride[i] = out_stride[i] * size;
    a.heads[i] = i == 0 ? hq : hkv;
  }
  if ((uintptr_t)rope->freq & 7) return DAG_ERR_ALIGN;
  a.pos = pos;
  a.freq = rope->freq;
  a.n_tokens = n_tokens;
  a.D = head_dim;
  a.rotary = rope->rotary_dim;
  a.factor = rope->factor;
  a.sign = transposed ? -1.f : 1.f;
  a.pairs = rope->layout == DAG_ROPE_PAIRS;
  return dtype == DAG_BF16 ? launch_rotary<true>(a, (hipStream_t)stream_) : launch_rotary<false>(a, (hipStream_t)stream_);
}
