// Decode attention over a paged KV cache held in 8 bits, a scale for each (page, KV head): a code c of a page stands for scale * c.
//
// dag_attn_decode_q8          : shared context of a sibling group | a branch's own pages (the description of dag_attn_decode).
// dag_attn_decode_segments_q8 : contexts as lists of KV segments (that of dag_attn_decode_segments).
//
// out = sum_j softmax_j(scale q . k_j) v_j.  With the key scale s of page(j) the exponent of key j is t_j = (scale log2(e) s) q . c_j,
// one product more a score, and with the value scale z its probability enters the second product as 2^(t_j - m + log2 z); the
// sum of the probabilities is without z.  The codes become bf16 in registers, which holds every e4m3 value, so nothing but
// the probabilities is rounded, as with a bf16 cache.  A step has to read 2 hkv D bytes a token, half of what that one needs.
//
// Pool formats (16 tokens a page) are operand images, as those of the bf16 cache:
//   K [P][hkv][D/16][16 slots][16 dims], V [P][hkv][D][16 slots]: a lane's 16 bytes are its operand of two MFMA steps.
// Scores are computed transposed (S^T = K Q^T), MFMA row i being slot r of page H, H = bit 2 of i, of the two pages of a block of 32 keys:
// a half of the wave then holds the 16 slots of one page, whose scales are one register, and its sums are the operand of
// O^T = V^T P^T as they are, two steps of eight slots of either page.
#include <type_traits>

#include "common.h"
#include "decode_plan.h"
#include "seg_plan.h"

namespace {

struct Q8Cache {
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  const float* k_scale;
  const float* v_scale;
  int n_pages, hkv;
};

struct Q8DecodeArgs {
  Q8Cache kv;
  const int32_t* group_branch_off;
  const int32_t* shared_page_off;
  const int32_t* shared_pages;
  const int32_t* shared_len;
  const int32_t* branch_page_off;
  const int32_t* branch_pages;
  const int32_t* branch_len;
  const uint16_t* q;
  uint16_t* out;
  float* part_o;   // [place][hq][D]: a branch's slices of the shared context, then (from first_own on) those of its own pages
  float* part_ml;  // [place][hq][2]: reference in the exponent's units, sum
  int first_own;
  int n_live, hq, hkv, G;
  int rb_max, chunk_a, splits_a, chunk_b, splits_b, items_a;
  float sc;        // softmax_scale * log2(e)
};

struct Q8SegArgs {
  SegArgs s;
  Q8Cache kv;
};

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) float f32x8;
// Eight codes as bf16 (exact: e4m3 has four significant bits).
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return __builtin_bit_cast(bf16x8, x);
}

template <int D>
struct Block {         // 32 keys (two pages)
  u32x4 k[D / 32];     // k[s]: dims 16 (2 s + H) .. of the key of MFMA row L
  u32x4 v[D / 32];     // v[db]: the slots of page H of dimension 32 db + L
};

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const uint8_t* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_block(Block<D>& b, const Q8Cache& c, int pages, int rel, int last_rel, int hk, int L, int H) {
  const int pg0 = __builtin_amdgcn_readlane(pages, rel & 63), pg1 = __builtin_amdgcn_readlane(pages, min(rel + 1, last_rel) & 63);
  const int slot = (L & 3) + 4 * (L >> 3);
  const size_t base0 = ((size_t)pg0 * c.hkv + hk) * (D * PAGE), base1 = ((size_t)pg1 * c.hkv + hk) * (D * PAGE);
  const uint8_t* const kp = c.k_pool + ((L >> 2) & 1 ? base1 : base0) + H * 256 + slot * 16;
  const uint8_t* const vp = c.v_pool + (H ? base1 : base0) + L * 16;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.k[s] = load16<ONCE>(kp + s * 512);
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.v[s] = load16<ONCE>(vp + s * 512);
}

// A block some of whose tokens are hidden from some rows only (the new tokens of a node): a value that is no number may not reach the rows
// that do not see it, and a probability of zero does not keep it from them.  Such codes are cleared, and the sums of the rows that
// see one become no number: a product of "is none" and "is seen" finds them.
template <int D>
__device__ __forceinline__ void hide_not_numbers(Block<D>& b, f32x16* O, int key0, int lim, int H) {
  uint32_t any = 0;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int w = 0; w < 4; ++w) any |= (b.v[db][w] & 0x7f7f7f7fu) + 0x01010101u;
  if (__builtin_amdgcn_ballot_w64((any & 0x80808080u) != 0) == 0) return;
  f32x8 seen[2];
#pragma unroll
  for (int r = 0; r < 16; ++r) seen[r >> 3][r & 7] = key0 + 16 * H + r < lim ? 1.f : 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    uint32_t one[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t none = (((b.v[db][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
      b.v[db][w] &= ~(none * 0xffu);
      one[w] = none * 0x38u;  // the code of one
    }
    f32x16 n;
#pragma unroll
    for (int r = 0; r < 16; ++r) n[r] = 0.f;
    n = mfma32(codes_to_bf16(one[0], one[1]), __builtin_convertvector(seen[0], bf16x8), n);
    n = mfma32(codes_to_bf16(one[2], one[3]), __builtin_convertvector(seen[1], bf16x8), n);
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = n[r] > 0.f ? NAN : O[db][r];
  }
}

// The exponent's reference m is raised only where a score is more than this above it (log2): the rescale of the sums stays rare.
constexpr float Q8_TH = 3.f;

// One block: scores, probabilities, their product with the values.  ks: key scale of the lane's page times |softmax scale| log2(e), lv: log2 of
// its value scale.  A lane's 16 scores are of one page, so their largest is found among the plain products, one multiply-add gives
// the exponent with the value scale in it, and the sum of a lane loses that factor again once.
// key0: first key of the block; keys from `lim` on are hidden from this lane's row; len: the smallest lim of the wave; slots from vlen on
// hold no token.
template <int D, typename QF>
__device__ __forceinline__ void compute_block(Block<D>& b, QF&& qop, f32x16* O, float& m, float& l, float ks, float lv, int key0, int len,
                                              int lim, int vlen, int H) {
  f32x16 S;
#pragma unroll
  for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    S = mfma32(codes_to_bf16(b.k[s][0], b.k[s][1]), qop(2 * s), S);
    S = mfma32(codes_to_bf16(b.k[s][2], b.k[s][3]), qop(2 * s + 1), S);
  }
  if (key0 + 32 > len) {
#pragma unroll
    for (int r = 0; r < 16; ++r) S[r] = key0 + 16 * H + r < lim ? S[r] : -INFINITY;
  }
  float bm = S[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) bm = fmaxf(bm, S[r]);
  bm *= ks;
  bm = fmaxf(bm, __shfl_xor(bm, 32));
  if (__builtin_amdgcn_ballot_w64(bm > m + Q8_TH) != 0) {
    const float m_new = fmaxf(m, bm), alpha = __builtin_amdgcn_exp2f(m - m_new);
    l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[db][r] *= alpha;
    m = m_new;
  }
  f32x8 p0, p1;
  float sum = 0.f;
  const float ref = lv - m;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    p0[r] = __builtin_amdgcn_exp2f(fmaf(S[r], ks, ref));
    p1[r] = __builtin_amdgcn_exp2f(fmaf(S[8 + r], ks, ref));
    sum += p0[r] + p1[r];
  }
  l = fmaf(sum, __builtin_amdgcn_exp2f(-lv), l);
  // (rounded to bf16, as the probabilities over a bf16 cache are)
  const bf16x8 pb0 = __builtin_convertvector(p0, bf16x8), pb1 = __builtin_convertvector(p1, bf16x8);
  if (key0 + 32 > vlen) {  // slots without a token may hold codes that are no number
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int n = vlen - (key0 + 16 * H + 4 * w);  // slots of this word that hold one
      const uint32_t mask = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << 8 * n) - 1u;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) b.v[db][w] &= mask;
    }
  }
  if (key0 + 32 > len && len < vlen) hide_not_numbers<D>(b, O, key0, lim, H);
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    O[db] = mfma32(codes_to_bf16(b.v[db][0], b.v[db][1]), pb0, O[db]);
    O[db] = mfma32(codes_to_bf16(b.v[db][2], b.v[db][3]), pb1, O[db]);
  }
}

// Pages [p0, p1) of one list against the wave's 32 rows, two pages at a time, the next two on their way meanwhile (four of them are no
// faster).  What bounds it is how the pages come from memory: pages that nobody else reads pass the caches by (ONCE; 16 groups of 8 over
// 8192 | 1024 tokens 114 -> 101 us), and 1,300 to 1,800 waves ask for them, those of the KV heads of a page next to each other (-> 94 us =
// 5.7 TB/s; 2,048 waves 99, 3,072 102 to 123; the loads alone of 2,048 waves take 98.6).
template <int D, bool ONCE, typename QF>
__device__ __forceinline__ void stream_slice(const Q8Cache& c, const int32_t* pages, int p0, int p1, int len, int lim, int vlen, int hk,
                                             float sc, int lane, QF&& qop, f32x16* O, float& m, float& l) {
  const int L = lane & 31, H = lane >> 5, np = p1 - p0;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
  m = -1e30f;
  l = 0.f;
  int pg = 0;
  float ksv = 0.f, lvv = 0.f;
  auto window = [&](int rel) __attribute__((always_inline)) {  // of 64 pages, a lane each: id (clamped to the pool) and scales
    pg = min(max(pages[p0 + min(rel + lane, np - 1)], 0), c.n_pages - 1);
    ksv = c.k_scale[(size_t)pg * c.hkv + hk] * fabsf(sc);
    lvv = __builtin_amdgcn_logf(c.v_scale[(size_t)pg * c.hkv + hk]);
  };
  auto of_page = [&](float x, int rel) __attribute__((always_inline)) {  // of page rel + H
    const float a = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), rel & 63));
    const float b = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), min(rel + 1, np - 1) & 63));
    return H ? b : a;
  };
  struct Ahead {
    Block<D> b;
    float ks, lv;
  };
  Ahead x0, x1;
  auto load = [&](Ahead& x, int rel) __attribute__((always_inline)) {
    if (rel >= np) return;
    if ((rel & 63) == 0) {
      window(rel);
      asm volatile("" ::"v"(ksv), "v"(lvv));  // arrived: a wait for them later would also wait for the blocks in flight
    }
    x.ks = of_page(ksv, rel);
    x.lv = of_page(lvv, rel);
    load_block<D, ONCE>(x.b, c, pg, rel, np - 1, hk, L, H);
  };
  auto compute = [&](Ahead& x, int rel) __attribute__((always_inline)) {
    compute_block<D>(x.b, qop, O, m, l, x.ks, x.lv, (p0 + rel) * PAGE, len, lim, vlen, H);
  };
  load(x0, 0);
  for (int rel = 0;;) {
    load(x1, rel + 2);
    compute(x0, rel);
    if ((rel += 2) >= np) break;
    load(x0, rel + 2);
    compute(x1, rel);
    if ((rel += 2) >= np) break;
  }
}

// Query operands of the wave's rows in LDS: step 2 s + u has dims 16 (2 s + H) + 8 u .. of row L, with the sign of the softmax scale.
template <int D>
__device__ __forceinline__ void stage_q(bf16x8* qs, const uint16_t* row, float sc, int lane) {
  const uint16_t* const p = row + 16 * (lane >> 5);
  const uint32_t sign = sc < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    u32x4 x = *(const u32x4*)(p + 32 * (s >> 1) + 8 * (s & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] ^= sign;
    qs[s * 64 + lane] = __builtin_bit_cast(bf16x8, x);
  }
}

template <int D>
__device__ __forceinline__ void store_part(float* part_o, float* part_ml, size_t at, const f32x16* O, float m, float l, int H) {
  float* const po = part_o + at * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *(f32x4*)(po + 32 * db + 8 * r4 + 4 * H) = f32x4{O[db][4 * r4], O[db][4 * r4 + 1], O[db][4 * r4 + 2], O[db][4 * r4 + 3]};
  if (H == 0) *(float2*)(part_ml + at * 2) = make_float2(m, l);
}

// A wave to a work item: a slice of a group's shared pages against 32 of its (branch, query head) rows of a KV head, or a slice of a
// branch's own pages against its rows.
template <int D, bool ONCE>
__global__ void __launch_bounds__(64, 2) k_q8_decode(Q8DecodeArgs a) {
  __shared__ bf16x8 qs[(D / 16) * 64];
  const int lane = threadIdx.x, L = lane & 31, H = lane >> 5;
  const bool shared = (int)blockIdx.x < a.items_a;
  int x = shared ? blockIdx.x : blockIdx.x - a.items_a;
  const int hk = x % a.hkv;
  x /= a.hkv;
  const int splits = shared ? a.splits_a : a.splits_b, split = x % splits;
  x /= splits;
  int row0 = 0;
  if (shared) {
    row0 = x % a.rb_max * 32;
    x /= a.rb_max;
  }
  const int branch0 = shared ? a.group_branch_off[x] : x;
  const int nrows = shared ? (a.group_branch_off[x + 1] - branch0) * a.G : a.G;
  const int32_t* const pages = shared ? a.shared_pages + a.shared_page_off[x] : a.branch_pages + a.branch_page_off[x];
  const int len = shared ? a.shared_len[x] : a.branch_len[x], chunk = shared ? a.chunk_a : a.chunk_b;
  if (row0 >= nrows) return;
  const int npages = (len + PAGE - 1) / PAGE, p0 = split * chunk, p1 = min(p0 + chunk, npages);
  const int row = row0 + L;
  const bool row_ok = row < nrows;
  const int rr = row_ok ? row : row0, branch = branch0 + rr / a.G, head = hk * a.G + rr % a.G;
  if (branch < 0 || branch >= a.n_live) return;  // (offsets that point behind the branches)
  const size_t at = (size_t)((shared ? 0 : a.first_own) + branch * splits + split) * a.hq + head;
  if (p0 >= p1) {  // nothing there: a partial without weight
    if (row_ok && H == 0) *(float2*)(a.part_ml + at * 2) = make_float2(-1e30f, 0.f);
    return;
  }
  stage_q<D>(qs, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
  auto qop = [&](int s) { return qs[s * 64 + lane]; };
  f32x16 O[D / 32];
  float m, l;
  stream_slice<D, ONCE>(a.kv, pages, p0, p1, len, len, len, hk, a.sc, lane, qop, O, m, l);
  l += __shfl_xor(l, 32);
  if (row_ok) store_part<D>(a.part_o, a.part_ml, at, O, m, l, H);
}

// The same for the items that k_seg_plan listed.
template <int D, bool ONCE>
__global__ void __launch_bounds__(64, 2) k_q8_decode_seg(Q8SegArgs args) {
  __shared__ bf16x8 qs[(D / 16) * 64];
  const SegArgs& a = args.s;
  const int lane = threadIdx.x, L = lane & 31, H = lane >> 5;
  const int hk = blockIdx.x % a.hkv, idx = blockIdx.x / a.hkv;
  if (idx >= a.totals[0]) return;
  const SegItem it = a.items[idx];
  const int slice = (it.nsplit >> 23) & 0x1fe, nsplit = it.nsplit & 0xffffff;
  const int npages = min((it.len + PAGE - 1) / PAGE, a.chunk * a.splits);
  int p1 = __builtin_amdgcn_readfirstlane(min(it.p0 + slice, npages));
  if (it.row0 >= it.nrows || it.p0 >= p1) return;  // (never listed)
  const int row = it.row0 + L;
  const bool row_ok = row < it.nrows;
  const int rr = row_ok ? row : it.row0;
  const int entry = it.e0 + rr / a.G, head = hk * a.G + rr % a.G, place = it.place + rr / a.G * nsplit;
  const bool there = entry >= 0 && entry < a.total_readers;
  const bool store_ok = row_ok && there && place < a.splits * a.total_readers;  // (reader lists longer than announced: no partial)
  const size_t at = (size_t)place * a.hq + head;
  int lim = it.len, lim_min = it.len;
  if (a.seg_reader_len) {
    lim = min(max(there ? a.seg_reader_len[entry] : 0, 0), it.len);
    int lim_max = lim;
    lim_min = lim;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      lim_max = max(lim_max, __shfl_xor(lim_max, o));
      lim_min = min(lim_min, __shfl_xor(lim_min, o));
    }
    p1 = min(p1, (lim_max + PAGE - 1) / PAGE);
    if (it.p0 >= p1) {
      if (store_ok && H == 0) *(float2*)(a.part_ml + at * 2) = make_float2(-1e30f, 0.f);
      return;
    }
  }
  const int branch = there ? min(max(a.seg_readers[entry], 0), a.n_live - 1) : 0;
  stage_q<D>(qs, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
  auto qop = [&](int s) { return qs[s * 64 + lane]; };
  f32x16 O[D / 32];
  float m, l;
  stream_slice<D, ONCE>(args.kv, a.seg_pages + it.page_off, it.p0, p1, lim_min, lim, it.len, hk, a.sc, lane, qop, O, m, l);
  l += __shfl_xor(l, 32);
  if (store_ok) store_part<D>(a.part_o, a.part_ml, at, O, m, l, H);
}

// A wave to a (branch, query head): its partials are put together by their references, 64 at a time a lane each has reference and
// sum of.  No weight anywhere: zeros.  place(i): where partial i lies, -1 for none.
template <int D, typename F>
__device__ __forceinline__ void merge_parts(const float* part_o, const float* part_ml, int hq, int head, int n, F&& place, uint16_t* out, int lane) {
  constexpr int PER = D / 64, BATCH = 8;
  float acc[PER], top = -1e30f, total = 0.f;
#pragma unroll
  for (int t = 0; t < PER; ++t) acc[t] = 0.f;
  for (int b = 0; b < n; b += 64) {
    float m = -1e30f, l = 0.f;
    uint32_t at = 0;
    if (b + lane < n) {
      const int p = place(b + lane);
      if (p >= 0) {
        at = (uint32_t)p * (uint32_t)hq + (uint32_t)head;
        const float2 ml = *(const float2*)(part_ml + (size_t)at * 2);
        if (!(ml.y <= 0.f)) {  // (not a number: it reaches the result)
          m = ml.x;
          l = ml.y;
        }
      }
    }
    const float mn = fmaxf(top, dag_wave_max(m)), keep = __builtin_amdgcn_exp2f(top - mn);
    const bool live = !(l <= 0.f);
    const float wgt = live ? __builtin_amdgcn_exp2f(m - mn) : 0.f;
    total = total * keep + dag_wave_sum(l * wgt);
    top = mn;
#pragma unroll
    for (int t = 0; t < PER; ++t) acc[t] *= keep;
    for (unsigned long long left = __builtin_amdgcn_ballot_w64(live); left;) {
      float w[BATCH], x[BATCH][PER];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int j = left ? __builtin_ctzll(left) : 0;
        w[i] = left ? __shfl(wgt, j) : 0.f;
        const float* const o = part_o + (size_t)(uint32_t)__shfl((int)at, j) * D + lane * PER;
        const bool there = left != 0;
        left &= left - 1;
#pragma unroll
        for (int t = 0; t < PER; ++t) x[i][t] = there ? o[t] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
#pragma unroll
        for (int t = 0; t < PER; ++t) acc[t] = fmaf(w[i], x[i][t], acc[t]);
    }
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* const o = out + lane * PER;
  if constexpr (PER == 2) *(uint32_t*)o = dag_pack_bf2(acc[0] * inv, acc[1] * inv);
  else o[0] = (uint16_t)dag_f2bf(acc[0] * inv);
}

template <int D>
__global__ void __launch_bounds__(64) k_q8_merge(Q8DecodeArgs a) {
  const int r = blockIdx.x / a.hq, head = blockIdx.x % a.hq;
  auto place = [&](int i) { return i < a.splits_a ? r * a.splits_a + i : a.first_own + r * a.splits_b + i - a.splits_a; };
  merge_parts<D>(a.part_o, a.part_ml, a.hq, head, a.splits_a + a.splits_b, place, a.out + (size_t)blockIdx.x * D, threadIdx.x);
}

template <int D>
__global__ void __launch_bounds__(64) k_q8_merge_seg(Q8SegArgs args) {
  const SegArgs& a = args.s;
  const int r = blockIdx.x / a.hq, head = blockIdx.x % a.hq;
  const int e0 = a.branch_entry_off[r], splits = a.splits > 0 ? a.totals[2] : 0;
  auto place = [&](int i) {
    const int entry = a.branch_entries[e0 + i / splits];
    if (entry < 0 || entry >= a.total_readers) return -1;
    const int p = a.entry_first[entry] + i % splits;
    const int behind = min(entry + 1 < a.total_readers ? a.entry_first[entry + 1] : a.totals[1], a.splits * a.total_readers);
    return p >= 0 && p < behind ? p : -1;
  };
  merge_parts<D>(a.part_o, a.part_ml, a.hq, head, (a.branch_entry_off[r + 1] - e0) * splits, place, a.out + (size_t)blockIdx.x * D, threadIdx.x);
}

int q8_cache(const dag_kv_q8_t* kv, Q8Cache* c) {
  if (!kv) return DAG_ERR_NULL;
  if (kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  *c = Q8Cache{(const uint8_t*)kv->k_pool, (const uint8_t*)kv->v_pool, kv->k_scale, kv->v_scale, kv->n_pages, kv->hkv};
  return DAG_OK;
}
int q8_pointers(const Q8Cache& c) {
  if (!c.k_pool || !c.v_pool || !c.k_scale || !c.v_scale) return DAG_ERR_NULL;
  return dag_aligned16(c.k_pool) && dag_aligned16(c.v_pool) && ((uintptr_t)c.k_scale & 3) == 0 && ((uintptr_t)c.v_scale & 3) == 0 ? DAG_OK : DAG_ERR_ALIGN;
}

}  // namespace

extern "C" size_t dag_decode_q8_workspace_bytes(const dag_decode_desc_t* desc, int32_t hq, int32_t hkv, int32_t head_dim) {
  Q8Plan p;
  return make_q8_plan(desc, hq, hkv, head_dim, &p) == DAG_OK ? p.bytes : 0;
}

extern "C" int dag_attn_decode_q8(const dag_decode_desc_t* d, const dag_kv_q8_t* kv, const void* q, void* out, int32_t hq, float softmax_scale,
                                  void* ws, size_t ws_bytes, void* stream_) {
  Q8DecodeArgs a;
  int rc = q8_cache(kv, &a.kv);
  if (rc != DAG_OK) return rc;
  Q8Plan p;
  const int D = kv->head_dim;
  rc = make_q8_plan(d, hq, kv->hkv, D, &p);
  if (rc != DAG_OK) return rc;
  if (d->n_live == 0) return DAG_OK;
  if (!q || !out) return DAG_ERR_NULL;
  if (p.items_a > 0 && (!d->group_branch_off || !d->shared_page_off || !d->shared_pages || !d->shared_len)) return DAG_ERR_NULL;
  if (p.items_b > 0 && (!d->branch_page_off || !d->branch_pages || !d->branch_len)) return DAG_ERR_NULL;
  if (p.items_a + p.items_b > 0) {
    rc = q8_pointers(a.kv);
    if (rc != DAG_OK) return rc;
    if (a.kv.n_pages < 1) return DAG_ERR_BAD_LEN;
  }
  if (!dag_aligned16(q) || !dag_aligned16(out)) return DAG_ERR_ALIGN;
  if (!ws || ws_bytes < p.bytes) return DAG_ERR_WORKSPACE;
  char* const base = (char*)dag_align_up((size_t)(uintptr_t)ws, 256);
  a.group_branch_off = d->group_branch_off;
  a.shared_page_off = d->shared_page_off;
  a.shared_pages = d->shared_pages;
  a.shared_len = d->shared_len;
  a.branch_page_off = d->branch_page_off;
  a.branch_pages = d->branch_pages;
  a.branch_len = d->branch_len;
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.part_o = (float*)base;
  a.part_ml = (float*)(base + p.off_ml);
  a.first_own = d->n_live * p.splits_a;
  a.n_live = d->n_live;
  a.hq = hq;
  a.hkv = kv->hkv;
  a.G = hq / kv->hkv;
  a.rb_max = p.rb_max;
  a.chunk_a = p.chunk_a;
  a.splits_a = p.splits_a;
  a.chunk_b = p.chunk_b;
  a.splits_b = p.splits_b;
  a.items_a = p.items_a;
  a.sc = softmax_scale * 1.4426950408889634f;
  hipStream_t stream = (hipStream_t)stream_;
  if (p.items_a + p.items_b > 0) {
    auto* const kernel = p.rb_max <= 1 ? (D == 128 ? k_q8_decode<128, true> : k_q8_decode<64, true>)
                                       : (D == 128 ? k_q8_decode<128, false> : k_q8_decode<64, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items_a + p.items_b)), dim3(64), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(D == 128 ? k_q8_merge<128> : k_q8_merge<64>, dim3((unsigned)(d->n_live * hq)), dim3(64), 0, stream, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

extern "C" size_t dag_decode_segments_q8_workspace_bytes(const dag_decode_seg_desc_t* desc, int32_t hq, int32_t hkv, int32_t head_dim) {
  SegPlan p;
  return make_seg_plan(desc, hq, hkv, head_dim, DecodeKnobs{0, 0, 0}, &p) == DAG_OK ? p.bytes : 0;
}

extern "C" int dag_attn_decode_segments_q8(const dag_decode_seg_desc_t* d, const dag_kv_q8_t* kv, const void* q, void* out, int32_t hq,
                                           float softmax_scale, void* ws, size_t ws_bytes, void* stream_) {
  Q8SegArgs args = {};
  int rc = q8_cache(kv, &args.kv);
  if (rc != DAG_OK) return rc;
  SegPlan p;
  const int D = kv->head_dim, hkv = kv->hkv;
  rc = make_seg_plan(d, hq, hkv, D, DecodeKnobs{0, 0, 0}, &p);
  if (rc != DAG_OK) return rc;
  if (d->n_live == 0) return DAG_OK;
  if (!q || !out || !d->branch_entry_off || !d->branch_entries) return DAG_ERR_NULL;
  if (d->n_segments > 0 && (!d->seg_page_off || !d->seg_pages || !d->seg_len || !d->seg_reader_off || !d->seg_readers)) return DAG_ERR_NULL;
  if (p.items > 0) {
    rc = q8_pointers(args.kv);
    if (rc != DAG_OK) return rc;
    if (args.kv.n_pages < 1) return DAG_ERR_BAD_LEN;
  }
  if (!dag_aligned16(q) || !dag_aligned16(out)) return DAG_ERR_ALIGN;
  if ((int64_t)d->n_live * hq > INT32_MAX) return DAG_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < p.bytes) return DAG_ERR_WORKSPACE;
  char* const base = (char*)dag_align_up((size_t)(uintptr_t)ws, 256);
  SegArgs& a = args.s;
  a.seg_page_off = d->seg_page_off;
  a.seg_pages = d->seg_pages;
  a.seg_len = d->seg_len;
  a.seg_reader_off = d->seg_reader_off;
  a.seg_readers = d->seg_readers;
  a.seg_reader_len = d->seg_reader_len;
  a.branch_entry_off = d->branch_entry_off;
  a.branch_entries = d->branch_entries;
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.part_o = (float*)(base + p.off_o);
  a.part_ml = (float*)(base + p.off_ml);
  a.items = (SegItem*)(base + p.off_items);
  a.totals = (int32_t*)(base + p.off_total);
  a.entry_first = (int32_t*)(base + p.off_first);
  a.item_cap = (int)p.items;
  a.n_segments = d->n_segments;
  a.n_live = d->n_live;
  a.hq = hq;
  a.hkv = hkv;
  a.G = hq / hkv;
  a.rb_max = p.rb_max;
  a.chunk = p.chunk;
  a.splits = p.splits;
  a.total_readers = d->total_readers;
  a.fixed = false;
  a.weight = (float)hkv * (float)D / 128.f;
  const int64_t most_pages = (int64_t)d->n_segments * p.rb_max * d->max_seg_pages * hkv * D;
  a.few = p.chunk == 8 && most_pages < (d->max_seg_pages <= SEG_SHORT ? SEG_PAGES_16_SHORT : SEG_PAGES_16) * 128;
  a.sc = softmax_scale * 1.4426950408889634f;
  hipStream_t stream = (hipStream_t)stream_;
  if (p.items > 0) {
    const int64_t waves = dag_ceil_div(d->n_segments, 64);
    hipLaunchKernelGGL(k_seg_plan, dim3(1), dim3((unsigned)(waves * 64 < PLAN_THREADS ? waves * 64 : PLAN_THREADS)), 0, stream, a);
    DAG_LAUNCH_CHECK();
    auto* const kernel = p.rb_max <= 1 ? (D == 128 ? k_q8_decode_seg<128, true> : k_q8_decode_seg<64, true>)
                                       : (D == 128 ? k_q8_decode_seg<128, false> : k_q8_decode_seg<64, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items * hkv)), dim3(64), 0, stream, args);
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(D == 128 ? k_q8_merge_seg<128> : k_q8_merge_seg<64>, dim3((unsigned)(d->n_live * hq)), dim3(64), 0, stream, args);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}
