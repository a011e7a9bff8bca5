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

__device__ __forceinline__ float other_half(float x) { return __uint_as_float(dag_other_group<32>(__float_as_uint(x))); }  // of lane ^ 32

template <int D>
struct Block {         // 32 keys (two pages)
  u32x4 k[D / 32];     // k[s]: dims 16 (2 s + H) .. of the key of MFMA row L
  u32x4 v[D / 32];     // v[db]: the slots of page H of dimension 32 db + L
};

template <int D>
__device__ __forceinline__ void load_block(Block<D>& b, const Q8Cache& c, int pages, int rel, int last_rel, int hk, int L, int H) {
  const int pg0 = __builtin_amdgcn_readlane(pages, min(rel, last_rel) & 63), pg1 = __builtin_amdgcn_readlane(pages, min(rel + 1, last_rel) & 63);
  const int slot = (L & 3) + 4 * (L >> 3);
  const size_t base0 = ((size_t)pg0 * c.hkv + hk) * (D * PAGE), base1 = ((size_t)pg1 * c.hkv + hk) * (D * PAGE);
  const uint8_t* const kp = c.k_pool + ((L >> 2) & 1 ? base1 : base0) + H * 256 + slot * 16;
  const uint8_t* const vp = c.v_pool + (H ? base1 : base0) + L * 16;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.k[s] = __builtin_nontemporal_load((const u32x4*)(kp + s * 512));
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.v[s] = __builtin_nontemporal_load((const u32x4*)(vp + s * 512));
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

// The reference to at least bm, the sums with it.
template <int D>
__device__ __forceinline__ void raise(f32x16* O, float& m, float& l, float bm) {
  const float m_new = fmaxf(m, bm), alpha = __builtin_amdgcn_exp2f(m - m_new);
  l *= alpha;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] *= alpha;
  m = m_new;
}

// Slots from vlen on hold no token: their codes may be no numbers, which a probability of zero does not keep from the sums.
template <int D>
__device__ __forceinline__ void clear_behind(Block<D>& b, int key0, int vlen, int H) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = vlen - (key0 + 16 * H + 4 * w);  // slots of this word that hold one
    const uint32_t mask = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << 8 * n) - 1u;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) b.v[db][w] &= mask;
  }
}

// U blocks together: scores, probabilities, their product with the values.  ks: key scale of the lane's page times |softmax scale| log2(e),
// lv: log2 of its value scale.  A lane's 16 scores of a block are of one page, so their largest is found among the plain products, one
// multiply-add gives the exponent with the value scale in it, and the sum of a lane loses that factor again once.
// key0: first key of the first block; keys from `lim` on are hidden from this lane's row; len: the smallest lim of the wave; slots from vlen on
// hold no token.  What bounds a wave by itself is the chain from the scores to the second product: two blocks share it.
template <int D, int U, bool LIMITS, typename QF, typename VF>
__device__ __forceinline__ void compute_blocks(Block<D> (&b)[U], QF&& q, VF&& values, f32x16* O, float& m, float& l, const float (&ks)[U],
                                               const float (&lv)[U], int key0, int len, int lim, int vlen, int H) {
  f32x16 S[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[u][r] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
#pragma unroll
    for (int u = 0; u < U; ++u) S[u] = mfma32(codes_to_bf16(b[u].k[s][0], b[u].k[s][1]), q(2 * s), S[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) S[u] = mfma32(codes_to_bf16(b[u].k[s][2], b[u].k[s][3]), q(2 * s + 1), S[u]);
  }
  values(b);
  if (key0 + 32 * U > len) {
    asm volatile("");  // (a branch: the compiler would compare and select in every block)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[u][r] = key0 + 32 * u + 16 * H + r < lim ? S[u][r] : -INFINITY;
  }
  float bm = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x = S[u][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) x = fmaxf(x, S[u][r]);
    bm = fmaxf(bm, x * ks[u]);
  }
  bm = fmaxf(bm, other_half(bm));
  if (__builtin_amdgcn_ballot_w64(bm > m + Q8_TH) != 0) raise<D>(O, m, l, bm);
  bf16x8 p[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float ref = lv[u] - m;
    f32x8 x[2];
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r >> 3][r & 7] = __builtin_amdgcn_exp2f(fmaf(S[u][r], ks[u], ref));
      sum[r >> 3] += x[r >> 3][r & 7];
    }
    l = fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-lv[u]), l);
    // (rounded to bf16, as the probabilities over a bf16 cache are)
    p[u][0] = __builtin_convertvector(x[0], bf16x8);
    p[u][1] = __builtin_convertvector(x[1], bf16x8);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int first = key0 + 32 * u;
    if (first + 32 > vlen) clear_behind<D>(b[u], first, vlen, H);
    if constexpr (LIMITS)
      if (first + 32 > len && len < vlen) hide_not_numbers<D>(b[u], O, first, lim, H);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) O[db] = mfma32(codes_to_bf16(b[u].v[db][2 * i], b[u].v[db][2 * i + 1]), p[u][i], O[db]);
}

// Pages [p0, p1) of one list against the wave's 32 rows, two pages at a time, the next two on their way meanwhile (four of them are no
// faster).  What bounds it is how the pages come from memory: pages that nobody else reads pass the caches by (ONCE; 16 groups of 8 over
// 8192 | 1024 tokens 114 -> 101 us), and 1,300 to 1,800 waves ask for them, those of the KV heads of a page next to each other (-> 94 us =
// 5.7 TB/s; 2,048 waves 99, 3,072 102 to 123; the loads alone of 2,048 waves take 98.6).
template <int D, bool LIMITS>
__device__ __forceinline__ void stream_slice(const Q8Cache& c, const int32_t* pages, int p0, int p1, int len, int lim, int vlen, int hk,
                                             float sc, int lane, const bf16x8 (&q)[D / 16], f32x16* O, float& m, float& l) {
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
    const float a = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), min(rel, np - 1) & 63));
    const float b = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), min(rel + 1, np - 1) & 63));
    return H ? b : a;
  };
  struct Ahead {
    Block<D> b[1];
    float ks[1], lv[1];
  };
  Ahead x0, x1;
  auto load = [&](Ahead& x, int rel) __attribute__((always_inline)) {
    if ((rel & 63) == 0 && rel < np) {
      window(rel);
      asm volatile("" ::"v"(ksv), "v"(lvv));  // arrived: a wait for them later would also wait for the blocks in flight
    }
    x.ks[0] = of_page(ksv, rel);
    x.lv[0] = of_page(lvv, rel);
    load_block<D>(x.b[0], c, pg, rel, np - 1, hk, L, H);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&](Ahead& x, int rel) __attribute__((always_inline)) {
    compute_blocks<D, 1, LIMITS>(x.b, [&](int s) { return q[s]; }, [](auto&) {}, O, m, l, x.ks, x.lv, (p0 + rel) * PAGE, len, lim, vlen, H);
    __builtin_amdgcn_sched_barrier(0);
  };
  // No load behind a condition: the wait for a block would then be one for the block behind it as well.  What is loaded behind the slice is
  // its last page again, which nobody uses.
  load(x0, 0);
  for (int rel = 0; rel < np; rel += 4) {
    load(x1, rel + 2);
    compute(x0, rel);
    load(x0, rel + 4);
    if (rel + 2 < np) compute(x1, rel + 2);
  }
}

// Query operands of the lane's row: step 2 s + u has dims 16 (2 s + H) + 8 u .., with the sign of the softmax scale.
template <int D>
__device__ __forceinline__ void load_q(bf16x8 (&q)[D / 16], const uint16_t* row, float sc, int lane) {
  const uint16_t* const p = row + 16 * (lane >> 5);
  const uint32_t sign = sc < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    u32x4 x = *(const u32x4*)(p + 32 * (s >> 1) + 8 * (s & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] ^= sign;
    q[s] = __builtin_bit_cast(bf16x8, x);
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
template <int D>
__global__ void __launch_bounds__(64, 2) k_q8_decode(Q8DecodeArgs a) {
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
  bf16x8 q[D / 16];
  load_q<D>(q, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
  f32x16 O[D / 32];
  float m, l;
  stream_slice<D, false>(a.kv, pages, p0, p1, len, len, len, hk, a.sc, lane, q, O, m, l);
  l += other_half(l);
  if (row_ok) store_part<D>(a.part_o, a.part_ml, at, O, m, l, H);
}

// The same for the items that k_seg_plan listed.
template <int D, bool LIMITS>
__global__ void __launch_bounds__(64, 2) k_q8_decode_seg(Q8SegArgs args) {
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
  if constexpr (LIMITS) {
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
  bf16x8 q[D / 16];
  load_q<D>(q, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
  f32x16 O[D / 32];
  float m, l;
  stream_slice<D, LIMITS>(args.kv, a.seg_pages + it.page_off, it.p0, p1, lim_min, lim, it.len, hk, a.sc, lane, q, O, m, l);
  l += other_half(l);
  if (store_ok) store_part<D>(a.part_o, a.part_ml, at, O, m, l, H);
}

// Lists with more than 32 rows of a KV head: a workgroup of eight waves takes up to eight blocks of 32 rows together, so that a page comes
// from memory once for all of them.  Tiles of four pages (two units of 32 keys) go straight into a ring in LDS, codes as they are (a page is
// the operand image), and every wave makes its own operands of them.  Up to four blocks: the waves w, w + blocks, .. share a block, its
// units in turn; five to seven: waves 0 to 3 have one each and the others share what is left, so that the SIMDs have the same
// to do.  Waves of one block put their sums together in LDS at the end.
// A wave is a pipeline: in one run of instructions the scores of its next unit and the exponentials of this one, in the next run
// this one's product with the values and the next one's maximum.  One after the other, the matrix and the vector pipe take turns in both waves of a
// SIMD, which the tiles keep in step: 1,700 cycles a unit, of which they need 520 and 960 (two groups of 32 over 32768 | 640,
// 5 heads on one: 93 us, so FIGURE).
constexpr int WG_WAVES = 8, WG_TILE = 4, WG_RING = 8;
static_assert(WG_ROWS == 32 * WG_WAVES && WG_MOST_PAGES >= 9 << 4, "");
constexpr int WG_SCALES = 192;  // pages of a slice: three windows of 64
constexpr int K_PAD = 128;  // bytes behind a page's keys: the 16 slots of two pages that are read together lie on all banks
template <int D>
constexpr int wg_lds_bytes() {  // the ring, or the sums of the waves in its place
  constexpr int tiles = WG_RING * WG_TILE * (2 * D * PAGE + K_PAD) + WG_SCALES * 8, sums = WG_WAVES * (D / 2 + 2) * 64 * 4;
  return tiles > sums ? tiles : sums;
}

struct WgShare {  // of a wave: its block, which of the waves of the block it is, how many there are, the first one, what lies between them
  int block, sub, parts, first, step;
  int most;  // largest number of waves of a block
};
__device__ __forceinline__ WgShare wg_share(int w, int blocks) {
  if (blocks > 4) {
    const int left = blocks - 4, b = (w - 4) % left;
    const int most = (WG_WAVES - 4 + left - 1) / left;
    return w < 4 ? WgShare{w, 0, 1, w, 1, most} : WgShare{4 + b, (w - 4) / left, (WG_WAVES - 4 - b + left - 1) / left, 4 + b, left, most};
  }
  return WgShare{w % blocks, w / blocks, (WG_WAVES - w % blocks + blocks - 1) / blocks, w % blocks, blocks, (WG_WAVES + blocks - 1) / blocks};
}

// What a unit needs of LDS in one round trip: the next unit's scales and keys, this one's values.  (Reads and their wait in one block: to the
// compiler a register that a read has been told to fill holds its value already.)
__device__ __forceinline__ void lds_unit(u32x2& scales, u32x4 (&k)[4], u32x4 (&v)[4], uint32_t s_at, uint32_t k_at, uint32_t v_at) {
  asm volatile(
      "ds_read_b64 %0, %9\n\t"
      "ds_read_b128 %1, %10\n\tds_read_b128 %2, %10 offset:512\n\tds_read_b128 %3, %10 offset:1024\n\tds_read_b128 %4, %10 offset:1536\n\t"
      "ds_read_b128 %5, %11\n\tds_read_b128 %6, %11 offset:512\n\tds_read_b128 %7, %11 offset:1024\n\tds_read_b128 %8, %11 offset:1536\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(scales), "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
      : "v"(s_at), "v"(k_at), "v"(v_at));
}
__device__ __forceinline__ void lds_unit(u32x2& scales, u32x4 (&k)[2], u32x4 (&v)[2], uint32_t s_at, uint32_t k_at, uint32_t v_at) {
  asm volatile(
      "ds_read_b64 %0, %5\n\tds_read_b128 %1, %6\n\tds_read_b128 %2, %6 offset:512\n\t"
      "ds_read_b128 %3, %7\n\tds_read_b128 %4, %7 offset:512\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(scales), "=&v"(k[0]), "=&v"(k[1]), "=&v"(v[0]), "=&v"(v[1])
      : "v"(s_at), "v"(k_at), "v"(v_at));
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14)); }

template <int D, bool LIMITS>
__device__ __forceinline__ void wg_stream(const Q8Cache& c, const int32_t* pages, int p0, int p1, int len, int lim, int vlen, int hk, float sc,
                                          unsigned char* smem, int w, int lane, int sub, int parts, int most_parts, const bf16x8 (&q)[D / 16], f32x16* O, float& m,
                                          float& l) {
  constexpr int PB = D * PAGE, KB = PB + K_PAD, PLACE = WG_TILE * (KB + PB);
  const int L = lane & 31, H = lane >> 5, np = p1 - p0, nt = (np + WG_TILE - 1) / WG_TILE, nu = (np + 1) / 2;
  static_assert(WG_MOST_PAGES <= WG_SCALES, "");
  auto page_of = [&](int i) { return min(max(pages[p0 + min(i + lane, np - 1)], 0), c.n_pages - 1); };
  const int pg0 = page_of(0), pg1 = page_of(64), pg2 = page_of(128);
  // Scales of the slice's pages to LDS, behind the ring: the waves take turns with the windows of 64.
  float2* const scales = (float2*)(smem + WG_RING * PLACE);
  const int mine64 = w < 3 ? w : 0, pgs = mine64 == 0 ? pg0 : mine64 == 1 ? pg1 : pg2;
  const float ks_here = c.k_scale[(size_t)pgs * c.hkv + hk] * fabsf(sc), vs_here = c.v_scale[(size_t)pgs * c.hkv + hk];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) asm volatile("" ::"v"(q[s]));
  // A wave brings 1 KiB of the keys and of the values of a page of the tile, at dimension 64 of either.
  constexpr int LOADS = D / 64;
  const int mine = D == 128 ? w >> 1 : w & 3, at = D == 128 ? (w & 1) * 1024 : 0;
  auto pick = [](int x, int y, int z, int i) __attribute__((always_inline)) {  // (by value: a choice between captured ones is one of addresses)
    return __builtin_amdgcn_readlane(i < 64 ? x : i < 128 ? y : z, i & 63);
  };
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= nt) return;
    const size_t src = ((size_t)pick(pg0, pg1, pg2, min(WG_TILE * t + mine, np - 1)) * c.hkv + hk) * PB + at + lane * 16;
    unsigned char* const place = smem + t % WG_RING * PLACE;
    typedef __attribute__((address_space(1))) const void* from_t;
    typedef __attribute__((address_space(3))) void* to_t;
    if (D == 128 || w < 4) __builtin_amdgcn_global_load_lds((from_t)(c.k_pool + src), (to_t)(place + mine * KB + at), 16, 0, 0);
    if (D == 128 || w >= 4) __builtin_amdgcn_global_load_lds((from_t)(c.v_pool + src), (to_t)(place + WG_TILE * KB + mine * PB + at), 16, 0, 0);
  };
  // Tile t is there for everybody.  A wave still has to read the values of its last unit, `parts` units in front of its next one: in a tile
  // up to (parts + 1) / 2 in front of t, which no tile may replace that is asked for up to here.
  const int ahead = WG_RING - 1 - (most_parts + 1) / 2;
  auto arrive = [&](int t) __attribute__((always_inline)) {
    static_assert(WG_RING == 8, "");
    switch (min(nt - 1 - t, ahead - 1)) {  // tiles under way behind it
      case 0: wait_vmcnt<0>(); break;
      case 1: wait_vmcnt<LOADS>(); break;
      case 2: wait_vmcnt<2 * LOADS>(); break;
      case 3: wait_vmcnt<3 * LOADS>(); break;
      case 4: wait_vmcnt<4 * LOADS>(); break;
      default: wait_vmcnt<5 * LOADS>();
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    issue(t + ahead);
  };
  for (int t = 0; t < ahead; ++t) issue(t);
  if (w < 3) scales[64 * w + lane] = make_float2(ks_here, __builtin_amdgcn_logf(vs_here));
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)smem;
  const uint32_t koff = ring + ((L >> 2) & 1) * KB + H * 256 + ((L & 3) + 4 * (L >> 3)) * 16, voff = ring + WG_TILE * KB + H * PB + L * 16;
  const uint32_t soff = ring + WG_RING * PLACE + H * 8;
  // What lies behind the slice in its last unit is its last page again, hidden like what lies behind the list.
  len = min(len, p1 * PAGE);
  lim = min(lim, p1 * PAGE);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
  m = -1e30f;
  l = 0.f;
  f32x16 S;
#pragma unroll
  for (int r = 0; r < 16; ++r) S[r] = -INFINITY;
  float ks = 1.f, lv = 0.f;
  // This wave's unit u, whose scores are in S, and the scores of unit n behind it.  (The first call has no unit u yet: hidden scores, and the
  // values of unit n.)
  auto unit = [&](int u, int n) __attribute__((always_inline)) {
    Block<D> b[1];
    u32x2 next;
    const int tu = u >> 1, tn = n >> 1;
    lds_unit(next, b[0].k, b[0].v, soff + 16 * n, koff + tn % WG_RING * PLACE + (n & 1) * 2 * KB, voff + tu % WG_RING * PLACE + (u & 1) * 2 * PB);
    const float ref = lv - m;
    f32x16 T;
    f32x8 x[2];
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) T[r] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      T = mfma32(codes_to_bf16(b[0].k[s >> 1][2 * (s & 1)], b[0].k[s >> 1][2 * (s & 1) + 1]), q[s], T);
#pragma unroll
      for (int r = s * 256 / D; r < (s + 1) * 256 / D; ++r) {
        x[r >> 3][r & 7] = __builtin_amdgcn_exp2f(fmaf(S[r], ks, ref));
        sum[r >> 3] += x[r >> 3][r & 7];
      }
    }
    l = fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-lv), l);
    bf16x8 p[2] = {__builtin_convertvector(x[0], bf16x8), __builtin_convertvector(x[1], bf16x8)};
    // (done here, beside the scores: the compiler would move it behind the branches below, to where it is used)
    asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(l));
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {  // vector instructions (0x2), one MFMA (0x8), in turn
      __builtin_amdgcn_sched_group_barrier(0x002, 4 + 64 / (D / 16), 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    ks = __uint_as_float(next[0]);
    lv = __uint_as_float(next[1]);
    const int key_n = (p0 + 2 * n) * PAGE, key_u = (p0 + 2 * u) * PAGE;
    if (key_n + 32 > len) {
      asm volatile("");
#pragma unroll
      for (int r = 0; r < 16; ++r) T[r] = key_n + 16 * H + r < lim ? T[r] : -INFINITY;
    }
    if (key_u + 32 > vlen) {
      asm volatile("");
      clear_behind<D>(b[0], key_u, vlen, H);
    }
    if constexpr (LIMITS)
      if (key_u + 32 > len && len < vlen) hide_not_numbers<D>(b[0], O, key_u, lim, H);
    float bm = T[0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) O[db] = mfma32(codes_to_bf16(b[0].v[db][2 * i], b[0].v[db][2 * i + 1]), p[i], O[db]);
#pragma unroll
    for (int r = 1; r < 16; ++r) bm = fmaxf(bm, T[r]);
    bm *= ks;
    bm = fmaxf(bm, other_half(bm));
    if (__builtin_amdgcn_ballot_w64(bm > m + Q8_TH) != 0) raise<D>(O, m, l, bm);
    S = T;
  };
  int u = -1, n = sub, t = 0;  // (a unit past the last one: nothing but the end of the pipeline)
  auto reach = [&](int tile) __attribute__((always_inline)) {
    for (; t <= tile; ++t) arrive(t);
  };
#pragma unroll 1
  for (; n < nu; n += parts) {
    reach(n >> 1);
    unit(u < 0 ? n : u, n);
    u = n;
  }
  reach(nt - 1);
  if (u >= 0) unit(u, u);
  __syncthreads();
}

// The rest of an item: sums of the waves of a block put together, a range of dimensions each, and stored.  (The ring is free.)
template <int D>
__device__ __forceinline__ void wg_store(float* smem, const WgShare& s, int w, int lane, f32x16* O, float m, float l, bool row_ok, float* part_o,
                                         float* part_ml, size_t at) {
  constexpr int DB = D / 32, EACH = (16 * DB + 2) * 64;
  const int H = lane >> 5;
  l += other_half(l);
  if (s.parts > 1) {
    float* const mine = smem + w * EACH + lane;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) mine[(16 * db + r) * 64] = O[db][r];
    mine[16 * DB * 64] = m;
    mine[(16 * DB + 1) * 64] = l;
  }
  __syncthreads();
  if (s.parts > 1) {
    float top = -1e30f;
    for (int p = 0; p < s.parts; ++p) top = fmaxf(top, smem[(s.first + p * s.step) * EACH + 16 * DB * 64 + lane]);
    float total = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      if (db % s.parts == s.sub)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
    for (int p = 0; p < s.parts; ++p) {
      const float* const theirs = smem + (s.first + p * s.step) * EACH + lane;
      const float wgt = __builtin_amdgcn_exp2f(theirs[16 * DB * 64] - top);
      total = fmaf(theirs[(16 * DB + 1) * 64], wgt, total);
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (db % s.parts == s.sub)
#pragma unroll
          for (int r = 0; r < 16; ++r) O[db][r] = fmaf(theirs[(16 * db + r) * 64], wgt, O[db][r]);
    }
    m = top;
    l = total;
  }
  if (!row_ok) return;
  float* const po = part_o + at * D;
#pragma unroll
  for (int db = 0; db < DB; ++db)
    if (db % s.parts == s.sub)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *(f32x4*)(po + 32 * db + 8 * r4 + 4 * H) = f32x4{O[db][4 * r4], O[db][4 * r4 + 1], O[db][4 * r4 + 2], O[db][4 * r4 + 3]};
  if (H == 0 && s.sub == 0) *(float2*)(part_ml + at * 2) = make_float2(m, l);
}

// Workgroups with own items, a wave each, then with shared ones.
template <int D>
__global__ void __launch_bounds__(64 * WG_WAVES, 2) k_q8_decode_wg(Q8DecodeArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, L = lane & 31;
  f32x16 O[D / 32];
  float m, l;
  const int own = gridDim.x - a.items_a;
  if ((int)blockIdx.x >= own) {
    int x = blockIdx.x - own;
    const int hk = x % a.hkv;
    x /= a.hkv;
    const int rb = x % a.rb_max;
    x /= a.rb_max;
    const int split = x % a.splits_a, g = x / a.splits_a;
    const int branch0 = a.group_branch_off[g], nrows = (a.group_branch_off[g + 1] - branch0) * a.G, len = a.shared_len[g];
    const int row0 = rb * WG_ROWS;
    if (row0 >= nrows) return;
    const int p0 = split * a.chunk_a, p1 = min(p0 + a.chunk_a, (len + PAGE - 1) / PAGE);
    const WgShare s = wg_share(w, min((nrows - row0 + 31) / 32, WG_WAVES));
    const int row = row0 + 32 * s.block + L;
    const bool row_ok = row < nrows;
    const int rr = row_ok ? row : row0, branch = min(max(branch0 + rr / a.G, 0), a.n_live - 1), head = hk * a.G + rr % a.G;
    const size_t at = (size_t)(branch * a.splits_a + split) * a.hq + head;
    if (p0 >= p1) {
      if (row_ok && s.sub == 0 && lane < 32) *(float2*)(a.part_ml + at * 2) = make_float2(-1e30f, 0.f);
      return;
    }
    bf16x8 q[D / 16];
    load_q<D>(q, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
    wg_stream<D, false>(a.kv, a.shared_pages + a.shared_page_off[g], p0, p1, len, len, len, hk, a.sc, smem, w, lane, s.sub, s.parts, s.most, q, O, m, l);
    wg_store<D>((float*)smem, s, w, lane, O, m, l, row_ok, a.part_o, a.part_ml, at);
    return;
  }
  int x = blockIdx.x * WG_WAVES + w;
  const int hk = x % a.hkv;
  x /= a.hkv;
  const int split = x % a.splits_b, branch = x / a.splits_b;
  if (branch >= a.n_live) return;
  const int len = a.branch_len[branch], p0 = split * a.chunk_b, p1 = min(p0 + a.chunk_b, (len + PAGE - 1) / PAGE);
  const size_t at = (size_t)(a.first_own + branch * a.splits_b + split) * a.hq + hk * a.G + min(L, a.G - 1);
  if (p0 >= p1) {
    if (lane < a.G) *(float2*)(a.part_ml + at * 2) = make_float2(-1e30f, 0.f);
    return;
  }
  bf16x8 q[D / 16];
  load_q<D>(q, a.q + ((size_t)branch * a.hq + hk * a.G + min(L, a.G - 1)) * D, a.sc, lane);
  stream_slice<D, false>(a.kv, a.branch_pages + a.branch_page_off[branch], p0, p1, len, len, len, hk, a.sc, lane, q, O, m, l);
  l += other_half(l);
  if (L < a.G) store_part<D>(a.part_o, a.part_ml, at, O, m, l, lane >> 5);
}

template <int D, bool LIMITS>
__global__ void __launch_bounds__(64 * WG_WAVES, 2) k_q8_decode_seg_wg(Q8SegArgs args) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const SegArgs& a = args.s;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, L = lane & 31;
  const int hk = blockIdx.x % a.hkv, idx = blockIdx.x / a.hkv;
  if (idx >= a.totals[0]) return;
  const SegItem it = a.items[idx];
  const int slice = (it.nsplit >> 23) & 0x1fe, nsplit = it.nsplit & 0xffffff;
  const int npages = min((it.len + PAGE - 1) / PAGE, a.chunk * a.splits), p1 = min(it.p0 + slice, npages);  // (a slice has 9 << 4 pages at most)
  const int row0 = it.row0;
  if (row0 >= it.nrows || it.p0 >= p1) return;  // (never listed)
  const WgShare s = wg_share(w, min((it.nrows - row0 + 31) / 32, WG_WAVES));
  const int row = row0 + 32 * s.block + L;
  const bool row_ok = row < it.nrows;
  const int rr = row_ok ? row : row0;
  const int entry = it.e0 + rr / a.G, head = hk * a.G + rr % a.G, place = it.place + rr / a.G * nsplit;
  const bool there = entry >= 0 && entry < a.total_readers;
  const bool store_ok = row_ok && there && place < a.splits * a.total_readers;
  const size_t at = (size_t)place * a.hq + head;
  int lim = it.len, lim_min = it.len;
  if constexpr (LIMITS) {
    lim = min(max(there ? a.seg_reader_len[entry] : 0, 0), it.len);
    lim_min = lim;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) lim_min = min(lim_min, __shfl_xor(lim_min, o));
  }
  const int branch = there ? min(max(a.seg_readers[entry], 0), a.n_live - 1) : 0;
  bf16x8 q[D / 16];
  load_q<D>(q, a.q + ((size_t)branch * a.hq + head) * D, a.sc, lane);
  f32x16 O[D / 32];
  float m, l;
  wg_stream<D, LIMITS>(args.kv, a.seg_pages + it.page_off, it.p0, p1, lim_min, lim, it.len, hk, a.sc, smem, w, lane, s.sub, s.parts, s.most, q, O, m, l);
  wg_store<D>((float*)smem, s, w, lane, O, m, l, store_ok, a.part_o, a.part_ml, at);
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
    if (p.wg) {
      auto* const kernel = D == 128 ? k_q8_decode_wg<128> : k_q8_decode_wg<64>;
      const int lds = D == 128 ? wg_lds_bytes<128>() : wg_lds_bytes<64>();
      DAG_HIP_CHECK(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items_a + dag_ceil_div(p.items_b, WG_WAVES))), dim3(64 * WG_WAVES), lds, stream, a);
    } else {
      hipLaunchKernelGGL((D == 128 ? k_q8_decode<128> : k_q8_decode<64>), dim3((unsigned)(p.items_a + p.items_b)), dim3(64), 0, stream, a);
    }
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(D == 128 ? k_q8_merge<128> : k_q8_merge<64>, dim3((unsigned)(d->n_live * hq)), dim3(64), 0, stream, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

extern "C" size_t dag_decode_segments_q8_workspace_bytes(const dag_decode_seg_desc_t* desc, int32_t hq, int32_t hkv, int32_t head_dim) {
  SegPlan p;
  bool wg;
  return make_q8_seg_plan(desc, hq, hkv, head_dim, &p, &wg) == DAG_OK ? p.bytes : 0;
}

extern "C" int dag_attn_decode_segments_q8(const dag_decode_seg_desc_t* d, const dag_kv_q8_t* kv, const void* q, void* out, int32_t hq,
                                           float softmax_scale, void* ws, size_t ws_bytes, void* stream_) {
  Q8SegArgs args = {};
  int rc = q8_cache(kv, &args.kv);
  if (rc != DAG_OK) return rc;
  SegPlan p;
  const int D = kv->head_dim, hkv = kv->hkv;
  bool wg;
  rc = make_q8_seg_plan(d, hq, hkv, D, &p, &wg);
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
  a.row_shift = wg ? 8 : 5;
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
    if (wg) {
      auto* const kernel = a.seg_reader_len ? (D == 128 ? k_q8_decode_seg_wg<128, true> : k_q8_decode_seg_wg<64, true>)
                                            : (D == 128 ? k_q8_decode_seg_wg<128, false> : k_q8_decode_seg_wg<64, false>);
      const int lds = D == 128 ? wg_lds_bytes<128>() : wg_lds_bytes<64>();
      DAG_HIP_CHECK(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items * hkv)), dim3(64 * WG_WAVES), lds, stream, args);
    } else {
      auto* const kernel = a.seg_reader_len ? (D == 128 ? k_q8_decode_seg<128, true> : k_q8_decode_seg<64, true>)
                                            : (D == 128 ? k_q8_decode_seg<128, false> : k_q8_decode_seg<64, false>);
      hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items * hkv)), dim3(64), 0, stream, args);
    }
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(D == 128 ? k_q8_merge_seg<128> : k_q8_merge_seg<64>, dim3((unsigned)(d->n_live * hq)), dim3(64), 0, stream, args);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}
