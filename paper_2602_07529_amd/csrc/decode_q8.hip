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
  int most_a, most_b;  // tokens of a list by the host's bounds: what a length has beyond them is not read
  float sc;        // softmax_scale * log2(e)
};

struct Q8SegArgs {
  SegArgs s;
  Q8Cache kv;
  int most;  // tokens of a segment by the host's bound
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

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const uint8_t* p) {  // ONCE: passes the caches by
  if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
// pages: of 64 pages, a lane each; rel, rel + 1: the two of the block, last: the slice's last one
template <int D, bool ONCE>
__device__ __forceinline__ void load_block(Block<D>& b, const Q8Cache& c, int pages, int rel, int last, int hk, int L, int H) {
  const int pg0 = __builtin_amdgcn_readlane(pages, min(rel, last) & 63), pg1 = __builtin_amdgcn_readlane(pages, min(rel + 1, last) & 63);
  const size_t base0 = ((size_t)pg0 * c.hkv + hk) * (D * PAGE), base1 = ((size_t)pg1 * c.hkv + hk) * (D * PAGE);
  const uint8_t* const kp = c.k_pool + (L >> 2 & 1 ? base1 : base0) + H * 256 + ((L & 3) + 4 * (L >> 3)) * 16;
  const uint8_t* const vp = c.v_pool + (H ? base1 : base0) + L * 16;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.k[s] = load16<ONCE>(kp + s * 512);
#pragma unroll
  for (int s = 0; s < D / 32; ++s) b.v[s] = load16<ONCE>(vp + s * 512);
}

// Sums of a wave: 32 rows, a lane has a column (row L) of them.
template <int D>
struct Sums {
  f32x16 O[D / 32];
  float m, l;
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
    m = -1e30f;
    l = 0.f;
  }
};

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

// A block some of whose tokens are hidden from some rows only (the new tokens of a node): a value that is no number may not reach the rows
// that do not see it, and a probability of zero does not keep it from them.  Such codes are cleared, and the sums of the rows that
// see one become no number: a product of "is none" and "is seen" finds them.
template <int D>
__device__ __forceinline__ void hide_not_numbers(Block<D>& b, Sums<D>& sums, int key0, int lim, int H) {
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
    for (int r = 0; r < 16; ++r) sums.O[db][r] = n[r] > 0.f ? NAN : sums.O[db][r];
  }
}

// The exponent's reference m is raised only where a score is more than this above it (log2): the rescale of the sums stays rare.
constexpr float Q8_TH = 3.f;

// A block: scores, probabilities, their product with the values.  ks: key scale of the lane's page times |softmax scale| log2(e),
// lv: log2 of its value scale.  A lane's 16 scores are of one page, so their largest is found among the plain products, one
// multiply-add gives the exponent with the value scale in it, and the sum of a lane loses that factor again once.  (The exponential's results
// reach down to 2^-149: on a page of zeros, scale 2^-100, a key loses at most 2^-50 of the largest in the sum, 2^31 of them 2^-19.)
// key0: first key of the block; keys from `lim` on are hidden from the lane's row; len: the smallest lim of the wave; slots from vlen on hold
// no token.  A wave by itself takes 1,005 cycles for a block at head dimension 128, two waves of a SIMD 512 each, as long as the 16 MFMAs.
template <int D, bool LIMITS>
__device__ __forceinline__ void compute_block(Block<D>& b, const bf16x8 (&q)[D / 16], Sums<D>& sums, float ks, float lv, int key0, int len, int lim,
                                              int vlen, int H) {
  f32x16 S;
#pragma unroll
  for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) S = mfma32(codes_to_bf16(b.k[s >> 1][2 * (s & 1)], b.k[s >> 1][2 * (s & 1) + 1]), q[s], S);
  if (key0 + 32 > len) {
    asm volatile("");  // (a branch: the compiler would compare and select in every block)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[r] = key0 + 16 * H + r < lim ? S[r] : -INFINITY;
    if constexpr (LIMITS)
      if (key0 + 16 * H >= lim) {  // (scales of a page that the row sees nothing of)
        ks = 1.f;
        lv = 0.f;
      }
  }
  float bm = S[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) bm = fmaxf(bm, S[r]);
  bm *= ks;
  bm = fmaxf(bm, other_half(bm));
  if (__builtin_amdgcn_ballot_w64(bm > sums.m + Q8_TH) != 0) {
    const float m_new = fmaxf(sums.m, bm), alpha = __builtin_amdgcn_exp2f(sums.m - m_new);
    sums.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums.O[db][r] *= alpha;
    sums.m = m_new;
  }
  const float ref = lv - sums.m;
  f32x8 x[2];
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    x[r >> 3][r & 7] = __builtin_amdgcn_exp2f(fmaf(S[r], ks, ref));
    sum[r >> 3] += x[r >> 3][r & 7];
  }
  sums.l = fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-lv), sums.l);
  // (rounded to bf16, as the probabilities over a bf16 cache are)
  const bf16x8 p[2] = {__builtin_convertvector(x[0], bf16x8), __builtin_convertvector(x[1], bf16x8)};
  if (key0 + 32 > vlen) clear_behind<D>(b, key0, vlen, H);
  if constexpr (LIMITS)
    if (key0 + 32 > len && len < vlen) hide_not_numbers<D>(b, sums, key0, lim, H);
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) sums.O[db] = mfma32(codes_to_bf16(b.v[db][2 * e], b.v[db][2 * e + 1]), p[e], sums.O[db]);
}

// Page ids (clamped to the pool) and scales of 64 pages of a slice, a lane each.
struct Window {
  int pg;
  float ks, lv;
  __device__ __forceinline__ void ask(const Q8Cache& c, const int32_t* pages, int rel, int np, int hk, int lane) {
    pg = min(max(pages[min(rel + lane, np - 1)], 0), c.n_pages - 1);
    ks = c.k_scale[(size_t)pg * c.hkv + hk];
    lv = c.v_scale[(size_t)pg * c.hkv + hk];
  }
  __device__ __forceinline__ void have(float sc) {
    ks *= fabsf(sc);
    ks = ks < 1.2e-38f ? 1.2e-38f : ks;  // (not zero: hidden keys have scores of minus infinity; no number stays none)
    lv = __builtin_amdgcn_logf(lv);
    asm volatile("" ::"v"(ks), "v"(lv));  // (arrived: a wait for them later would also wait for the blocks in flight)
  }
  static __device__ __forceinline__ float of(float x, int rel, int np, int H) {  // of page rel + H
    const float a = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), min(rel, np - 1) & 63));
    const float b = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), min(rel + 1, np - 1) & 63));
    return H ? b : a;
  }
};

// Pages [p0, p1) of one list against the wave's 32 rows, added to its sums, two pages at a time, the next two on their way meanwhile.
// What bounds it is how the pages come from memory: a page that nobody else reads (ONCE) passes the caches by (16 groups of 8 over
// 8192 | 1024 tokens 114 -> 101 us), and 1,300 to 1,800 waves ask for them, those of the KV heads of a page next to each other (-> 94 us =
// 5.7 TB/s; 2,048 waves 99, 3,072 102 to 123; the loads alone of 2,048 waves take 98.6).  Four pages ahead are no faster.
template <int D, bool LIMITS, bool ONCE>
__device__ __forceinline__ void stream_slice(const Q8Cache& c, const int32_t* pages, int p0, int p1, int len, int lim, int vlen, int hk,
                                             float sc, int lane, const bf16x8 (&q)[D / 16], Sums<D>& sums) {
  const int L = lane & 31, H = lane >> 5, np = p1 - p0;
  Window win;
  struct Ahead {
    Block<D> b;
    float ks, lv;
  };
  Ahead x[2];
  auto load = [&](Ahead& y, int rel) __attribute__((always_inline)) {
    const bool first = (rel & 63) == 0 && rel < np;
    if (first) win.ask(c, pages + p0, rel, np, hk, lane);
    load_block<D, ONCE>(y.b, c, win.pg, rel, np - 1, hk, L, H);
    if (first) win.have(sc);
    y.ks = Window::of(win.ks, rel, np, H);
    y.lv = Window::of(win.lv, rel, np, H);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto compute = [&](Ahead& y, int rel) __attribute__((always_inline)) {
    compute_block<D, LIMITS>(y.b, q, sums, y.ks, y.lv, (p0 + rel) * PAGE, len, lim, vlen, H);
    __builtin_amdgcn_sched_barrier(0);
  };
  // No load behind a condition: the wait for a block would then be one for the block behind it as well (107 us instead of 98 for three levels
  // of segments).  What is loaded behind the slice is its last page again, which nobody uses.
  load(x[0], 0);
  for (int rel = 0;;) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load(x[1 - i], rel + 2);
      compute(x[i], rel);
      if ((rel += 2) >= np) return;
    }
  }
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
template <int D>
__device__ __forceinline__ void load_q(bf16x8 (&q)[D / 16], const uint16_t* row, float sc, int lane) {
  fetch_q<D>(q, row, lane);
  sign_q<D>(q, sc);
}

template <int D>
__device__ __forceinline__ void store_part(float* part_o, float* part_ml, size_t at, const Sums<D>& sums, int H) {
  const f32x16(&O)[D / 32] = sums.O;
  const float m = sums.m, l = sums.l + other_half(sums.l);
  float* const po = part_o + at * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *(f32x4*)(po + 32 * db + 8 * r4 + 4 * H) = f32x4{O[db][4 * r4], O[db][4 * r4 + 1], O[db][4 * r4 + 2], O[db][4 * r4 + 3]};
  if (H == 0) *(float2*)(part_ml + at * 2) = make_float2(m, l);
}

// A slice of one list against 32 of its rows, those from row0 on: rows(i) says which query row the i-th is and where its partial goes.
struct Row {
  const uint16_t* q;
  size_t at;   // of its partial
  int lim;     // tokens of the list that it sees
  bool store;
};
template <int D, bool LIMITS, bool ONCE, typename RF>
__device__ __forceinline__ void run_item(const Q8Cache& c, const int32_t* pages, int p0, int p1, int vlen, int hk, float sc, int row0, int nrows, float* part_o,
                                         float* part_ml, int lane, RF&& rows) {
  const int L = lane & 31, H = lane >> 5;
  const bool there = row0 + L < nrows;
  const Row row = rows(there ? row0 + L : row0);
  int len = vlen;
  if constexpr (LIMITS) {  // the slice ends where its rows see no further
    int most = row.lim;
    len = row.lim;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      len = min(len, __shfl_xor(len, o));
      most = max(most, __shfl_xor(most, o));
    }
    p1 = __builtin_amdgcn_readfirstlane(min(p1, (most + PAGE - 1) / PAGE));
  }
  if (p0 >= p1) {  // nothing there: a partial without weight
    if (there && row.store && H == 0) *(float2*)(part_ml + row.at * 2) = make_float2(-1e30f, 0.f);
    return;
  }
  bf16x8 q[D / 16];
  load_q<D>(q, row.q, sc, lane);
  Sums<D> sums;
  sums.start();
  stream_slice<D, LIMITS, ONCE>(c, pages, p0, p1, len, LIMITS ? row.lim : vlen, vlen, hk, sc, lane, q, sums);
  if (there && row.store) store_part<D>(part_o, part_ml, row.at, sums, H);
}

// A wave to a work item: a slice of a group's shared pages against 32 of its (branch, query head) rows of a KV head, or a slice of a branch's
// own pages against its rows.  WIDE: groups have more rows; their waves read the same pages at about the same time, and what they wait for is
// memory: each has two pages on their way, so five blocks of rows have ten, of which two are different.  Two groups of 32 over
// 32768 | 640, 5 heads on one: 83 us (88 when these were built in its place: workgroups of a wave to a block that find the pages in the L1 98, the
// pages in a ring in LDS, 80 KB on their way, 95, because the waves of a SIMD then do the same at the same time, 64 rows to a wave 90 to 101).
// The KV head is the fast index, so the blocks of rows of a page meet in one L2 where the heads are a multiple of 8 (the XCDs are eight and take
// workgroups in turn).  As many bytes in fewer heads come over for several XCDs: 8 heads 218 MiB read, 83 us; 4 350 and 89; 2 617 and 115; 1 733 and 143.
template <int D, bool WIDE>
__global__ void __launch_bounds__(64, 2) k_q8_decode(Q8DecodeArgs a) {
  const int lane = threadIdx.x;
  const bool shared = (int)blockIdx.x < a.items_a;
  int x = shared ? blockIdx.x : blockIdx.x - a.items_a;
  const int hk = x % a.hkv;
  x /= a.hkv;
  int row0 = 0;
  if (shared) {
    row0 = x % a.rb_max * 32;
    x /= a.rb_max;
  }
  const int splits = shared ? a.splits_a : a.splits_b, split = x % splits;
  x /= splits;
  const int branch0 = shared ? a.group_branch_off[x] : x;
  const int nrows = shared ? (a.group_branch_off[x + 1] - branch0) * a.G : a.G;
  const int32_t* const pages = shared ? a.shared_pages + a.shared_page_off[x] : a.branch_pages + a.branch_page_off[x];
  const int len = shared ? min(a.shared_len[x], a.most_a) : min(a.branch_len[x], a.most_b), chunk = shared ? a.chunk_a : a.chunk_b;
  if (row0 >= nrows) return;
  const int p0 = split * chunk, p1 = min(p0 + chunk, (len + PAGE - 1) / PAGE);
  auto rows = [&](int row) __attribute__((always_inline)) {
    const int branch = min(max(branch0 + row / a.G, 0), a.n_live - 1), head = hk * a.G + row % a.G;
    return Row{a.q + ((size_t)branch * a.hq + head) * D, (size_t)((shared ? 0 : a.first_own) + branch * splits + split) * a.hq + head, len, true};
  };
  run_item<D, false, !WIDE>(a.kv, pages, p0, p1, len, hk, a.sc, row0, nrows, a.part_o, a.part_ml, lane, rows);
}

// The same for the items that k_seg_plan listed.
template <int D, bool WIDE, bool LIMITS>
__global__ void __launch_bounds__(64, 2) k_q8_decode_seg(Q8SegArgs args) {
  const SegArgs& a = args.s;
  const int lane = threadIdx.x, hk = blockIdx.x % a.hkv, idx = blockIdx.x / a.hkv;
  if (idx >= a.totals[0]) return;
  const SegItem it = a.items[idx];
  const int slice = (it.nsplit >> 23) & 0x1fe, nsplit = it.nsplit & 0xffffff;
  const int len = min(it.len, args.most), p1 = min(it.p0 + slice, (len + PAGE - 1) / PAGE);
  if (it.row0 >= it.nrows) return;  // (never listed)
  auto rows = [&](int row) __attribute__((always_inline)) {
    const int entry = it.e0 + row / a.G, head = hk * a.G + row % a.G, place = it.place + row / a.G * nsplit;
    const bool there = entry >= 0 && entry < a.total_readers;  // (reader lists longer than announced: no partial)
    const int branch = there ? min(max(a.seg_readers[entry], 0), a.n_live - 1) : 0;
    int lim = len;
    if constexpr (LIMITS) lim = min(max(there ? a.seg_reader_len[entry] : 0, 0), len);
    return Row{a.q + ((size_t)branch * a.hq + head) * D, (size_t)place * a.hq + head, lim, there && place < a.splits * a.total_readers};
  };
  run_item<D, LIMITS, !WIDE>(args.kv, a.seg_pages + it.page_off, it.p0, p1, len, hk, a.sc, it.row0, it.nrows, a.part_o, a.part_ml, lane, rows);
}

constexpr int WHOLE_WAVES = 8;

// Steps over short contexts: a workgroup to a (branch, KV head), whose eight waves share the pages of all lists that the branch reads and put
// their sums together in LDS: one launch and no partials in memory, which is what such steps consist of otherwise.  Every branch reads
// the shared pages for itself.  lists(base, pages, seen): pages of list base + lane, and how many tokens the branch sees of it.
// What bounds it is the chain of loads up to the first page, each of which takes about as long as the arithmetic of a wave: they stand
// in as few steps as the description allows, none behind a condition.
template <int D, bool ONCE, typename A, typename F>
__device__ __forceinline__ void whole_branch(const A& a, const Q8Cache& kv, int n_lists, F&& lists, bf16x8 (&q)[D / 16], int r, int hk, float* smem, int w,
                                             int lane) {
  const int L = lane & 31, G = a.G;
  Sums<D> sums;
  sums.start();
  bool some = false;
  for (int base = 0; base == 0 || base < n_lists; base += 64) {
    const int32_t* pages;
    int seen;
    lists(base, pages, seen);
    if (base == 0) sign_q<D>(q, a.sc);
    const int np = (seen + PAGE - 1) / PAGE, units = (np + 1) / 2;
    const int behind = dag_wave_scan(units), all = __builtin_amdgcn_readlane(behind, 63), front = behind - units;
    const int u0 = (int)((int64_t)all * w / WHOLE_WAVES), u1 = (int)((int64_t)all * (w + 1) / WHOLE_WAVES);
    some |= u0 < u1;
    for (uint64_t left = __builtin_amdgcn_ballot_w64(max(front, u0) < min(behind, u1)); left; left &= left - 1) {
      const int i = __builtin_ctzll(left), at = __builtin_amdgcn_readlane(front, i);
      const int n = __builtin_amdgcn_readlane(np, i), tokens = __builtin_amdgcn_readlane(seen, i);
      const int32_t* const list = (const int32_t*)dag_readlane((int64_t)(uintptr_t)pages, i);
      const int p0 = 2 * max(u0 - at, 0), p1 = min(2 * (u1 - at), n);
      stream_slice<D, false, ONCE>(kv, list, p0, p1, tokens, tokens, tokens, hk, a.sc, lane, q, sums);
    }
  }
  const float m = sums.m, l = sums.l + other_half(sums.l);
  const f32x16(&O)[D / 32] = sums.O;
  constexpr int ROW = D + 4;
  float* const ml = smem + WHOLE_WAVES * G * ROW;
  if (L < G) {
    if (some) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *(f32x4*)(smem + (w * G + L) * ROW + 32 * db + 8 * r4 + 4 * (lane >> 5)) = f32x4{O[db][4 * r4], O[db][4 * r4 + 1], O[db][4 * r4 + 2], O[db][4 * r4 + 3]};
    }
    if (lane < 32) *(float2*)(ml + (w * G + L) * 2) = make_float2(m, some ? l : 0.f);
  }
  __syncthreads();
  for (int x = w * 64 + lane; x < G * (D / 4); x += 64 * WHOLE_WAVES) {
    const int row = x / (D / 4), c = x % (D / 4) * 4;
    float top = -1e30f, total = 0.f;
    for (int i = 0; i < WHOLE_WAVES; ++i) top = fmaxf(top, ml[(i * G + row) * 2]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < WHOLE_WAVES; ++i) {
      const float2 of = *(const float2*)(ml + (i * G + row) * 2);
      if (of.y == 0.f) continue;
      const float wgt = __builtin_amdgcn_exp2f(of.x - top);
      const f32x4 o = *(const f32x4*)(smem + (i * G + row) * ROW + c);
      total = fmaf(of.y, wgt, total);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(o[e], wgt, acc[e]);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    *(u32x2*)(a.out + ((size_t)r * a.hq + hk * G + row) * D + c) = u32x2{dag_pack_bf2(acc[0] * inv, acc[1] * inv), dag_pack_bf2(acc[2] * inv, acc[3] * inv)};
  }
}
inline int whole_lds_bytes(int G, int D) { return WHOLE_WAVES * G * (D + 6) * 4; }

template <int D, typename A>
__device__ __forceinline__ const uint16_t* whole_row(const A& a, int r, int hk, int lane) {
  return a.q + ((size_t)r * a.hq + hk * a.G + min(lane & 31, a.G - 1)) * D;
}

// (ONCE: q8_whole_cached.  Arrays that the description does not have are replaced by q, whose memory may be read, by the host.)
template <int D, bool ONCE>
__global__ void __launch_bounds__(64 * WHOLE_WAVES, 2) k_q8_whole(Q8DecodeArgs a, int n_groups) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hk = blockIdx.x % a.hkv, r = blockIdx.x / a.hkv;
  bf16x8 q[D / 16];
  fetch_q<D>(q, whole_row<D>(a, r, hk, lane), lane);
  const int own_at = a.branch_page_off[r], own_len = a.branch_len[r];
  int g = -1;  // the group of the branch
  for (int base = 0; base < n_groups; base += 64) {
    const int at = min(base + lane, n_groups - 1), from = a.group_branch_off[at], to = a.group_branch_off[at + 1];
    const uint64_t found = __builtin_amdgcn_ballot_w64((from <= r) & (r < to));
    if (found) g = min(base + __builtin_ctzll(found), n_groups - 1);
  }
  const int shared_at = a.shared_page_off[max(g, 0)], shared_len = a.shared_len[max(g, 0)];
  const int seen = max(lane == 0 ? (g >= 0 ? min(shared_len, a.most_a) : 0) : lane == 1 ? min(own_len, a.most_b) : 0, 0);
  auto lists = [&](int, const int32_t*& list, int& n) __attribute__((always_inline)) {
    list = lane == 0 ? a.shared_pages + shared_at : a.branch_pages + own_at;
    n = seen;
  };
  whole_branch<D, ONCE>(a, a.kv, 2, lists, q, r, hk, (float*)smem, w, lane);
}

// Over segments, up to 64 of them: lane i has entry i of the branch (of the next 64, if it names segments more than once).
template <int D>
__global__ void __launch_bounds__(64 * WHOLE_WAVES, 2) k_q8_whole_seg(Q8SegArgs args) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const SegArgs& a = args.s;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hk = blockIdx.x % a.hkv, r = blockIdx.x / a.hkv;
  bf16x8 q[D / 16];
  fetch_q<D>(q, whole_row<D>(a, r, hk, lane), lane);
  const int last = a.seg_reader_off[min(lane, a.n_segments - 1) + 1], end = lane < a.n_segments ? last : INT32_MAX;  // of the entries of segment `lane`
  const int e0 = a.branch_entry_off[r], entries = max(a.branch_entry_off[r + 1] - e0, 0);
  auto lists = [&](int base, const int32_t*& list, int& seen) __attribute__((always_inline)) {
    const int n = min(entries - base, 64), entry = n > 0 ? a.branch_entries[e0 + base + min(lane, n - 1)] : -1;
    int seg = -1;
    for (int i = 0; i < n; ++i) {
      const int e = __builtin_amdgcn_readlane(entry, i), s = __popcll(__builtin_amdgcn_ballot_w64(end <= e));
      if (lane == i && e >= 0 && e < a.total_readers && s < a.n_segments) seg = s;
    }
    const int at = max(seg, 0), page_off = a.seg_page_off[at], len = min(a.seg_len[at], args.most);
    const int sees = a.seg_reader_len && n > 0 && a.total_readers > 0 ? a.seg_reader_len[min(max(entry, 0), a.total_readers - 1)] : len;
    list = a.seg_pages + page_off;
    seen = seg >= 0 ? max(min(sees, len), 0) : 0;
  };
  whole_branch<D, true>(a, args.kv, entries, lists, q, r, hk, (float*)smem, w, lane);
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
// (of a softmax scale that is infinite no score is a number)
float q8_softmax_scale(float x) { return fabsf(x) < INFINITY ? x * 1.4426950408889634f : NAN; }
// Tokens of so many pages (sums of a few more stay in 32 bits).
int tokens_of(int pages) { return (pages < (INT32_MAX - 64) / PAGE ? pages : (INT32_MAX - 64) / PAGE) * PAGE; }
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
  a.most_a = p.items_a > 0 ? tokens_of(d->max_shared_pages) : 0;
  a.most_b = tokens_of(d->max_branch_pages);
  a.sc = q8_softmax_scale(softmax_scale);
  hipStream_t stream = (hipStream_t)stream_;
  if (p.whole) {
    if (p.items_b == 0) a.branch_page_off = a.branch_len = (const int32_t*)q;
    if (p.items_a == 0) a.shared_page_off = a.shared_len = (const int32_t*)q;
    auto* const kernel = q8_whole_cached(d, a.hkv) ? (D == 128 ? k_q8_whole<128, false> : k_q8_whole<64, false>)
                                                   : (D == 128 ? k_q8_whole<128, true> : k_q8_whole<64, true>);
    const int lds = whole_lds_bytes(a.G, D);
    if (lds > 65536) DAG_HIP_CHECK(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(d->n_live * a.hkv)), dim3(64 * WHOLE_WAVES), lds, stream, a, p.items_a > 0 ? d->n_groups : 0);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  if (p.items_a + p.items_b > 0) {
    auto* const kernel = p.rb_max > 1 ? (D == 128 ? k_q8_decode<128, true> : k_q8_decode<64, true>) : (D == 128 ? k_q8_decode<128, false> : k_q8_decode<64, false>);
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
  args.most = tokens_of(d->max_seg_pages);
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
  const bool wide = p.rb_max > 1;
  a.weight = (float)hkv * (float)D / 128.f;
  a.pages_128 = wide ? Q8_SEG_WIDE_128 : (float)SEG_PAGES_128;
  const int64_t most_pages = (int64_t)d->n_segments * p.rb_max * d->max_seg_pages * hkv * D;
  a.few = p.chunk == 8 && most_pages < (d->max_seg_pages <= SEG_SHORT ? SEG_PAGES_16_SHORT : SEG_PAGES_16) * 128;
  a.sc = q8_softmax_scale(softmax_scale);
  hipStream_t stream = (hipStream_t)stream_;
  if (p.items > 0 && q8_whole_segments(d, hkv, D)) {
    auto* const kernel = D == 128 ? k_q8_whole_seg<128> : k_q8_whole_seg<64>;
    const int lds = whole_lds_bytes(a.G, D);
    if (lds > 65536) DAG_HIP_CHECK(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(d->n_live * hkv)), dim3(64 * WHOLE_WAVES), lds, stream, args);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  if (p.items > 0) {
    const int64_t waves = dag_ceil_div(d->n_segments, 64);
    hipLaunchKernelGGL(k_seg_plan, dim3(1), dim3((unsigned)(waves * 64 < PLAN_THREADS ? waves * 64 : PLAN_THREADS)), 0, stream, a);
    DAG_LAUNCH_CHECK();
    auto pick = [&](auto d_c) {
      constexpr int N = decltype(d_c)::value;
      return a.seg_reader_len ? (wide ? k_q8_decode_seg<N, true, true> : k_q8_decode_seg<N, false, true>)
                              : (wide ? k_q8_decode_seg<N, true, false> : k_q8_decode_seg<N, false, false>);
    };
    auto* const kernel = D == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.items * hkv)), dim3(64), 0, stream, args);
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(D == 128 ? k_q8_merge_seg<128> : k_q8_merge_seg<64>, dim3((unsigned)(d->n_live * hq)), dim3(64), 0, stream, args);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}
