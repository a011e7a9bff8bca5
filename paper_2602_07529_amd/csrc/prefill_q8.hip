// dag_attn_prefill_paged_q8: the new tokens of nodes against the pages of their contexts in an 8-bit cache.
//
// out_i = sum_j p_ij v_j / sum_j p_ij with p_ij = exp(scale q_i . k_j), over the slots j of the node's list of pages that hold a token and do
// not lie behind new token i.  A code c of a page stands for its scale times c; the key scale goes into the exponent,
// t_j = (scale log2(e) s) q . c_j, and so does the value scale z, p'_j = 2^(t_j - m + log2 z), which the sum of the probabilities
// takes out again (value_exponent: all of it but what is left over of a tiny one, which the values get).
//
// Many pairs (k_q8_chunk).  A work item is 32 NW (row, query head) pairs of a node and KV head, row after row, against a stretch of its pages, 32
// pairs to a wave.  A tile is four pages.  The threads fetch codes into registers a tile ahead of their use and put them into LDS as bf16, which
// holds every e4m3 value: once for eight waves, not once a wave.  A wave works in steps of 32 keys, and a step is a straight run of three things that
// do not wait for each other: the scores of the next 32 keys, the exponentials of these, the product of the ones before with their values; slot by
// slot, a matrix product (transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane has one pair and its probabilities are operands as they lie),
// the read of an operand four products ahead, an element of the exponentials.  The reference in the exponent is looked after behind the fact: only
// where a block's probabilities sum to 2^30 is the maximum taken and the block done again (their size does not matter to bf16 and fp32).
// Masks only where a tile has a page that is not full or reaches behind a wave's first row.  A value that is no number is not looked for in the
// tiles: where the sums of a wave turn out to hold none, it goes over its pages once more (sums_again).
// What bounds it: the matrix pipes and the power limit, as the bf16 form (1.8 GHz).  16 nodes of 2048 new tokens behind 8192, 32 / 8 heads of 128:
// 4.5 to 4.65 ms, 1.1 PFLOP/s (a library product of 8192^3 in bf16 1.39); the first form, a barrier and whole blocks a tile, codes to
// bf16 by every wave, took 6.8.  Scores as 8-bit products, q in two e4m3 parts, are 9 % faster (4.1), but that pipe's sums are off by 2^-19 of the
// sum of their terms' magnitudes, the bf16 one's by 2^-24: not kept.  Eight waves to a workgroup or four, of which a compute unit holds one at dimension 128 as well: 4.6
// / 7.9 ms.  Probabilities are rounded to bf16 for the second product: in 32 bits it takes sixteen times as long, in two parts
// of bf16 twice, and fp16, of three bits more, has them down to 2^-14 of the largest only (many keys behind a large one of small values).  Outputs are off by
// 0.0023 of their size (2-norm), of which their own rounding is 0.0016.
//
// Few pairs (k_q8_chunk_few, nodes of up to 128): a workgroup's four waves share a stretch of the pages for 32 pairs, each a run of its own,
// straight from memory into registers, and add their sums up in LDS.  One token behind 64,000, 32 / 8 heads: 36 us (130 MB); three nodes of nine behind 1500: 14.5,
// of which what a step of a wave takes, half a microsecond to one, is the most.
//
// Contexts are cut among workgroups by what that costs (cut); a second launch puts the stretches together.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "q8_ops.h"

namespace {

constexpr int PAGE = DAG_PAGE_SIZE;
constexpr int TILE = 4;          // pages
constexpr int MAX_SPLITS = 64;   // (the lanes of the wave that puts them together)

struct ChunkArgs {
  Q8Cache kv;
  const int32_t* q_off;
  const int32_t* ctx_page_off;
  const int32_t* ctx_pages;
  const int32_t* ctx_page_len;
  const int32_t* own_page;
  const int32_t* own_len;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  float* part_o;   // [slot][KV head][split][pair][D]
  float* part_ml;  // the same [2]: reference in the exponent's units, sum
  int n_nodes, n_rows, max_new, max_ctx_pages, hq, G;
  int splits, slice;  // stretches of a context, tiles in each
  int blocks;         // of 32 pairs to a node (nodes with few pairs)
  int few_rows;       // pairs that a block of them may have
  int few_most;       // pairs of a node up to which they are
  float sc;           // softmax_scale * log2(e)
  float back;         // what takes a logarithm to base 2 of a sum of exponentials back: the inverse of the factor that is in sc, as it was rounded
};

// New tokens of a node times query heads of a KV head, up to which they are k_q8_chunk_few's.  It reads a context for every 32 of them, k_q8_chunk for every 256.  Few /
// many, 32 / 8 heads of 128, us: 64 pairs, 2 nodes behind 300 9.5 / 14.5, 48 behind 4000 102 / 182, 120 behind 1500 111 / 155; 96 pairs 9.4 / 16.7, 137 / 175, 145 / 193;
// 128 pairs 9.5 / 17.3, 171 / 185, 173 / 175.  16 / 4 heads of 64, 128 pairs: 7.4 / 14.6, 56 / 104, 56 / 86; as many KV heads as heads, or one, alike: 0.45 to 1.01.
constexpr int FEW_PAIRS = 128;

// The pairs pair0 .. of a node, n new tokens from row0 on; pages / np: its list, nstart: place of its first new token in it.
struct Place {
  int row0, n, pair0, pages, np, nstart;
};
__device__ __forceinline__ int64_t first_row(const ChunkArgs& a, int i) { return min(max(a.q_off[i], 0), a.n_rows); }
__device__ __forceinline__ void node_place(const ChunkArgs& a, int i, Place* p) {
  const int64_t r0 = first_row(a, i), r1 = first_row(a, i + 1);
  p->row0 = (int)r0;
  p->n = (int)max(min(r1 - r0, (int64_t)a.max_new), (int64_t)0);
  p->pages = a.ctx_page_off[i];
  p->np = min(max(a.ctx_page_off[i + 1] - p->pages, 0), a.max_ctx_pages);
  p->nstart = a.own_page[i] * PAGE + a.own_len[i] - (int)(r1 - r0);
}
// Slot x holds pairs PAIRS (x - first slot of the node) .. of the node with the largest first slot up to x, the first slot of node i being
// floor(G q_off[i] / PAIRS) + i: at least as many as its pairs fill, and known without a scan.
template <int PAIRS>
__device__ __forceinline__ bool find_place(const ChunkArgs& a, int64_t slot, int lane, Place* p) {
  int lo = 0, hi = a.n_nodes;
  while (hi > lo) {  // 64 nodes of [lo, hi) a turn; the last one whose first slot is not behind
    const int step = (hi - lo + 63) / 64;
    const int64_t i = lo + lane * (int64_t)step;
    const bool ok = i < hi && first_row(a, (int)i) * a.G / PAIRS + i <= slot;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(ok));
    if (n == 0) return false;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
    if (step == 1) break;
  }
  node_place(a, lo, p);
  const int64_t pair0 = (slot - ((int64_t)p->row0 * a.G / PAIRS + lo)) * PAIRS;
  if (pair0 >= (int64_t)p->n * a.G || p->n * a.G <= a.few_most) return false;
  p->pair0 = (int)pair0;
  return true;
}
// Slot x of the nodes with few pairs: block x % blocks of 32 pairs of node x / blocks.
__device__ __forceinline__ bool few_place(const ChunkArgs& a, int64_t slot, Place* p) {
  node_place(a, (int)(slot / a.blocks), p);
  p->pair0 = (int)(slot % a.blocks) * 32;
  return p->n * a.G <= a.few_most && p->pair0 < p->n * a.G;
}

__device__ __forceinline__ void lds_barrier() {  // (loads from memory stay on their way)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ uint32_t slots_mask(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << 8 * n) - 1u; }  // the first n of four

// Of a page for its scores and probabilities: key scale with the softmax's, log2 of the value scale.
__device__ __forceinline__ float2 page_scales(const ChunkArgs& a, float ks, float vs, int len) {
  ks *= fabsf(a.sc);
  ks = ks < 1.2e-38f ? 1.2e-38f : ks;  // (not zero: hidden keys have scores of minus infinity; no number stays none)
  return len == 0 ? make_float2(1.f, 0.f) : make_float2(ks, value_log2(vs));  // (nobody looks at the scales of a page without tokens)
}

constexpr int NW = 8;  // waves of a workgroup of many pairs
template <int D>
struct Lds {
  uint8_t k[3][TILE * D * PAGE * 2];  // [page][half of a piece][piece of 16 dims][slot][8 dims]
  uint8_t v[3][TILE * D * PAGE * 2];  // [page][half of the slots][dim][8 slots]
  float2 page[4][TILE];               // key scale with the softmax's, what the exponent gets of the value scale
  float left[4][TILE];                // what the values get of it
  int len[4][TILE];                   // tokens
};

// A wave's pairs once more, page by page from memory, where a value that is no number was among those that it multiplied: it may not reach
// the rows that do not see it, and a probability of zero does not keep it from them.  Such values are cleared here, and the sums of the rows
// that see one become no number: a product of "is none" and "is seen" finds them.
template <int D>
__device__ __forceinline__ bool no_number(const f32x16 (&O)[D / 32]) {  // has been among the values
  float any = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) any = fmaf(O[db][r], 0.f, any);
  return __builtin_amdgcn_ballot_w64(any != any) != 0;
}
template <int D>
__device__ __forceinline__ void sums_again(const ChunkArgs& a, const Place& pl, int p0, int p1, int hk, int row, int head, int lim, int L, int H,
                                        f32x16 (&O)[D / 32], float& m, float& l) {
  bf16x8 q[D / 16];
  fetch_q<D>(q, a.q + ((size_t)(pl.row0 + row) * a.hq + head) * D, L + 32 * H);
  sign_q<D>(q, a.sc);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
  m = -1e30f;
  l = 0.f;
  for (int pg0 = p0; pg0 < p1; pg0 += 2) {
    int64_t at[2];
    int len[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const size_t e = (size_t)pl.pages + min(pg0 + i, p1 - 1);
      at[i] = (int64_t)min(max(a.ctx_pages[e], 0), a.kv.n_pages - 1) * a.kv.hkv + hk;
      len[i] = pg0 + i < p1 ? min(max(a.ctx_page_len[e], 0), PAGE) : 0;
    }
    const size_t mine = H ? at[1] : at[0], key = L >> 2 & 1 ? at[1] : at[0];
    const int plen = H ? len[1] : len[0], n = min(plen, lim - (pg0 + H) * PAGE + 1);
    float2 page = page_scales(a, a.kv.k_scale[mine], a.kv.v_scale[mine], plen);
    float left;  // (of the page, not of the row: the lane has values for all rows)
    page.y = value_exponent(page.y, &left);
    if (n <= 0) page = make_float2(1.f, 0.f);
    f32x16 S;
#pragma unroll
    for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const u32x4 c = *(const u32x4*)(a.kv.k_pool + key * (D * PAGE) + s * 512 + H * 256 + ((L & 3) + 4 * (L >> 3)) * 16);
      S = mfma32(codes_to_bf16(c[0], c[1]), q[2 * s], S);
      S = mfma32(codes_to_bf16(c[2], c[3]), q[2 * s + 1], S);
    }
    float bm = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      S[r] = r < n ? S[r] * page.x : -INFINITY;
      bm = fmaxf(bm, S[r]);
    }
    bm = fmaxf(bm, other_half(bm));
    const float m_new = fmaxf(m, bm), alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    f32x8 x[2], seen[2];
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r >> 3][r & 7] = __builtin_amdgcn_exp2f(S[r] + (page.y - m));
      sum += x[r >> 3][r & 7];
      seen[r >> 3][r & 7] = r < n ? 1.f : 0.f;
    }
    l = fmaf(l, alpha, sum * __builtin_amdgcn_exp2f(-page.y));
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      u32x4 c = *(const u32x4*)(a.kv.v_pool + mine * (D * PAGE) + (32 * db + L) * 16), one;
      f32x16 none;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        O[db][r] *= alpha;
        none[r] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t bad = (((c[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
        one[e] = bad * 0x38u & slots_mask(plen - 4 * e);  // the code of one
        c[e] &= ~(bad * 0xffu) & slots_mask(plen - 4 * e);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        none = mfma32(codes_to_bf16(one[2 * e], one[2 * e + 1]), __builtin_convertvector(seen[e], bf16x8), none);
        O[db] = mfma32(codes_to_bf16(c[2 * e], c[2 * e + 1], left), __builtin_convertvector(x[e], bf16x8), O[db]);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) O[db][r] = none[r] > 0.f ? NAN : O[db][r];
    }
  }
}

template <int D>
__device__ __forceinline__ void store_part(const ChunkArgs& a, size_t at, const f32x16 (&O)[D / 32], float m, float l, int H) {
  float* const po = a.part_o + at * D;
  if (l != 0.f)  // (nobody reads it otherwise)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) *(f32x4*)(po + 32 * db + 8 * r + 4 * H) = f32x4{O[db][4 * r], O[db][4 * r + 1], O[db][4 * r + 2], O[db][4 * r + 3]};
  if (H == 0) *(float2*)(a.part_ml + at * 2) = make_float2(m, l);
}
template <int D>
__device__ __forceinline__ void store_out(const ChunkArgs& a, size_t at, const f32x16 (&O)[D / 32], float m, float l, int H) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      u32x2 y;
      y[0] = dag_pack_bf2(O[db][4 * r] * inv, O[db][4 * r + 1] * inv);
      y[1] = dag_pack_bf2(O[db][4 * r + 2] * inv, O[db][4 * r + 3] * inv);
      *(u32x2*)(a.out + at * D + 32 * db + 8 * r + 4 * H) = y;
    }
  if (a.lse && H == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * a.back;
}

constexpr float TOP_SUM = 1073741824.f;  // of a block's probabilities relative to the reference: 2^30

template <int D>
__global__ void __launch_bounds__(64 * NW, 2) k_q8_chunk(ChunkArgs a) {
  constexpr int PAIRS = 32 * NW, THREADS = 64 * NW, PIECES = (TILE * D + THREADS - 1) / THREADS;  // 16-byte pieces of the keys of a tile to a thread
  constexpr bool HALF = TILE * D < THREADS;  // the upper half of the waves fetches the values, the lower one the keys
  static_assert(!HALF || 2 * TILE * D == THREADS, "");
  __shared__ __attribute__((aligned(16))) Lds<D> lds;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, L = lane & 31, H = lane >> 5;
  const int hkv = a.kv.hkv, hk = blockIdx.x % hkv, split = blockIdx.x / hkv % a.splits;
  const int64_t slot = blockIdx.x / hkv / a.splits;
  Place pl;
  if (!find_place<PAIRS>(a, slot, lane, &pl)) return;
  const int n_pairs = min(PAIRS, pl.n * a.G - pl.pair0);
  const int pair = min(pl.pair0 + 32 * w + L, pl.n * a.G - 1), row = pair / a.G, head = hk * a.G + pair % a.G;
  const int lim = pl.nstart + row;  // the last place that the row sees
  const int lim_first = pl.nstart + min(pl.pair0 + 32 * w, pl.n * a.G - 1) / a.G;
  const int lim_last = pl.nstart + (pl.pair0 + n_pairs - 1) / a.G;
  const int nt = lim_last < 0 ? 0 : min((pl.np + TILE - 1) / TILE, lim_last / (TILE * PAGE) + 1);
  const int t0 = min(split * a.slice, nt), t1 = min(t0 + a.slice, nt);
  const bool idle = 32 * w >= n_pairs;

  f32x16 O[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
  float m = -1e30f, l = 0.f;

  if (t0 < t1) {
    bf16x8 q[D / 16];
    fetch_q<D>(q, a.q + ((size_t)(pl.row0 + row) * a.hq + head) * D, lane);
    sign_q<D>(q, a.sc);
    // ids and tokens of 64 pages, a lane each, and of the 64 behind them
    int win_pg, win_len, next_pg, next_len;
    auto ask = [&](int rel) __attribute__((always_inline)) {
      const int i = rel + lane;
      next_pg = a.ctx_pages[(size_t)pl.pages + min(i, pl.np - 1)];
      next_len = i < pl.np ? a.ctx_page_len[(size_t)pl.pages + min(i, pl.np - 1)] : 0;
    };
    auto have = [&]() __attribute__((always_inline)) {
      win_pg = min(max(next_pg, 0), a.kv.n_pages - 1);
      win_len = min(max(next_len, 0), PAGE);
    };
    u32x4 kpiece[PIECES], vpiece[PIECES];
    int held[PIECES];
    float ks = 0.f, vs = 0.f;
    int len = 0;
    const bool my_k = !HALF || w < NW / 2, my_v = !HALF || w >= NW / 2;
    const int wv = HALF ? w & (NW / 2 - 1) : w;  // the wave's place among those that fetch
    auto fetch = [&](const uint8_t* pool, int t, int i, u32x4& to, int* n) __attribute__((always_inline)) {
      const int x = wv * 64 + i * THREADS, j = x / D, at = (TILE * t + j) & 63;
      const int pg = __builtin_amdgcn_readlane(win_pg, at);
      if (n) *n = __builtin_amdgcn_readlane(win_len, at);
      to = *(const u32x4*)(pool + ((size_t)pg * hkv + hk) * (D * PAGE) + (uint32_t)((x % D + lane) * 16));
    };
    auto load_k = [&](int t) __attribute__((always_inline)) {  // tile t of the context
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (my_k) fetch(a.kv.k_pool, t, i, kpiece[i], nullptr);
      const int at = (TILE * t + (w & (TILE - 1))) & 63;
      const size_t ph = (size_t)__builtin_amdgcn_readlane(win_pg, at) * hkv + hk;
      len = __builtin_amdgcn_readlane(win_len, at);
      ks = a.kv.k_scale[ph];
      vs = a.kv.v_scale[ph];
    };
    auto load_v = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (my_v) fetch(a.kv.v_pool, t, i, vpiece[i], &held[i]);
    };
    auto store_k = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int x = wv * 64 + i * THREADS;
        if (!my_k) break;
        uint8_t* const to = lds.k[buf] + x / D * (D * 32) + (x % D + lane) * 16;
        *(bf16x8*)to = codes_to_bf16(kpiece[i][0], kpiece[i][1]);
        *(bf16x8*)(to + D * 16) = codes_to_bf16(kpiece[i][2], kpiece[i][3]);
      }
      if (w < TILE && lane == 0) {
        float2 page = page_scales(a, ks, vs, len);
        page.y = value_exponent(page.y, &lds.left[t & 3][w]);
        lds.page[t & 3][w] = page;
        lds.len[t & 3][w] = len;
      }
    };
    float left[PIECES];
    auto ask_left = [&](int t) __attribute__((always_inline)) {  // (a barrier behind store_k of the tile, and some time in front of store_v)
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (my_v) left[i] = lds.left[t & 3][(wv * 64 + i * THREADS) / D];
    };
    auto store_v = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        if (!my_v) break;
        const int x = wv * 64 + i * THREADS;
        u32x4 c = vpiece[i];
        if (held[i] < PAGE) {  // slots without a token may hold any codes
#pragma unroll
          for (int e = 0; e < 4; ++e) c[e] &= slots_mask(held[i] - 4 * e);
        }
        uint8_t* const to = lds.v[buf] + x / D * (D * 32) + (x % D + lane) * 16;
        *(bf16x8*)to = codes_to_bf16(c[0], c[1], left[i]);
        *(bf16x8*)(to + D * 16) = codes_to_bf16(c[2], c[3], left[i]);
      }
    };
    const int koff = (L >> 2 & 1) * (D * 32) + H * 256 + ((L & 3) + 4 * (L >> 3)) * 16, voff = H * (D * 32) + L * 16;
    constexpr int NK = D / 16, NV = D / 16, SLOTS = D / 8;  // operands of a block's keys and values, matrix products of a step
    int v_old = 0, v_now = 0, v_next = 1;  // buffers of tiles t - 1 (values), t and t + 1
    constexpr int AHEAD = 4;  // operands of either on their way
    u32x4 kop[AHEAD], vop[AHEAD];
    auto read_k = [&](int i, int buf, int b) __attribute__((always_inline)) {
      kop[i % AHEAD] = *(const u32x4*)(lds.k[buf] + 2 * b * (D * 32) + koff + (i & 1) * (D * 16) + (i >> 1) * 512);
    };
    auto read_v = [&](int i, int buf, int b) __attribute__((always_inline)) {
      vop[i % AHEAD] = *(const u32x4*)(lds.v[buf] + 2 * b * (D * 32) + voff + i / (D / 32) * (D * 16) + i % (D / 32) * 512);
    };
    auto score = [&](f32x16& S, int j) __attribute__((always_inline)) {  // product j of a block's scores
      if (j == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = 0.f;
      }
      S = mfma32(__builtin_bit_cast(bf16x8, kop[j % AHEAD]), q[j], S);
    };
    auto product = [&](int i, const u32x4(&p)[2]) __attribute__((always_inline)) {
      O[i % (D / 32)] = mfma32(__builtin_bit_cast(bf16x8, vop[i % AHEAD]), __builtin_bit_cast(bf16x8, p[i / (D / 32)]), O[i % (D / 32)]);
    };
    u32x4 P[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) P[i >> 1][i & 1] = u32x4{0, 0, 0, 0};
    // One step: the scores of block g + 1 from the operands that are there, the probabilities of block g = (t, b) and the product of those of
    // block g - 1 with their values, slot by slot: a matrix product, the read of an operand of the next step into the place of the one just
    // used, some of the exponentials.  stage: called behind the second slot.
    auto step = [&](f32x16& S, f32x16& S_next, u32x4(&p)[2], const u32x4(&p_before)[2], float2 page, int t, int b, bool masked, auto&& stage) __attribute__((always_inline)) {
      float pks = page.x, plv = page.y;
      if (masked) {
        const int n = min(lds.len[t & 3][2 * b + H], lim - (TILE * t + 2 * b + H) * PAGE + 1);  // slots that the row sees
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = r < n ? S[r] : -INFINITY;
        if (n <= 0) pks = 1.f, plv = 0.f;
      }
      const float inv = __builtin_amdgcn_exp2f(-plv);
      float ref = plv - m, sum[2] = {0.f, 0.f};
      float x[16];
      // (elements of slot i; the last two slots have none left, so that their sum is there when it is asked for: 853 -> 832 us for 64 joins of 131)
      auto of_slot = [&](int i, auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i < SLOTS - 2 && r >= i * 16 / (SLOTS - 2) && r < (i + 1) * 16 / (SLOTS - 2)) f(r);
      };
      auto soft_a = [&](int i) __attribute__((always_inline)) { of_slot(i, [&](int r) __attribute__((always_inline)) { x[r] = fmaf(S[r], pks, ref); }); };
      auto soft_b = [&](int i) __attribute__((always_inline)) { of_slot(i, [&](int r) __attribute__((always_inline)) { x[r] = __builtin_amdgcn_exp2f(x[r]); }); };
      auto soft_c = [&](int i) __attribute__((always_inline)) {
        of_slot(i, [&](int r) __attribute__((always_inline)) {
          sum[r & 1] += x[r];
          // (rounded to bf16, as the probabilities over a bf16 cache are)
          if (r & 1) p[r >> 3][(r & 7) >> 1] = dag_pack_bf2(x[r - 1], x[r]);
        });
      };
      constexpr int LAG = 2;
#pragma unroll
      for (int i = 0; i < LAG; ++i) soft_a(i);
#pragma unroll
      for (int i = 0; i < LAG - 1; ++i) soft_b(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        const int j = i >> 1;
        if ((i & 1) == 0) {
          score(S_next, j);
          if (j + AHEAD < NK) read_k(j + AHEAD, b ? v_next : v_now, 1 - b);  // of this block g + 1, then of the next one
          else read_k(j + AHEAD - NK, v_next, b);
        } else {
          product(j, p_before);
          if (j + AHEAD < NV) read_v(j + AHEAD, b ? v_now : v_old, 1 - b);  // of this block g - 1, then of the next one
          else read_v(j + AHEAD - NV, v_now, b);
        }
        // (an element's multiply-add, exponential, sum and rounding in slots behind one another: none waits for the one in front)
        soft_a(i + LAG);
        soft_b(i + LAG - 1);
        soft_c(i);
        __builtin_amdgcn_sched_barrier(0);
        if (i == 1) {
          stage();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      float more = (sum[0] + sum[1]) * inv;
      asm volatile("" : "+v"(S_next));  // (here, not where they are used: the compiler would put all their products in one place)
      if (__builtin_amdgcn_ballot_w64(!(more < TOP_SUM)) != 0) {  // the reference follows, and the block once more
        float bm = S[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) bm = fmaxf(bm, S[r]);
        bm *= pks;
        bm = fmaxf(bm, other_half(bm));
        const float m_new = fmaxf(m, bm), alpha = __builtin_amdgcn_exp2f(m - m_new);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) O[db][r] *= alpha;
        m = m_new;
        ref = plv - m;
        sum[0] = sum[1] = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float y = __builtin_amdgcn_exp2f(fmaf(S[r], pks, ref)), z = __builtin_amdgcn_exp2f(fmaf(S[r + 1], pks, ref));
          sum[0] += y;
          sum[1] += z;
          p[r >> 3][(r & 7) >> 1] = dag_pack_bf2(y, z);
          __builtin_amdgcn_sched_barrier(0);
        }
        more = (sum[0] + sum[1]) * inv;
      }
      l += more;
    };

    // Tile t reads the keys of tile t + 1 and its own values; the keys of tile t + 2 and the values of t + 1 come into LDS, those of t + 3 and
    // t + 2 are fetched.  (What is fetched behind the stretch is never used: its pages are those of the list, or the last one again.)
    uint64_t full = 0;  // pages of the window that are full
    auto window = [&](int t) __attribute__((always_inline)) {  // before the pages of tile t are fetched
      if ((TILE * t & 63) == 0) {
        have();
        ask(TILE * t + 64);
      }
    };
    auto is_full = [&](int t) __attribute__((always_inline)) {
      full = __builtin_amdgcn_ballot_w64(win_len == PAGE);
      return (full >> (TILE * t & 63) & ((1 << TILE) - 1)) == (1 << TILE) - 1 && (t + 1) * (TILE * PAGE) - 1 <= lim_first;
    };
    ask(TILE * t0 & ~63);
    have();
    ask((TILE * t0 & ~63) + 64);
    bool f0, f1, f2, f3;  // whether nothing of tiles t .. t + 3 is hidden
    load_k(t0);
    load_v(t0);
    f0 = is_full(t0);
    store_k(t0, 0);
    lds_barrier();
    ask_left(t0);
    store_v(0);
    window(t0 + 1);
    load_k(t0 + 1);
    load_v(t0 + 1);
    f1 = is_full(t0 + 1);
    store_k(t0 + 1, 1);
    window(t0 + 2);
    load_k(t0 + 2);
    f2 = is_full(t0 + 2);
    lds_barrier();
    f32x16 S0, S1;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_k(i, 0, 0);
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      score(S0, j);
      if (j + AHEAD < NK) read_k(j + AHEAD, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_k(i, 0, 1);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_v(i, 0, 1);  // (the first product is of zeros)
    float2 page0 = lds.page[t0 & 3][H], page1 = lds.page[t0 & 3][2 + H];
    for (int t = t0; t < t1; ++t) {
      lds_barrier();
      ask_left(t + 1);
      if (idle) {  // no row is this wave's: it fetches its share and leaves the matrix pipe to the others
        store_v(v_next);
        load_v(t + 2);
        store_k(t + 2, 3 - v_now - v_next);
        window(t + 3);
        load_k(t + 3);
      } else {
        step(S0, S1, P[0], P[1], page0, t, 0, !f0, [&]() __attribute__((always_inline)) {
          store_v(v_next);
          load_v(t + 2);
          page0 = lds.page[(t + 1) & 3][H];
        });
        step(S1, S0, P[1], P[0], page1, t, 1, !f0, [&]() __attribute__((always_inline)) {
          store_k(t + 2, 3 - v_now - v_next);
          window(t + 3);
          load_k(t + 3);
          f3 = is_full(t + 3);
          page1 = lds.page[(t + 1) & 3][2 + H];
        });
      }
      v_old = v_now;
      v_now = v_next;
      v_next = v_next == 2 ? 0 : v_next + 1;
      f0 = f1;
      f1 = f2;
      f2 = f3;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      product(i, P[1]);
      if (i + AHEAD < NV) read_v(i + AHEAD, v_old, 1);
    }
    if (no_number<D>(O)) {
      sums_again<D>(a, pl, TILE * t0, min(TILE * t1, pl.np), hk, row, head, lim, L, H, O, m, l);
    }
    l += other_half(l);
  }

  if (32 * w + L >= n_pairs) return;
  if (a.splits > 1) store_part<D>(a, (((size_t)slot * hkv + hk) * a.splits + split) * PAIRS + 32 * w + L, O, m, l, H);
  else store_out<D>(a, (size_t)(pl.row0 + row) * a.hq + head, O, m, l, H);
}

// Few pairs: 32 of them to a workgroup, whose waves share a stretch of the pages, each a run of its own, straight from memory, and put their sums
// together in LDS.  What bounds it is how the pages come: two blocks of two pages of a wave are on their way.
constexpr int FEW_WAVES = 4;
template <int D>
__global__ void __launch_bounds__(64 * FEW_WAVES, 2) k_q8_chunk_few(ChunkArgs a) {
  extern __shared__ __attribute__((aligned(16))) float s_o[];  // [wave][pair][D + 4], of as many pairs as a block may have
  __shared__ float2 s_ml[FEW_WAVES][32];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, L = lane & 31, H = lane >> 5;
  const int hkv = a.kv.hkv, hk = blockIdx.x % hkv, split = blockIdx.x / hkv % a.splits;
  const int64_t slot = blockIdx.x / hkv / a.splits;
  Place pl;
  if (!few_place(a, slot, &pl)) return;
  const int n_pairs = min(32, pl.n * a.G - pl.pair0);
  const int pair = min(pl.pair0 + L, pl.n * a.G - 1), row = pair / a.G, head = hk * a.G + pair % a.G;
  const int lim = pl.nstart + row, lim_first = pl.nstart + pl.pair0 / a.G, lim_last = pl.nstart + (pl.pair0 + n_pairs - 1) / a.G;
  const int np = lim_last < 0 ? 0 : min(pl.np, lim_last / PAGE + 1), slice = a.slice * TILE;
  const int s0 = min(split * slice, np), s1 = min(s0 + slice, np), each = ((s1 - s0 + FEW_WAVES - 1) / FEW_WAVES + 1) & ~1;
  const int p0 = min(s0 + w * each, s1), p1 = min(p0 + each, s1);

  f32x16 O[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[db][r] = 0.f;
  float m = -1e30f, l = 0.f;
  if (p0 < p1) {
    struct Ahead {
      u32x4 k[D / 32], v[D / 32];
      float ks, lv;
      int len[2];
    } x[2];
    // 64 pages, a lane each
    int pg, len;
    float2 scales;
    auto load = [&](Ahead& y, int rel) __attribute__((always_inline)) {  // pages p0 + rel, + 1
      const bool first = (rel & 63) == 0 && p0 + rel < p1;
      if (first) {
        const int i = p0 + rel + lane;
        const size_t e = (size_t)pl.pages + min(i, p1 - 1);
        pg = min(max(a.ctx_pages[e], 0), a.kv.n_pages - 1);
        len = i < p1 ? min(max(a.ctx_page_len[e], 0), PAGE) : 0;
        const size_t ph = (size_t)pg * hkv + hk;
        scales = make_float2(a.kv.k_scale[ph], a.kv.v_scale[ph]);
      }
      size_t base[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) base[i] = ((size_t)__builtin_amdgcn_readlane(pg, (rel + i) & 63) * hkv + hk) * (D * PAGE);
      const uint8_t* const kp = a.kv.k_pool + (L >> 2 & 1 ? base[1] : base[0]) + H * 256 + ((L & 3) + 4 * (L >> 3)) * 16;
      const uint8_t* const vp = a.kv.v_pool + (H ? base[1] : base[0]) + L * 16;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) y.k[s] = *(const u32x4*)(kp + s * 512);
#pragma unroll
      for (int s = 0; s < D / 32; ++s) y.v[s] = *(const u32x4*)(vp + s * 512);
      if (first) {
        scales = page_scales(a, scales.x, scales.y, len);
        asm volatile("" ::"v"(scales.x), "v"(scales.y));  // (arrived: a wait for them later would also wait for the blocks in flight)
      }
      auto of = [&](float z, int i) __attribute__((always_inline)) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(z), (rel + i) & 63)); };
      y.ks = H ? of(scales.x, 1) : of(scales.x, 0);
      y.lv = H ? of(scales.y, 1) : of(scales.y, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) y.len[i] = p0 + rel + i < p1 ? __builtin_amdgcn_readlane(len, (rel + i) & 63) : 0;
      __builtin_amdgcn_sched_barrier(0);
    };
    load(x[0], 0);
    bf16x8 q[D / 16];
    fetch_q<D>(q, a.q + ((size_t)(pl.row0 + row) * a.hq + head) * D, lane);
    sign_q<D>(q, a.sc);
    auto compute = [&](Ahead& y, int rel) __attribute__((always_inline)) {
      f32x16 S;
#pragma unroll
      for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) S = mfma32(codes_to_bf16(y.k[s >> 1][2 * (s & 1)], y.k[s >> 1][2 * (s & 1) + 1]), q[s], S);
      float pks = y.ks, left, plv = value_exponent(y.lv, &left);  // (left: of the page, not of the row)
      const int pos = (p0 + rel) * PAGE;
      if (y.len[0] < PAGE || y.len[1] < PAGE || pos + 2 * PAGE - 1 > lim_first) {
        asm volatile("");  // (a branch: the compiler would compare and select in every block)
        const int plen = H ? y.len[1] : y.len[0], n = min(plen, lim - (pos + H * PAGE) + 1);  // slots that the row sees
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = r < n ? S[r] : -INFINITY;
        if (n <= 0) pks = 1.f, plv = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // slots without a token may hold any codes
          const uint32_t mask = slots_mask(plen - 4 * e);
#pragma unroll
          for (int db = 0; db < D / 32; ++db) y.v[db][e] &= mask;
        }
      }
      float bm = S[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) bm = fmaxf(bm, S[r]);
      bm *= pks;
      bm = fmaxf(bm, other_half(bm));
      if (__builtin_amdgcn_ballot_w64(bm > m + 3.f) != 0) {
        const float m_new = fmaxf(m, bm), alpha = __builtin_amdgcn_exp2f(m - m_new);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) O[db][r] *= alpha;
        m = m_new;
      }
      const float ref = plv - m;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // (one half behind the other: registers)
        f32x8 e;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          e[r] = __builtin_amdgcn_exp2f(fmaf(S[8 * h + r], pks, ref));
          sum += e[r];
        }
        const bf16x8 p = __builtin_convertvector(e, bf16x8);  // (rounded to bf16, as the probabilities over a bf16 cache are)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) O[db] = mfma32(codes_to_bf16(y.v[db][2 * h], y.v[db][2 * h + 1], left), p, O[db]);
        __builtin_amdgcn_sched_barrier(0);
      }
      l = fmaf(sum, __builtin_amdgcn_exp2f(-plv), l);
      __builtin_amdgcn_sched_barrier(0);
    };
    // (no load and no block behind a condition: what is fetched behind the run is of pages of the window, and counts as pages without tokens)
    for (int rel = 0; rel < p1 - p0; rel += 4) {
      load(x[1], rel + 2);
      compute(x[0], rel);
      load(x[0], rel + 4);
      compute(x[1], rel + 2);
    }
    if (no_number<D>(O)) sums_again<D>(a, pl, p0, p1, hk, row, head, lim, L, H, O, m, l);
    l += other_half(l);
  }

  // The sums of all waves, added up in their order: 2 FEW_WAVES threads to a pair.
  constexpr int LINE = D + 4, EACH = D / (2 * FEW_WAVES);
  if (H == 0) s_ml[w][L] = make_float2(m, l);
  if (L < a.few_rows && l != 0.f) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(f32x4*)&s_o[(w * a.few_rows + L) * LINE + 32 * db + 8 * r + 4 * H] = f32x4{O[db][4 * r], O[db][4 * r + 1], O[db][4 * r + 2], O[db][4 * r + 3]};
  }
  __syncthreads();
  const int mine = tid / (2 * FEW_WAVES), d0 = tid % (2 * FEW_WAVES) * EACH;
  if (mine >= n_pairs) return;
  float top = -1e30f, total = 0.f, weight[FEW_WAVES], o[EACH] = {};
#pragma unroll
  for (int i = 0; i < FEW_WAVES; ++i) top = fmaxf(top, s_ml[i][mine].y != 0.f ? s_ml[i][mine].x : -1e30f);
#pragma unroll
  for (int i = 0; i < FEW_WAVES; ++i) {
    const float2 ml = s_ml[i][mine];
    weight[i] = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    total = fmaf(ml.y, weight[i], total);
    if (ml.y != 0.f) {
#pragma unroll
      for (int e = 0; e < EACH; e += 4) {
        const f32x4 y = *(const f32x4*)&s_o[(i * a.few_rows + mine) * LINE + d0 + e];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[e + j] = fmaf(y[j], weight[i], o[e + j]);
      }
    }
  }
  if (a.splits > 1) {
    const size_t at = (((size_t)slot * hkv + hk) * a.splits + split) * 32 + mine;
#pragma unroll
    for (int e = 0; e < EACH; e += 4) *(f32x4*)(a.part_o + at * D + d0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
    if (d0 == 0) *(float2*)(a.part_ml + at * 2) = make_float2(top, total);
    return;
  }
  const int p = pl.pair0 + mine;
  const size_t at = (size_t)(pl.row0 + p / a.G) * a.hq + hk * a.G + p % a.G;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint32_t y[EACH / 2];
#pragma unroll
  for (int e = 0; e < EACH / 2; ++e) y[e] = dag_pack_bf2(o[2 * e] * inv, o[2 * e + 1] * inv);
#pragma unroll
  for (int e = 0; e < EACH / 2; e += 2) *(u32x2*)(a.out + at * D + d0 + 2 * e) = u32x2{y[e], y[e + 1]};
  if (a.lse && d0 == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * a.back;
}

// Puts the stretches of a context together, in their order: a wave to a pair, a lane to a stretch and then to D / 64 dims.
template <int D, int PAIRS, bool FEW>
__global__ void __launch_bounds__(256) k_q8_chunk_merge(ChunkArgs a) {
  constexpr int EACH = D / 64;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hkv = a.kv.hkv;
  const int part = blockIdx.x % (PAIRS / 4), hk = blockIdx.x / (PAIRS / 4) % hkv;
  const int64_t slot = blockIdx.x / (PAIRS / 4) / hkv;
  Place pl;
  if (!(FEW ? few_place(a, slot, &pl) : find_place<PAIRS>(a, slot, lane, &pl))) return;
  const int mine = part * 4 + w, pair = pl.pair0 + mine;
  if (pair >= pl.n * a.G) return;
  const size_t at = ((size_t)slot * hkv + hk) * a.splits * PAIRS + mine;
  float2 ml = make_float2(-1e30f, 0.f);
  if (lane < a.splits) ml = *(const float2*)(a.part_ml + (at + (size_t)lane * PAIRS) * 2);
  const float top = dag_wave_max(ml.y != 0.f ? ml.x : -1e30f), weight = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
  const float total = dag_wave_sum(ml.y * weight);
  float o[EACH] = {};
  const uint64_t there = __builtin_amdgcn_ballot_w64(ml.y != 0.f);  // (the others have not been written)
  constexpr int AHEAD = 8;
  for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
    float x[AHEAD][EACH];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const float* const from = a.part_o + (at + (size_t)min(s0 + i, a.splits - 1) * PAIRS) * D + EACH * lane;
#pragma unroll
      for (int e = 0; e < EACH; ++e) x[i][e] = from[e];
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int s = s0 + i;
      if (s >= a.splits || !(there >> s & 1)) continue;
      const float f = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(weight), s));
#pragma unroll
      for (int e = 0; e < EACH; ++e) o[e] = fmaf(x[i][e], f, o[e]);
    }
  }
  const int row = pair / a.G, head = hk * a.G + pair % a.G;
  const size_t to = (size_t)(pl.row0 + row) * a.hq + head;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  if constexpr (EACH == 2) *(uint32_t*)(a.out + to * D + 2 * lane) = dag_pack_bf2(o[0] * inv, o[EACH - 1] * inv);
  else a.out[to * D + lane] = (uint16_t)dag_pack_bf2(o[0] * inv, 0.f);
  if (a.lse && lane == 0) a.lse[to] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * a.back;
}

// How the contexts are cut: `splits` stretches of `slice` tiles, for `slots` blocks of `pairs` pairs.
struct Cut {
  int64_t slots;
  int splits, slice, pairs;
  size_t parts(int hkv) const { return splits > 1 ? (size_t)slots * hkv * splits * pairs : 0; }
};
struct Plan {
  Cut few, many;  // slots 0: not launched
  int blocks, few_rows;
  size_t floats(int hkv, int D) const { return (few.parts(hkv) + many.parts(hkv)) * (D + 2); }
};
// As many stretches as take the least time: rounds of the workgroups that the device holds at once, each as long as its steps through a stretch
// and what a workgroup costs apart from them, then the second launch and the partial results, which are written and read.  In microseconds.
// Against calls cut in 1 to 64, what it takes / the fastest, 32 / 8 heads of 128: one token behind 2000 9.8 / 9.8, behind 64000 36 / 32 (in 24); eight nodes of 8 behind 8000
// 34.6 / 31.6; 128 tokens behind 30000 81 / 80 (uncut 701), 1024 behind 31000 481 / 480 (uncut 748); four nodes of 500 behind 10000, where the host's bound
// on the items is one over a round, 360 / 305; 64 of 121 behind 6000 uncut, as fastest.
struct Cost {
  double tile, each, merge;
  int at_once;
};
double cut(Cut* c, double items, int64_t tiles, int D, const Cost& cost) {
  double best = 1e300;
  c->splits = 1;
  c->slice = (int)std::max<int64_t>(tiles, 1);
  for (int s = 1; s <= MAX_SPLITS && s <= std::max<int64_t>(tiles, 1); ++s) {
    const int64_t slice = dag_ceil_div(std::max<int64_t>(tiles, 1), s);
    if (dag_ceil_div(std::max<int64_t>(tiles, 1), slice) != s) continue;
    double time = std::ceil(items * s / cost.at_once) * (slice * cost.tile + cost.each);
    if (s > 1) time += cost.merge + items * s * c->pairs * (D + 2) * 8. / 4e6;
    if (time < best * 0.97) {
      best = time;
      c->splits = s;
      c->slice = (int)slice;
    }
  }
  return best;
}
// By the host's bounds.  The device has 256 compute units.
bool plan(const dag_paged_prefill_desc_t* d, int64_t n_rows, int hq, int hkv, int D, Plan* p) {
  const int64_t G = hq / hkv, tiles = dag_ceil_div(d->max_ctx_pages, TILE), most = d->max_new * G;
  const bool none = d->max_new == 0 || d->n_nodes == 0 || n_rows == 0;
  p->few = p->many = Cut{0, 1, 1, 32};
  p->blocks = (int)std::max<int64_t>(1, dag_ceil_div(std::min<int64_t>(most, FEW_PAIRS), 32));
  p->few_rows = (int)std::max<int64_t>(1, std::min<int64_t>(most, 32));
  // (few new tokens in all: a node with more is a tile kernel's, which has a slot for it wherever there is one)
  // (a single node whose bound is past them is one of many pairs, whatever it has: a launch less)
  if (!none && (most <= FEW_PAIRS || d->n_nodes > 1)) {
    p->few.slots = (int64_t)d->n_nodes * p->blocks;
    // (eight waves to a workgroup in place of a cut: three nodes of nine behind 1500 16.7 us, cut 14.2; one token behind 2000 11.2, 9.4)
    cut(&p->few, (double)std::min<int64_t>(p->few.slots, n_rows * G / 32 + d->n_nodes) * hkv, tiles, D, Cost{0.4, 5., 4., 512});
  }
  if (!none && most > FEW_PAIRS) {
    p->many.pairs = 32 * NW;
    p->many.slots = n_rows * G / p->many.pairs + d->n_nodes;  // (the last node's last one is below: find_place)
    const double items = d->n_nodes == 1 ? (double)dag_ceil_div(n_rows * G, p->many.pairs) : (double)n_rows * G / p->many.pairs + 0.5 * d->n_nodes;
    cut(&p->many, items * hkv, tiles, D, Cost{D / 64., 6., 5., 256});
  }
  for (const Cut* c : {&p->few, &p->many}) {  // (threads of a launch, 256 or 512 a workgroup, are counted in 32 bits)
    const int64_t most = (int64_t)1 << (c == &p->few ? 23 : 22), merge = (int64_t)1 << 23;
    if (c->slots > most || hkv > most || c->slots * hkv * c->splits > most || (c->splits > 1 && c->slots * hkv * (c->pairs / 4) > merge)) return false;
  }
  return true;
}

bool bounds_ok(const dag_paged_prefill_desc_t* d, int64_t n_rows, int32_t hq, int32_t hkv, int32_t head_dim) {
  return d && d->n_nodes >= 0 && d->max_new >= 0 && d->max_ctx_pages >= 0 && d->max_ctx_pages <= (1 << 26) && n_rows >= 0 && n_rows <= INT32_MAX && hkv >= 1 &&
         hq >= 1 && hq % hkv == 0 && hq / hkv <= 256 && (int64_t)d->max_new * (hq / hkv) <= INT32_MAX && (head_dim == 64 || head_dim == 128);
}

template <int D>
int launch_many(const ChunkArgs& a, const Cut& c, hipStream_t stream) {
  hipLaunchKernelGGL(k_q8_chunk<D>, dim3((unsigned)(c.slots * a.kv.hkv * c.splits)), dim3(64 * NW), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (c.splits > 1) {
    hipLaunchKernelGGL((k_q8_chunk_merge<D, 32 * NW, false>), dim3((unsigned)(c.slots * a.kv.hkv * (32 * NW / 4))), dim3(256), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}
template <int D>
int launch(ChunkArgs a, const Plan& p, hipStream_t stream) {
  a.blocks = p.blocks;
  a.few_rows = p.few_rows;
  a.few_most = p.few.slots > 0 ? FEW_PAIRS : 0;
  auto use = [&](const Cut& c, float* part) {
    a.splits = c.splits;
    a.slice = c.slice;
    a.part_o = part;
    a.part_ml = part + c.parts(a.kv.hkv) * D;
  };
  float* const ws = a.part_o;
  if (p.many.slots > 0) {
    use(p.many, ws);
    const int rc = launch_many<D>(a, p.many, stream);
    if (rc != DAG_OK) return rc;
  }
  if (p.few.slots == 0) return DAG_OK;
  use(p.few, ws + p.many.parts(a.kv.hkv) * (D + 2));
  const size_t lds = (size_t)FEW_WAVES * a.few_rows * (D + 4) * sizeof(float);
  static_assert((size_t)FEW_WAVES * 32 * (D + 4) * sizeof(float) <= 68 << 10, "");
  if (lds > 65536 && hipFuncSetAttribute((const void*)k_q8_chunk_few<D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return DAG_ERR_HIP;
  hipLaunchKernelGGL(k_q8_chunk_few<D>, dim3((unsigned)(p.few.slots * a.kv.hkv * p.few.splits)), dim3(64 * FEW_WAVES), lds, stream, a);
  DAG_LAUNCH_CHECK();
  if (p.few.splits > 1) {
    hipLaunchKernelGGL((k_q8_chunk_merge<D, 32, true>), dim3((unsigned)(p.few.slots * a.kv.hkv * 8)), dim3(256), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}

}  // namespace

extern "C" size_t dag_prefill_paged_q8_workspace_bytes(const dag_paged_prefill_desc_t* d, int64_t n_rows, int32_t hq, int32_t hkv, int32_t head_dim) {
  Plan p;
  if (!bounds_ok(d, n_rows, hq, hkv, head_dim) || d->page_size != PAGE || !plan(d, n_rows, hq, hkv, head_dim, &p)) return 0;
  return p.floats(hkv, head_dim) * sizeof(float);
}

extern "C" int dag_attn_prefill_paged_q8(const dag_paged_prefill_desc_t* d, const dag_kv_q8_t* kv, const void* q, int64_t n_rows, void* out, float* lse,
                                         int32_t hq, float softmax_scale, void* ws, size_t ws_bytes, void* stream_) {
  if (!d || !kv) return DAG_ERR_NULL;
  if (d->n_nodes < 0 || d->max_new < 0 || d->max_ctx_pages < 0 || kv->n_pages < 0 || n_rows < 0) return DAG_ERR_BAD_LEN;
  Plan p;
  if (d->page_size != PAGE || !bounds_ok(d, n_rows, hq, kv->hkv, kv->head_dim) || !plan(d, n_rows, hq, kv->hkv, kv->head_dim, &p)) return DAG_ERR_UNSUPPORTED;
  if (p.few.slots == 0 && p.many.slots == 0) return DAG_OK;  // no new token anywhere
  const bool pages = d->max_ctx_pages > 0;
  if (pages && kv->n_pages == 0) return DAG_ERR_BAD_LEN;
  if (!q || !out || !d->q_off || !d->ctx_page_off || !d->own_page || !d->own_len) return DAG_ERR_NULL;
  if (pages && (!d->ctx_pages || !d->ctx_page_len || !kv->k_pool || !kv->v_pool || !kv->k_scale || !kv->v_scale)) return DAG_ERR_NULL;
  if (!dag_aligned16(q) || !dag_aligned16(out) || !dag_aligned16(kv->k_pool) || !dag_aligned16(kv->v_pool) || ((uintptr_t)kv->k_scale & 3) ||
      ((uintptr_t)kv->v_scale & 3) || ((uintptr_t)lse & 3))
    return DAG_ERR_ALIGN;
  const size_t need = p.floats(kv->hkv, kv->head_dim) * sizeof(float);
  if (need > 0 && (!ws || ws_bytes < need)) return DAG_ERR_WORKSPACE;
  if (need > 0 && !dag_aligned16(ws)) return DAG_ERR_ALIGN;
  ChunkArgs a = {};
  a.kv = Q8Cache{(const uint8_t*)kv->k_pool, (const uint8_t*)kv->v_pool, kv->k_scale, kv->v_scale, kv->n_pages, kv->hkv};
  a.q_off = d->q_off;
  a.ctx_page_off = d->ctx_page_off;
  a.ctx_pages = d->ctx_pages;
  a.ctx_page_len = d->ctx_page_len;
  a.own_page = d->own_page;
  a.own_len = d->own_len;
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.part_o = (float*)ws;
  a.n_nodes = d->n_nodes;
  a.n_rows = (int)n_rows;
  a.max_new = d->max_new;
  a.max_ctx_pages = d->max_ctx_pages;
  a.hq = hq;
  a.G = hq / kv->hkv;
  a.sc = std::isfinite(softmax_scale) ? softmax_scale * 1.4426950408889634f : NAN;
  a.back = (float)(a.sc != 0.f && std::isfinite(a.sc) ? (double)softmax_scale / (double)a.sc : 0.69314718055994530942);
  return kv->head_dim == 128 ? launch<128>(a, p, (hipStream_t)stream_) : launch<64>(a, p, (hipStream_t)stream_);
}
