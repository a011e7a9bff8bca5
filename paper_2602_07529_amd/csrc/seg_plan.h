// Work items of decode over segments, for both formats of the cache: the description as the kernels take it, and the kernel that
// lists the items (step 1 of the three).
#pragma once
#include "common.h"
#include "decode_plan.h"

namespace {

// Decode over lists of KV segments: a segment is a page list with a token count and the set of
// live branches that read it; a branch's context is the union of the segments it reads.
struct SegItem {  // one work item: a slice of a segment's pages against one 32-row block of its readers' rows
  int32_t page_off, len, e0, nrows, row0;
  int32_t p0, place;  // first page of the slice; place of its partial of reader e0
  int32_t nsplit;     // slices of the segment, pages of a slice / 2 in the highest eight bits (unless SegArgs::fixed)
};
static_assert(sizeof(SegItem) == SEG_ITEM_BYTES, "");
struct SegArgs {
  const int32_t* seg_page_off;
  const int32_t* seg_pages;
  const int32_t* seg_len;
  const int32_t* seg_reader_off;
  const int32_t* seg_readers;
  const int32_t* seg_reader_len;  // optional: leading tokens of the segment each reader-list entry sees
  const int32_t* branch_entry_off;
  const int32_t* branch_entries;
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  uint16_t* out;
  float* part_o;   // [splits * total_readers][hq][D]: the slices of every reader-list entry one after another
  float* part_ml;  // [splits * total_readers][hq][2]
  SegItem* items;        // [item_cap] compact list of (segment, row block, slice), written by k_seg_plan
  int32_t* totals;       // number of list entries, place behind the last partial, most slices of a segment
  int32_t* entry_first;  // [total_readers] place of the first partial of each reader-list entry (the next one's: behind its last)
  int item_cap;
  int n_segments, n_live, hq, hkv, G;
  int rb_max;      // 32-row blocks per (segment, kv head)
  int chunk, splits, total_readers;  // pages of a slice and slices of a segment that the workspace has room for
  bool fixed;      // slices of `chunk` pages, whatever there is to read
  bool few;        // by the host's bounds the slices have eight pages
  float weight;    // of a page: hkv * D / 128
  float pages_128; // from which a slice gets 128 of them
  float sc, th;
};

// Segment form, step 1: the work items.  Segment lengths and reader counts live in device memory,
// so a launch sized by the host bounds would consist mostly of items that find nothing to do, and
// those cost time even when they exit at once (they sit between the real items in the dispatch
// order and hold wave slots while their loads return).  One workgroup therefore writes the compact
// list: for every segment, in the caller's order, its slices x row blocks (exclusive scan of the
// counts), and for every reader-list entry the place of its first partial.
//
// The list also settles how long slices are (rules and figures: SEG_PAGES_16 and what follows it).  What that costs is exchanges between
// the waves: one for what there is to read, and the scan of the counts tells whether the lists have room for slices of that length.  294 segments:
// 6.2 us; with the host's slices, which need neither, 4.8; with an exchange for each length that is tried 7.2.  28 segments: 3.4, 3.1, 3.4.
constexpr int PLAN_THREADS = 1024;
__global__ void __launch_bounds__(PLAN_THREADS) k_seg_plan(SegArgs a) {
  __shared__ uint32_t s_all[2][4][PLAN_THREADS / 64];  // (in turn: a barrier between two exchanges)
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, threads = blockDim.x, room = a.splits * a.total_readers;
  struct Seg {
    int len, e0, nr, npages, rbs;
  };
  auto segment = [&](int s) __attribute__((always_inline)) {
    Seg g = {0, 0, 0, 0, 0};
    if (s < a.n_segments) {
      g.len = max(a.seg_len[s], 0);
      g.e0 = a.seg_reader_off[s];
      g.nr = max(a.seg_reader_off[s + 1] - g.e0, 0);
      g.npages = min((int)(((uint32_t)g.len + PAGE - 1) / PAGE), a.chunk * a.splits);
      g.rbs = min((g.nr * a.G + 31) / 32, a.rb_max);
    }
    return g;
  };
  const Seg mine = segment(tid);
  static_assert(PLAN_THREADS == 16 * 64, "");
  int turn = 0;
  auto exchange = [&](uint32_t x) __attribute__((always_inline)) {  // 16 lanes have a value of all waves each: that of lane 0, 1, 2, 3
    uint32_t* const all = &s_all[turn & 1][0][0];
    ++turn;
    if (lane < 4) all[lane * (PLAN_THREADS / 64) + w] = x;
    __syncthreads();
    return (lane & 15) < threads / 64 ? all[lane] : 0u;
  };
  auto of_lane = [](float x, int from) __attribute__((always_inline)) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), from));
  };
  struct Sums {
    float x, y, top;
  };
  auto gather = [&](Sums s) __attribute__((always_inline)) {  // sums over all threads (exact up to 2^24), the maximum of the last value
    s = Sums{dag_wave_sum(s.x), dag_wave_sum(s.y), dag_wave_max(s.top)};
    if (threads > 64) {
      const float v = __uint_as_float(exchange(__float_as_uint(lane == 0 ? s.x : lane == 1 ? s.y : s.top)));
      const float sum = dag_wave_sum<8>(v);
      s = Sums{of_lane(sum, 0), of_lane(sum, 16), of_lane(dag_wave_max<8>(v), 32)};
    }
    return s;
  };
  // slices of a segment of at most 2^k pages (an eighth more of the longer ones), and the pages of them if all are alike and even
  // (a 32-key block never straddles two)
  auto longest_slice = [](int k) __attribute__((always_inline)) { return (1 << k) >= SEG_STRETCH ? 9 << (k - 3) : 1 << k; };
  auto slices_of = [&](int npages, int k) __attribute__((always_inline)) {
    const uint32_t x = (uint32_t)(npages + longest_slice(k) - 1);
    return (int)((1 << k) >= SEG_STRETCH ? (x >> (k - 3)) / 9 : x >> k);
  };
  auto slice_of = [&](int npages, int k) __attribute__((always_inline)) {
    const int n = slices_of(npages, k);
    return n > 0 ? (int)((uint32_t)(npages + n - 1) / (uint32_t)n + 1) & ~1 : 1;
  };
  auto fits = [](float n, int most) { return n < 16777216.f ? n <= (float)most : n * 1.001f < (float)most; };
  const bool at_once = a.n_segments <= threads;
  const int host = 31 - __builtin_clz(a.chunk);  // (of a power of two, unless a.fixed)
  int k = a.few ? 3 : host;
  float longest = (float)(a.chunk * a.splits);
  if (!a.few && !a.fixed) {
    Sums sums = {};
    for (int s = tid; s < a.n_segments; s += threads) {
      const Seg g = s == tid ? mine : segment(s);
      sums.x += (float)g.rbs * (float)g.npages;
      sums.y += (float)g.nr * (float)g.npages;
      sums.top = fmaxf(sums.top, (float)g.npages);
    }
    sums = gather(sums);
    longest = sums.top;
    const float pages = sums.x * a.weight;
    k = pages < (longest <= SEG_SHORT ? SEG_PAGES_16_SHORT : SEG_PAGES_16) ? 3 : pages < SEG_PAGES_32 ? 4 : pages < SEG_PAGES_64 ? 5 : pages < a.pages_128 ? 6 : 7;
    for (; k < host; ++k) {
      const float one = 1.f / (float)longest_slice(k);
      if (!fits(sums.x * one, a.item_cap) || !fits(sums.y * one, room)) continue;
      if (at_once) break;  // (the places tell)
      Sums n = {};
      for (int s = tid; s < a.n_segments; s += threads) {
        const Seg g = s == tid ? mine : segment(s);
        const float nsp = (float)slices_of(g.npages, k);
        n.x += nsp * (float)g.rbs;
        n.y += nsp * (float)g.nr;
      }
      n = gather(n);
      if (fits(n.x, a.item_cap) && fits(n.y, room)) break;
    }
  }
  int start0 = 0, first0 = 0;  // items and partials of the segments in front
  for (int base = 0; base < a.n_segments; base += threads) {
    const int s = base + tid;
    const Seg g = base == 0 ? mine : segment(s);
    int slice, nsp, cnt, parts, start, first;
    for (;; ++k) {
      slice = a.fixed ? a.chunk : slice_of(g.npages, k);
      nsp = (int)((uint32_t)(g.npages + slice - 1) / (uint32_t)slice);
      cnt = nsp * g.rbs;
      parts = nsp * g.nr;
      start = dag_wave_scan(cnt);
      first = dag_wave_scan(parts);
      int items = __builtin_amdgcn_readlane(start, 63), places = __builtin_amdgcn_readlane(first, 63);
      start += start0 - cnt;
      first += first0 - parts;
      if (threads > 64) {
        const uint32_t v = exchange(lane == 0 ? items : places);
        const int front = dag_wave_sum<8>((lane & 15) < w ? (int)v : 0), sum = dag_wave_sum<8>((int)v);
        start += __builtin_amdgcn_readlane(front, 0);
        first += __builtin_amdgcn_readlane(front, 16);
        items = __builtin_amdgcn_readlane(sum, 0);
        places = __builtin_amdgcn_readlane(sum, 16);
      }
      if (a.few || !at_once || k >= host || ((uint32_t)items <= (uint32_t)a.item_cap && (uint32_t)places <= (uint32_t)room)) {
        start0 += items;
        first0 += places;
        break;
      }
    }
    if (s < a.n_segments) {
      int at = start;
      const int page_off = a.seg_page_off[s], code = a.fixed ? nsp : nsp | slice << 23;
      for (int sp = nsp - 1; sp >= 0; --sp)
        for (int rb = 0; rb < g.rbs; ++rb, ++at)
          if (at < a.item_cap) a.items[at] = SegItem{page_off, g.len, g.e0, g.nr * a.G, rb * 32, sp * slice, first + sp, code};
      for (int e = 0; e < g.nr; ++e) {
        if (g.e0 + e >= 0 && g.e0 + e < a.total_readers) a.entry_first[g.e0 + e] = first + e * nsp;
        if (g.e0 + e == a.total_readers - 1) a.totals[1] = first + (e + 1) * nsp;
      }
      const int end = g.e0 + g.nr;  // (fewer entries listed than announced: the last one's partials end here all the same)
      if (s + 1 == a.n_segments && end >= 0 && end < a.total_readers) a.entry_first[end] = first + parts;
    }
  }
  if (tid == 0) {
    a.totals[0] = min(start0, a.item_cap);
    // most slices of a segment, at least (one of more than 2^24 pages is longer than any pool)
    a.totals[2] = a.fixed || a.few ? a.splits : ((int)longest + (1 << k) - 1) >> k;
  }
}

}  // namespace
