// Pages that several rows hold, worked out on the GPU: dag_kv_fork, dag_kv_release_shared, dag_kv_compact, and the copies they ask for.
//
// A page has one holder and extra[p] more.  A fork holds its parent's full pages once more and takes a page of its own for what is left of the
// prefix; a release takes holders off and frees the pages that have none left; a compaction moves the k-th used page from the number U of
// used ones on to the k-th free page in front of it.  All of it is prefix sums and sums of ones, which do not depend on an order; what bounds the
// calls is launches and the loads behind one another, what bounds the copies is bytes.
#include <algorithm>

#include "kv_rows.h"

namespace {

constexpr int LIST_THREADS = 256, PAGE_THREADS = 256;

struct PagesArgs {
  dag_kv_rows_t rows;
  dag_kv_rows_t to;  // compaction: what table and free list become
  const int32_t* parent;
  const int32_t* child;
  const int32_t* fork_len;
  const int32_t* ended;
  const int32_t* row_len;
  int32_t* row_len_out;
  const int32_t* extra;
  int32_t* extra_out;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* refused;
  int32_t* page_map;
  int32_t* n_copies;
  int n_forks;
  // workspace
  int32_t* claim;   // [n_rows] fork: the first one that asks for the row; release: pages that the row frees, then where they go
  int32_t* tokens;  // [n_forks] of the child, -1: refused
  uint64_t* last;   // [n_pages] the last place (+ 1) from which the page is given back
  int32_t* times;   // [n_pages] how often it is
  uint32_t* bits;   // [n_pages / 32] free pages
  int32_t* rank;    // [1 + n_pages / 32] used pages; for each word, pages that move in front of its own
};

__device__ __forceinline__ int pages_held(const PagesArgs& a, int r) { return (int)min(pages_of(max(a.row_len[r], 0)), (int64_t)a.rows.max_row_pages); }
__device__ __forceinline__ int free_pages(const PagesArgs& a) { return min(max(a.free_count[0], 0), a.rows.n_pages); }
__device__ __forceinline__ bool in_pool(const PagesArgs& a, int p) { return (uint32_t)p < (uint32_t)a.rows.n_pages; }
// (written by atomics of other waves: past the caches of the compute unit)
template <typename T>
__device__ __forceinline__ T fresh(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A barrier behind which what the workgroup's waves have written and added up is where fresh() looks for it.
__device__ __forceinline__ void settle() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Which forks there are, their tokens and pages; by one workgroup.
__device__ __forceinline__ void fork_rows(const PagesArgs& a) {
  const int me = threadIdx.x, n_rows = a.rows.n_rows;
  for (int r = me; r < n_rows; r += ROW_THREADS) {
    a.claim[r] = INT32_MAX;
    if (a.row_len_out != a.row_len) a.row_len_out[r] = max(a.row_len[r], 0);
  }
  settle();
  for (int f = me; f < a.n_forks; f += ROW_THREADS) {
    const int p = a.parent[f], c = a.child[f];
    if ((uint32_t)p < (uint32_t)n_rows && (uint32_t)c < (uint32_t)n_rows && a.row_len[c] <= 0) atomicMin(a.claim + c, f);
  }
  settle();
  const int count = free_pages(a);
  int64_t front = 0, refused = 0;
  for (int base = 0; base < a.n_forks; base += ROW_THREADS) {
    const int f = base + me;
    int n = 0, p = 0;
    bool ok = false;
    if (f < a.n_forks) {
      const int c = a.child[f];
      p = a.parent[f];
      ok = (uint32_t)p < (uint32_t)n_rows && (uint32_t)c < (uint32_t)n_rows && fresh(a.claim + c) == f;
      if (ok) {
        n = (int)min((int64_t)max(a.row_len[p], 0), (int64_t)a.rows.max_row_pages * PAGE);
        if (a.fork_len) n = min(n, max(a.fork_len[f], 0));
      }
    }
    const bool need = ok && n % PAGE != 0;
    int64_t x[1] = {need}, all[1];
    block_scan(x, all);
    if (need && front + x[0] >= count) ok = false;
    int64_t y[1] = {f < a.n_forks && !ok}, bad[1];
    block_scan(y, bad);
    if (f < a.n_forks) {
      a.tokens[f] = ok ? n : -1;
      a.copy_src[f] = ok && need ? a.rows.table[(size_t)p * a.rows.max_row_pages + n / PAGE] : -1;
      a.copy_dst[f] = ok && need ? a.rows.free_pages[count - 1 - (front + x[0])] : -1;
    }
    front += all[0];
    refused += bad[0];
  }
  // (a parent without tokens may be a child: lengths are written when all have been read)
  for (int f = me; f < a.n_forks; f += ROW_THREADS)
    if (a.tokens[f] >= 0) a.row_len_out[a.child[f]] = a.tokens[f];
  if (me == 0) {
    a.free_count_out[0] = (int32_t)(count - min(front, (int64_t)count));
    if (a.refused) a.refused[0] = (int32_t)refused;
  }
}

__device__ __forceinline__ void fork_extra(const PagesArgs& a, int64_t at, int64_t step) {
  if (a.extra_out == a.extra) return;
  for (int64_t p = at; p < a.rows.n_pages; p += step) a.extra_out[p] = a.extra[p];
}
// The child's line of fork f, by `step` threads.
__device__ __forceinline__ void fork_line(const PagesArgs& a, int f, int at, int step) {
  const int n = a.tokens[f];
  if (n <= 0) return;
  const int32_t* const from = a.rows.table + (size_t)a.parent[f] * a.rows.max_row_pages;
  int32_t* const to = a.rows.table + (size_t)a.child[f] * a.rows.max_row_pages;
  for (int i = at; i < n / PAGE; i += step) {
    const int p = from[i];
    to[i] = p;
    if (in_pool(a, p)) atomicAdd(a.extra_out + p, 1);
  }
  if (at == 0 && n % PAGE != 0) to[n / PAGE] = a.copy_dst[f];
}

// In two launches (workgroup 0: the forks; the others take the holders over), or small tables in one, by one workgroup.
__global__ void __launch_bounds__(ROW_THREADS) k_kv_fork_rows(PagesArgs a) {
  if (blockIdx.x == 0) fork_rows(a);
  else fork_extra(a, (int64_t)(blockIdx.x - 1) * ROW_THREADS + threadIdx.x, (int64_t)(gridDim.x - 1) * ROW_THREADS);
}
__global__ void __launch_bounds__(LIST_THREADS) k_kv_fork_lines(PagesArgs a) {
  for (int f = blockIdx.x; f < a.n_forks; f += gridDim.x) fork_line(a, f, threadIdx.x, LIST_THREADS);
}
__global__ void __launch_bounds__(ROW_THREADS) k_kv_fork_whole(PagesArgs a) {
  fork_extra(a, threadIdx.x, ROW_THREADS);
  fork_rows(a);
  settle();
  for (int f = threadIdx.x / 64; f < a.n_forks; f += ROW_THREADS / 64) fork_line(a, f, threadIdx.x & 63, 64);
}

// Release, in phases that each need the one in front whole: by one workgroup with barriers between them, or a launch each.
// What one thread of `step` does, from `at` on.
__device__ __forceinline__ void release_clear(const PagesArgs& a, int64_t at, int64_t step) {
  for (int64_t p = at; p < a.rows.n_pages; p += step) {
    a.times[p] = 0;
    a.last[p] = 0;
  }
}
// (a wave to a row)
__device__ __forceinline__ void release_count(const PagesArgs& a, int64_t at, int64_t step, int lane) {
  for (int64_t r = at; r < a.rows.n_rows; r += step) {
    if (a.ended[r] == 0) continue;
    const int n = pages_held(a, (int)r);
    for (int i = lane; i < n; i += 64) {
      const int64_t place = r * a.rows.max_row_pages + i;
      const int p = a.rows.table[place];
      if (!in_pool(a, p)) continue;
      atomicAdd(a.times + p, 1);
      atomicMax((unsigned long long*)(a.last + p), (unsigned long long)place + 1);
    }
  }
}
// Pages that row r frees, the entries that give a page back last and leave it without a holder: how many, or (WRITE) into the free list from `to` on.
template <bool WRITE>
__device__ __forceinline__ int release_row(const PagesArgs& a, int64_t r, int to, int lane) {
  const int n = a.ended[r] == 0 ? 0 : pages_held(a, (int)r);
  for (int base = 0; base < n; base += 64) {
    const int i = base + lane;
    const int64_t place = r * a.rows.max_row_pages + i;
    const int p = i < n ? a.rows.table[place] : -1;
    const bool mine = in_pool(a, p) && fresh(a.last + p) == (uint64_t)place + 1 && fresh(a.times + p) > max(a.extra[p], 0);
    const uint64_t all = __builtin_amdgcn_ballot_w64(mine);
    const int at = to + __builtin_popcountll(all & ((1ull << lane) - 1));
    if (WRITE && mine && at < a.rows.n_pages) a.rows.free_pages[at] = p;
    to += __builtin_popcountll(all);
  }
  return to;
}
__device__ __forceinline__ void release_rows(const PagesArgs& a, int64_t at, int64_t step, int lane) {
  for (int64_t r = at; r < a.rows.n_rows; r += step) {
    const int n = release_row<false>(a, r, 0, lane);
    if (lane == 0) a.claim[r] = n;
  }
}
// The free list of the rows [r0, r0 + ROW_WAVES), a wave each, behind the sums of all rows in front.
constexpr int ROW_WAVES = ROW_THREADS / 64;
__device__ __forceinline__ void release_write(const PagesArgs& a, int64_t r0) {
  __shared__ int s_to[ROW_WAVES];
  int64_t front = free_pages(a);
  for (int64_t base = 0; base < r0 + ROW_WAVES; base += ROW_THREADS) {
    const int64_t r = base + threadIdx.x;
    int64_t x[1] = {r < a.rows.n_rows ? fresh(a.claim + r) : 0}, all[1];
    block_scan(x, all);
    if (r >= r0 && r < r0 + ROW_WAVES) s_to[r - r0] = (int)(front + x[0]);
    front += all[0];
  }
  __syncthreads();
  const int64_t r = r0 + threadIdx.x / 64;
  if (r < a.rows.n_rows) release_row<true>(a, r, s_to[threadIdx.x / 64], threadIdx.x & 63);
  __syncthreads();
}
// When nobody reads them any more: holders, lengths and the number of free pages.
__device__ __forceinline__ void release_end(const PagesArgs& a, int64_t at, int64_t step) {
  for (int64_t p = at; p < a.rows.n_pages; p += step) a.extra_out[p] = max(max(a.extra[p], 0) - fresh(a.times + p), 0);
  for (int64_t r = at; r < a.rows.n_rows; r += step) a.row_len_out[r] = a.ended[r] != 0 ? 0 : max(a.row_len[r], 0);
}
// By one workgroup: the sums of the pages that rows free, the number of free pages.  PLACES: the sums in front of every row in its place.
template <bool PLACES>
__device__ __forceinline__ void release_scan(const PagesArgs& a) {
  int64_t front = free_pages(a);
  for (int64_t base = 0; base < a.rows.n_rows; base += ROW_THREADS) {
    const int64_t r = base + threadIdx.x;
    int64_t x[1] = {r < a.rows.n_rows ? fresh(a.claim + r) : 0}, all[1];
    block_scan(x, all);
    if (PLACES && r < a.rows.n_rows) a.claim[r] = (int32_t)(front + x[0]);
    front += all[0];
  }
  if (threadIdx.x == 0) a.free_count_out[0] = (int32_t)min(front, (int64_t)a.rows.n_pages);
}
__device__ __forceinline__ void release_lists(const PagesArgs& a, int64_t at, int64_t step, int lane) {
  for (int64_t r = at; r < a.rows.n_rows; r += step) release_row<true>(a, r, fresh(a.claim + r), lane);
}

__global__ void __launch_bounds__(ROW_THREADS) k_kv_release_whole(PagesArgs a) {
  const int me = threadIdx.x, lane = me & 63, w = me >> 6;
  release_clear(a, me, ROW_THREADS);
  settle();
  release_count(a, w, ROW_WAVES, lane);
  settle();
  release_rows(a, w, ROW_WAVES, lane);
  settle();
  release_scan<true>(a);
  settle();
  release_lists(a, w, ROW_WAVES, lane);
  settle();
  release_end(a, me, ROW_THREADS);
}

enum { CLEAR, COUNT, ROWS, WRITE, END, SCAN, LISTS, LAST };
template <int PHASE>
__global__ void __launch_bounds__(ROW_THREADS) k_kv_release_phase(PagesArgs a) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  const int lane = threadIdx.x & 63;
  if constexpr (PHASE == CLEAR) release_clear(a, at, step);
  if constexpr (PHASE == COUNT) release_count(a, at / 64, step / 64, lane);
  if constexpr (PHASE == ROWS) release_rows(a, at / 64, step / 64, lane);
  if constexpr (PHASE == WRITE) release_write(a, (int64_t)blockIdx.x * ROW_WAVES);
  if constexpr (PHASE == END) {  // (workgroup 0 adds the pages up; their number may be written where it was read, so not before)
    if (blockIdx.x == 0) release_scan<false>(a);
    else release_end(a, at - blockDim.x, step - blockDim.x);
  }
  // (many rows: every workgroup of WRITE would go through all of them)
  if constexpr (PHASE == SCAN) release_scan<true>(a);
  if constexpr (PHASE == LISTS) release_lists(a, at / 64, step / 64, lane);
  if constexpr (PHASE == LAST) release_end(a, at, step);
}

// Compaction: which pages are free, how many used ones move, from where to where.  One workgroup; a thread has a run of words of 32 pages.
constexpr int LDS_WORDS = 8192;  // 262144 pages
__device__ __forceinline__ void compact_pages(const PagesArgs& a) {
  __shared__ uint32_t s_bits[LDS_WORDS];
  const int me = threadIdx.x, n_pages = a.rows.n_pages, words = (n_pages + 31) / 32;
  const bool lds = words <= LDS_WORDS;
  for (int i = me; i < words; i += ROW_THREADS) {
    if (lds) s_bits[i] = 0;
    else a.bits[i] = 0;
  }
  settle();
  const int count = free_pages(a);
  constexpr int AHEAD = 4;
  for (int base = me; base < count; base += AHEAD * ROW_THREADS) {
    int p[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) p[i] = a.rows.free_pages[min(base + i * ROW_THREADS, count - 1)];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (!in_pool(a, p[i])) continue;
      if (lds) atomicOr(s_bits + p[i] / 32, 1u << p[i] % 32);
      else atomicOr(a.bits + p[i] / 32, 1u << p[i] % 32);
    }
  }
  settle();
  auto bits = [&](int i) { return lds ? s_bits[i] : fresh(a.bits + i); };
  const int each = (words + ROW_THREADS - 1) / ROW_THREADS, w0 = min(me * each, words), w1 = min(w0 + each, words);
  int64_t f[1] = {0}, n_free[1];
  for (int i = w0; i < w1; ++i) f[0] += __builtin_popcount(bits(i));
  block_scan(f, n_free);
  const int used = n_pages - (int)n_free[0];
  // pages of word i in front of `used`, and those of the pool
  auto front = [=](int i) { return i * 32 >= used ? 0u : i * 32 + 32 <= used ? 0xffffffffu : (1u << (used - i * 32)) - 1u; };
  auto there = [=](int i) { return i * 32 + 32 <= n_pages ? 0xffffffffu : (1u << (n_pages - i * 32)) - 1u; };
  int64_t x[2] = {0, 0}, all[2];
  for (int i = w0; i < w1; ++i) {
    const uint32_t b = bits(i);
    x[0] += __builtin_popcount(b & front(i));
    x[1] += __builtin_popcount(~b & there(i) & ~front(i));
  }
  block_scan(x, all);
  int to = (int)x[0], from = (int)x[1];
  for (int i = w0; i < w1; ++i) {
    const uint32_t b = bits(i);
    if (lds) a.bits[i] = b;
    a.rank[i + 1] = from;
    for (uint32_t m = b & front(i); m; m &= m - 1) a.copy_dst[to++] = 32 * i + __builtin_ctz(m);
    for (uint32_t m = ~b & there(i) & ~front(i); m; m &= m - 1) a.copy_src[from++] = 32 * i + __builtin_ctz(m);
  }
  if (me == 0) {
    a.n_copies[0] = (int32_t)all[0];
    a.rank[0] = used;
  }
}

// Then the lists of the pages and the lines of the rows (a wave to a row).  WHOLE: in the workgroup that has worked the places out.
template <bool WHOLE>
struct Places {
  const PagesArgs& a;
  int used, n_pages;
  __device__ __forceinline__ uint32_t bits(int w) const { return WHOLE ? fresh(a.bits + w) : a.bits[w]; }
  __device__ __forceinline__ bool is_free(int p) const { return bits(p / 32) >> p % 32 & 1; }
  __device__ __forceinline__ int operator()(int p) const {  // of a used page
    if (p < used) return p;
    const uint32_t b = ~bits(p / 32) & (0xffffffffu << max(used - (p & ~31), 0)) & ((1u << p % 32) - 1u);
    return a.copy_dst[a.rank[p / 32 + 1] + __builtin_popcount(b)];
  }
};
template <bool WHOLE>
__device__ __forceinline__ void compact_lists(const PagesArgs& a, int64_t at, int64_t step) {
  const int n_pages = a.rows.n_pages, used = a.rank[0], count = n_pages - used;
  const Places<WHOLE> place{a, used, n_pages};
  for (int64_t i = at; i < n_pages; i += step) {
    const int p = (int)i;
    const bool none = place.is_free(p);
    const int to = none ? -1 : place(p);
    a.page_map[p] = to;
    if (p < count) a.to.free_pages[p] = n_pages - 1 - p;
    // (a free page in front of `used` is written by the page that moves there)
    if (!none) {
      const int n = a.extra[p];
      if (to != p) a.extra_out[p] = 0;
      a.extra_out[to] = n;
    } else if (p >= used) {
      a.extra_out[p] = 0;
    }
  }
}
template <bool WHOLE>
__device__ __forceinline__ void compact_lines(const PagesArgs& a, int64_t at, int64_t step, int lane) {
  const Places<WHOLE> place{a, a.rank[0], a.rows.n_pages};
  for (int64_t r = at; r < a.rows.n_rows; r += step) {
    const int n = pages_held(a, (int)r);
    for (int i = lane; i < n; i += 64) {
      const size_t e = (size_t)r * a.rows.max_row_pages + i;
      const int p = a.rows.table[e];
      a.to.table[e] = in_pool(a, p) && !place.is_free(p) ? place(p) : p;
    }
  }
}
__global__ void __launch_bounds__(ROW_THREADS) k_kv_compact_pages(PagesArgs a) { compact_pages(a); }
__global__ void __launch_bounds__(PAGE_THREADS) k_kv_compact_lists(PagesArgs a, int page_blocks) {  // the first workgroups: pages, the others: rows
  constexpr int WAVES = PAGE_THREADS / 64;
  if ((int)blockIdx.x < page_blocks) compact_lists<false>(a, (int64_t)blockIdx.x * PAGE_THREADS + threadIdx.x, (int64_t)page_blocks * PAGE_THREADS);
  else compact_lines<false>(a, (int64_t)(blockIdx.x - page_blocks) * WAVES + threadIdx.x / 64, (int64_t)(gridDim.x - page_blocks) * WAVES, threadIdx.x & 63);
}
__global__ void __launch_bounds__(ROW_THREADS) k_kv_compact_whole(PagesArgs a) {
  compact_pages(a);
  settle();
  compact_lists<true>(a, threadIdx.x, ROW_THREADS);
  compact_lines<true>(a, threadIdx.x / 64, ROW_THREADS / 64, threadIdx.x & 63);
}

struct CopyArgs {
  const int32_t* src;
  const int32_t* dst;
  const int32_t* count;
  char* pool[2];
  float* scale[2];
  int64_t page_bytes;
  int n, n_pages, hkv;
};
// A wave has 4 KiB of a page of a pool, four pieces of a lane on their way.
constexpr int COPY_BYTES = 4096;
__global__ void __launch_bounds__(256) k_kv_copy_pages(CopyArgs a) {
  const int lane = threadIdx.x & 63, chunks = (int)((a.page_bytes + COPY_BYTES - 1) / COPY_BYTES);
  const int n = a.count ? min(max(a.count[0], 0), a.n) : a.n;
  const int64_t waves = (int64_t)gridDim.x * 4, units = (int64_t)n * 2 * chunks;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += waves) {
    const int e = (int)(u / (2 * chunks)), x = (int)(u % (2 * chunks)), v = x >= chunks, chunk = x - v * chunks;
    const int src = a.src[e], dst = a.dst[e];
    if ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages) continue;
    const char* const from = a.pool[v] + (int64_t)src * a.page_bytes;
    char* const to = a.pool[v] + (int64_t)dst * a.page_bytes;
    u32x4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = chunk * (int64_t)COPY_BYTES + i * 1024 + lane * 16;
      if (at < a.page_bytes) y[i] = *(const u32x4*)(from + at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = chunk * (int64_t)COPY_BYTES + i * 1024 + lane * 16;
      if (at < a.page_bytes) *(u32x4*)(to + at) = y[i];
    }
    if (chunk == 0 && a.scale[v])
      for (int h = lane; h < a.hkv; h += 64) a.scale[v][(int64_t)dst * a.hkv + h] = a.scale[v][(int64_t)src * a.hkv + h];
  }
}

int copy_pages(const CopyArgs& a, hipStream_t stream) {
  if (a.n == 0 || a.n_pages == 0) return DAG_OK;
  const int64_t waves = (int64_t)a.n * 2 * dag_ceil_div(a.page_bytes, COPY_BYTES);
  hipLaunchKernelGGL(k_kv_copy_pages, dim3((unsigned)std::min<int64_t>(dag_ceil_div(waves, 4), 2048)), dim3(256), 0, stream, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

// One workgroup does a call as a whole as long as its turns take no longer than the launches do: with two lines of the table (rows, or the children of
// forks) to a wave, up to 4096 pages (2048 to compact) and 4096 entries (2048 of forks).  Whole / in launches, replayed: 24 rows of 64 and 833 pages, 6 forks 5.3 / 7.0 us, release
// 8.0 / 11.1, compaction 9.0 / 9.4; 32 rows of 128 and 2003 pages 7.0 / 7.4, 12.3 / 13.6, 11.9 / 11.2; 64 rows of 48 (16 forks) 5.9 / 7.1, 12.6 / 11.8,
// 11.5 / 10.3; 128 rows of 64 and 3589 pages 10.6 / 7.0, 25.3 / 12.4, 15.4 / 10.6; 150 rows of 12 (30 forks) 7.3 / 7.4, 25.1 / 11.9, 14.5 / 10.2.
inline bool by_one(int64_t lines, const dag_kv_rows_t* rows, int64_t most_entries, int64_t most_pages) {
  return lines <= 2 * ROW_WAVES && lines * rows->max_row_pages <= most_entries && rows->n_pages <= most_pages;
}
// Workgroups of a launch at most (its threads are counted in 32 bits); they go on with the rows or forks that are left.
constexpr int64_t MOST_BLOCKS = 1 << 20;

size_t words_of(int32_t n_pages) { return ((size_t)n_pages + 31) / 32; }

int check_pages(const dag_kv_rows_t* rows, const void* ws, size_t ws_bytes, int64_t n_forks) {
  if (!rows) return DAG_ERR_NULL;
  // (rows and forks are counted in 32 bits, a workgroup's threads past the last one too)
  if (rows->n_rows < 0 || rows->max_row_pages < 0 || rows->n_pages < 0 || rows->n_pages > INT32_MAX / PAGE || rows->max_row_pages > INT32_MAX / PAGE ||
      rows->n_rows > INT32_MAX / PAGE || n_forks < 0 || n_forks > INT32_MAX / PAGE)
    return DAG_ERR_BAD_LEN;
  if (rows->page_size != PAGE) return DAG_ERR_UNSUPPORTED;
  if ((rows->n_rows > 0 && rows->max_row_pages > 0 && !rows->table) || (rows->n_pages > 0 && !rows->free_pages)) return DAG_ERR_NULL;
  if (!ws || ws_bytes < dag_kv_pages_workspace_bytes(rows->n_rows, rows->n_pages, (int32_t)n_forks)) return DAG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 7) return DAG_ERR_ALIGN;
  return DAG_OK;
}

PagesArgs pages_args(const dag_kv_rows_t* rows, void* ws) {
  PagesArgs a = {};
  a.rows = *rows;
  a.last = (uint64_t*)ws;
  a.times = (int32_t*)(a.last + rows->n_pages);
  a.claim = a.times + rows->n_pages;
  a.tokens = a.claim + rows->n_rows;
  a.bits = (uint32_t*)ws;  // (of another call than those)
  a.rank = (int32_t*)(a.bits + words_of(rows->n_pages));
  return a;
}

}  // namespace

extern "C" size_t dag_kv_pages_workspace_bytes(int32_t n_rows, int32_t n_pages, int32_t n_forks) {
  if (n_rows < 0 || n_pages < 0 || n_forks < 0) return 0;
  return (size_t)n_pages * 12 + ((size_t)n_rows + n_forks) * 4 + 256;
}

extern "C" int dag_kv_fork(const dag_kv_rows_t* rows, int32_t n_forks, const int32_t* parent, const int32_t* child, const int32_t* fork_len,
                           const int32_t* row_len, int32_t* row_len_out, const int32_t* extra, int32_t* extra_out, const int32_t* free_count,
                           int32_t* free_count_out, int32_t* copy_src, int32_t* copy_dst, int32_t* refused, void* ws, size_t ws_bytes, void* stream_) {
  const int rc = check_pages(rows, ws, ws_bytes, n_forks);
  if (rc != DAG_OK) return rc;
  if (!free_count || !free_count_out || (rows->n_rows > 0 && (!row_len || !row_len_out)) || (rows->n_pages > 0 && (!extra || !extra_out)) ||
      (n_forks > 0 && (!parent || !child || !copy_src || !copy_dst)))
    return DAG_ERR_NULL;
  PagesArgs a = pages_args(rows, ws);
  a.parent = parent;
  a.child = child;
  a.fork_len = fork_len;
  a.row_len = row_len;
  a.row_len_out = row_len_out;
  a.extra = extra;
  a.extra_out = extra_out;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  a.copy_src = copy_src;
  a.copy_dst = copy_dst;
  a.refused = refused;
  a.n_forks = n_forks;
  hipStream_t stream = (hipStream_t)stream_;
  if (by_one(n_forks, rows, 2048, 4096)) {
    hipLaunchKernelGGL(k_kv_fork_whole, dim3(1), dim3(ROW_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  const int64_t copies = extra == extra_out ? 0 : std::min<int64_t>(dag_ceil_div(rows->n_pages, ROW_THREADS), 256);
  hipLaunchKernelGGL(k_kv_fork_rows, dim3((unsigned)(1 + copies)), dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (n_forks > 0) {
    hipLaunchKernelGGL(k_kv_fork_lines, dim3((unsigned)std::min<int64_t>(n_forks, MOST_BLOCKS)), dim3(LIST_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}

extern "C" int dag_kv_release_shared(const dag_kv_rows_t* rows, const int32_t* ended, const int32_t* row_len, int32_t* row_len_out, const int32_t* extra,
                                     int32_t* extra_out, const int32_t* free_count, int32_t* free_count_out, void* ws, size_t ws_bytes, void* stream_) {
  const int rc = check_pages(rows, ws, ws_bytes, 0);
  if (rc != DAG_OK) return rc;
  if (!free_count || !free_count_out || (rows->n_rows > 0 && (!ended || !row_len || !row_len_out)) || (rows->n_pages > 0 && (!extra || !extra_out)))
    return DAG_ERR_NULL;
  PagesArgs a = pages_args(rows, ws);
  a.ended = ended;
  a.row_len = row_len;
  a.row_len_out = row_len_out;
  a.extra = extra;
  a.extra_out = extra_out;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  hipStream_t stream = (hipStream_t)stream_;
  if (by_one(rows->n_rows, rows, 4096, 4096)) {
    hipLaunchKernelGGL(k_kv_release_whole, dim3(1), dim3(ROW_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  const unsigned by_page = (unsigned)std::max<int64_t>(1, std::min<int64_t>(dag_ceil_div(rows->n_pages, 256), 2048));
  const unsigned by_row = (unsigned)std::max<int64_t>(1, std::min<int64_t>(dag_ceil_div(rows->n_rows, 4), 2048));
  hipLaunchKernelGGL(k_kv_release_phase<CLEAR>, dim3(by_page), dim3(256), 0, stream, a);
  DAG_LAUNCH_CHECK();
  hipLaunchKernelGGL(k_kv_release_phase<COUNT>, dim3(by_row), dim3(256), 0, stream, a);
  DAG_LAUNCH_CHECK();
  hipLaunchKernelGGL(k_kv_release_phase<ROWS>, dim3(by_row), dim3(256), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (rows->n_rows > 4 * ROW_THREADS) {
    hipLaunchKernelGGL(k_kv_release_phase<SCAN>, dim3(1), dim3(ROW_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
    hipLaunchKernelGGL(k_kv_release_phase<LISTS>, dim3(by_row), dim3(256), 0, stream, a);
    DAG_LAUNCH_CHECK();
    hipLaunchKernelGGL(k_kv_release_phase<LAST>, dim3(by_page), dim3(256), 0, stream, a);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  if (rows->n_rows > 0) {
    hipLaunchKernelGGL(k_kv_release_phase<WRITE>, dim3((unsigned)dag_ceil_div(rows->n_rows, ROW_WAVES)), dim3(ROW_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(k_kv_release_phase<END>, dim3((unsigned)std::min<int64_t>(1 + dag_ceil_div(std::max(rows->n_pages, rows->n_rows), ROW_THREADS), 1025)),
                     dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  return DAG_OK;
}

extern "C" int dag_kv_compact(const dag_kv_rows_t* rows, const dag_kv_rows_t* rows_out, const int32_t* row_len, const int32_t* extra, int32_t* extra_out,
                              const int32_t* free_count, int32_t* page_map, int32_t* copy_src, int32_t* copy_dst, int32_t* n_copies, void* ws,
                              size_t ws_bytes, void* stream_) {
  const int rc = check_pages(rows, ws, ws_bytes, 0);
  if (rc != DAG_OK) return rc;
  if (!rows_out || !free_count || !n_copies || (rows->n_rows > 0 && !row_len) || (rows->n_pages > 0 && (!extra || !extra_out || !page_map)) ||
      (rows->n_pages > 1 && (!copy_src || !copy_dst)))
    return DAG_ERR_NULL;
  if (rows_out->n_rows != rows->n_rows || rows_out->max_row_pages != rows->max_row_pages || rows_out->n_pages != rows->n_pages) return DAG_ERR_BAD_LEN;
  if (rows_out->page_size != PAGE) return DAG_ERR_UNSUPPORTED;
  if ((rows->n_rows > 0 && rows->max_row_pages > 0 && !rows_out->table) || (rows->n_pages > 0 && !rows_out->free_pages)) return DAG_ERR_NULL;
  PagesArgs a = pages_args(rows, ws);
  a.to = *rows_out;
  a.row_len = row_len;
  a.extra = extra;
  a.extra_out = extra_out;
  a.free_count = free_count;
  a.page_map = page_map;
  a.copy_src = copy_src;
  a.copy_dst = copy_dst;
  a.n_copies = n_copies;
  hipStream_t stream = (hipStream_t)stream_;
  if (by_one(rows->n_rows, rows, 4096, 2048)) {
    hipLaunchKernelGGL(k_kv_compact_whole, dim3(1), dim3(ROW_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  hipLaunchKernelGGL(k_kv_compact_pages, dim3(1), dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  const int page_blocks = (int)std::min<int64_t>(dag_ceil_div(rows->n_pages, PAGE_THREADS), 1024);
  const int64_t blocks = page_blocks + std::min<int64_t>(dag_ceil_div(rows->n_rows, PAGE_THREADS / 64), MOST_BLOCKS);
  if (blocks > 0) {
    hipLaunchKernelGGL(k_kv_compact_lists, dim3((unsigned)blocks), dim3(PAGE_THREADS), 0, stream, a, page_blocks);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}

extern "C" int dag_kv_copy_pages_q8(const dag_kv_q8_t* kv, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* count, void* stream_) {
  if (!kv) return DAG_ERR_NULL;
  if (n < 0 || kv->n_pages < 0) return DAG_ERR_BAD_LEN;
  if (kv->hkv < 1 || (kv->head_dim != 64 && kv->head_dim != 128)) return DAG_ERR_UNSUPPORTED;
  if (n == 0) return DAG_OK;
  if (!src || !dst || !kv->k_pool || !kv->v_pool || !kv->k_scale || !kv->v_scale) return DAG_ERR_NULL;
  if (!dag_aligned16(kv->k_pool) || !dag_aligned16(kv->v_pool) || ((uintptr_t)kv->k_scale & 3) || ((uintptr_t)kv->v_scale & 3)) return DAG_ERR_ALIGN;
  const CopyArgs a = {src, dst, count, {(char*)kv->k_pool, (char*)kv->v_pool}, {kv->k_scale, kv->v_scale}, (int64_t)kv->hkv * kv->head_dim * PAGE, n,
                      kv->n_pages, kv->hkv};
  return copy_pages(a, (hipStream_t)stream_);
}

extern "C" int dag_kv_copy_pages(void* k_pool, void* v_pool, int32_t n_pages, int32_t hkv, int32_t head_dim, const int32_t* src, const int32_t* dst, int32_t n,
                                 const int32_t* count, void* stream_) {
  if (n < 0 || n_pages < 0) return DAG_ERR_BAD_LEN;
  if (hkv < 1 || (head_dim != 64 && head_dim != 128)) return DAG_ERR_UNSUPPORTED;
  if (n == 0) return DAG_OK;
  if (!src || !dst || !k_pool || !v_pool) return DAG_ERR_NULL;
  if (!dag_aligned16(k_pool) || !dag_aligned16(v_pool)) return DAG_ERR_ALIGN;
  const CopyArgs a = {src, dst, count, {(char*)k_pool, (char*)v_pool}, {nullptr, nullptr}, (int64_t)hkv * head_dim * PAGE * 2, n, n_pages, hkv};
  return copy_pages(a, (hipStream_t)stream_);
}
