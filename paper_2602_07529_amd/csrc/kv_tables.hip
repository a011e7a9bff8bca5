// Pages, slots and positions of rows (branches, nodes) that grow, worked out on the GPU: dag_kv_release, dag_kv_tables.
//
// A row r with n_r tokens holds ceil(n_r / 16) pages of its line of the table; free pages lie on a stack.  New tokens w_r need
// need_r = ceil((n_r + w_r) / 16) - ceil(n_r / 16) pages; with S_r = sum of need over the rows in front, row r takes the pages
// S_r .. S_r + need_r - 1 from the top of the stack, if that many are there.  Everything else follows from the prefix sums of need, w and the
// pages held.  Up to ONE_ROWS rows a call is one launch: every workgroup works out the sums of all rows, side by side, and writes the lists of a
// few of them.  Lengths and the number of free pages may be written where they were read, so the workgroup that comes last writes
// them, when all have read.  More rows: a scan by one workgroup, then a launch that writes the lists.  What bounds it is launches and the
// chain of loads behind one another (length, free page or line, lists), not bytes.
#include "common.h"

namespace {

constexpr int PAGE = DAG_PAGE_SIZE;
constexpr int ROW_THREADS = 1024, LIST_THREADS = 256;
constexpr int ONE_ROWS = ROW_THREADS, ONE_WAVES = ROW_THREADS / 64;

struct TableArgs {
  dag_kv_rows_t rows;
  const int32_t* new_len;
  const int32_t* ended;
  const int32_t* row_len;
  int32_t* row_len_out;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* new_off;
  int32_t* slots;
  const int32_t* pos0;
  int32_t* pos;
  int32_t* page_off;
  int32_t* pages;
  int32_t* refused;
  int64_t max_new, max_pages;
  int32_t* first;  // [n_rows] workspace: top of the stack for the row's first new page, -1: refused (or: place of its first page given back)
  int32_t* held;   // [n_rows] workspace: tokens before
  uint32_t* ticket;  // workspace: zero between calls
};

__device__ __forceinline__ int64_t pages_of(int64_t n) { return (n + PAGE - 1) / PAGE; }

// Sums over the threads in front of this one of N values each, and over all threads.
template <int N>
__device__ __forceinline__ void block_scan(int64_t (&x)[N], int64_t (&all)[N]) {
  __shared__ int64_t s_wave[N][ROW_THREADS / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t incl[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    incl[i] = dag_wave_scan(x[i]);
    if (lane == 63) s_wave[i][w] = incl[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t v = lane < (int)(blockDim.x >> 6) ? s_wave[i][lane] : 0, s = dag_wave_scan(v);
    all[i] = dag_readlane(s, 63);
    x[i] = incl[i] - x[i] + (w > 0 ? dag_readlane(s, w - 1) : 0);
  }
  __syncthreads();
}

// Sums of many rows by one workgroup, PER_THREAD of them to a thread, as a turn is loads and scans behind one another (release and tables of 4096
// rows, replayed: 29.6 us with one to a thread, 25.1 with four).
constexpr int PER_THREAD = 4;

__global__ void __launch_bounds__(ROW_THREADS) k_kv_release_rows(TableArgs a) {
  const int width = a.rows.max_row_pages, n_rows = a.rows.n_rows;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  int64_t front = 0;
  for (int64_t base = 0; base < n_rows; base += PER_THREAD * ROW_THREADS) {
    const int64_t r0 = base + PER_THREAD * threadIdx.x;
    int len[PER_THREAD];
    bool end[PER_THREAD];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      const int64_t r = min(r0 + i, (int64_t)n_rows - 1);
      len[i] = max(a.row_len[r], 0);
      end[i] = r0 + i < n_rows && a.ended[r] != 0;
    }
    int64_t gone[1] = {0}, all[1];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) gone[0] += end[i] ? min(pages_of(len[i]), (int64_t)width) : 0;
    block_scan(gone, all);
    int64_t at = count + front + gone[0];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      const int64_t r = r0 + i;
      if (r >= n_rows) break;
      const int64_t n = end[i] ? min(pages_of(len[i]), (int64_t)width) : 0;
      a.first[r] = (int32_t)at;
      a.held[r] = (int32_t)n;
      a.row_len_out[r] = end[i] ? 0 : len[i];
      at += n;
    }
    front += all[0];
  }
  if (threadIdx.x == 0) a.free_count_out[0] = (int32_t)min(count + front, (int64_t)a.rows.n_pages);
}

__global__ void __launch_bounds__(LIST_THREADS) k_kv_release_pages(TableArgs a) {
  const int r = blockIdx.x, n = a.held[r], at = a.first[r];
  const int32_t* const line = a.rows.table + (size_t)r * a.rows.max_row_pages;
  for (int j = threadIdx.x; j < n; j += LIST_THREADS)
    if (at + j < a.rows.n_pages) a.rows.free_pages[at + j] = line[j];
}

__global__ void __launch_bounds__(ROW_THREADS) k_kv_table_rows(TableArgs a) {
  const int width = a.rows.max_row_pages, n_rows = a.rows.n_rows;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  int64_t front_need = 0, front_new = 0, front_pages = 0, taken = 0, refused = 0;
  for (int64_t base = 0; base < n_rows; base += PER_THREAD * ROW_THREADS) {
    const int64_t r0 = base + PER_THREAD * threadIdx.x;
    int64_t len[PER_THREAD], want[PER_THREAD], need[PER_THREAD];
    bool fits[PER_THREAD];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      const int64_t r = min(r0 + i, (int64_t)n_rows - 1);
      const int x = a.row_len[r], y = a.new_len[r];
      const bool there = r0 + i < n_rows;
      len[i] = there ? max(x, 0) : 0;
      want[i] = there ? max(y, 0) : 0;
    }
    int64_t x[2] = {0, 0}, all[2];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      fits[i] = len[i] + want[i] <= (int64_t)width * PAGE;
      need[i] = fits[i] ? pages_of(len[i] + want[i]) - pages_of(len[i]) : 0;
      x[0] += need[i];
      x[1] += want[i];
    }
    block_scan(x, all);
    int64_t y[3] = {0, 0, 0}, sums[3], start = front_need + x[0];
    int32_t first[PER_THREAD], now[PER_THREAD];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      const bool ok = fits[i] && (need[i] == 0 || start + need[i] <= count);
      first[i] = !ok ? -1 : need[i] == 0 ? 0 : (int32_t)(count - 1 - start);
      now[i] = (int32_t)(len[i] + (ok ? want[i] : 0));
      start += need[i];
      y[0] += min(pages_of(now[i]), (int64_t)width);
      y[1] += !ok && want[i] > 0 ? 1 : 0;
      y[2] += ok ? need[i] : 0;
    }
    block_scan(y, sums);
    int64_t at = front_new + x[1], page_at = front_pages + y[0];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
      const int64_t r = r0 + i;
      if (r >= n_rows) break;
      a.row_len_out[r] = now[i];
      a.new_off[r] = (int32_t)at;
      if (a.page_off) a.page_off[r] = (int32_t)page_at;
      a.first[r] = first[i];
      a.held[r] = (int32_t)len[i];
      at += want[i];
      page_at += min(pages_of(now[i]), (int64_t)width);
    }
    front_need += all[0];
    front_new += all[1];
    front_pages += sums[0];
    refused += sums[1];
    taken += sums[2];
  }
  if (threadIdx.x == 0) {
    a.new_off[n_rows] = (int32_t)front_new;
    if (a.page_off) a.page_off[n_rows] = (int32_t)front_pages;
    if (a.refused) a.refused[0] = (int32_t)refused;
    a.free_count_out[0] = (int32_t)(count - taken);
  }
}

// Slots, positions and pages of row r, by `step` threads.  held: tokens before, now: behind, top: where its first new page lies on the stack
// (-1: refused); its new tokens are n from t0 on, its pages in the list from p0 on.
__device__ __forceinline__ void write_row(const TableArgs& a, int r, int held, int now, int top, int64_t t0, int n, int64_t p0, int tid, int step) {
  const int width = a.rows.max_row_pages, has = (int)pages_of(held), pages = (int)min(pages_of(now), (int64_t)width);
  int32_t* const line = a.rows.table + (size_t)r * width;
  const int32_t* const stack = a.rows.free_pages;
  auto page = [=](int p) { return *(p < has ? line + p : stack + max(top - (p - has), 0)); };  // (one load, not two under conditions)
  const int first = a.pos && a.pos0 ? a.pos0[r] : 0;
  constexpr int AHEAD = 4;  // loads on their way together
  for (int j = tid; j < n; j += AHEAD * step) {
    int id[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) id[i] = top < 0 ? 0 : page((held + min(j + i * step, n - 1)) / PAGE);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int q = j + i * step, at = held + q;
      if (q >= n || t0 + q >= a.max_new) break;
      a.slots[t0 + q] = top < 0 ? -1 : id[i] * PAGE + at % PAGE;
      if (a.pos) a.pos[t0 + q] = first + at;
    }
  }
  for (int p = (a.pages ? 0 : has) + tid; p < pages; p += AHEAD * step) {
    int id[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) id[i] = page(min(p + i * step, pages - 1));
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int q = p + i * step;
      if (q >= pages) break;
      if (q >= has) line[q] = id[i];
      if (a.pages && p0 + q < a.max_pages) a.pages[p0 + q] = id[i];
    }
  }
}

__global__ void __launch_bounds__(LIST_THREADS) k_kv_table_lists(TableArgs a) {
  const int r = blockIdx.x, t0 = a.new_off[r];
  write_row(a, r, a.held[r], a.row_len_out[r], a.first[r], t0, a.new_off[r + 1] - t0, a.page_off ? a.page_off[r] : 0, threadIdx.x, LIST_THREADS);
}

// Whether this workgroup is the last one to come here.
__device__ __forceinline__ bool comes_last(uint32_t* ticket) {
  __shared__ bool s_last;
  if (gridDim.x == 1) return true;
  if (threadIdx.x == 0) s_last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;  // (zero again behind the last one)
  __syncthreads();
  return s_last;
}

// All in one launch, per_row waves to a row.  Release and tables together, replayed from a graph, one launch each against two:
// 128 rows of one new token 10.5 us against 11.3, 256 prompts of 4099 tokens 15.4 / 16.7, 1024 rows of 1 12.0 / 12.6, 4096 rows (scans of four
// turns in every workgroup) 30.0 / 25.1; called one by one, where a launch costs the host 3.4 us, 128 rows 16.2 / 20.7.
__global__ void __launch_bounds__(ROW_THREADS) k_kv_tables_one(TableArgs a, int per_row) {
  struct Mine {
    int64_t t0, p0;
    int held, now, top, n;
  };
  __shared__ Mine s_row[ONE_WAVES];
  const int width = a.rows.max_row_pages, n_rows = a.rows.n_rows, here = ONE_WAVES / per_row, row0 = blockIdx.x * here;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  const int me = threadIdx.x;
  const bool there = me < n_rows;
  int64_t len = 0, want = 0, need = 0;
  bool fits = true;
  if (there) {
    len = max(a.row_len[me], 0);
    want = max(a.new_len[me], 0);
    fits = len + want <= (int64_t)width * PAGE;
    if (fits) need = pages_of(len + want) - pages_of(len);
  }
  int64_t x[2] = {need, want}, all[2];
  block_scan(x, all);
  const bool ok = fits && (need == 0 || x[0] + need <= count);
  const int64_t now = len + (ok ? want : 0), listed = there ? min(pages_of(now), (int64_t)width) : 0;
  int64_t y[3] = {listed, there && !ok && want > 0 ? 1 : 0, ok ? need : 0}, sums[3];
  block_scan(y, sums);
  if (there && me >= row0 && me < row0 + here) {
    a.new_off[me] = (int32_t)x[1];
    if (a.page_off) a.page_off[me] = (int32_t)y[0];
    s_row[me - row0] = Mine{x[1], y[0], (int)len, (int)now, ok ? (int)(need == 0 ? 0 : count - 1 - x[0]) : -1, (int)want};
  }
  __syncthreads();
  if (comes_last(a.ticket)) {
    if (there) a.row_len_out[me] = (int)now;
    if (me == 0) {
      a.new_off[n_rows] = (int32_t)all[1];
      if (a.page_off) a.page_off[n_rows] = (int32_t)sums[0];
      if (a.refused) a.refused[0] = (int32_t)sums[1];
      a.free_count_out[0] = (int32_t)(count - sums[2]);
    }
  }
  const int i = (threadIdx.x >> 6) / per_row, r = row0 + i;
  if (r < n_rows) {
    const Mine m = s_row[i];
    write_row(a, r, m.held, m.now, m.top, m.t0, m.n, m.p0, threadIdx.x % (64 * per_row), 64 * per_row);
  }
}

__global__ void __launch_bounds__(ROW_THREADS) k_kv_release_one(TableArgs a, int per_row) {
  __shared__ int s_at[ONE_WAVES], s_n[ONE_WAVES];
  const int width = a.rows.max_row_pages, n_rows = a.rows.n_rows, here = ONE_WAVES / per_row, row0 = blockIdx.x * here;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  const int me = threadIdx.x;
  const bool there = me < n_rows;
  int64_t gone[1] = {0}, all[1];
  int kept = 0;
  if (there) {
    const int len = max(a.row_len[me], 0);
    if (a.ended[me] != 0) gone[0] = min(pages_of(len), (int64_t)width);
    else kept = len;
  }
  const int n_mine = (int)gone[0];
  block_scan(gone, all);
  if (there && me >= row0 && me < row0 + here) {
    s_at[me - row0] = (int)(count + gone[0]);
    s_n[me - row0] = n_mine;
  }
  __syncthreads();
  if (comes_last(a.ticket)) {
    if (there) a.row_len_out[me] = kept;
    if (me == 0) a.free_count_out[0] = (int32_t)min(count + all[0], (int64_t)a.rows.n_pages);
  }
  const int i = (threadIdx.x >> 6) / per_row, r = row0 + i;
  if (r >= n_rows) return;
  const int32_t* const line = a.rows.table + (size_t)r * width;
  const int at = s_at[i], n = s_n[i];
  for (int j = threadIdx.x % (64 * per_row); j < n; j += 64 * per_row)
    if (at + j < a.rows.n_pages) a.rows.free_pages[at + j] = line[j];
}

int check_rows(const dag_kv_rows_t* rows, const void* ws, size_t ws_bytes) {
  if (!rows) return DAG_ERR_NULL;
  if (rows->n_rows < 0 || rows->max_row_pages < 0 || rows->n_pages < 0 || rows->n_pages > INT32_MAX / PAGE ||
      rows->max_row_pages > INT32_MAX / PAGE)
    return DAG_ERR_BAD_LEN;
  if (rows->page_size != PAGE) return DAG_ERR_UNSUPPORTED;
  if (rows->n_rows == 0) return DAG_OK;
  if ((rows->max_row_pages > 0 && !rows->table) || (rows->n_pages > 0 && !rows->free_pages)) return DAG_ERR_NULL;
  if (!ws || ws_bytes < dag_kv_tables_workspace_bytes(rows->n_rows)) return DAG_ERR_WORKSPACE;
  if ((uintptr_t)ws & 3) return DAG_ERR_ALIGN;
  return DAG_OK;
}

void place(TableArgs& a, const dag_kv_rows_t* rows, void* ws) {
  a.rows = *rows;
  a.ticket = (uint32_t*)ws;
  a.first = (int32_t*)ws + 1;
  a.held = a.first + rows->n_rows;
}
// Waves to a row of so many tokens and pages on average: four turns of a wave where there is no more than that to do, and no more workgroups than
// the chip holds at once (each works out all sums).
int waves_per_row(int64_t work, int n_rows) {
  const int64_t each = work / n_rows;
  const int most = n_rows <= 256 ? ONE_WAVES : 4;
  const int want = each <= 256 ? 1 : each <= 1024 ? 4 : ONE_WAVES;
  return want < most ? want : most;
}

}  // namespace

extern "C" size_t dag_kv_tables_workspace_bytes(int32_t n_rows) { return n_rows < 0 ? 0 : (size_t)n_rows * 8 + 256; }

extern "C" int dag_kv_release(const dag_kv_rows_t* rows, const int32_t* ended, const int32_t* row_len, int32_t* row_len_out,
                              const int32_t* free_count, int32_t* free_count_out, void* ws, size_t ws_bytes, void* stream_) {
  const int rc = check_rows(rows, ws, ws_bytes);
  if (rc != DAG_OK) return rc;
  if (!free_count || !free_count_out) return DAG_ERR_NULL;
  if (rows->n_rows > 0 && (!ended || !row_len || !row_len_out)) return DAG_ERR_NULL;
  TableArgs a = {};
  place(a, rows, ws);
  a.ended = ended;
  a.row_len = row_len;
  a.row_len_out = row_len_out;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  hipStream_t stream = (hipStream_t)stream_;
  if (rows->n_rows > 0 && rows->n_rows <= ONE_ROWS) {
    const int per_row = waves_per_row((int64_t)rows->n_rows * rows->max_row_pages / 2, rows->n_rows);  // (most rows do not end)
    hipLaunchKernelGGL(k_kv_release_one, dim3((unsigned)dag_ceil_div(rows->n_rows, ONE_WAVES / per_row)), dim3(ROW_THREADS), 0, stream, a, per_row);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  hipLaunchKernelGGL(k_kv_release_rows, dim3(1), dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (rows->n_rows > 0) {
    hipLaunchKernelGGL(k_kv_release_pages, dim3((unsigned)rows->n_rows), dim3(LIST_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}

extern "C" int dag_kv_tables(const dag_kv_rows_t* rows, const int32_t* new_len, const int32_t* row_len, int32_t* row_len_out,
                             const int32_t* free_count, int32_t* free_count_out, int32_t* new_off, int32_t* slots, int64_t max_new,
                             const int32_t* pos0, int32_t* pos, int32_t* page_off, int32_t* pages, int64_t max_pages, int32_t* refused, void* ws,
                             size_t ws_bytes, void* stream_) {
  const int rc = check_rows(rows, ws, ws_bytes);
  if (rc != DAG_OK) return rc;
  if (max_new < 0 || max_new > INT32_MAX || max_pages < 0 || max_pages > INT32_MAX) return DAG_ERR_BAD_LEN;
  if (!free_count || !free_count_out || !new_off || (max_new > 0 && !slots) || (pages && !page_off)) return DAG_ERR_NULL;
  if (rows->n_rows > 0 && (!new_len || !row_len || !row_len_out)) return DAG_ERR_NULL;
  TableArgs a = {};
  place(a, rows, ws);
  a.new_len = new_len;
  a.row_len = row_len;
  a.row_len_out = row_len_out;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  a.new_off = new_off;
  a.slots = slots;
  a.pos0 = pos0;
  a.pos = pos;
  a.page_off = page_off;
  a.pages = pages;
  a.refused = refused;
  a.max_new = max_new;
  a.max_pages = max_pages;
  hipStream_t stream = (hipStream_t)stream_;
  if (rows->n_rows > 0 && rows->n_rows <= ONE_ROWS) {
    const int64_t lines = (int64_t)rows->n_rows * rows->max_row_pages, listed = !pages ? 0 : lines < max_pages ? lines : max_pages;
    const int per_row = waves_per_row(max_new + listed, rows->n_rows);
    hipLaunchKernelGGL(k_kv_tables_one, dim3((unsigned)dag_ceil_div(rows->n_rows, ONE_WAVES / per_row)), dim3(ROW_THREADS), 0, stream, a, per_row);
    DAG_LAUNCH_CHECK();
    return DAG_OK;
  }
  hipLaunchKernelGGL(k_kv_table_rows, dim3(1), dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (rows->n_rows > 0) {
    hipLaunchKernelGGL(k_kv_table_lists, dim3((unsigned)rows->n_rows), dim3(LIST_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}
