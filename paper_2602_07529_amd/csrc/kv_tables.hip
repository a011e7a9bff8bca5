// Pages, slots and positions of rows (branches, nodes) that grow, worked out on the GPU: dag_kv_release, dag_kv_tables.
//
// A row r with n_r tokens holds ceil(n_r / 16) pages of its line of the table; free pages lie on a stack.  New tokens w_r need
// need_r = ceil((n_r + w_r) / 16) - ceil(n_r / 16) pages; with S_r = sum of need over the rows in front, row r takes the pages
// S_r .. S_r + need_r - 1 from the top of the stack, if that many are there.  Everything else follows from the prefix sums of need, w and the
// pages held, so a call is a scan by one workgroup (rows) and a launch that writes lists (tokens, pages), whatever order its
// workgroups run in.
#include "common.h"

namespace {

constexpr int PAGE = DAG_PAGE_SIZE;
constexpr int ROW_THREADS = 1024, LIST_THREADS = 256;

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

__global__ void __launch_bounds__(ROW_THREADS) k_kv_release_rows(TableArgs a) {
  const int width = a.rows.max_row_pages;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  int64_t front = 0;
  for (int base = 0; base < a.rows.n_rows; base += blockDim.x) {
    const int r = base + threadIdx.x;
    int64_t gone[1] = {0}, all[1];
    int len = 0;
    bool end = false;
    if (r < a.rows.n_rows) {
      len = max(a.row_len[r], 0);
      end = a.ended[r] != 0;
      if (end) gone[0] = min(pages_of(len), (int64_t)width);
    }
    const int n = (int)gone[0];
    block_scan(gone, all);
    if (r < a.rows.n_rows) {
      a.first[r] = (int32_t)(count + front + gone[0]);
      a.held[r] = n;
      a.row_len_out[r] = end ? 0 : len;
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
  const int width = a.rows.max_row_pages;
  const int64_t count = min(max(a.free_count[0], 0), a.rows.n_pages);
  int64_t front_need = 0, front_new = 0, front_pages = 0, taken = 0, refused = 0;
  for (int base = 0; base < a.rows.n_rows; base += blockDim.x) {
    const int r = base + threadIdx.x;
    const bool there = r < a.rows.n_rows;
    int64_t len = 0, want = 0, need = 0;
    bool fits = true;
    if (there) {
      len = max(a.row_len[r], 0);
      want = max(a.new_len[r], 0);
      fits = len + want <= (int64_t)width * PAGE;
      if (fits) need = pages_of(len + want) - pages_of(len);
    }
    int64_t x[2] = {need, want}, all[2];
    block_scan(x, all);
    const int64_t start = front_need + x[0];
    const bool ok = fits && (need == 0 || start + need <= count);
    const int64_t now = len + (ok ? want : 0), listed = there ? min(pages_of(now), (int64_t)width) : 0;
    int64_t y[3] = {listed, there && !ok && want > 0 ? 1 : 0, ok ? need : 0}, sums[3];
    block_scan(y, sums);
    if (there) {
      a.row_len_out[r] = (int32_t)now;
      a.new_off[r] = (int32_t)(front_new + x[1]);
      if (a.page_off) a.page_off[r] = (int32_t)(front_pages + y[0]);
      a.first[r] = ok ? (int32_t)(count - 1 - start) : -1;
      if (ok && need == 0) a.first[r] = 0;
      a.held[r] = (int32_t)len;
    }
    front_need += all[0];
    front_new += all[1];
    front_pages += sums[0];
    refused += sums[1];
    taken += sums[2];
  }
  if (threadIdx.x == 0) {
    a.new_off[a.rows.n_rows] = (int32_t)front_new;
    if (a.page_off) a.page_off[a.rows.n_rows] = (int32_t)front_pages;
    if (a.refused) a.refused[0] = (int32_t)refused;
    a.free_count_out[0] = (int32_t)(count - taken);
  }
}

__global__ void __launch_bounds__(LIST_THREADS) k_kv_table_lists(TableArgs a) {
  const int r = blockIdx.x, width = a.rows.max_row_pages, step = LIST_THREADS * gridDim.y, tid = blockIdx.y * LIST_THREADS + threadIdx.x;
  const int len = a.held[r], top = a.first[r], now = a.row_len_out[r];
  const int64_t t0 = a.new_off[r];
  const int n = a.new_off[r + 1] - (int)t0, has = (int)pages_of(len), pages = (int)min(pages_of(now), (int64_t)width);
  int32_t* const line = a.rows.table + (size_t)r * width;
  auto page = [&](int p) { return p < has ? line[p] : a.rows.free_pages[max(top - (p - has), 0)]; };
  for (int j = tid; j < n; j += step) {
    if (t0 + j >= a.max_new) break;
    const int at = len + j;
    a.slots[t0 + j] = top < 0 ? -1 : page(at / PAGE) * PAGE + at % PAGE;
    if (a.pos) a.pos[t0 + j] = (a.pos0 ? a.pos0[r] : 0) + at;
  }
  const int64_t p0 = a.page_off ? a.page_off[r] : 0;
  for (int p = (a.pages ? 0 : has) + tid; p < pages; p += step) {
    const int id = page(p);
    if (p >= has) line[p] = id;
    if (a.pages && p0 + p < a.max_pages) a.pages[p0 + p] = id;
  }
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

}  // namespace

extern "C" size_t dag_kv_tables_workspace_bytes(int32_t n_rows) { return n_rows < 0 ? 0 : (size_t)n_rows * 8 + 256; }

extern "C" int dag_kv_release(const dag_kv_rows_t* rows, const int32_t* ended, const int32_t* row_len, int32_t* row_len_out,
                              const int32_t* free_count, int32_t* free_count_out, void* ws, size_t ws_bytes, void* stream_) {
  const int rc = check_rows(rows, ws, ws_bytes);
  if (rc != DAG_OK) return rc;
  if (!free_count || !free_count_out) return DAG_ERR_NULL;
  if (rows->n_rows > 0 && (!ended || !row_len || !row_len_out)) return DAG_ERR_NULL;
  TableArgs a = {};
  a.rows = *rows;
  a.ended = ended;
  a.row_len = row_len;
  a.row_len_out = row_len_out;
  a.free_count = free_count;
  a.free_count_out = free_count_out;
  a.first = (int32_t*)ws;
  a.held = a.first + rows->n_rows;
  hipStream_t stream = (hipStream_t)stream_;
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
  a.rows = *rows;
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
  a.first = (int32_t*)ws;
  a.held = a.first + rows->n_rows;
  hipStream_t stream = (hipStream_t)stream_;
  hipLaunchKernelGGL(k_kv_table_rows, dim3(1), dim3(ROW_THREADS), 0, stream, a);
  DAG_LAUNCH_CHECK();
  if (rows->n_rows > 0) {
    hipLaunchKernelGGL(k_kv_table_lists, dim3((unsigned)rows->n_rows), dim3(LIST_THREADS), 0, stream, a);
    DAG_LAUNCH_CHECK();
  }
  return DAG_OK;
}
