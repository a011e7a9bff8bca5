// What the kernels over tables of rows and pages share.
#pragma once
#include "common.h"

namespace {

constexpr int PAGE = DAG_PAGE_SIZE;
constexpr int ROW_THREADS = 1024;

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

}  // namespace
