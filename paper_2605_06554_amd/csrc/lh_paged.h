// lh_paged.h -- shape facts and launchers of the paged calls (serving).
#pragma once

#include "lh_common.h"

namespace lh {

// Inclusive sum over the workgroup's threads, in thread order, plus `carry`; `part` holds a word per
// wave. Every thread calls it.
template <int NT>
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t carry, int64_t* part) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  if (lane == 63) part[w] = x;
  __syncthreads();
  for (int i = 0; i < w; ++i) carry += part[i];
  __syncthreads();
  return x + carry;
}

}  // namespace lh

// A step's bounds, checked once per call on the host (include/lighthouse.h: lh_paged).
struct LhPaged {
  int64_t T, pages;
  int32_t R, max_blocks, page, shift;  // page = 1 << shift
  int32_t Hq, Hkv, D, G;               // G = Hq / Hkv
  int32_t dtype;
  float scale;
};

constexpr int32_t kPagedMaxRequests = 4096;

hipError_t lh_launch_page_plan(const LhPaged& s, const int32_t* cached, const int32_t* fresh,
                               const int32_t* free_pages, const int32_t* n_free, int32_t* table, int32_t* cu_q,
                               int32_t* kv_len, int32_t* slots, int32_t* pos, int32_t* balance, int32_t* n_taken,
                               hipStream_t st);
hipError_t lh_launch_page_write(const LhPaged& s, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                const int32_t* slots, void* kpages, void* vpages, hipStream_t st);
size_t lh_sdpa_paged_ws_bytes(const LhPaged& s);
hipError_t lh_launch_sdpa_paged(const LhPaged& s, const void* q, int64_t q_stride, const void* kpages,
                                const void* vpages, const int32_t* table, const int32_t* cu_q,
                                const int32_t* kv_len, void* o, float* lse, void* ws, hipStream_t st);
