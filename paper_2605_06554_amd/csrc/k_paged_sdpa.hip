// k_paged_sdpa.hip -- attention of a step's new tokens over a paged K/V cache (include/lighthouse.h,
// serving).
#include <math.h>

#include "lh_paged.h"

namespace lh {

struct PagedArgs {
  const void *q, *kp, *vp;
  const int32_t *table, *cu_q, *kv_len;
  void* o;
  float* lse;
  int64_t q_stride, T, pages;
  int32_t R, max_blocks, shift, Hq, Hkv, G;
  float scale;
};

__device__ __forceinline__ int32_t clip(int64_t x, int64_t hi) { return (int32_t)(x < 0 ? 0 : x > hi ? hi : x); }

// A wave per (row, query head): 8 keys at a time, 8 lanes a key.
template <typename T, int D>
__global__ void __launch_bounds__(64) paged_plain(const PagedArgs a) {
  constexpr int E = D / 8;
  const int lane = threadIdx.x, sub = lane & 7, key = lane >> 3;
  const int64_t t = blockIdx.x / a.Hq;
  const int h = blockIdx.x % a.Hq, g = h / a.G;
  // the request of row t: the last one that begins at or before it and ends behind it
  int r = -1;
  for (int r0 = 0; r0 < a.R && r < 0; r0 += 64) {
    const int x = r0 + lane;
    const bool in = x < a.R && clip(a.cu_q[x], a.T) <= t && t < clip(a.cu_q[x + 1], a.T);
    const uint64_t m = __ballot(in);
    if (m) r = r0 + __ffsll((unsigned long long)m) - 1;
  }
  if (r < 0) return;
  const int32_t first = clip(a.cu_q[r], a.T), n = clip(a.cu_q[r + 1], a.T) - first;
  const int32_t len = clip(a.kv_len[r], (int64_t)a.max_blocks << a.shift);
  const int32_t keys = len - n + (int32_t)(t - first) + 1;  // keys of this row
  const T* q = (const T*)a.q + t * a.q_stride + (int64_t)h * D + sub * E;
  float qr[E], acc[E], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) qr[e] = Elem<T>::load(q + e) * a.scale, acc[e] = 0.0f;
  for (int j0 = 0; j0 < keys; j0 += 8) {
    const int j = j0 + key;
    const int jc = j < keys ? j : keys - 1;
    const int32_t id = clip(a.table[(int64_t)r * a.max_blocks + (jc >> a.shift)], a.pages - 1);
    const int64_t at = (((((int64_t)id * a.Hkv + g) << a.shift) + (jc & ((1 << a.shift) - 1))) * D) + sub * E;
    const T *k = (const T*)a.kp + at, *v = (const T*)a.vp + at;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += qr[e] * Elem<T>::load(k + e);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) s += __shfl_xor(s, d, 64);
    if (j < keys) {
      const float mn = fmaxf(m, s), al = m == -INFINITY ? 0.0f : expf(m - mn), p = s == -INFINITY ? 0.0f : expf(s - mn);
      m = mn, l = l * al + p;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] * al + p * Elem<T>::load(v + e);
    }
  }
  // the 8 key lanes' statistics and sums
  float mt = m;
#pragma unroll
  for (int d = 8; d < 64; d <<= 1) mt = fmaxf(mt, __shfl_xor(mt, d, 64));
  const float w = m == -INFINITY ? 0.0f : expf(m - mt);
  l *= w;
#pragma unroll
  for (int d = 8; d < 64; d <<= 1) l += __shfl_xor(l, d, 64);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    acc[e] *= w;
#pragma unroll
    for (int d = 8; d < 64; d <<= 1) acc[e] += __shfl_xor(acc[e], d, 64);
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  if (key == 0) {
    T* o = (T*)a.o + (t * a.Hq + h) * D + sub * E;
#pragma unroll
    for (int e = 0; e < E; ++e) Elem<T>::store(o + e, keys > 0 ? acc[e] * (l == l ? inv : l) : 0.0f);
    if (sub == 0 && a.lse) a.lse[t * a.Hq + h] = mt + logf(l);
  }
}

}  // namespace lh

using namespace lh;

size_t lh_sdpa_paged_ws_bytes(const LhPaged& s) { return 0; }

hipError_t lh_launch_sdpa_paged(const LhPaged& s, const void* q, int64_t q_stride, const void* kpages,
                                const void* vpages, const int32_t* table, const int32_t* cu_q,
                                const int32_t* kv_len, void* o, float* lse, void* ws, hipStream_t st) {
  const PagedArgs a{q, kpages, vpages, table, cu_q, kv_len, o, lse, q_stride, s.T, s.pages,
                    s.R, s.max_blocks, s.shift, s.Hq, s.Hkv, s.G, s.scale};
  const dim3 grid((unsigned)(s.T * s.Hq));
  if (s.dtype == LH_BF16) {
    if (s.D == 128) hipLaunchKernelGGL((paged_plain<bf16_t, 128>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((paged_plain<bf16_t, 64>), grid, dim3(64), 0, st, a);
  } else {
    if (s.D == 128) hipLaunchKernelGGL((paged_plain<float, 128>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((paged_plain<float, 64>), grid, dim3(64), 0, st, a);
  }
  return hipGetLastError();
}
