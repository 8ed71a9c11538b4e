// k_paged_sdpa.hip -- attention of a step's new tokens over a paged K/V cache (include/lighthouse.h, serving):
// the choice of the kernel, its workspace, and the joining of the tiles that the cut of the work divides.
#include <float.h>
#include <math.h>

#include "lh_mfma.h"
#include "lh_paged_sdpa.h"

namespace lh {

// Joins the parts of the tiles that were cut: a workgroup per tile and four rows; a wave per row where the
// parts are few, else the four waves share a row's parts.
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_join(const PagedArgs a, int TM) {
  constexpr int E = D / 64;
  __shared__ float acc_s[4][D], l_s[4];
  const int lw = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const PartDesc d = a.desc[lw];
  const int y0 = blockIdx.y * 4;
  if (y0 >= d.rows) return;
  const int count = d.last - lw + 1;
  const bool share = count > 8;
  for (int y = share ? 0 : w; y < (share ? 4 : w + 1); ++y) {
    const int row = y0 + y;
    if (row >= d.rows) break;
    const int p0 = share ? w : 0, dp = share ? 4 : 1;
    auto slot = [&](int p) __attribute__((always_inline)) { return (p == 0 ? 2 * (int64_t)lw + 1 : 2 * (int64_t)(lw + p)) * TM + row; };
    float mt = -INFINITY;
    for (int p = lane; p < count; p += 64) mt = fmaxf(mt, a.stat[slot(p)].x);
#pragma unroll
    for (int z = 32; z > 0; z >>= 1) mt = fmaxf(mt, __shfl_xor(mt, z, 64));
    float acc[E], l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll 8
    for (int p = p0; p < count; p += dp) {
      const int64_t at = slot(p);
      const float2 st = a.stat[at];
      const float wt = st.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st.x - mt);
      l += st.x == -INFINITY ? st.y : wt * st.y;
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = a.part[at * D + lane * E + e];
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += wt * x[e];
    }
    if (share) {
#pragma unroll
      for (int e = 0; e < E; ++e) acc_s[w][lane * E + e] = acc[e];
      if (lane == 0) l_s[w] = l;
      __syncthreads();
      l = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        l += l_s[z];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += acc_s[z][lane * E + e];
      }
      __syncthreads();
      if (w != 0) continue;
    }
    const int gr = d.row0 + row, tok = gr / a.G;
    const int64_t at = (int64_t)(d.first + tok) * a.Hq + d.head * a.G + (gr - tok * a.G);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) Elem<T>::store((T*)a.o + at * D + lane * E + e, acc[e] * inv);
    if (a.lse && lane == 0) a.lse[at] = l == 0.0f ? -INFINITY : (mt + __log2f(l)) * kLn2;
  }
}


// The variant that serves a step, by its rows a request (an average: of a step, the host knows only its bounds).
static PagedVariant variant_of(const LhPaged& s) {
  const int64_t rows = s.T * s.G / s.R;
  if (s.dtype == LH_BF16 && rows > 64) return lh_paged_tile_variant(s, rows > 192 ? 12 : 4);
  return lh_paged_rows_variant(s, rows > 16 ? 32 : 16);
}

template <typename T, int D>
static void launch_join(const LhPaged& s, const PagedArgs& a, int TM, hipStream_t st) {
  const int64_t rows = s.T * s.G < TM ? s.T * s.G : TM;
  hipLaunchKernelGGL((paged_join<T, D>), dim3((unsigned)a.W, (unsigned)((rows + 3) / 4)), dim3(256), 0, st, a, TM);
}

}  // namespace lh

using namespace lh;

size_t lh_sdpa_paged_ws_bytes(const LhPaged& s) {
  const PagedVariant v = variant_of(s);
  return paged_ws(v.W, v.TM, s.D).total;
}

hipError_t lh_launch_sdpa_paged(const LhPaged& s, const void* q, int64_t q_stride, const void* kpages,
                                const void* vpages, const int32_t* table, const int32_t* cu_q,
                                const int32_t* kv_len, void* o, float* lse, void* ws, hipStream_t st) {
  const PagedVariant v = variant_of(s);
  const PagedWs w = paged_ws(v.W, v.TM, s.D);
  PagedArgs a{};
  a.q = q, a.kp = kpages, a.vp = vpages, a.table = table, a.cu_q = cu_q, a.kv_len = kv_len, a.o = o, a.lse = lse;
  a.q_stride = q_stride, a.T = s.T, a.pages = s.pages;
  a.R = s.R, a.max_blocks = s.max_blocks, a.shift = s.shift, a.Hq = s.Hq, a.Hkv = s.Hkv, a.G = s.G;
  a.sl2 = fmaxf(s.scale * kLog2e, FLT_MIN);  // (0 times a masked logit would be NaN)
  a.desc = (PartDesc*)ws;
  a.stat = (float2*)((char*)ws + w.stat);
  a.part = (float*)((char*)ws + w.part);
  a.W = (int32_t)v.W;
  v.launch(a, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (s.dtype == LH_BF16) {
    if (s.D == 128) launch_join<bf16_t, 128>(s, a, v.TM, st);
    else launch_join<bf16_t, 64>(s, a, v.TM, st);
  } else {
    if (s.D == 128) launch_join<float, 128>(s, a, v.TM, st);
    else launch_join<float, 64>(s, a, v.TM, st);
  }
  return hipGetLastError();
}
