// k_paged_sdpa.hip -- attention of a step's new tokens over a paged K/V cache (include/lighthouse.h, serving):
// the choice of the kernel, its workspace, and the joining of the tiles that the cut of the work divides.
#include <float.h>
#include <math.h>

#include "lh_mfma.h"
#include "lh_paged_sdpa.h"

namespace lh {

// Joins the parts of the tiles that were cut: 16 lanes to a row and group of parts, which reads its parts FEW at a time,
// all in flight at once, with a running maximum; S groups share the parts of a row and are joined in LDS, in order.
// Small tiles (of the rows kernel) take S = 4 and a workgroup to 4 rows, large ones S = 1 and 16 rows. Bound by the
// latency of two dependent loads (which tile, its parts) and the launch, and by HBM where tiles are large.
template <bool SMALL>
struct JoinCfg {
  static constexpr int S = SMALL ? 4 : 1, FEW = SMALL ? 4 : 8, ROWS = 16 / S;
};

template <typename T, int D, bool SMALL>
__global__ void __launch_bounds__(256) paged_join(const PagedArgs a, int TM) {
  using C = JoinCfg<SMALL>;
  constexpr int E = D / 16;  // columns a lane
  __shared__ __align__(16) float acc_s[SMALL ? 16 : 1][D];
  __shared__ float m_s[16], l_s[16];
  const int lw = blockIdx.x, y0 = blockIdx.y * C::ROWS;
  const PartDesc d = a.desc[lw];
  if (y0 >= d.rows) return;
  const int count = uni(d.last) - lw + 1, grp = threadIdx.x >> 4, c = (threadIdx.x & 15) * E;
  const int row = y0 + grp / C::S, sub = grp % C::S;
  const bool real = row < d.rows;
  float acc[E], l = 0.0f, m = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  // A part with the maximum -inf has no weights: its sum is 0, or NaN where all its logits are.
  auto weight = [&](float x, float top) __attribute__((always_inline)) { return x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x - top); };
  if (real) {
    for (int p0 = sub; p0 < count; p0 += C::S * C::FEW) {
      float2 st[C::FEW];
      float4 x[C::FEW][E / 4];
#pragma unroll
      for (int i = 0; i < C::FEW; ++i) {
        const int p = p0 + C::S * i;
        st[i] = make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int z = 0; z < E / 4; ++z) x[i][z] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p < count) {
          const int64_t at = (2 * (int64_t)(lw + p) + (p == 0 ? 1 : 0)) * TM + row;
          st[i] = a.stat[at];
#pragma unroll
          for (int z = 0; z < E / 4; ++z) x[i][z] = *reinterpret_cast<const float4*>(a.part + at * D + c + 4 * z);
        }
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < C::FEW; ++i) top = fmaxf(top, st[i].x);
      const float al = weight(m, top);
      m = top, l *= al;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= al;
#pragma unroll
      for (int i = 0; i < C::FEW; ++i) {
        const float wt = weight(st[i].x, top);
        l += wt * st[i].y;
#pragma unroll
        for (int z = 0; z < E / 4; ++z) {
          acc[4 * z] += wt * x[i][z].x, acc[4 * z + 1] += wt * x[i][z].y;
          acc[4 * z + 2] += wt * x[i][z].z, acc[4 * z + 3] += wt * x[i][z].w;
        }
      }
    }
  }
  if constexpr (SMALL) {
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(&acc_s[grp][c + e]) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    if (c == 0) m_s[grp] = m, l_s[grp] = l;
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int z = 1; z < 4; ++z) m = fmaxf(m, m_s[grp + z]);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const float wt = weight(m_s[grp + z], m);
      l += wt * l_s[grp + z];
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += wt * acc_s[grp + z][c + e];
    }
  }
  if (!real) return;
  const int gr = d.row0 + row, tok = gr / a.G;
  const int64_t at = (int64_t)(d.first + tok) * a.Hq + d.head * a.G + (gr - tok * a.G);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] *= inv;
  T* const o = (T*)a.o + at * D + c;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(o + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
  } else {
    uint32_t y[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) y[e] = (uint32_t)f2bf(acc[2 * e]) | ((uint32_t)f2bf(acc[2 * e + 1]) << 16);
    if constexpr (E == 8) *reinterpret_cast<uint4*>(o) = make_uint4(y[0], y[1], y[2], y[3]);
    else *reinterpret_cast<uint2*>(o) = make_uint2(y[0], y[1]);
  }
  if (a.lse && c == 0) a.lse[at] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// The variant that serves a step, by its rows a request (an average: of a step, the host knows only its bounds). Eight
// requests of 16,000 cached tokens, 32 heads on 8, us, by rows a request: rows kernel (32 a tile), tiles of 128, 256
// and 384: 16 rows 98 (16 a tile), 106, 119, 127; 48 128, 112, 119, 125; 96 291, 125, 126, 132; 128 201, 134, 130, 137;
// 256 349, 194, 176, 182; 384 537, 329, 291, 233; 512 664, 346, 306, 348; 1024 1293, 628, 577, 628; one request of
// 8192 rows 672, 358, 321, 318. Between 256 and 384 the rows that the last tile leaves idle decide. (D = 128; D = 64 takes the
// same lines. A step of unequal requests goes by its average as well: 127 single tokens and a chunk of 512 at 16,000 cached
// have 19 rows a request and take the rows kernel, 1837 us, where a call for each of the two kinds takes 1237 and 173.)
static PagedVariant variant_of(const LhPaged& s, int64_t rows) {
  if (s.dtype != LH_BF16 || rows <= 32) return lh_paged_rows_variant(s, rows);
  if (rows <= 112) return lh_paged_tile_variant(s, 4);
  const int64_t in8 = (rows + 255) / 256 * 256, in12 = (rows + 383) / 384 * 384;
  return lh_paged_tile_variant(s, rows > 256 && in12 * 32 <= in8 * 33 ? 12 : 8);
}
static PagedVariant variant_of(const LhPaged& s) { return variant_of(s, s.T * s.G / s.R); }

template <typename T, int D, bool SMALL>
static void launch_join(const LhPaged& s, const PagedArgs& a, int TM, hipStream_t st) {
  const int64_t rows = s.T * s.G < TM ? s.T * s.G : TM, per = JoinCfg<SMALL>::ROWS;
  hipLaunchKernelGGL((paged_join<T, D, SMALL>), dim3((unsigned)a.W, (unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a, TM);
}
template <typename T, int D>
static void launch_join(const LhPaged& s, const PagedArgs& a, int TM, hipStream_t st) {
  if (sizeof(T) == 4 || TM <= 32) launch_join<T, D, true>(s, a, TM, st);
  else if constexpr (sizeof(T) == 2) launch_join<T, D, false>(s, a, TM, st);
}

}  // namespace lh

using namespace lh;

// The most that a step of up to R requests and T rows needs. (Steps of fewer requests or rows may take a variant of larger
// parts, and one workspace serves them all.) The variants by the fewest rows a request that select them.
size_t lh_sdpa_paged_ws_bytes(const LhPaged& s) {
  size_t most = 0;
  for (const int64_t rows : {1, 17, 33, 113, 257}) {
    if (rows > 1 && rows > s.T * s.G) break;
    const PagedVariant v = variant_of(s, rows);
    const size_t bytes = paged_ws(v.W, v.TM, s.D).total;
    most = bytes > most ? bytes : most;
  }
  return most;
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
