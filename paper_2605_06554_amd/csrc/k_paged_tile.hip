// k_paged_tile.hip -- attention over a paged cache, bf16, for requests of many rows (chunks of prompts, whole
// prompts; rows, cut and parts: lh_paged_sdpa.h). Tiles of 32 NW rows, a wave to 32 of them.
//
// The arithmetic and the LDS tiles are those of the layer's forward kernel (k_sdpa_mfma.hip: layouts,
// swizzle, two-slot ring filled by global_load_lds): S^T = K Q^T, a lane owning one row, 64 keys a tile; P is
// rounded to bf16 for its product, everything else of the softmax is fp32. (The roundings are independent and no larger than
// that of o itself, so the 2-norm error is at most sqrt(2) of the output's where V has no common sign: 2.0e-3 to 2.4e-3, and
// 1.7e-3 with P as two bf16 values, as in lh_paged_rows.h. Here the matrix unit has no time to spare for the second
// product: the chunk below takes 1150 us with it and 858 without, two prompts of 7000 to 8192 tokens 645 and 500.)
// What differs:
//   - A tile of 64 keys is filled page by page: the 4 or 8 rows that one load instruction copies lie in one
//     page (pages hold 16 tokens or more), so their address is one scalar base, read from the table a tile
//     ahead, and a fixed offset a lane. The tile with the request's last key reads that key again for the
//     rows behind it, which hold anything.
//   - The keys of a tile are a part's share of them, and the rows of a part of a tile go to the workspace.
//   - Rows whose mask leaves nothing, and values of V that are not finite: what is masked does not reach a row.
// 12 waves have 168 registers each: at D = 128 they spill 5, two of which are read again in every masked tile (1 without MIX, read
// once); the others spill none.
//
// Bound by the matrix and vector units side by side, at a clock that their power sets (1.7 to 2.0 GHz): a chunk of 2048
// tokens at 96,000 cached, 8 heads of 128, 256 rows a tile: 835 to 870 us, 940 to 980 TFLOP/s (a large library product
// reaches 1177), matrix units busy 44% of the cycles, 1.1 GB fetched (0.41 GB without a second reading; L2 and the
// parts' common progress hold the rest). Tried on this loop and not kept: three and four slots of the ring (869 us
// became 884 and 890), logits of the next tile under the softmax of this one (836 became 901 to 920), six waves a
// workgroup and two of them a CU (829 became 1150).
#include <math.h>

#include "lh_paged_lds.h"
#include "lh_paged_rows.h"

namespace lh {

template <int D, int NW>
struct TileCfg {
  static constexpr int TM = 32 * NW, FK = 64;
  static constexpr int EU = NW == 4 ? 2 : NW / 4;          // waves a SIMD
  static constexpr int64_t W = 256 * (NW == 4 ? 2 : 1);    // two workgroups of 4 waves a CU (64 KB of LDS each), else one
  static constexpr int LPW = (FK * D / 512 + NW - 1) / NW;  // 1 KB load instructions a wave, for each of K and V
  static constexpr int RPB = 512 / D;                       // rows of one
};

// The ring as the memory of rows_tile.
template <int D, int NW>
struct TileLds {
  using M = TileLdsMap<D, NW>;
  static_assert(M::sound(), "a wave's words and another's part may be in use at the same time");
  static constexpr int PER = M::PER;
  static constexpr bool kOwnWords = M::kOwnWords;
  float* ring[M::ARRAYS];
  float (*stat)[16];
  __device__ __forceinline__ float* at(int i, int off) const { return (i == 0 ? ring[0] : i == 1 ? ring[1] : i == 2 ? ring[2] : ring[3]) + off; }
  __device__ __forceinline__ float* part(int w) const { return at(M::part_array(w), M::part_off(w)); }
  __device__ __forceinline__ float* words(int w) const { return at(M::words_array(w), M::words_off(w)); }
  __device__ __forceinline__ float* ms(int w) const { return stat[w]; }
  __device__ __forceinline__ float* ls(int w) const { return stat[NW + w]; }
};

// lane_offsets of a tile's rows, from three registers: the k-step and the column block change bits of a lane's
// offset that the swizzle leaves alone or flips, so they come in by an exclusive or. (All 16 held: 16 registers
// spilled, and a reload in the loop waits for the tile in flight.)
template <int D>
struct LaneBase {
  int row0, trl0, trh0;
  __device__ __forceinline__ explicit LaneBase(int lane) {
    const LaneOff<D> o = lane_offsets<D>(lane, 0);
    row0 = o.row[0], trl0 = o.trl[0], trh0 = o.trh[0];
  }
  __device__ __forceinline__ int row(int kk) const { return row0 ^ (kk << 5); }
  __device__ __forceinline__ int trl(int d) const { return trl0 ^ (d << 6); }
  __device__ __forceinline__ int trh(int d) const { return trh0 ^ (d << 6); }
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row0), "+v"(trl0), "+v"(trh0)); }  // nothing formed ahead
};

// MIX: tiles of 16 rows or fewer go through rows_tile. (Without, nothing is lost for it where there is one request: the
// loop takes 1% less.)
template <int D, int NW, bool MIX>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(TileCfg<D, NW>::EU, TileCfg<D, NW>::EU)))
paged_tile(const PagedArgs a) {
  using C = TileCfg<D, NW>;
  constexpr int TM = C::TM, FK = C::FK, RB = 2 * D, NT = 64 * NW, LPW = C::LPW;
  __shared__ __align__(16) bf16_t Ks0[FK * D], Ks1[FK * D], Vs0[FK * D], Vs1[FK * D];
  __shared__ int64_t scan[NW];
  __shared__ typename Walk<TM, 8, MIX ? 5 : 0>::Found found;
  __shared__ int32_t more;
  __shared__ float stat[2 * NW][16];
  const int tid = threadIdx.x, w = uni(tid >> 6);
  // The way along the part waits in LDS while a tile is worked on: in registers (the results of divisions live in
  // vector registers, uniform or not) it made the loop spill 22.
  __shared__ Walk<TM, 8, MIX ? 5 : 0> way;
  {
    Walk<TM, 8, MIX ? 5 : 0> wk;
    if (!wk.template begin<NT>(a, scan, &found)) return;
    if (tid == 0) way = wk;
  }
  for (;;) {
    __syncthreads();  // the way is known, and the ring is free: the last tile's waves are done
    // (formed in every tile: held across the tiles, what follows from the lane made the loop spill 16 registers)
    int lane = tid & 63;
    asm volatile("" : "+v"(lane));
    const int hh = lane >> 5, r32 = lane & 31;
    LaneBase<D> lo(lane);
    // this lane's row and bytes of the 1 KB blocks that it copies (a block too many repeats another's: same bytes)
    auto block_of = [&](int j) __attribute__((always_inline)) {
      const int b = j * NW + w;
      return b < FK / C::RPB ? b : b - FK / C::RPB;
    };
    const int rib = lane / (D / 8);
    int ch[LPW];
  #pragma unroll
    for (int j = 0; j < LPW; ++j) ch[j] = ((lane % (D / 8)) ^ swz<D>(block_of(j) * C::RPB + rib)) << 4;
    const int h = uni(way.h), row0 = uni(way.t) * TM, all_rows = uni(way.rq.rows), base = uni(way.rq.base), first = uni(way.rq.first);
    const int rows = all_rows - row0 < TM ? all_rows - row0 : TM;
    const int keys = uni(base + (row0 + rows - 1) / a.G + 1);  // that any row of the tile sees
    const int safe = uni(base + row0 / a.G + 1);               // that all of them see
    int t0, t1;
    way.blocks(keys > 0 ? (keys + FK - 1) / FK : 0, t0, t1);
    t0 = uni(t0), t1 = uni(t1);
    if (MIX && rows <= 16) {
      // Rows for one MFMA: the waves share the keys instead, as in the rows kernel (a wave alone with 64 keys at a
      // time takes 2 us for them, 16 GB/s a CU).
      RowsItem it;
      it.r = uni(way.r), it.h = h, it.row0 = row0, it.rows = rows, it.all_rows = all_rows, it.first = first;
      it.base = base, it.keys = keys, it.safe = safe;
      const int nb = keys > 0 ? (keys + 31) / 32 : 0;
      it.b0 = 2 * t0, it.b1 = 2 * t1 < nb ? 2 * t1 : nb;
      it.whole = way.whole(), it.slot = way.slot();
      rows_tile<bf16_t, D, 1, NW, true, TM>(a, it, TileLds<D, NW>{{(float*)Ks0, (float*)Ks1, (float*)Vs0, (float*)Vs1}, stat});
    } else {
      const int64_t ids = (int64_t)uni(way.r) * a.max_blocks;  // the request's row of the table
      const int last = (keys - 1) >> a.shift;  // the last page in use (of a tile with a key)

      // this lane's row, and what its wave's rows see
      const int row = row0 + 32 * w + r32, myrow = row < all_rows ? row : all_rows - 1, tok = myrow / a.G;
      const int pos = base + tok;
      const bool idle = 32 * w >= rows;  // no row of the wave is one
      const int wsafe = uni(base + (row0 + 32 * w) / a.G);  // position of the wave's first row
      const int wlast = idle ? -1 : uni(__shfl(pos, 31, 64));  // of its last one

      int32_t pg[LPW];  // pages of the next tile to be loaded
      auto next_pages = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
          const int b = (kt * FK + block_of(j) * C::RPB) >> a.shift;
          pg[j] = page_id(a.table, ids + (b < last ? b : last), a.pages);
        }
      };
      auto load_kv = [&](int slot, int kt) __attribute__((always_inline)) {
        bf16_t* const kt_ = slot ? Ks1 : Ks0;
        bf16_t* const vt_ = slot ? Vs1 : Vs0;
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
          int k0 = kt * FK + block_of(j) * C::RPB;  // rows behind the last key read it again
          k0 = k0 < keys ? k0 : keys - 1;
          const int most = keys - 1 - k0;
          const int64_t at = ((((int64_t)pg[j] * a.Hkv + h) << a.shift) + (k0 & ((1 << a.shift) - 1))) * RB;
          const int off = (rib < most ? rib : most) * RB + ch[j];
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((const char*)a.kp + at + off),
                                           (__attribute__((address_space(3))) void*)(kt_ + block_of(j) * 512), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((const char*)a.vp + at + off),
                                           (__attribute__((address_space(3))) void*)(vt_ + block_of(j) * 512), 16, 0, 0);
        }
        if (kt + 1 < t1) next_pages(kt + 1);
      };

      if (t0 < t1) {
        next_pages(t0);
        load_kv(0, t0);
      }
      bf16x8 qreg[D / 16];
      {
        const bf16_t* qr = (const bf16_t*)a.q + (int64_t)(first + tok) * a.q_stride + (int64_t)(h * a.G + myrow - tok * a.G) * D;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) qreg[kk] = *reinterpret_cast<const bf16x8*>(qr + 16 * kk + 8 * hh);
      }
      f32x16 oacc[D / 32];
#pragma unroll
      for (int d = 0; d < D / 32; ++d) oacc[d] = f32x16{};
      float m_run = -INFINITY, l_run = 0.0f;
      bool oddly = false;  // a value of V was taken out of a tile

      auto step = [&](auto slotc, int kt) __attribute__((always_inline)) {
        constexpr int SL = decltype(slotc)::value;
        bf16_t* const Kt = SL ? Ks1 : Ks0;
        bf16_t* const Vt = SL ? Vs1 : Vs0;
        sync_tiles<0>();  // tile kt landed in every wave; tile kt - 1 is done
        lo.fresh();
        const int k0 = kt * FK;
        // Values of V that are not finite may be of keys that some rows see and others do not, and 0 times them
        // is NaN: all waves look for them where a row of the tile is masked, and take them out.
        if (k0 + FK > safe) {
          bool mine = false;
          int i = tid;
          asm volatile("" : "+v"(i));  // (no address of it is formed ahead of the loop)
#pragma unroll 1
          for (; i < FK * D / 8; i += NT) {
            const u32x4 y = *reinterpret_cast<const u32x4*>(Vt + i * 8);
            const uint32_t x[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) mine |= (x[c] & 0x7f80u) == 0x7f80u || (x[c] & 0x7f800000u) == 0x7f800000u;
          }
          if (__syncthreads_or(mine)) {
            oddly = true;
            i = tid;
            asm volatile("" : "+v"(i));
#pragma unroll 1
            for (; i < FK * D; i += NT)
              if ((Vt[i] & 0x7f80u) == 0x7f80u) Vt[i] = 0;
            __syncthreads();
          }
        }
        if (kt + 1 < t1) load_kv(SL ^ 1, kt + 1);
        const bool skip = k0 > wlast;  // every key is behind the wave's rows
        f32x16 sacc[2];
        if (!skip) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) sacc[kb] = f32x16{};
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) sacc[kb] = mfma32(row8(Kt, kb * 32 * RB + lo.row(kk)), qreg[kk], sacc[kb]);
          if (k0 + FK - 1 > wsafe) {
            const int sees = pos - k0 - 4 * hh;  // (against constants: 32 keys a lane held across the loop were spilled)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (kb * 32 + 8 * (i >> 2) + (i & 3) > sees) sacc[kb][i] = -INFINITY;
          }
        }
        if (skip) return;
        float mloc = sacc[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mloc = fmaxf(mloc, sacc[kb][i]);
        mloc = fmaxf(mloc, __shfl_xor(mloc, 32, 64)) * a.sl2;
        if (mloc > m_run + kRescale) {  // new running maximum of the row: rescale what was accumulated
          const float alpha = __builtin_amdgcn_exp2f(m_run - mloc);
          l_run *= alpha;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[d][i] *= alpha;
          m_run = mloc;
        }
        const float mm = m_run == -INFINITY ? 0.0f : m_run;  // no key yet: all weights are 0
        float la = 0.0f, lb = 0.0f;
        auto soft = [&](int st) __attribute__((always_inline)) {
          float f[8];
#pragma unroll
          for (int y = 0; y < 8; ++y) f[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[st >> 1][8 * (st & 1) + y], a.sl2, -mm));
          la += (f[0] + f[1]) + (f[2] + f[3]);
          lb += (f[4] + f[5]) + (f[6] + f[7]);
          return cvt8(f);
        };
        bf16x8 pcur = soft(0);
        asm volatile("" ::"v"(la), "v"(lb));  // the first step's sums stay ahead of the interleaving
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          bf16x8 pnext = pcur;
          if (st + 1 < 4) pnext = soft(st + 1);
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
            oacc[d] = mfma32(tr8(Vt, 16 * st * RB + lo.trl(d), 16 * st * RB + lo.trh(d)), pcur, oacc[d]);
          if (st + 1 < 4) {
            // groups: DS reads (mask 0x100), MFMA (0x008), VALU (0x002), transcendental (0x400)
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              if (d + 1 < D / 32) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
              __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
              __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          pcur = pnext;
        }
        l_run += la + lb;
      };
      for (int kt = t0; kt < t1; kt += 2) {
        step(IC<0>{}, kt);
        if (kt + 1 < t1) step(IC<1>{}, kt + 1);
      }

      if (oddly) {
        // What was taken out is added to the rows that see its key: the masked tiles once more, with codes in V's
        // place (1 for +inf, 64 for -inf, 4096 for NaN). A product with the rows' view of the keys (1 or 0) counts
        // them, 16 keys at a time, so that the counts do not overlap.
        for (int kt = safe / FK > t0 ? safe / FK : t0; kt < t1; ++kt) {
          __syncthreads();
          next_pages(kt);
          load_kv(0, kt);
          sync_tiles<0>();
#pragma unroll 1
          for (int i = tid; i < FK * D; i += NT) {
            const uint32_t x = Vs0[i];
            Vs0[i] = (x & 0x7f80u) != 0x7f80u ? 0 : x & 0x7fu ? 0x4580u : x >> 15 ? 0x4280u : 0x3f80u;
          }
          __syncthreads();
#pragma unroll 1
          for (int st = 0; st < 4; ++st) {
            float see[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) see[y] = 8 * (y >> 2) + (y & 3) <= pos - kt * FK - 16 * st - 4 * hh ? 1.0f : 0.0f;
            const bf16x8 s8 = cvt8(see);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
              __builtin_amdgcn_sched_barrier(0);
              const f32x16 cnt = mfma32(tr8(Vs0, 16 * st * RB + lo.trl(d), 16 * st * RB + lo.trh(d)), s8, f32x16{});
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int c = (int)cnt[i];
                oacc[d][i] += c == 0 ? 0.0f : c >> 12 || ((c & 63) && (c >> 6)) ? NAN : c & 63 ? INFINITY : -INFINITY;
              }
            }
          }
        }
      }

      const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
      if (row < all_rows) {
        if (way.whole()) {
          int orow = row;
          asm volatile("" : "+v"(orow));  // (formed again here, not held through the loop)
          const int otok = orow / a.G;
          const int64_t out = (int64_t)(first + otok) * a.Hq + h * a.G + (orow - otok * a.G);
          const float inv = l_tot == 0.0f ? 0.0f : 1.0f / l_tot;
          bf16_t* const o = (bf16_t*)a.o + out * D;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t w0 = (uint32_t)f2bf(oacc[d][4 * y] * inv) | ((uint32_t)f2bf(oacc[d][4 * y + 1] * inv) << 16);
              const uint32_t w1 = (uint32_t)f2bf(oacc[d][4 * y + 2] * inv) | ((uint32_t)f2bf(oacc[d][4 * y + 3] * inv) << 16);
              *reinterpret_cast<uint2*>(o + 32 * d + 8 * y + 4 * hh) = make_uint2(w0, w1);
            }
          if (a.lse && hh == 0) a.lse[out] = l_tot == 0.0f ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
        } else {
          const int64_t at = way.slot() * TM + 32 * w + r32;
          float* const o = a.part + at * D;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              *reinterpret_cast<float4*>(o + 32 * d + 8 * y + 4 * hh) =
                  make_float4(oacc[d][4 * y], oacc[d][4 * y + 1], oacc[d][4 * y + 2], oacc[d][4 * y + 3]);
          if (hh == 0) a.stat[at] = make_float2(m_run, l_tot);
        }
      }
    }
    __syncthreads();  // (the way was read)
    if (tid == 0) {
      Walk<TM, 8, MIX ? 5 : 0> wk = way;
      wk.describe(a, rows, row0);
      more = wk.next(a);
      way = wk;
    }
    __syncthreads();
    if (!more) return;
  }
}

template <int D, int NW, bool MIX>
static void launch_tile(const PagedArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((paged_tile<D, NW, MIX>), dim3((unsigned)TileCfg<D, NW>::W), dim3(64 * NW), 0, st, a);
}
template <int D, bool MIX>
static PagedVariant variant(int waves) {
  if (waves <= 4) return {TileCfg<D, 4>::W, 128, launch_tile<D, 4, MIX>};
  if (waves <= 8) return {TileCfg<D, 8>::W, 256, launch_tile<D, 8, MIX>};
  return {TileCfg<D, 12>::W, 384, launch_tile<D, 12, MIX>};
}

}  // namespace lh

PagedVariant lh_paged_tile_variant(const LhPaged& s, int waves) {
  if (s.R > 1) return s.D == 128 ? lh::variant<128, true>(waves) : lh::variant<64, true>(waves);
  return s.D == 128 ? lh::variant<128, false>(waves) : lh::variant<64, false>(waves);
}
