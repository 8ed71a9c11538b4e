// lh_paged_rows.h -- attention of a tile of 16 or 32 rows over a paged cache (rows, cut and parts:
// lh_paged_sdpa.h). With one new token a tile has G rows, the product with them costs a 16-row MFMA whatever G
// is, and the time is that of the bytes of K and V.
//
// Within a part, the waves of a workgroup take its blocks of keys in turn, each with a running maximum and sum of
// its own, and are joined in LDS at the end of the tile.
//
// Registers only. A wave's loop uses no LDS and no barrier:
//   bf16, MFMA 16x16x32, lane l, n = l % 16, g = l / 16: A[m = n][k = 8 g + 0..7], B[k = 8 g + 0..7][n],
//   C[m = 4 g + i][n], i = 0..3.
//   S^T = K Q^T: a lane reads 16 bytes of key n of 16 keys (64 consecutive bytes a row and load).
//   O^T = V^T P^T: the k order is the keys 4 g + 0..3 and 16 + 4 g + 0..3 of a 32-key block, the order
//   in which the lane holds S^T, so P is the operand as it is computed. V^T's operand is 8 keys of one column;
//   a lane reads D / 16 consecutive columns of those 8 keys (whole rows a wave) and transposes
//   them in registers, one v_perm_b32 for two values; its columns are d = (D / 16) m + s of MFMA s, which
//   permutes the columns of O^T and not the sums, and hands a lane consecutive columns to store.
//   fp32, MFMA 16x16x4: A[m = n][k = g] one value; the k order of step c of 4 is column 16 kk + 4 g + c (a
//   16-byte read), and of V step i the key 4 g + i, whose columns need no transpose at all.
// The loads of the next block's K are issued when the last ones were multiplied, the same for V.
//
// Bound by HBM: 64 decoding requests of 482,000 keys, 32 heads on 8, D = 128, bf16: 308 us for 1.98 GB (2.0 GB fetched),
// 6.4 TB/s; one request at 262,143 keys 162 us, 6.6 TB/s (a large copy moves 5.1). Short steps are bound by the chain
// of dependent loads before the first product (lengths, table, keys), 3 us of 8 for one request of 777 keys. In fp32 with
// many rows by the fp32 matrix rate: 8 requests of 64 tokens at 16,000 keys, 32 heads on 8: 106 TFLOP/s (a large
// library product 154).
#pragma once

#include <math.h>

#include "lh_mfma.h"
#include "lh_paged_sdpa.h"

namespace lh {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32v4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32v2;

template <typename T, int D, int RT>
struct RowsCfg {
  static constexpr int KB = sizeof(T) == 2 ? 32 : 16;                  // keys of a block
  static constexpr int DL = D / 16;                                    // columns of V that a lane reads
  static constexpr int KV = KB / 16 * D / (sizeof(T) == 2 ? 32 : 16);  // 16-byte reads of K a lane and block
  static constexpr int NV = KB / 4;                                    // keys of V a lane and block
  static constexpr int VW = DL * sizeof(T) / 4;                        // 32-bit words of one of them
};

template <bool NT, typename V>
__device__ __forceinline__ V load(const char* p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

template <typename T, int D, int RT>
struct Wave {
  using C = RowsCfg<T, D, RT>;
  f32x4 acc[RT][C::DL];
  float m[RT], l[RT];  // of row n; the sum is this lane's share
  u32v4 q[RT][D * sizeof(T) / 64];
  u32v4 k[C::KV];
  uint32_t v[C::NV][C::VW];
};

// One part of one tile: rows row0 .. row0 + rows - 1 (16 RT at most) of a request over blocks b0 .. b1 - 1 of its keys.
struct RowsItem {
  int r, h, row0, rows, all_rows, first, base, keys, safe;  // keys: that any row sees; safe: that all of them see
  int b0, b1;
  bool whole;    // all of the tile's keys: the rows are the outputs
  int64_t slot;  // else where the part's rows go
};

// The NW waves of a workgroup on it. Lds: part(w), 16 D floats of wave w (PER of them at a time); words(w), 8 D floats of a
// wave alone, inside part(w) where kOwnWords (a wave that is done writes its part while others use their words), else
// anywhere, and a barrier stands before the first part; ms(w), ls(w), 16 floats each. Rows of a
// part are swizzled (16-byte chunk c of row n at c ^ n). TM: rows that a part has room for in the workspace.
template <typename T, int D, int RT, int NW, bool NT, int TM, typename Lds>
__device__ __forceinline__ void rows_tile(const PagedArgs& a, const RowsItem& it, const Lds& lds) {
  using C = RowsCfg<T, D, RT>;
  constexpr int DL = C::DL, KB = C::KB, RB = D * (int)sizeof(T);
  constexpr bool B16 = sizeof(T) == 2;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (what follows from the lane is formed anew for every tile, not held across them)
  const int lane = tid & 63, w = uni(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int h = it.h, row0 = it.row0, rows = it.rows, keys = it.keys, safe = it.safe, b1 = it.b1;
  Wave<T, D, RT> s;

  // ---- this wave's blocks
  int pos[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    int row = row0 + rt * 16 + n;
    row = row < it.all_rows ? row : it.all_rows - 1;
    const int tok = row / a.G;
    pos[rt] = it.base + tok;
    const T* qp = (const T*)a.q + (int64_t)(it.first + tok) * a.q_stride + (int64_t)(h * a.G + row - tok * a.G) * D;
#pragma unroll
    for (int c = 0; c < RB / 64; ++c) s.q[rt][c] = *reinterpret_cast<const u32v4*>((const char*)qp + c * 64 + g * 16);
    s.m[rt] = -INFINITY, s.l[rt] = 0.0f;
#pragma unroll
    for (int e = 0; e < DL; ++e) s.acc[rt][e] = f32x4{};
  }
  const int64_t ids = (int64_t)it.r * a.max_blocks;  // the request's row of the table
  const int last = (keys - 1) >> a.shift;  // the last page in use (keys > 0 wherever it is used)
  // A block's pages are looked up a block ahead of its loads; K and V lie at the same place of their pools.
  int32_t pg[KB / 16];
  int64_t off[KB / 16];  // bytes from the pool's start to 16 keys
  auto look_up = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < KB / 16; ++c) {
      const int b = (j + 16 * c) >> a.shift;
      pg[c] = page_id(a.table, ids + (b < last ? b : last), a.pages);
    }
  };
  auto place = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < KB / 16; ++c)
      off[c] = ((((int64_t)pg[c] * a.Hkv + h) << a.shift) + ((j + 16 * c) & ((1 << a.shift) - 1))) * RB;
  };
  auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < KB / 16; ++c) {
      const char* p = (const char*)a.kp + off[c];
#pragma unroll
      for (int i = 0; i < RB / 64; ++i)
        s.k[c * (RB / 64) + i] = load<NT, u32v4>(p + n * RB + g * 16 + i * 64);
    }
  };
  auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < KB / 16; ++c) {
      const char* p = (const char*)a.vp + off[c];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char* pv = p + (4 * g + i) * RB + n * (DL * (int)sizeof(T));
        if constexpr (C::VW == 2) {
          const u32v2 y = load<NT, u32v2>(pv);
          s.v[4 * c + i][0] = y[0], s.v[4 * c + i][1] = y[1];
        } else {
#pragma unroll
          for (int z = 0; z < C::VW / 4; ++z) {
            const u32v4 y = load<NT, u32v4>(pv + 16 * z);
#pragma unroll
            for (int o = 0; o < 4; ++o) s.v[4 * c + i][4 * z + o] = y[o];
          }
        }
      }
    }
  };
  // O^T += V^T P^T; p[rt]: this lane's weights of its keys
  auto pv = [&](const float (*p)[C::NV]) __attribute__((always_inline)) {
    if constexpr (B16) {
      // The weights as the sum of two bf16 values, whose products are both formed: the matrix unit has time for it
      // beside the loads, and o is off by its own rounding alone (2-norm 1.65e-3; with the weights rounded once 2.3e-3).
      // The first is cut off, not rounded, and the last bit set: the second is above 0 wherever the weight is, so that
      // an infinite value of V keeps its sign in both products. (In all within 2^-16 of the weight.)
      bf16x8 pb[RT], pl[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        u32v4 hi;
        float rest[C::NV];
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
          const uint32_t x = __float_as_uint(p[rt][i]);
          rest[i] = __uint_as_float(x | 1u) - __uint_as_float(x & 0xffff0000u);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          hi[c] = __builtin_amdgcn_perm(__float_as_uint(p[rt][2 * c + 1]), __float_as_uint(p[rt][2 * c]), 0x07060302u);
        pb[rt] = __builtin_bit_cast(bf16x8, hi);
        pl[rt] = cvt8(rest);
      }
#pragma unroll
      for (int e = 0; e < DL; ++e) {
        u32v4 y;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          y[c] = __builtin_amdgcn_perm(s.v[2 * c + 1][e / 2], s.v[2 * c][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          s.acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y), pb[rt], s.acc[rt][e], 0, 0, 0);
          s.acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y), pl[rt], s.acc[rt][e], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < DL; ++e)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            s.acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(s.v[i][e]), p[rt][i], s.acc[rt][e], 0, 0, 0);
    }
  };
  // Takes the values of V that are not finite out of the registers and adds them to the rows that see their
  // key. (They may be of keys that some rows see and others do not, and 0 times them would be NaN.) A product
  // with the rows' view of the keys (1 or 0) counts them, 1 for +inf, 64 for -inf, 4096 for NaN: of
  // at most 32 keys, so the counts do not overlap. A rare path that must not cost the loop registers: the
  // words go through the wave's part of the LDS, and the columns are a loop that is not unrolled.
  auto odd_values = [&](int j0) __attribute__((always_inline)) {
    uint32_t* const mine = reinterpret_cast<uint32_t*>(lds.words(w)) + lane;
    constexpr int HW = C::VW / 2;  // words of a key at a time: 32 D bytes a wave
    static_assert(C::NV * HW * 64 * 4 <= 32 * D, "the words fit");
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int i = 0; i < C::NV; ++i)
#pragma unroll
        for (int z = 0; z < HW; ++z) {
          uint32_t& y = s.v[i][half * HW + z];
          mine[(i * HW + z) * 64] = y;
          if constexpr (B16) {
            if ((y & 0x7f80u) == 0x7f80u) y &= 0xffff0000u;
            if ((y & 0x7f800000u) == 0x7f800000u) y &= 0x0000ffffu;
          } else {
            if ((y & 0x7f800000u) == 0x7f800000u) y = 0;
          }
        }
#pragma unroll 1
      for (int e = 0; e < DL / 2; ++e) {
        float code[C::NV], see[C::NV];
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
          const uint32_t y = mine[(i * HW + (B16 ? e / 2 : e)) * 64];
          const uint32_t x = B16 ? (e & 1 ? y & 0xffff0000u : y << 16) : y;
          code[i] = (x & 0x7f800000u) != 0x7f800000u ? 0.0f : x & 0x7fffffu ? 4096.0f : x >> 31 ? 64.0f : 1.0f;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
          for (int i = 0; i < C::NV; ++i) see[i] = j0 + 16 * (i / 4) + 4 * g + i % 4 <= pos[rt] ? 1.0f : 0.0f;
          f32x4 cnt = {};
          if constexpr (B16) {
            cnt = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cvt8(code), cvt8(see), cnt, 0, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) cnt = __builtin_amdgcn_mfma_f32_16x16x4f32(code[i], see[i], cnt, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = (int)cnt[i];
            const float add = c == 0 ? 0.0f : c >> 12 || ((c & 63) && (c >> 6)) ? NAN : c & 63 ? INFINITY : -INFINITY;
#pragma unroll
            for (int y = 0; y < DL / 2; ++y) s.acc[rt][half * (DL / 2) + y][i] += y == e ? add : 0.0f;
          }
        }
      }
    }
  };
  int blk = it.b0 + w;
  if (blk < b1) {
    look_up(blk * KB);
    place(blk * KB);
    load_k();
    load_v();
    look_up((blk + NW) * KB);
  }
  for (; blk < b1; blk += NW) {
    const int j0 = blk * KB, next = (blk + NW) * KB;
    const bool more = blk + NW < b1;
    f32x4 sc[RT][KB / 16];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int c = 0; c < KB / 16; ++c) {
        sc[rt][c] = f32x4{};
#pragma unroll
        for (int i = 0; i < RB / 64; ++i) {
          const u32v4 kk = s.k[c * (RB / 64) + i], qq = s.q[rt][i];
          if constexpr (B16) {
            sc[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), __builtin_bit_cast(bf16x8, qq),
                                                                 sc[rt][c], 0, 0, 0);
          } else {
#pragma unroll
            for (int o = 0; o < 4; ++o)
              sc[rt][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kk[o]), __uint_as_float(qq[o]), sc[rt][c], 0, 0, 0);
          }
        }
      }
    if (more) {
      place(next);
      load_k();
      look_up(next + NW * KB);
    }
    const bool masked = j0 + KB > safe;
    if (masked) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < KB / 16; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (j0 + 16 * c + 4 * g + i > pos[rt]) sc[rt][c][i] = -INFINITY;
    }
    float p[RT][C::NV];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = sc[rt][0][0];
#pragma unroll
      for (int c = 0; c < KB / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[rt][c][i]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64)) * a.sl2;
      const bool grown = top > s.m[rt] + kRescale;  // each row by its own: no row's bits depend on another's
      if (__any(grown)) {
        const float al = !grown ? 1.0f : s.m[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(s.m[rt] - top);
        s.m[rt] = grown ? top : s.m[rt], s.l[rt] *= al;
#pragma unroll
        for (int e = 0; e < DL; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) s.acc[rt][e][i] *= al;
      }
      const float mm = s.m[rt] == -INFINITY ? 0.0f : s.m[rt];  // no key yet: all weights are 0
#pragma unroll
      for (int c = 0; c < KB / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[rt][4 * c + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rt][c][i], a.sl2, -mm));
          s.l[rt] += p[rt][4 * c + i];
        }
    }
    bool odd = false;
    if (masked) {  // rows behind the last key hold anything: they count as 0
#pragma unroll
      for (int i = 0; i < C::NV; ++i) {
        const bool in = j0 + 16 * (i / 4) + 4 * g + i % 4 < keys;
#pragma unroll
        for (int z = 0; z < C::VW; ++z) {
          uint32_t& y = s.v[i][z];
          y = in ? y : 0u;
          odd |= (y & 0x7f800000u) == 0x7f800000u || (B16 && (y & 0x7f80u) == 0x7f80u);
        }
      }
    }
    if (__any(odd)) odd_values(j0);
    pv(p);
    if (more) load_v();
  }

  // ---- the waves joined, PER of them at a time
  constexpr int PER = Lds::PER;
  static_assert(Lds::kOwnWords ? PER == NW : true, "every wave has a part of its own");
  if constexpr (!Lds::kOwnWords) __syncthreads();  // no wave needs its words any more
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float l = s.l[rt];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) lds.ms(w)[n] = s.m[rt], lds.ls(w)[n] = l;
    const int rn = tid >> 4, c0 = (tid & 15) * DL, row = rt * 16 + rn;
    const bool mine = tid < 256 && row < rows;  // a thread to DL columns of a row
    float mt = -INFINITY, lt = 0.0f, out[DL];
#pragma unroll
    for (int e = 0; e < DL; ++e) out[e] = 0.0f;
#pragma unroll
    for (int w0 = 0; w0 < NW; w0 += PER) {
      if (w >= w0 && w < w0 + PER) {
        float* const p = lds.part(w - w0) + n * D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < DL; e += 4)
            *reinterpret_cast<f32x4*>(p + (((DL * (4 * g + i) + e) / 4 ^ n) << 2)) =
                f32x4{s.acc[rt][e][i], s.acc[rt][e + 1][i], s.acc[rt][e + 2][i], s.acc[rt][e + 3][i]};
      }
      __syncthreads();
      if (mine) {
        if (w0 == 0) {
#pragma unroll
          for (int y = 0; y < NW; ++y) mt = fmaxf(mt, lds.ms(y)[rn]);
        }
#pragma unroll
        for (int y = w0; y < w0 + PER && y < NW; ++y) {
          // (a wave without a key has 0; one whose logits are all NaN has the maximum -inf and a sum of NaN)
          const float my = lds.ms(y)[rn], wt = my == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(my - mt);
          lt += wt * lds.ls(y)[rn];
          const float* const p = lds.part(y - w0) + rn * D;
#pragma unroll
          for (int e = 0; e < DL; e += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p + (((c0 + e) / 4 ^ rn) << 2));
#pragma unroll
            for (int z = 0; z < 4; ++z) out[e + z] += wt * x[z];
          }
        }
      }
      if (w0 + PER < NW || rt + 1 < RT) __syncthreads();
    }
    if (mine) {
      if (it.whole) {
        const int gr = row0 + row, tok = gr / a.G;
        const int64_t at = (int64_t)(it.first + tok) * a.Hq + h * a.G + (gr - tok * a.G);
        const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
        T* o = (T*)a.o + at * D + c0;
        if constexpr (B16) {
          uint32_t y[DL / 2];
#pragma unroll
          for (int e = 0; e < DL / 2; ++e) y[e] = (uint32_t)f2bf(out[2 * e] * inv) | ((uint32_t)f2bf(out[2 * e + 1] * inv) << 16);
          if constexpr (DL == 8) *reinterpret_cast<u32v4*>(o) = u32v4{y[0], y[1], y[2], y[3]};
          else *reinterpret_cast<u32v2*>(o) = u32v2{y[0], y[1]};
        } else {
#pragma unroll
          for (int e = 0; e < DL; e += 4)
            *reinterpret_cast<f32x4*>(o + e) = f32x4{out[e] * inv, out[e + 1] * inv, out[e + 2] * inv, out[e + 3] * inv};
        }
        if (a.lse && c0 == 0) a.lse[at] = lt == 0.0f ? -INFINITY : (mt + __log2f(lt)) * kLn2;
      } else {
        float* o = a.part + (it.slot * TM + row) * D + c0;
#pragma unroll
        for (int e = 0; e < DL; e += 4) *reinterpret_cast<f32x4*>(o + e) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
        if (c0 == 0) a.stat[it.slot * TM + row] = make_float2(mt, lt);
      }
    }
  }
}

}  // namespace lh
