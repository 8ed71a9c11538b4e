// k_paged_sdpa.hip -- attention of a step's new tokens over a paged K/V cache (include/lighthouse.h,
// serving): the rows kernel, for requests of few rows (decoding, drafts) and all of fp32.
//
// Rows. Query head hq = g G + x of token i of a request attends over KV head g like the other heads of the
// group, so the group's heads and the request's tokens make one list of rows, row = i G + x, whose K and V
// are read once: a tile is TM = 16 RT of them. With one new token that is G rows, and the product with
// them costs a 16-row MFMA whatever G is; the kernel is bound by the bytes of K and V.
//
// Split. A step's work is one line of units (keys to be read, tile after tile, head after head, request
// after request), cut into as many equal parts as the chip has room for workgroups; a workgroup takes
// one part, which may begin and end inside a tile's keys. So one request of a long context and hundreds of
// short ones fill the chip alike, and no length need be known to the host. Within a part, the four waves
// take its blocks of keys in turn, each with a running maximum and sum of its own, and are joined in LDS
// at the end of the tile; a tile cut across workgroups leaves its parts (fp32) in the workspace, and a second
// launch joins them in order: results depend on the lengths alone.
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
// The loads of the next block's K are issued when the last ones were multiplied, the same for V, and
// 12 waves a CU hide one another's latency.
#include <math.h>

#include "lh_paged.h"

namespace lh {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32v4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32v2;

__device__ __forceinline__ bf16x8 cvt8(const float* f) {
  typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
  const f32x8 v = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
  return __builtin_convertvector(v, bf16x8);
}

struct PagedArgs {
  const void *q, *kp, *vp;
  const int32_t *table, *cu_q, *kv_len;
  void* o;
  float* lse;
  int64_t q_stride, T, pages;
  int32_t R, max_blocks, shift, Hq, Hkv, G;
  float sl2;  // scale log2(e): logits are kept in log2 units
  // workspace
  struct PartDesc* desc;  // [W]
  float2* stat;           // [2 W][TM] maximum and sum
  float* part;            // [2 W][TM][D]
  int32_t W;
};

// A tile whose parts begin in workgroup w: rows and where they go, and the last workgroup with a part.
struct PartDesc {
  int32_t rows, row0, first, head, last;  // rows = 0: no tile
  int32_t pad[3];
};

constexpr float kLn2p = 0.6931471805599453f;
constexpr float kLog2ep = 1.4426950408889634f;
constexpr float kGrow = 8.0f;    // the accumulator is rescaled when a row's maximum grows by more than 2^8
constexpr int32_t kOver = 64;    // what a tile costs besides its keys, in keys
constexpr int32_t kLeast = 256;  // keys below which a part is not worth a workgroup

__device__ __forceinline__ int32_t clip(int64_t x, int64_t hi) { return (int32_t)(x < 0 ? 0 : x > hi ? hi : x); }
__device__ __forceinline__ int32_t uni(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uni64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// What a request asks for. Lengths and offsets are clipped into their ranges.
template <int TM>
struct Req {
  int32_t first, n, len, base, rows, tiles;  // base: position of the first new token
  __device__ __forceinline__ Req(const PagedArgs& a, int r) {
    first = clip(a.cu_q[r], a.T);
    n = clip((int64_t)clip(a.cu_q[r + 1], a.T) - first, a.T);
    len = clip(a.kv_len[r], (int64_t)a.max_blocks << a.shift);
    base = len - n;
    rows = n * a.G;
    tiles = (int32_t)(((int64_t)rows + TM - 1) / TM);
  }
  // Units of tile t: the keys up to its last row (by whole tokens), and the constant.
  __device__ __forceinline__ int64_t step(const PagedArgs& a) const { return a.G < TM ? TM / a.G : 1; }
  __device__ __forceinline__ int64_t fixed() const { return (base > 0 ? base : 0) + kOver; }
  __device__ __forceinline__ int64_t units(const PagedArgs& a, int64_t t) const { return fixed() + (t + 1) * step(a); }
  __device__ __forceinline__ int64_t before(const PagedArgs& a, int64_t t) const {  // of tiles 0 .. t - 1
    return t * fixed() + step(a) * (t * (t + 1) / 2);
  }
};

struct Cut {  // the line of units in n equal parts
  int64_t q, rem;
  int32_t n;
  __device__ __forceinline__ int64_t start(int64_t w) const { return q * w + rem * w / n; }
};

template <typename T, int D, int RT>
struct RowsCfg {
  static constexpr int NW = 4, TM = 16 * RT, KB = sizeof(T) == 2 ? 32 : 16;  // keys of a block
  static constexpr int DL = D / 16;                                           // columns of V that a lane reads
  static constexpr int KV = KB / 16 * D / (sizeof(T) == 2 ? 32 : 16);         // 16-byte reads of K a lane and block
  static constexpr int NV = KB / 4;                                           // keys of V a lane and block
  static constexpr int VW = DL * sizeof(T) / 4;                               // 32-bit words of one of them
  static constexpr int EU = RT == 1 ? 3 : 2;  // workgroups a CU
  static constexpr int64_t W = 256 * EU;
};

template <typename T, int D, int RT>
struct Wave {
  using C = RowsCfg<T, D, RT>;
  f32x4 acc[RT][C::DL];
  float m[RT], l[RT];  // of row n; the sum is this lane's share
  u32v4 q[RT][D * sizeof(T) / 64];
  u32v4 k[C::KV];
  uint32_t v[C::NV][C::VW];
};

template <typename T, int D, int RT>
__global__ void __launch_bounds__(256, (RowsCfg<T, D, RT>::EU)) paged_rows(const PagedArgs a) {
  using C = RowsCfg<T, D, RT>;
  constexpr int TM = C::TM, DL = C::DL, KB = C::KB, RB = D * (int)sizeof(T);
  constexpr bool B16 = sizeof(T) == 2;
  constexpr int LD = D + 4;  // a row of the LDS parts, padded by 16 bytes
  __shared__ __align__(16) float parts[C::NW][16][LD];
  __shared__ float ms[C::NW][16], ls[C::NW][16];
  __shared__ int64_t scan[C::NW];
  __shared__ int32_t found_r;
  __shared__ int64_t found_x;
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6), n = lane & 15, g = lane >> 4;

  // where this workgroup's part begins
  int64_t total = 0;
  int64_t cost = 0, upto = 0;
  for (int r0 = 0; r0 < a.R; r0 += 256) {
    cost = 0;
    if (r0 + tid < a.R) {
      const Req<TM> rq(a, r0 + tid);
      cost = rq.before(a, rq.tiles) * a.Hkv;
    }
    upto = block_scan<256>(cost, total, scan);
    if (tid == 255) scan[0] = upto;
    __syncthreads();
    total = uni64(scan[0]);
    __syncthreads();
  }
  Cut cut;
  {
    const int64_t most = (total + kLeast - 1) / kLeast;
    int32_t parts_n = most < a.W ? (int32_t)((most + 7) & ~7) : a.W;
    cut.n = parts_n < 8 ? 8 : parts_n;
    cut.q = total / cut.n, cut.rem = total - cut.q * cut.n;
  }
  const int b = blockIdx.x;
  // neighbouring parts on one XCD (workgroups go to the 8 XCDs in turn): they read the same keys
  const int32_t lw = b < cut.n ? (b % 8) * (cut.n / 8) + b / 8 : b;
  if (tid == 0) a.desc[lw].rows = 0;
  if (lw >= cut.n) return;
  int64_t x = cut.start(lw);
  const int64_t x1 = cut.start(lw + 1);
  if (x >= x1) return;
  if (a.R > 256) {  // the request of unit x: the sums again, chunk by chunk
    int64_t sum = 0;
    for (int r0 = 0; r0 < a.R; r0 += 256) {
      cost = 0;
      if (r0 + tid < a.R) {
        const Req<TM> rq(a, r0 + tid);
        cost = rq.before(a, rq.tiles) * a.Hkv;
      }
      upto = block_scan<256>(cost, sum, scan);
      if (upto - cost <= x && x < upto) found_r = r0 + tid, found_x = x - (upto - cost);
      if (tid == 255) scan[0] = upto;
      __syncthreads();
      sum = uni64(scan[0]);
      __syncthreads();
    }
  } else if (upto - cost <= x && x < upto) {
    found_r = tid, found_x = x - (upto - cost);
  }
  __syncthreads();
  int r = uni(found_r);
  int64_t u0 = uni64(found_x);  // unit of the tile
  Req<TM> rq(a, r);
  int h, t = 0;
  {
    const int64_t each = rq.before(a, rq.tiles);
    h = (int)(u0 / each);
    u0 -= h * each;
    int hi = rq.tiles;  // before(t) <= u0 < before(hi)
    while (hi - t > 1) {
      const int mid = t + (hi - t) / 2;
      if (rq.before(a, mid) <= u0) t = mid;
      else hi = mid;
    }
    u0 -= rq.before(a, t);
  }

  Wave<T, D, RT> s;
  for (;;) {
    const int64_t units = rq.units(a, t);
    int64_t u1 = u0 + (x1 - x);
    if (u1 > units) u1 = units;
    const int row0 = t * TM, rows = rq.rows - row0 < TM ? rq.rows - row0 : TM;
    const int keys = rq.base + (row0 + rows - 1) / a.G + 1;  // that any row of the tile sees
    const int safe = rq.base + row0 / a.G + 1;               // that all of them see
    const int nb = keys > 0 ? (keys + KB - 1) / KB : 0;
    const int b0 = (int)((int64_t)nb * u0 / units), b1 = u1 == units ? nb : (int)((int64_t)nb * u1 / units);

    // ---- this wave's blocks
    int pos[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      int row = row0 + rt * 16 + n;
      row = row < rq.rows ? row : rq.rows - 1;
      const int tok = row / a.G;
      pos[rt] = rq.base + tok;
      const T* qp = (const T*)a.q + (int64_t)(rq.first + tok) * a.q_stride + (int64_t)(h * a.G + row - tok * a.G) * D;
#pragma unroll
      for (int c = 0; c < RB / 64; ++c) s.q[rt][c] = *reinterpret_cast<const u32v4*>((const char*)qp + c * 64 + g * 16);
      s.m[rt] = -INFINITY, s.l[rt] = 0.0f;
#pragma unroll
      for (int e = 0; e < DL; ++e) s.acc[rt][e] = f32x4{};
    }
    const int32_t* ids = a.table + (int64_t)r * a.max_blocks;
    const int last = (keys - 1) >> a.shift;  // the last page in use (keys > 0 wherever it is used)
    auto at = [&](int j) __attribute__((always_inline)) {  // bytes from the pool's start to 16 keys from j
      int b_ = j >> a.shift;
      b_ = b_ < last ? b_ : last;
      const int32_t id = clip(uni(ids[b_]), a.pages - 1);
      return ((((int64_t)id * a.Hkv + h) << a.shift) + (j & ((1 << a.shift) - 1))) * RB;
    };
    auto load_k = [&](int j) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < KB / 16; ++c) {
        const char* p = (const char*)a.kp + at(j + 16 * c);
#pragma unroll
        for (int i = 0; i < RB / 64; ++i)
          s.k[c * (RB / 64) + i] = *reinterpret_cast<const u32v4*>(p + n * RB + g * 16 + i * 64);
      }
    };
    auto load_v = [&](int j) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < KB / 16; ++c) {
        const char* p = (const char*)a.vp + at(j + 16 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const char* pv = p + (4 * g + i) * RB + n * (DL * (int)sizeof(T));
          if constexpr (C::VW == 2) {
            const u32v2 y = *reinterpret_cast<const u32v2*>(pv);
            s.v[4 * c + i][0] = y[0], s.v[4 * c + i][1] = y[1];
          } else {
#pragma unroll
            for (int z = 0; z < C::VW / 4; ++z) {
              const u32v4 y = *reinterpret_cast<const u32v4*>(pv + 16 * z);
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
        bf16x8 pb[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) pb[rt] = cvt8(p[rt]);  // one rounding, to the type of V
#pragma unroll
        for (int e = 0; e < DL; ++e) {
          u32v4 y;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            y[c] = __builtin_amdgcn_perm(s.v[2 * c + 1][e / 2], s.v[2 * c][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            s.acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y), pb[rt], s.acc[rt][e], 0, 0, 0);
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
      uint32_t* const mine = reinterpret_cast<uint32_t*>(&parts[w][0][0]) + lane;
      static_assert(C::NV * C::VW * 64 <= 16 * LD, "the words of a block fit a wave's part");
#pragma unroll
      for (int i = 0; i < C::NV; ++i)
#pragma unroll
        for (int z = 0; z < C::VW; ++z) {
          uint32_t& y = s.v[i][z];
          mine[(i * C::VW + z) * 64] = y;
          if constexpr (B16) {
            if ((y & 0x7f80u) == 0x7f80u) y &= 0xffff0000u;
            if ((y & 0x7f800000u) == 0x7f800000u) y &= 0x0000ffffu;
          } else {
            if ((y & 0x7f800000u) == 0x7f800000u) y = 0;
          }
        }
#pragma unroll 1
      for (int e = 0; e < DL; ++e) {
        float code[C::NV], see[C::NV];
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
          const uint32_t y = mine[(i * C::VW + (B16 ? e / 2 : e)) * 64];
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
            for (int y = 0; y < DL; ++y) s.acc[rt][y][i] += y == e ? add : 0.0f;
          }
        }
      }
    };
    int blk = b0 + w;
    if (blk < b1) {
      load_k(blk * KB);
      load_v(blk * KB);
    }
    for (; blk < b1; blk += C::NW) {
      const int j0 = blk * KB, next = (blk + C::NW) * KB;
      const bool more = blk + C::NW < b1;
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
      if (more) load_k(next);
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
        const bool grown = top > s.m[rt] + kGrow;  // each row by its own: no row's bits depend on another's
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
      if (more) load_v(next);
    }

    // ---- the four waves joined
    const bool whole = u0 == 0 && u1 == units;
    const int64_t slot = 2 * (int64_t)lw + (u0 > 0 ? 0 : 1);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float l = s.l[rt];
      l += __shfl_xor(l, 16, 64);
      l += __shfl_xor(l, 32, 64);
      if (g == 0) ms[w][n] = s.m[rt], ls[w][n] = l;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < DL; e += 4)
          *reinterpret_cast<f32x4*>(&parts[w][n][DL * (4 * g + i) + e]) =
              f32x4{s.acc[rt][e][i], s.acc[rt][e + 1][i], s.acc[rt][e + 2][i], s.acc[rt][e + 3][i]};
      __syncthreads();
      const int rn = tid >> 4, c0 = (tid & 15) * DL, row = rt * 16 + rn;
      if (row < rows) {
        float mt = ms[0][rn], lt = 0.0f, out[DL];
#pragma unroll
        for (int y = 1; y < C::NW; ++y) mt = fmaxf(mt, ms[y][rn]);
#pragma unroll
        for (int e = 0; e < DL; ++e) out[e] = 0.0f;
#pragma unroll
        for (int y = 0; y < C::NW; ++y) {
          const float wt = ms[y][rn] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ms[y][rn] - mt);
          if (ms[y][rn] != -INFINITY || ls[y][rn] != 0.0f) {  // (a NaN sum comes with a maximum of -inf where all logits are NaN)
            lt += ms[y][rn] == -INFINITY ? ls[y][rn] : wt * ls[y][rn];
#pragma unroll
            for (int e = 0; e < DL; ++e) out[e] += wt * parts[y][rn][c0 + e];
          }
        }
        if (whole) {
          const int gr = row0 + row, tok = gr / a.G;
          const int64_t at_ = (int64_t)(rq.first + tok) * a.Hq + h * a.G + (gr - tok * a.G);
          const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
          T* o = (T*)a.o + at_ * D + c0;
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
          if (a.lse && (tid & 15) == 0) a.lse[at_] = lt == 0.0f ? -INFINITY : (mt + __log2f(lt)) * kLn2p;
        } else {
          float* o = a.part + (slot * TM + row) * D + c0;
#pragma unroll
          for (int e = 0; e < DL; e += 4) *reinterpret_cast<f32x4*>(o + e) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
          if ((tid & 15) == 0) a.stat[slot * TM + row] = make_float2(mt, lt);
        }
      }
      __syncthreads();
    }
    if (!whole && u0 == 0 && tid == 0) {  // the tile's parts begin here: up to the workgroup with its last unit
      const int64_t end = x + units;
      int lo = lw, hi = cut.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (cut.start(mid) < end) lo = mid;
        else hi = mid;
      }
      a.desc[lw] = PartDesc{rows, row0, rq.first, h, lo, {0, 0, 0}};
    }

    x += u1 - u0;
    if (x >= x1) return;
    u0 = 0;
    if (++t < rq.tiles) continue;
    t = 0;
    if (++h < a.Hkv) continue;
    h = 0;
    do {
      if (++r >= a.R) return;
      rq = Req<TM>(a, r);
    } while (rq.tiles == 0);
  }
}

// Joins the parts of the tiles that were cut: a workgroup per tile and four rows; a wave per row where the
// parts are few, else the four waves share a row's parts.
template <typename T, int D, int TM>
__global__ void __launch_bounds__(256) paged_join(const PagedArgs a) {
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
    if (a.lse && lane == 0) a.lse[at] = l == 0.0f ? -INFINITY : (mt + __log2f(l)) * kLn2p;
  }
}

struct RowsWs {
  size_t desc, stat, part, total;
};
template <typename T, int D, int RT>
static RowsWs rows_ws() {
  using C = RowsCfg<T, D, RT>;
  RowsWs w;
  w.desc = 0;
  w.stat = sizeof(PartDesc) * C::W;
  w.part = w.stat + sizeof(float2) * 2 * C::W * C::TM;
  w.total = w.part + sizeof(float) * 2 * C::W * C::TM * D;
  return w;
}

template <typename T, int D, int RT>
static hipError_t launch_rows(const LhPaged& s, PagedArgs a, void* ws, hipStream_t st) {
  using C = RowsCfg<T, D, RT>;
  const RowsWs w = rows_ws<T, D, RT>();
  a.desc = (PartDesc*)ws;
  a.stat = (float2*)((char*)ws + w.stat);
  a.part = (float*)((char*)ws + w.part);
  a.W = (int32_t)C::W;
  hipLaunchKernelGGL((paged_rows<T, D, RT>), dim3((unsigned)C::W), dim3(256), 0, st, a);
  const int64_t rows = s.T * s.G < C::TM ? s.T * s.G : C::TM;
  hipLaunchKernelGGL((paged_join<T, D, C::TM>), dim3((unsigned)C::W, (unsigned)((rows + 3) / 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

// f(IC<RT>) of the variant that serves the step: rows a request on average
template <typename T, int D, typename F>
static auto with_rows(const LhPaged& s, F&& f) {
  const int64_t rows = s.T * s.G / s.R;
  return rows > 16 ? f(rows_ws<T, D, 2>(), launch_rows<T, D, 2>) : f(rows_ws<T, D, 1>(), launch_rows<T, D, 1>);
}

template <typename F>
static auto with_variant(const LhPaged& s, F&& f) {
  if (s.dtype == LH_BF16) return s.D == 128 ? with_rows<bf16_t, 128>(s, f) : with_rows<bf16_t, 64>(s, f);
  return s.D == 128 ? with_rows<float, 128>(s, f) : with_rows<float, 64>(s, f);
}

}  // namespace lh

using namespace lh;

size_t lh_sdpa_paged_ws_bytes(const LhPaged& s) {
  return with_variant(s, [](const RowsWs& w, auto) { return w.total; });
}

hipError_t lh_launch_sdpa_paged(const LhPaged& s, const void* q, int64_t q_stride, const void* kpages,
                                const void* vpages, const int32_t* table, const int32_t* cu_q,
                                const int32_t* kv_len, void* o, float* lse, void* ws, hipStream_t st) {
  PagedArgs a{};
  a.q = q, a.kp = kpages, a.vp = vpages, a.table = table, a.cu_q = cu_q, a.kv_len = kv_len, a.o = o, a.lse = lse;
  a.q_stride = q_stride, a.T = s.T, a.pages = s.pages;
  a.R = s.R, a.max_blocks = s.max_blocks, a.shift = s.shift, a.Hq = s.Hq, a.Hkv = s.Hkv, a.G = s.G;
  a.sl2 = s.scale * kLog2ep;
  return with_variant(s, [&](const RowsWs&, auto launch) { return launch(s, a, ws, st); });
}
