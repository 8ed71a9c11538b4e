// lh_paged_sdpa.h -- what the paged attention kernels share: the rows of a request, the cut of a step's work
// into equal parts, and the parts of the tiles that a cut divides (k_paged_rows.hip, k_paged_tile.hip).
//
// Rows. Query head hq = g G + x of token i of a request attends over KV head g like the other heads of the
// group, so the group's heads and the request's tokens make one list of rows, row = i G + x, whose K and V
// are read once for a tile of TM rows.
//
// Cut. A step's work is one line of units (tile after tile, head after head, request after request; a tile's
// units are the keys that it reads, weighed by what a key costs it), cut into as many equal parts
// as the chip has room for workgroups. A part may begin and end inside a tile's keys. So one request of a long
// context and hundreds of short ones fill the chip alike, and no length need be known to the host. A tile that
// lies in several parts leaves each one's maximum, sum and unnormalised rows (fp32) in the workspace, and a second
// launch joins them in order: the results depend on the inputs alone.
#pragma once

#include "lh_paged.h"

namespace lh {

// A tile whose parts begin in workgroup w: its rows and where they go, and the last workgroup with a part.
struct PartDesc {
  int32_t rows, row0, first, head, last;  // rows = 0: no tile
  int32_t pad[3];
};

struct PagedArgs {
  const void *q, *kp, *vp;
  const int32_t *table, *cu_q, *kv_len;
  void* o;
  float* lse;
  int64_t q_stride, T, pages;
  int32_t R, max_blocks, shift, Hq, Hkv, G;
  float sl2;  // scale log2(e): logits are kept in log2 units
  // workspace. A workgroup has two parts at most: 2 w of the tile that it begins in, 2 w + 1 of the one it ends in
  PartDesc* desc;  // [W]
  float2* stat;    // [2 W][TM] maximum and sum
  float* part;     // [2 W][TM][D]
  int32_t W;       // workgroups
};

struct PagedWs {
  size_t stat, part, total;
};
inline PagedWs paged_ws(int64_t W, int TM, int D) {
  PagedWs w;
  w.stat = sizeof(PartDesc) * W;
  w.part = w.stat + sizeof(float2) * 2 * W * TM;
  w.total = w.part + sizeof(float) * 2 * W * TM * D;
  return w;
}

constexpr int32_t kCUs = 256;
template <int TM>
constexpr int32_t kOver = TM > 128 ? 160 : 64;  // what a tile costs besides its keys, in keys
// Keys below which a part is not worth a workgroup: with 128 in place of 256, tiles of 16 rows take 11.3 us and not 12.4 (one
// request, 777 keys) and 16.4 and not 17.7 (4 of 500), larger ones 24 and not 20 (32 rows, 8000 keys).
template <int TM>
constexpr int32_t kLeast = TM == 16 ? 128 : 256;

__device__ __forceinline__ int32_t clip(int64_t x, int64_t hi) { return (int32_t)(x < 0 ? 0 : x > hi ? hi : x); }
__device__ __forceinline__ int32_t uni(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uni64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// A page id by a scalar load, of an address that is the same for the whole wave (the table is written by
// earlier launches alone). A vector load would be waited for with the tiles in flight.
__device__ __forceinline__ int32_t page_id(const int32_t* table, int64_t i, int64_t pages) {
  return clip(((const __attribute__((address_space(4))) int32_t*)table)[i], pages - 1);
}

// What a request asks for. Lengths and offsets are clipped into their ranges. FW: what a key costs a tile
// whatever its rows, in 16ths of what it costs a full one; NR: what it costs 16 rows or fewer, if that differs.
template <int TM, int FW, int NR>
struct Req {
  int32_t first, n, base, rows, tiles, lastw;  // base: position of the first new token
  __device__ __forceinline__ Req() {}
  __device__ __forceinline__ Req(const PagedArgs& a, int r) {
    first = clip(a.cu_q[r], a.T);
    n = clip((int64_t)clip(a.cu_q[r + 1], a.T) - first, a.T);
    base = clip(a.kv_len[r], (int64_t)a.max_blocks << a.shift) - n;
    rows = n * a.G;
    tiles = (int32_t)(((int64_t)rows + TM - 1) / TM);
    const int32_t rest = rows - (tiles - 1) * TM;  // of the last tile
    lastw = NR > 0 && rest <= 16 ? NR : FW + ((16 - FW) * rest + TM - 1) / TM;
  }
  // Units of tile t: the keys up to its last row (by whole tokens; where a token has several tiles, each counts as one:
  // the host's bound on the sum allows for it) and a constant, in 16ths.
  __device__ __forceinline__ int64_t step(const PagedArgs& a) const { return a.G < TM ? TM / a.G : 1; }
  __device__ __forceinline__ int64_t past() const { return base > 0 ? base : 0; }
  __device__ __forceinline__ int64_t units(const PagedArgs& a, int64_t t) const {
    return (past() + (t + 1) * step(a)) * (t == tiles - 1 ? lastw : 16) + 16 * kOver<TM>;
  }
  __device__ __forceinline__ int64_t before(const PagedArgs& a, int64_t t) const {  // of tiles 0 .. t - 1, t < tiles
    return 16 * (t * (past() + kOver<TM>) + step(a) * (t * (t + 1) / 2));
  }
  __device__ __forceinline__ int64_t all(const PagedArgs& a) const {
    return tiles > 0 ? before(a, tiles - 1) + units(a, tiles - 1) : 0;
  }
};

// floor(a / b), a >= 0, b > 0. (The 64-bit integer division is longer, and several stand before the first load of a part.)
// The first quotient is off by 2^-52 of itself and one at most, so the rest is a few b's, whose quotient is exact but for
// one.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  int64_t q = (int64_t)((double)a / (double)b);
  int64_t r = a - q * b;
  const int64_t more = (int64_t)((double)r / (double)b);
  q += more, r -= more * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

struct Cut {  // the line of units in n equal parts, the first `rem` of them one longer
  int64_t q, rem;
  int32_t n;
  __device__ __forceinline__ int64_t start(int64_t w) const { return q * w + (w < rem ? w : rem); }
};

// A workgroup's way along its part.
template <int TM, int FW, int NR = 0>
struct Walk {
  Cut cut;
  int32_t lw;     // the workgroup's place in the line
  int64_t x, x1;  // units done and to do
  int r, h, t;    // the tile at hand: request, KV head, tile of its rows
  int64_t u0, u1, units;  // this part of the tile's units, and all of them
  Req<TM, FW, NR> rq;

  // Finds the part's beginning; false: the workgroup has none. Every thread of the NT calls it.
  struct Found {
    int64_t x;
    int32_t r;
    Req<TM, FW, NR> rq;
  };
  template <int NT>
  __device__ __forceinline__ bool begin(const PagedArgs& a, int64_t* scan, Found* found) {
    const int tid = threadIdx.x;
    int64_t total = 0, cost = 0, upto = 0;
    auto chunk = [&](int r0, int64_t& sum) __attribute__((always_inline)) {
      cost = 0;
      if (r0 + tid < a.R) {
        rq = Req<TM, FW, NR>(a, r0 + tid);
        cost = rq.all(a) * a.Hkv;
      }
      upto = block_scan<NT>(cost, sum, scan);
      if (tid == NT - 1) scan[0] = upto;
      __syncthreads();
      sum = uni64(scan[0]);
      __syncthreads();
    };
    for (int r0 = 0; r0 < a.R; r0 += NT) chunk(r0, total);
    const int64_t most = (total + 16 * kLeast<TM> - 1) / (16 * kLeast<TM>);  // (a power of two)
    // (between one and two workgroups a CU, those that share one would take twice as long)
    cut.n = most >= a.W ? a.W : most > kCUs ? kCUs : most <= 8 ? 8 : (int32_t)((most + 7) & ~7);
    cut.q = uni64(quotient(total, cut.n)), cut.rem = total - cut.q * cut.n;
    // neighbouring parts on one XCD (workgroups go to the 8 XCDs in turn): they read the same keys
    const int b = blockIdx.x;
    lw = b < cut.n ? (b % 8) * (cut.n / 8) + b / 8 : b;
    if (tid == 0) a.desc[lw].rows = 0;
    if (lw >= cut.n) return false;
    x = cut.start(lw), x1 = cut.start(lw + 1);
    if (x >= x1) return false;
    auto look = [&](int r0) __attribute__((always_inline)) {
      if (upto - cost <= x && x < upto) *found = Found{x - (upto - cost), r0 + tid, rq};
    };
    if (a.R <= NT) {
      look(0);
      __syncthreads();
    } else {
      int64_t sum = 0;
      for (int r0 = 0; r0 < a.R; r0 += NT) {
        chunk(r0, sum);
        look(r0);
        __syncthreads();
      }
    }
    r = uni(found->r);
    u0 = uni64(found->x);
    rq = found->rq;
    rq.first = uni(rq.first), rq.n = uni(rq.n), rq.base = uni(rq.base);
    rq.rows = uni(rq.rows), rq.tiles = uni(rq.tiles), rq.lastw = uni(rq.lastw);
    const int64_t each = rq.all(a);
    h = uni((int)quotient(u0, each));
    u0 -= h * each;
    t = 0;
    int hi = rq.tiles;  // before(t) <= u0, and u0 < before(hi) or hi is behind the last
    while (hi - t > 1) {
      const int mid = t + (hi - t) / 2;
      if (rq.before(a, mid) <= u0) t = mid;
      else hi = mid;
    }
    u0 -= rq.before(a, t);
    span(a);
    return true;
  }
  __device__ __forceinline__ void span(const PagedArgs& a) {
    units = rq.units(a, t);
    u1 = u0 + (x1 - x) < units ? u0 + (x1 - x) : units;
  }
  // On to the next tile; false: the part is done.
  __device__ __forceinline__ bool next(const PagedArgs& a) {
    x += u1 - u0;
    if (x >= x1) return false;
    u0 = 0;
    if (++t >= rq.tiles) {
      t = 0;
      if (++h >= a.Hkv) {
        h = 0;
        do {
          if (++r >= a.R) return false;
          rq = Req<TM, FW, NR>(a, r);
        } while (rq.tiles == 0);
      }
    }
    span(a);
    return true;
  }
  // This part's share [b0, b1) of the tile's nb blocks of keys. Parts that meet agree on the block between them: it is
  // the same expression of the same unit, does not fall where the unit grows, and is nb at most.
  __device__ __forceinline__ void blocks(int nb, int& b0, int& b1) const {
    b0 = u0 == 0 ? 0 : (int)((double)nb * (double)u0 / (double)units);
    b1 = u1 == units ? nb : (int)((double)nb * (double)u1 / (double)units);
  }
  __device__ __forceinline__ bool whole() const { return u0 == 0 && u1 == units; }
  __device__ __forceinline__ int64_t slot() const { return 2 * (int64_t)lw + (u0 > 0 ? 0 : 1); }
  // The first of a cut tile's parts says so (one thread).
  __device__ __forceinline__ void describe(const PagedArgs& a, int rows, int row0) const {
    if (whole() || u0 > 0) return;
    const int64_t end = x + units;
    int lo = lw, hi = cut.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (cut.start(mid) < end) lo = mid;
      else hi = mid;
    }
    a.desc[lw] = PartDesc{rows, row0, rq.first, h, lo, {0, 0, 0}};
  }
};

}  // namespace lh

// Launchers of the kernels (one for each variant of rows a tile), and of the joining of parts.
struct PagedVariant {
  int64_t W;
  int TM;
  void (*launch)(const lh::PagedArgs& a, hipStream_t st);
};
PagedVariant lh_paged_rows_variant(const LhPaged& s, int64_t rows);  // by the rows of a request
PagedVariant lh_paged_tile_variant(const LhPaged& s, int waves);    // waves of 32 rows: 4, 8 or 12 (bf16)
