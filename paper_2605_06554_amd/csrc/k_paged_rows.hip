// k_paged_rows.hip -- attention over a paged cache for requests of few rows (decoding, drafts) and for fp32: tiles
// of 16 or 32 rows (lh_paged_rows.h), workgroups of four waves, two of them a CU: 8 waves keep enough loads in
// flight (64 requests, 482,000 keys: 312 us with 8 waves a CU, 325 with 12, 327 with 4), and workgroups of their own
// keep loading while one joins its waves (12 waves in one workgroup: 372 us where four took 352).
#include "lh_paged_rows.h"

namespace lh {

constexpr int kRowsNW = 4, kRowsEU = 2;  // waves, and workgroups a CU
constexpr int64_t kRowsW = kCUs * kRowsEU;

template <int D>
struct RowsLds {
  static constexpr int PER = kRowsNW;
  static constexpr bool kOwnWords = true;
  float (*parts)[16 * D], (*stat)[16];
  __device__ __forceinline__ float* part(int w) const { return parts[w]; }
  __device__ __forceinline__ float* words(int w) const { return parts[w]; }
  __device__ __forceinline__ float* ms(int w) const { return stat[w]; }
  __device__ __forceinline__ float* ls(int w) const { return stat[kRowsNW + w]; }
};

// NT: K and V are loaded with the non-temporal hint.
template <typename T, int D, int RT, bool NT>
__global__ void __launch_bounds__(64 * kRowsNW, kRowsEU) paged_rows(const PagedArgs a) {
  constexpr int TM = 16 * RT, KB = RowsCfg<T, D, RT>::KB;
  __shared__ __align__(16) float parts[kRowsNW][16 * D];
  __shared__ float stat[2 * kRowsNW][16];
  __shared__ int64_t scan[kRowsNW];
  __shared__ typename Walk<TM, 16>::Found found;
  Walk<TM, 16> wk;
  if (!wk.template begin<64 * kRowsNW>(a, scan, &found)) return;
  do {
    RowsItem it;
    it.first = uni(wk.rq.first), it.base = uni(wk.rq.base), it.all_rows = uni(wk.rq.rows);
    it.r = uni(wk.r), it.h = uni(wk.h), it.row0 = uni(wk.t) * TM;
    it.rows = it.all_rows - it.row0 < TM ? it.all_rows - it.row0 : TM;
    it.keys = uni(it.base + (it.row0 + it.rows - 1) / a.G + 1);
    it.safe = uni(it.base + it.row0 / a.G + 1);
    int b0, b1;
    wk.blocks(it.keys > 0 ? (it.keys + KB - 1) / KB : 0, b0, b1);
    it.b0 = uni(b0), it.b1 = uni(b1);
    it.whole = wk.whole(), it.slot = wk.slot();
    rows_tile<T, D, RT, kRowsNW, NT, TM>(a, it, RowsLds<D>{parts, stat});
    if (threadIdx.x == 0) wk.describe(a, it.rows, it.row0);
    __syncthreads();  // the parts were read
  } while (wk.next(a));
}

template <typename T, int D, int RT, bool NT>
static PagedVariant variant() {
  return {kRowsW, 16 * RT, [](const PagedArgs& a, hipStream_t st) {
            hipLaunchKernelGGL((paged_rows<T, D, RT, NT>), dim3((unsigned)kRowsW), dim3(256), 0, st, a);
          }};
}
// A request of one tile reads its keys once, and the non-temporal hint is worth 8% of the time (6.1 against 5.6
// TB/s, 64 requests of 482,000 keys); one of several finds them in the caches (four tiles, fp32: 60 us, 67 with the hint).
// fp32 takes 32 rows a tile above 16 whatever the number of tiles: 39 us where 16 rows take 42 (8 requests of 16 tokens at 4000,
// 8 heads on 2), 69 and 70 (16 of 40 at 1000, 8 on 8); few and short ones lose by it, 30 and 20 (3 of 12 at 2200, 8 on 2).
// At D = 128 it spills 16 registers, outside the loop over the keys.
template <typename T, int D>
static PagedVariant variant(int64_t rows) {
  return rows > 32 ? variant<T, D, 2, false>() : rows > 16 ? variant<T, D, 2, true>() : variant<T, D, 1, true>();
}

}  // namespace lh

PagedVariant lh_paged_rows_variant(const LhPaged& s, int64_t rows) {
  if (s.dtype == LH_BF16) return s.D == 128 ? lh::variant<lh::bf16_t, 128>(rows) : lh::variant<lh::bf16_t, 64>(rows);
  return s.D == 128 ? lh::variant<float, 128>(rows) : lh::variant<float, 64>(rows);
}
