// k_paged.hip -- the bookkeeping of a serving step over a paged K/V cache: block tables, slot maps and
// positions from the requests' lengths (page_plan_kernel), and the new K and V rows into their
// slots (page_write_kernel).
#include "lh_paged.h"

namespace lh {

__device__ __forceinline__ int64_t blocks_of(int64_t tokens, int shift) {
  return (tokens + ((int64_t)1 << shift) - 1) >> shift;
}

struct PlanArgs {
  const int32_t *cached, *fresh, *free_pages, *n_free;
  int32_t *table, *cu_q, *kv_len, *slots, *pos, *balance, *n_taken;
  int64_t T, pages;
  int32_t R, max_blocks, shift;
};

// One launch. A page's place in the free list follows from two running sums over the requests (tokens,
// pages), and a token's request from a search in the first of them; both fit a workgroup's LDS, so
// every workgroup forms the sums for itself (R lengths, which the caches hold) and then maps
// its own range of tokens, and nothing waits for another workgroup. The table entry of a new page is
// written by its first token, which is always one of the step's.
// Bound by the latency of the launch and of the two scans: 64 requests of one token 4.0 us, 256 of 203,000 tokens 5.7.
constexpr int kPlanThreads = 256;  // a token a thread: with four, 203,000 tokens of 256 requests take 7.7 us and not 5.7

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanArgs a) {
  extern __shared__ int32_t lds[];
  __shared__ int64_t part[kPlanThreads / 64];
  __shared__ int64_t most[kPlanThreads / 64][2];
  int32_t* const cu = lds;             // [R + 1] first row of every request, clipped at T
  int32_t* const base = lds + a.R + 1;  // [R] pages handed out before the request; -1: it waits
  const int tid = threadIdx.x;
  int64_t n_free = a.n_free[0];
  n_free = n_free < 0 ? 0 : n_free > a.pages ? a.pages : n_free;
  int64_t rows = 0, pages = 0;  // sums up to the last chunk of requests
  int64_t taken = 0, asked = 0;  // pages handed out, and asked for by requests up to the last admitted one
  if (tid == 0) cu[0] = 0;
  for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
    const int r = r0 + tid;
    const bool real = r < a.R;
    const int64_t c = real ? a.cached[r] : 0, f = real ? a.fresh[r] : 0;
    const int64_t end = block_scan<kPlanThreads>(f > 0 ? f : 0, rows, part);
    const int64_t all = blocks_of(c + f, a.shift);
    const bool fits = real && c >= 0 && f >= 0 && all <= a.max_blocks && end <= a.T;
    const int64_t need = fits ? all - blocks_of(c, a.shift) : 0;
    const int64_t upto = block_scan<kPlanThreads>(need, pages, part);
    const bool ok = fits && (need == 0 || upto <= n_free);
    if (ok && need > 0) taken = upto;  // (grows with r)
    if (ok) asked = upto;
    if (real) {
      cu[r + 1] = (int32_t)(end < a.T ? end : a.T);
      base[r] = ok ? (int32_t)(need == 0 ? 0 : upto - need) : -1;
      if (blockIdx.x == 0) a.kv_len[r] = ok ? (int32_t)(c + f) : 0;
    }
    // the last thread's sums are the chunk's
    if (tid == kPlanThreads - 1) part[0] = end, part[1] = upto;
    __syncthreads();
    rows = part[0], pages = part[1];
    __syncthreads();
  }
  if (blockIdx.x == 0) {
    for (int r = tid; r <= a.R; r += kPlanThreads) a.cu_q[r] = cu[r];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const int64_t y = __shfl_xor(taken, d, 64), z = __shfl_xor(asked, d, 64);
      taken = taken > y ? taken : y, asked = asked > z ? asked : z;
    }
    if ((tid & 63) == 0) most[tid >> 6][0] = taken, most[tid >> 6][1] = asked;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < kPlanThreads / 64; ++i) {
        taken = taken > most[i][0] ? taken : most[i][0];
        asked = asked > most[i][1] ? asked : most[i][1];
      }
      const int64_t balance = n_free - asked;
      a.balance[0] = (int32_t)(balance < INT32_MIN ? INT32_MIN : balance);
      if (a.n_taken) a.n_taken[0] = (int32_t)taken;
    }
  }
  const int32_t total = cu[a.R];
  for (int64_t t = (int64_t)blockIdx.x * kPlanThreads + tid; t < a.T; t += (int64_t)gridDim.x * kPlanThreads) {
    int32_t slot = -1, pos = -1;
    if (t < total) {
      int lo = 0, hi = a.R;  // cu[lo] <= t < cu[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
      }
      const int32_t b = base[lo];
      if (b >= 0) {
        const int32_t c = a.cached[lo];
        pos = c + (int32_t)(t - cu[lo]);
        const int32_t block = pos >> a.shift, first = (int32_t)blocks_of(c, a.shift);
        int32_t* const entry = a.table + (int64_t)lo * a.max_blocks + block;
        int32_t id;
        if (block >= first) {
          id = a.free_pages[n_free - 1 - (b + block - first)];
          if ((pos & ((1 << a.shift) - 1)) == 0) *entry = id;
        } else {
          id = *entry;
        }
        if (id >= 0 && id < a.pages) slot = (id << a.shift) + (pos & ((1 << a.shift) - 1));
      }
    }
    a.slots[t] = slot;
    a.pos[t] = pos;
  }
}

// A thread moves one 16-byte chunk of a K row and the same chunk of the V row. Rows of a head are
// 128 to 512 consecutive bytes on both sides, so a wave reads and writes whole lines. Bound by
// HBM: each row is read and written once (24,548 tokens of 8 heads of 128 in bf16, 201 MB: 33 us, 6.0 TB/s; one
// token of each of 64 requests 2.6 us, the launch).
__global__ void __launch_bounds__(256)
page_write_kernel(const char* __restrict__ k, int64_t k_stride, const char* __restrict__ v, int64_t v_stride,
                  const int32_t* __restrict__ slots, char* __restrict__ kp, char* __restrict__ vp, uint32_t rows,
                  uint32_t Hkv, int32_t cshift, int32_t shift, int64_t n_slots) {
  const uint64_t chunks = (uint64_t)rows << cshift;
  const int32_t cmask = (1 << cshift) - 1, rb = 16 << cshift;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (uint64_t)gridDim.x * 256) {
    const uint32_t row = (uint32_t)(i >> cshift);
    const int32_t c = ((int32_t)i & cmask) * 16;
    const uint32_t t = row / Hkv, h = row - t * Hkv;
    const int32_t slot = slots[t];
    if (slot < 0 || slot >= n_slots) continue;
    const u32x4 x = load16_nt(k + (int64_t)t * k_stride + (int64_t)h * rb + c);
    const u32x4 y = load16_nt(v + (int64_t)t * v_stride + (int64_t)h * rb + c);
    const int64_t page = slot >> shift, in = slot & ((1 << shift) - 1);
    const int64_t to = (((page * Hkv + h) << shift) + in) * rb + c;
    *reinterpret_cast<u32x4*>(kp + to) = x;
    *reinterpret_cast<u32x4*>(vp + to) = y;
  }
}

}  // namespace lh

using namespace lh;

hipError_t lh_launch_page_plan(const LhPaged& s, const int32_t* cached, const int32_t* fresh,
                               const int32_t* free_pages, const int32_t* n_free, int32_t* table, int32_t* cu_q,
                               int32_t* kv_len, int32_t* slots, int32_t* pos, int32_t* balance, int32_t* n_taken,
                               hipStream_t st) {
  const PlanArgs a{cached, fresh, free_pages, n_free, table, cu_q, kv_len, slots, pos, balance, n_taken,
                   s.T, s.pages, s.R, s.max_blocks, s.shift};
  int64_t blocks = (s.T + kPlanThreads - 1) / kPlanThreads;
  if (blocks > 2048) blocks = 2048;
  hipLaunchKernelGGL(page_plan_kernel, dim3((unsigned)blocks), dim3(kPlanThreads), (2 * (size_t)s.R + 1) * 4, st, a);
  return hipGetLastError();
}

hipError_t lh_launch_page_write(const LhPaged& s, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                const int32_t* slots, void* kpages, void* vpages, hipStream_t st) {
  const int es = s.dtype == LH_BF16 ? 2 : 4;
  int cshift = 0;
  while ((16 << cshift) < s.D * es) ++cshift;
  const int64_t rows = s.T * s.Hkv, chunks = rows << cshift;
  int64_t blocks = (chunks + 255) / 256;
  if (blocks > (1 << 20)) blocks = 1 << 20;
  hipLaunchKernelGGL(page_write_kernel, dim3((unsigned)blocks), dim3(256), 0, st, (const char*)k, k_stride * es,
                     (const char*)v, v_stride * es, slots, (char*)kpages, (char*)vpages, (uint32_t)rows,
                     (uint32_t)s.Hkv, cshift, s.shift, s.pages << s.shift);
  return hipGetLastError();
}
