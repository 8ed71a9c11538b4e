// api_paged.cpp -- host side of the paged calls of the C ABI (include/lighthouse.h, serving):
// argument validation, workspace sizing and dispatch. Nothing is allocated and nothing synchronizes.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include "lh_paged.h"

namespace {

constexpr int64_t k2G = (int64_t)1 << 31, k1G = (int64_t)1 << 30;

lh_status make_paged(const lh_paged* pc, LhPaged* s) {
  if (!pc) return lh_fail(LH_E_NULL, "the step's description is NULL");
  if (pc->R < 1 || pc->R > kPagedMaxRequests)
    return lh_fail(LH_E_SHAPE, "R must be in [1, %d] (R=%d)", kPagedMaxRequests, pc->R);
  if (pc->T < 1 || pc->pages < 1 || pc->max_blocks < 1)
    return lh_fail(LH_E_SHAPE, "T, pages and max_blocks must be >= 1 (T=%lld, pages=%lld, max_blocks=%d)",
                   (long long)pc->T, (long long)pc->pages, pc->max_blocks);
  if (pc->page < 16 || pc->page > 1024 || (pc->page & (pc->page - 1)) != 0)
    return lh_fail(LH_E_PARAM, "page must be a power of two in [16, 1024] (page=%d)", pc->page);
  if (pc->Hq < 1 || pc->Hkv < 1 || pc->Hq % pc->Hkv != 0)
    return lh_fail(LH_E_PARAM, "need Hq >= 1, Hkv >= 1 and Hq %% Hkv == 0 (Hq=%d, Hkv=%d)", pc->Hq, pc->Hkv);
  if (pc->D != 64 && pc->D != 128) return lh_fail(LH_E_PARAM, "head dim D must be 64 or 128 (D=%d)", pc->D);
  if (pc->dtype != LH_F32 && pc->dtype != LH_BF16)
    return lh_fail(LH_E_DTYPE, "dtype must be LH_F32 or LH_BF16 (%d)", pc->dtype);
  if (isnan(pc->scale) || isinf(pc->scale)) return lh_fail(LH_E_NONFINITE, "scale must be finite (0 selects 1/sqrt(D))");
  if (pc->scale < 0.0f) return lh_fail(LH_E_PARAM, "scale must be >= 0 (0 selects 1/sqrt(D))");
  if (pc->pages >= k2G / pc->page)
    return lh_fail(LH_E_SHAPE, "the cache has %lld * %d >= 2^31 slots", (long long)pc->pages, pc->page);
  // (the kernels count a request's keys and rows in 32 bits, and look up to a tile further)
  if (pc->max_blocks > k1G / pc->page)
    return lh_fail(LH_E_SHAPE, "a request could hold %d * %d > 2^30 tokens", pc->max_blocks, pc->page);
  if (pc->T > k1G / pc->Hq) return lh_fail(LH_E_SHAPE, "T * Hq = %lld * %d > 2^30", (long long)pc->T, pc->Hq);
  // The units of the cut of an attention's work (lh_paged_sdpa.h: Req) are counted in 64 bits, whatever cu_q and kv_len
  // hold, each request clipped into [0, T) rows of its own: tiles of 16 rows and up, and a tile's keys, which for the
  // G > 16 heads of a group grow by one a tile and not one a token.
  const int64_t G = pc->Hq / pc->Hkv, grow = pc->T * ((G + 15) / 16);
  const unsigned __int128 units = (unsigned __int128)pc->R * (uint64_t)(pc->T * pc->Hq + 16 * (int64_t)pc->Hkv) *
                                  (uint64_t)((int64_t)pc->max_blocks * pc->page + grow + 1024);
  if (units > ((unsigned __int128)1 << 62))
    return lh_fail(LH_E_SHAPE, "R * (T * Hq + 16 * Hkv) * (max_blocks * page + T * ceil(Hq / Hkv / 16) + 1024) is above 2^62");
  memset(s, 0, sizeof(*s));
  s->T = pc->T, s->pages = pc->pages, s->R = pc->R, s->max_blocks = pc->max_blocks, s->page = pc->page;
  while ((1 << s->shift) < s->page) ++s->shift;
  s->Hq = pc->Hq, s->Hkv = pc->Hkv, s->D = pc->D, s->G = pc->Hq / pc->Hkv;
  s->dtype = pc->dtype;
  s->scale = pc->scale != 0.0f ? pc->scale : (float)(1.0 / sqrt((double)pc->D));
  return LH_OK;
}

lh_status need(const void* p, const char* name, unsigned align) {
  if (!p) return lh_fail(LH_E_NULL, "%s is NULL", name);
  if (((uintptr_t)p & (align - 1)) != 0) return lh_fail(LH_E_ALIGN, "%s is not %u-byte aligned", name, align);
  return LH_OK;
}

// A stride between tokens of H heads, in elements.
lh_status need_stride(const LhPaged& s, int64_t stride, int32_t H, const char* name) {
  if (stride < (int64_t)H * s.D) return lh_fail(LH_E_SHAPE, "%s = %lld is less than %d * %d", name, (long long)stride, H, s.D);
  if (stride % (s.dtype == LH_BF16 ? 8 : 4) != 0)
    return lh_fail(LH_E_ALIGN, "%s = %lld elements is not a multiple of 16 bytes", name, (long long)stride);
  if (stride > ((int64_t)1 << 40)) return lh_fail(LH_E_SHAPE, "%s = %lld is out of range", name, (long long)stride);
  return LH_OK;
}

// An array of a call, in bytes. (No size is within 64 bits for all bounds that pass the checks.)
typedef unsigned __int128 u128;
struct Span {
  const char* name;
  const void* at;
  u128 bytes;
};
u128 rows_bytes(const LhPaged& s, int64_t stride, int32_t H) {
  return ((u128)(s.T - 1) * (uint64_t)stride + (uint64_t)H * s.D) * (s.dtype == LH_BF16 ? 2 : 4);
}
u128 pool_bytes(const LhPaged& s) {
  return (u128)(uint64_t)(s.pages * s.page) * (uint64_t)((int64_t)s.Hkv * s.D * (s.dtype == LH_BF16 ? 2 : 4));
}
// The last `n_out` of the arrays are written: none of them may share memory with another array. (Workgroups read
// the inputs while others write.)
template <int N>
lh_status need_apart(const Span (&x)[N], int n_out) {
  for (int i = N - n_out; i < N; ++i) {
    if (!x[i].at) continue;
    for (int j = 0; j < i; ++j) {
      const uintptr_t a = (uintptr_t)x[i].at, b = (uintptr_t)x[j].at;
      if (b && (u128)a < b + x[j].bytes && (u128)b < a + x[i].bytes)
        return lh_fail(LH_E_PARAM, "%s and %s overlap", x[j].name, x[i].name);
    }
  }
  return LH_OK;
}

lh_status status(hipError_t e, const char* what) {
  if (e == hipSuccess) return LH_OK;
  return lh_fail(LH_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define LH_TRY(x)                   \
  do {                              \
    lh_status _st = (x);            \
    if (_st != LH_OK) return _st;   \
  } while (0)

}  // namespace

extern "C" {

lh_status lh_paged_check(const lh_paged* pc) {
  LhPaged s;
  return make_paged(pc, &s);
}

lh_status lh_paged_workspace_bytes(const lh_paged* pc, size_t* bytes) {
  LhPaged s;
  LH_TRY(make_paged(pc, &s));
  if (!bytes) return lh_fail(LH_E_NULL, "bytes is NULL");
  *bytes = lh_sdpa_paged_ws_bytes(s);
  return LH_OK;
}

lh_status lh_page_plan(const lh_paged* pc, const int32_t* cached, const int32_t* fresh, const int32_t* free_pages,
                       const int32_t* n_free, int32_t* table, int32_t* cu_q, int32_t* kv_len, int32_t* slots,
                       int32_t* pos, int32_t* balance, int32_t* n_taken, void* stream) {
  LhPaged s;
  LH_TRY(make_paged(pc, &s));
  LH_TRY(need(cached, "cached", 4));
  LH_TRY(need(fresh, "fresh", 4));
  LH_TRY(need(free_pages, "free_pages", 4));
  LH_TRY(need(n_free, "n_free", 4));
  LH_TRY(need(table, "table", 4));
  LH_TRY(need(cu_q, "cu_q", 4));
  LH_TRY(need(kv_len, "kv_len", 4));
  LH_TRY(need(slots, "slots", 4));
  LH_TRY(need(pos, "pos", 4));
  LH_TRY(need(balance, "balance", 4));
  if (n_taken) LH_TRY(need(n_taken, "n_taken", 4));
  const u128 R = 4 * (u128)s.R, T = 4 * (u128)s.T;
  LH_TRY(need_apart({{"cached", cached, R}, {"fresh", fresh, R}, {"free_pages", free_pages, 4 * (u128)s.pages},
                     {"n_free", n_free, 4}, {"table", table, R * s.max_blocks}, {"cu_q", cu_q, R + 4},
                     {"kv_len", kv_len, R}, {"slots", slots, T}, {"pos", pos, T}, {"balance", balance, 4},
                     {"n_taken", n_taken, 4}}, 7));
  lh_fail(LH_OK, "%s", "");
  return status(lh_launch_page_plan(s, cached, fresh, free_pages, n_free, table, cu_q, kv_len, slots, pos, balance,
                                    n_taken, (hipStream_t)stream),
                "lh_page_plan");
}

lh_status lh_page_write(const lh_paged* pc, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                        const int32_t* slots, void* kpages, void* vpages, void* stream) {
  LhPaged s;
  LH_TRY(make_paged(pc, &s));
  LH_TRY(need(k, "k", 16));
  LH_TRY(need_stride(s, k_stride, s.Hkv, "k_stride"));
  LH_TRY(need(v, "v", 16));
  LH_TRY(need_stride(s, v_stride, s.Hkv, "v_stride"));
  LH_TRY(need(slots, "slots", 4));
  LH_TRY(need(kpages, "kpages", 16));
  LH_TRY(need(vpages, "vpages", 16));
  LH_TRY(need_apart({{"k", k, rows_bytes(s, k_stride, s.Hkv)}, {"v", v, rows_bytes(s, v_stride, s.Hkv)},
                     {"slots", slots, 4 * (u128)s.T}, {"kpages", kpages, pool_bytes(s)}, {"vpages", vpages, pool_bytes(s)}}, 2));
  lh_fail(LH_OK, "%s", "");
  return status(lh_launch_page_write(s, k, k_stride, v, v_stride, slots, kpages, vpages, (hipStream_t)stream),
                "lh_page_write");
}

lh_status lh_sdpa_paged(const lh_paged* pc, const void* q, int64_t q_stride, const void* kpages, const void* vpages,
                        const int32_t* table, const int32_t* cu_q, const int32_t* kv_len, void* o, float* lse,
                        void* ws, size_t ws_bytes, void* stream) {
  LhPaged s;
  LH_TRY(make_paged(pc, &s));
  LH_TRY(need(q, "q", 16));
  LH_TRY(need_stride(s, q_stride, s.Hq, "q_stride"));
  LH_TRY(need(kpages, "kpages", 16));
  LH_TRY(need(vpages, "vpages", 16));
  LH_TRY(need(table, "table", 4));
  LH_TRY(need(cu_q, "cu_q", 4));
  LH_TRY(need(kv_len, "kv_len", 4));
  LH_TRY(need(o, "o", 16));
  if (lse) LH_TRY(need(lse, "lse", 4));
  const size_t bytes = lh_sdpa_paged_ws_bytes(s);
  if (bytes > 0) {
    if (!ws) return lh_fail(LH_E_WORKSPACE, "workspace is NULL (%zu bytes needed)", bytes);
    if (((uintptr_t)ws & 255u) != 0) return lh_fail(LH_E_ALIGN, "workspace is not 256-byte aligned");
    if (ws_bytes < bytes) return lh_fail(LH_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, bytes);
  }
  LH_TRY(need_apart({{"q", q, rows_bytes(s, q_stride, s.Hq)}, {"kpages", kpages, pool_bytes(s)},
                     {"vpages", vpages, pool_bytes(s)}, {"table", table, 4 * (u128)s.R * s.max_blocks},
                     {"cu_q", cu_q, 4 * (u128)s.R + 4}, {"kv_len", kv_len, 4 * (u128)s.R},
                     {"o", o, rows_bytes(s, (int64_t)s.Hq * s.D, s.Hq)}, {"lse", lse, 4 * (u128)s.T * s.Hq},
                     {"ws", ws, bytes}}, 3));
  lh_fail(LH_OK, "%s", "");
  return status(lh_launch_sdpa_paged(s, q, q_stride, kpages, vpages, table, cu_q, kv_len, o, lse, ws,
                                     (hipStream_t)stream),
                "lh_sdpa_paged");
}

}  // extern "C"
