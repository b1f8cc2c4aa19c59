// Entry points of the attention operators.
#include "attend_plan.h"

namespace slh {

// The launches of a plan: the prefix and the own keys in one where the same kernel takes both.
static int attend_run(AttendArgs& a, const AttendPlan& p, bool paged, bool bf16, int d, void* ws, int64_t ws_bytes,
                      hipStream_t s) {
  if (p.bytes && (!ws || ((uintptr_t)ws) % 16 != 0 || ws_bytes < p.bytes)) return SLH_EINVAL;
  const int64_t own = p.own.tiles * p.own.splits * a.Hkv, pre = p.pre.tiles * p.pre.splits * a.Hkv;
  if (own + pre > AT_BLOCKS - 64) return SLH_EINVAL;
  if (p.bytes) {
    a.part_o = (float*)ws;
    a.part_ml = a.part_o + p.slots * a.rows * d;
  }
  a.splits = p.own.splits;
  a.pre_splits = p.pre.tiles ? p.pre.splits : 0;
  a.by_heads = at_divisor(a.Hkv);
  a.by_splits = at_divisor(a.splits);
  a.by_pre_splits = at_divisor(std::max(1, a.pre_splits));
  auto go = [&](int rows, int64_t blocks) {
    return rows >= AT_ROWS / 2 ? launch_attend_tiles(a, paged, bf16, rows, d, blocks, s)
                               : launch_attend_rows(a, paged, bf16, rows, d, blocks, s);
  };
  (void)hipGetLastError();
  a.pre_tiles = (int)p.pre.tiles;
  a.chain = p.chain;
  hipError_t e;
  if (pre && p.pre.rows == AT_ROWS && p.own.rows != AT_ROWS) {
    e = launch_attend_both(a, bf16, p.own.rows, d, pre, pre + own, s);
  } else if (pre && p.pre.rows != p.own.rows) {
    e = go(p.pre.rows, pre);
    if (e != hipSuccess) return SLH_EHIP;
    a.pre_tiles = 0;
    e = go(p.own.rows, own);
  } else {
    e = go(p.own.rows, pre + own);
  }
  if (e == hipSuccess && p.bytes) e = launch_attend_join(a, bf16, d, p.slots, s);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // namespace slh

extern "C" {

int64_t slh_attend_workspace(int64_t Tq, int64_t Tk, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                             int32_t causal) {
  using namespace slh;
  if (!attend_common_ok(SLH_BF16, B, Hq, Hkv, d, 1.0) || !attend_packed_ok(Tq, Tk, Hq / Hkv)) return SLH_EINVAL;
  return attend_plan_packed(Tq, Tk, B, Hq, Hkv, d, causal != 0).bytes;
}

int slh_attend(const void* q, int64_t q_st, int64_t q_sh, const void* k, int64_t k_st, int64_t k_sh,
               const void* v, int64_t v_st, int64_t v_sh, int32_t dtype, int64_t Tq, int64_t Tk,
               int32_t B, int32_t Hq, int32_t Hkv, int32_t d, const int32_t* cu_q,
               const int32_t* cu_k, double scale, int32_t causal, void* out, int64_t o_st,
               int64_t o_sh, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  const int g = Hq / Hkv;
  if (!attend_packed_ok(Tq, Tk, g)) return SLH_EINVAL;
  if (B == 0 || Tq == 0) return SLH_OK;
  if (!attend_rows_ok(q, q_st, q_sh) || !attend_rows_ok(out, o_st, o_sh) || !cu_q || !cu_k) return SLH_EINVAL;
  if (Tk > 0 && !(attend_rows_ok(k, k_st, k_sh) && attend_rows_ok(v, v_st, v_sh))) return SLH_EINVAL;
  AttendArgs a = {};
  a.q = (const uint16_t*)q, a.q_st = q_st, a.q_sh = q_sh;
  a.k = (const uint16_t*)k, a.k_st = k_st, a.k_sh = k_sh;
  a.v = (const uint16_t*)v, a.v_st = v_st, a.v_sh = v_sh;
  a.out = (uint16_t*)out, a.o_st = o_st, a.o_sh = o_sh, a.lse = lse;
  a.Hq = Hq, a.Hkv = Hkv, a.g = g, a.c = (float)(scale * 1.4426950408889634), a.scale = (float)scale, a.B = B, a.causal = causal != 0;
  a.cu_q = cu_q, a.cu_k = cu_k, a.Tq = Tq, a.Tk = Tk;
  a.rows = Tq * Hq;
  return attend_run(a, attend_plan_packed(Tq, Tk, B, Hq, Hkv, d, causal != 0), false, dtype == SLH_BF16, d, workspace,
                    workspace_bytes, (hipStream_t)stream);
}

int64_t slh_attend_paged_workspace(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d,
                                   int64_t max_len, int64_t prefix_len) {
  using namespace slh;
  if (!attend_common_ok(SLH_BF16, B, Hq, Hkv, d, 1.0) || !attend_paged_ok(B, n_q, Hq / Hkv, max_len, prefix_len))
    return SLH_EINVAL;
  return attend_plan_paged(B, n_q, Hq, Hkv, d, max_len, prefix_len).bytes;
}

int slh_attend_paged(const void* q, int64_t q_st, int64_t q_sh, const void* k_cache,
                     const void* v_cache, int32_t dtype, int64_t n_pages, int32_t page_size,
                     int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d,
                     const int32_t* page_table, int64_t ld_pages, int32_t max_pages,
                     const int32_t* lens, const int32_t* prefix_pages, int64_t prefix_len,
                     double scale, void* out, int64_t o_st, int64_t o_sh, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  const int g = Hq / Hkv;
  if (page_size < 1 || page_size > 65536 || (page_size & (page_size - 1))) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * Hkv > INT32_MAX / page_size) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages ||
      !attend_paged_ok(B, n_q, g, (int64_t)max_pages * page_size, prefix_len))
    return SLH_EINVAL;
  if (B == 0 || n_q == 0) return SLH_OK;
  if (!attend_rows_ok(q, q_st, q_sh) || !attend_rows_ok(out, o_st, o_sh) || !attend_rows_ok(k_cache, 0, 0) ||
      !attend_rows_ok(v_cache, 0, 0) || !lens || (max_pages > 0 && !page_table) || (prefix_len > 0 && !prefix_pages))
    return SLH_EINVAL;
  AttendArgs a = {};
  a.q = (const uint16_t*)q, a.q_st = q_st, a.q_sh = q_sh;
  a.k = (const uint16_t*)k_cache, a.v = (const uint16_t*)v_cache;
  a.out = (uint16_t*)out, a.o_st = o_st, a.o_sh = o_sh, a.lse = lse;
  a.Hq = Hq, a.Hkv = Hkv, a.g = g, a.c = (float)(scale * 1.4426950408889634), a.scale = (float)scale, a.B = B, a.causal = 1;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_pages = max_pages, a.lens = lens;
  a.prefix_pages = prefix_pages, a.n_q = n_q, a.prefix_len = (int)prefix_len;
  a.n_pages = (int)n_pages, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.rows = (int64_t)B * n_q * Hq;
  return attend_run(a, attend_plan_paged(B, n_q, Hq, Hkv, d, (int64_t)max_pages * page_size, prefix_len), true,
                    dtype == SLH_BF16, d, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
