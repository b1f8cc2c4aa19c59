// Entry point of the attention over a cache held in 8 bits.
#include "attend8.h"
#include "attend_plan.h"

namespace slh {

// As ATTEND_COSTS, for the kernels of 8-bit keys: steps of 16 and of 32 rows against few keys take less than those of 16-bit keys,
// whose loads they wait for.  us a call by the costs of 16-bit keys and by these:
//   8 sequences, prefix 1000, own 100, 28 / 4 heads          18.3   12.6 (in front of each sequence's own keys)
//   2, 40 new tokens each, own 4000, 40 / 8                   29.3   25.8 (blocks of 32 rows, not 128)
//   32, 5 new tokens, own 1500, 28 / 4                        20.6   18.1 (32, not 16)
//   8, own 8000, 28 / 4                                       17.9   16.3
// 13 other shapes (1 to 256 sequences): 0.93 to 1.02 of the time.  Against every choice of rows and splits in turn, on ten shapes, the
// plan's time is 1.06 of the best at most.
static const AttendCost ATTEND8_COSTS[3] = {
    {16, 1.8, 0.5, 0.63, 0.33}, {32, 2.5, 0.5, 0.65, 0.4}, {AT_ROWS, 3.0, 1.13, 1.75, 0.95}};
static const AttendKind ATTEND_8 = {ATTEND8_COSTS, 3, 1.0};

static bool attend8_sizes_ok(int B, int n_q, int Hq, int Hkv, int d, int64_t max_len, int64_t prefix_len) {
  return attend_common_ok(SLH_BF16, B, Hq, Hkv, d, 1.0) && attend_paged_ok(B, n_q, Hq / Hkv, max_len, prefix_len);
}

}  // namespace slh

extern "C" {

int64_t slh_attend_paged_e4m3_workspace(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d, int64_t max_len,
                                        int64_t prefix_len) {
  using namespace slh;
  if (!attend8_sizes_ok(B, n_q, Hq, Hkv, d, max_len, prefix_len)) return SLH_EINVAL;
  return attend_plan_paged(B, n_q, Hq, Hkv, d, max_len, prefix_len, ATTEND_8).bytes;
}

int slh_attend_paged_e4m3(const void* q, int64_t q_st, int64_t q_sh, const void* k_cache, const void* v_cache,
                          const void* k_scale, const void* v_scale, int32_t dtype, int64_t n_pages, int32_t page_size,
                          int32_t block, int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d,
                          const int32_t* page_table, int64_t ld_pages, int32_t max_pages, const int32_t* lens,
                          const int32_t* prefix_pages, int64_t prefix_len, double scale, void* out, int64_t o_st,
                          int64_t o_sh, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  const int g = Hq / Hkv;
  if (!c8_sizes_ok(n_pages, page_size, Hkv, block)) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || !attend_paged_ok(B, n_q, g, (int64_t)max_pages * page_size, prefix_len))
    return SLH_EINVAL;
  if (B == 0 || n_q == 0) return SLH_OK;
  if (!attend_rows_ok(q, q_st, q_sh) || !attend_rows_ok(out, o_st, o_sh) || !attend_rows_ok(k_cache, 0, 0) ||
      !attend_rows_ok(v_cache, 0, 0) || !k_scale || !v_scale || !lens || (max_pages > 0 && !page_table) ||
      (prefix_len > 0 && !prefix_pages))
    return SLH_EINVAL;
  Attend8Args x = {};
  AttendArgs& a = x.a;
  a.q = (const uint16_t*)q, a.q_st = q_st, a.q_sh = q_sh;
  a.k = (const uint16_t*)k_cache, a.v = (const uint16_t*)v_cache;
  x.held = AtHeld{(const uint8_t*)k_scale, (const uint8_t*)v_scale, __builtin_ctz((unsigned)block)};
  a.out = (uint16_t*)out, a.o_st = o_st, a.o_sh = o_sh, a.lse = lse;
  a.Hq = Hq, a.Hkv = Hkv, a.g = g, a.c = (float)(scale * 1.4426950408889634), a.scale = (float)scale, a.B = B, a.causal = 1;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_pages = max_pages, a.lens = lens;
  a.prefix_pages = prefix_pages, a.n_q = n_q, a.prefix_len = (int)prefix_len;
  a.n_pages = (int)n_pages, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.rows = (int64_t)B * n_q * Hq;
  const AttendPlan p = attend_plan_paged(B, n_q, Hq, Hkv, d, (int64_t)max_pages * page_size, prefix_len, ATTEND_8);
  if (p.bytes && (!workspace || ((uintptr_t)workspace) % 16 != 0 || workspace_bytes < p.bytes)) return SLH_EINVAL;
  const int64_t own = p.own.tiles * p.own.splits * Hkv, pre = p.pre.tiles * p.pre.splits * Hkv;
  if (own + pre > AT_BLOCKS - 64) return SLH_EINVAL;
  if (p.bytes) {
    a.part_o = (float*)workspace;
    a.part_ml = a.part_o + p.slots * a.rows * d;
  }
  a.splits = p.own.splits;
  a.pre_splits = p.pre.tiles ? p.pre.splits : 0;
  a.by_heads = at_divisor(Hkv);
  a.by_splits = at_divisor(a.splits);
  a.by_pre_splits = at_divisor(std::max(1, a.pre_splits));
  a.pre_tiles = (int)p.pre.tiles;
  a.chain = p.chain;
  const bool bf16 = dtype == SLH_BF16;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  auto go = [&](int rows, int64_t blocks) {
    return rows == AT_ROWS ? launch_tiles8(x, bf16, d, blocks, s) : launch_rows8(x, bf16, rows, d, blocks, s);
  };
  hipError_t e;
  if (pre && p.pre.rows == AT_ROWS && p.own.rows != AT_ROWS) {
    e = launch_both8(x, bf16, p.own.rows, d, pre, pre + own, s);
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

}  // extern "C"
