// Entry points of the attention operators: what the host can check, which kernel takes which
// rows, and over how many blocks the keys are split.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "attend.h"

namespace slh {

// compute units of the current device (asked for once a device)
static int attend_cus() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Which kernel takes a set of rows, in how many pieces of its keys.
struct AttendPart {
  int rows;               // of a block: AT_ROWS (k_attend), 32 or 16 (k_attend_rows)
  int splits;
  int64_t tiles;          // row tiles of a key/value head, all sequences together
};
struct AttendPlan {
  AttendPart own, pre;    // of the packed or the sequences' own keys; of the prefix (tiles 0: none)
  int slots;              // partial results of a row (1: none are written)
  int64_t bytes;
};

// Key splits for `blocks` blocks over `keys` keys: two blocks a compute unit, each with `least` keys
// or more.
static int attend_splits(int64_t blocks, int64_t keys, int least, int n_cu) {
  const int64_t fill = 2 * (int64_t)n_cu / std::max<int64_t>(1, blocks);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(fill, keys / least), 64));
}

static void attend_finish(AttendPlan& p, int64_t rows, int d) {
  p.slots = p.own.splits + (p.pre.tiles ? p.pre.splits : 0);
  p.bytes = p.slots > 1 ? p.slots * rows * (4 * (int64_t)d + 8) : 0;
}

static AttendPlan attend_plan_packed(int64_t Tq, int64_t Tk, int B, int Hq, int Hkv, int d) {
  const int n_cu = attend_cus();
  const int64_t rows = Tq * (Hq / Hkv), keys = Tk / std::max(1, B);
  AttendPlan p = {};
  p.own.rows = AT_ROWS;
  // the tiles that there are at least; the keys of the average sequence
  auto sure = [&](int r) { return std::max<int64_t>(B, (rows + r - 1) / r) * Hkv; };
  if (sure(AT_ROWS) < n_cu && sure(32) * keys < (int64_t)4096 * n_cu) p.own.rows = rows * Hkv > 32 * n_cu ? 32 : 16;
  const int r = p.own.rows;
  p.own.tiles = rows / r + B;
  p.own.splits = attend_splits(sure(r), keys, r == AT_ROWS ? 4 * 64 : 256, n_cu);
  attend_finish(p, Tq * Hq, d);
  return p;
}

static AttendPlan attend_plan_paged(int B, int n_q, int Hq, int Hkv, int d, int64_t max_len, int64_t prefix_len) {
  const int n_cu = attend_cus(), g = Hq / Hkv;
  auto part = [&](int64_t rows, int64_t sets, int64_t keys) {
    AttendPart p;
    p.rows = rows <= 16 ? 16 : rows <= 64 ? 32 : AT_ROWS;
    p.tiles = sets * ((rows + p.rows - 1) / p.rows);
    p.splits = attend_splits(p.tiles * Hkv, keys, 256, n_cu);
    return p;
  };
  AttendPlan p = {};
  p.own = part((int64_t)n_q * g, B, max_len);
  if (prefix_len > 0) p.pre = part((int64_t)B * n_q * g, 1, prefix_len);
  attend_finish(p, (int64_t)B * n_q * Hq, d);
  return p;
}

// The launches of a plan: the prefix and the own keys in one where the same kernel takes both.
static int attend_run(AttendArgs& a, const AttendPlan& p, bool paged, bool bf16, int d, void* ws, int64_t ws_bytes,
                      hipStream_t s) {
  if (p.bytes && (!ws || ((uintptr_t)ws) % 16 != 0 || ws_bytes < p.bytes)) return SLH_EINVAL;
  const int64_t own = p.own.tiles * p.own.splits * a.Hkv, pre = p.pre.tiles * p.pre.splits * a.Hkv;
  if (own + pre > INT32_MAX / 256) return SLH_EINVAL;
  if (p.bytes) {
    a.part_o = (float*)ws;
    a.part_ml = a.part_o + p.slots * a.rows * d;
  }
  a.splits = p.own.splits;
  a.pre_splits = p.pre.tiles ? p.pre.splits : 0;
  auto go = [&](int rows, int64_t blocks) {
    return rows == AT_ROWS ? launch_attend_tiles(a, paged, bf16, d, blocks, s)
                           : launch_attend_rows(a, paged, bf16, rows, d, blocks, s);
  };
  (void)hipGetLastError();
  a.pre_tiles = (int)p.pre.tiles;
  hipError_t e;
  if (pre && p.pre.rows != p.own.rows) {
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

static bool attend_rows_ok(const void* p, int64_t st, int64_t sh) {
  return p && ((uintptr_t)p) % 16 == 0 && st >= 0 && st <= AT_STRIDE && sh >= 0 && st % 8 == 0 && sh % 8 == 0;
}

static bool attend_packed_ok(int64_t Tq, int64_t Tk, int g) {
  return Tq >= 0 && Tk >= 0 && Tk <= INT32_MAX / 2 && Tq <= INT32_MAX / 2 && Tq * g <= INT32_MAX / 2;
}
static bool attend_paged_ok(int B, int n_q, int g, int64_t max_len, int64_t prefix_len) {
  return n_q >= 0 && (int64_t)B * n_q <= INT32_MAX / 2 && (int64_t)B * n_q * g <= INT32_MAX / 2 && max_len >= 0 &&
         max_len <= INT32_MAX / 4 && prefix_len >= 0 && prefix_len <= INT32_MAX / 4;
}
static bool attend_common_ok(int dtype, int64_t B, int Hq, int Hkv, int d, double scale) {
  if (dtype != SLH_BF16 && dtype != SLH_F16) return false;
  if (d != 64 && d != 80 && d != 96 && d != 128) return false;
  if (Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hkv > 65535 || Hq / Hkv > 1024) return false;
  return B >= 0 && B <= (1 << 20) && scale > 0.0 && !std::isinf(scale);
}

}  // namespace slh

extern "C" {

int64_t slh_attend_workspace(int64_t Tq, int64_t Tk, int32_t B, int32_t Hq, int32_t Hkv, int32_t d) {
  using namespace slh;
  if (!attend_common_ok(SLH_BF16, B, Hq, Hkv, d, 1.0) || !attend_packed_ok(Tq, Tk, Hq / Hkv)) return SLH_EINVAL;
  return attend_plan_packed(Tq, Tk, B, Hq, Hkv, d).bytes;
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
  return attend_run(a, attend_plan_packed(Tq, Tk, B, Hq, Hkv, d), false, dtype == SLH_BF16, d, workspace,
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
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * Hkv > INT32_MAX / std::max(1, page_size) || page_size < 1 || page_size > 65536 || (page_size & (page_size - 1)))
    return SLH_EINVAL;
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
