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
  int rows;               // of a block: AT_ROWS or half of it (k_attend), 32 or 16 (k_attend_rows)
  int splits;
  int64_t tiles;          // row tiles of a key/value head, all sequences together
  double us;
};
struct AttendPlan {
  AttendPart own, pre;    // of the packed or the sequences' own keys; of the prefix (tiles 0: none for itself)
  bool chain;             // the prefix in front of each sequence's own keys, no part for itself
  int slots;              // partial results of a row (1: none are written)
  int64_t bytes;
};

// What a launch costs, in microseconds, as measured with d = 128 on 256 compute units.  A block goes
// through its keys 64 at a time: a tile of k_attend, or a step of each wave of k_attend_rows.  `start`:
// of a block, for finding its rows and keys, its first loads and its last stores (and ATTEND_LAUNCH of the launch);
// `one`: a block's 64 keys where it has a compute unit to itself; `pair`: where another block is beside
// it; `full`: a unit's 64 keys of one block with all units busy for several rounds (power and caches are shared then).
// Over 62 packed shapes (16 to 10000 tokens, 0 to 9000 keys in front) the plan's time is on average 1.02 of the best
// of all kernels and 1 to 32 splits, over 45 paged ones 1.04 (sequences of equal lengths, tables as wide as those).  One
// split, us, queries x context, heads:
//                            16 rows   32 rows   64 rows   128 rows
//   256 x 0, 28 / 4            7.3       9.0       8.8      10.4
//   512 x 0, 28 / 4           15.3      12.7      12.3      15.4
//   1024 x 0, 28 / 4                    29.6      21.8      25.2
//   1024 x 2000, 40 / 8                 112       82.0      76.0
//   3000 x 0, 28 / 4                    136       88.7      80.9
struct AttendCost { int rows; double start, one, pair, full; };
static const AttendCost ATTEND_COSTS[4] = {
    {16, 1.8, 0.65, 0.8, 0.33}, {32, 2.5, 0.75, 0.95, 0.42}, {AT_ROWS / 2, 2.6, 0.78, 1.1, 0.55}, {AT_ROWS, 3.0, 1.13, 1.75, 0.95}};
static const double ATTEND_LAUNCH = 4.0;
static const double ATTEND_SECOND = 2.3;         // of a second launch, where it is the host that is waited for
// Partial results: another pass over memory, the end of the blocks that write them, and a launch.
static double attend_join_us(int64_t slots, int64_t rows, int d) {
  return slots > 1 ? 3.0 + 0.1 * (double)slots + 1.35 * (double)(slots * rows) * (4.0 * d + 8.0) / 3.5e6 : 0.0;
}

// The kernel and the splits (at most max_splits) that cost least for `sets` runs of `rows` rows a key/value head
// against `keys` keys each, of which a row tile sees `mean` on average.  out_rows: rows of a partial result.  also: other partial results of a row; same: the kernel of a launch
// that this one would join.  ahead: keys of a prefix, the same for all runs, that each goes through first (k_attend_rows).
static AttendPart attend_part(int64_t rows, int64_t sets, int Hkv, int64_t keys, double mean, int64_t out_rows,
                              int d, int n_cu, int also, int same, bool paged, int max_splits, int64_t ahead = 0) {
  AttendPart best = {};
  best.us = INFINITY;
  best.rows = 16, best.splits = 1;
  // part of a block's time does not shrink with d: 4 heads of 64, 256 rows against 2256 keys, 0.79 us a tile of 128
  // rows, 0.57 of 64, 0.52 of 32
  const double work = 0.4 + 0.6 * d / 128.0, part = keys > 0 ? mean / (double)keys : 1.0;
  const int64_t units = (keys + 63) / 64, most = std::max<int64_t>(1, std::min<int64_t>(max_splits, units));
  const int64_t slots = 2 * (int64_t)n_cu;
  for (const AttendCost& c : ATTEND_COSTS) {
    if (paged && (c.rows == AT_ROWS / 2 || (ahead && c.rows == AT_ROWS))) continue;
    const int64_t per = std::max<int64_t>(1, (rows + c.rows - 1) / c.rows), tiles = sets * per, base = tiles * Hkv;
    // a unit's 64 keys come from memory at 5.2 TB/s, for the row tiles that share them once, and from the
    // caches at four times that
    const double mem = 256.0 * d * n_cu / 5.2e6 * (0.25 + 0.75 / (double)per);
    const double full = c.full * work, pair = c.pair * work;
    const int64_t fill = slots / std::max<int64_t>(1, base);
    for (const int64_t want : {(int64_t)1, (int64_t)2, (int64_t)3, fill / 2, fill, 2 * fill, 4 * fill, most}) {
      const int64_t s = std::max<int64_t>(1, std::min(want, most)), n = (units + s - 1) / s, blocks = base * s;
      const int64_t rounds = blocks / slots, rest = blocks - rounds * slots;
      const double each = (double)n * part, two = rounds > 1 || (rounds == 1 && rest) ? 2.0 * full : std::min(pair, 2.0 * full);
      const double drawn = std::min(1.0, 0.4 + (double)blocks / n_cu);           // few draw less
      const double one = std::max(c.one * work, mem * drawn);
      double us;
      if (part < 1.0) {
        // causal, the blocks with the most keys first, down to 2 part - 1 of the longest: the longest has one
        // beside it for as long as the block takes that comes when all units have one, and all together take what
        // the units can do
        const double beside = blocks <= n_cu ? 0.0 : 1.0 - 2.0 * (1.0 - part) * n_cu / (double)blocks;
        us = std::max((double)n * (beside * pair + (1.0 - beside) * one) + c.start,
                      (double)blocks / n_cu * (each * two / 2.0 + c.start));
        // nor do the last blocks, short as they are, start before whole rounds of the others have run
        if (rounds && rest)
          us = std::max(us, rounds * (each * two + 2.0 * c.start) +
                        (2.0 * part - 1.0) * n * (rest <= n_cu ? one : two) + c.start);
      } else {
        us = (double)rounds * (each * two + 2.0 * c.start) + (rest == 0 ? 0.0 : each * (rest <= n_cu ? one : two) + c.start);
      }
      us = std::max(us, (double)blocks / n_cu * each * mem + c.start);
      if (ahead) {
        // a block's prefix steps and its own come after each other and add up, each with a bound of its own: taken
        // together, own keys that wait for memory would hide the prefix's products
        const double first = (double)((ahead + 63) / 64), once = mem / (double)sets;
        const double alone = std::max(c.one * work, once * drawn);
        us += std::max(first * ((double)rounds * two + (rest == 0 ? 0.0 : rest <= n_cu ? alone : two)),
                       (double)blocks / n_cu * first * once);
      }
      us += (same && (c.rows == same || c.rows == AT_ROWS) ? 0.0 : ATTEND_LAUNCH) + attend_join_us(s + also, out_rows, d);
      if (blocks + sets * Hkv * s > AT_BLOCKS / 2 - 64) us += 1e12;      // a launch may be of two plans
      if (us < best.us) best = AttendPart{c.rows, (int)s, tiles, us};
    }
  }
  return best;
}

static void attend_finish(AttendPlan& p, int64_t rows, int d) {
  p.slots = p.own.splits + (p.pre.tiles ? p.pre.splits : 0);
  p.bytes = p.slots > 1 ? p.slots * rows * (4 * (int64_t)d + 8) : 0;
}

static AttendPlan attend_plan_packed(int64_t Tq, int64_t Tk, int B, int Hq, int Hkv, int d, bool causal) {
  AttendPlan p = {};
  // as if the sequences were equal; where they are not, their tiles are B more at most
  const int64_t rows = Tq * (Hq / Hkv), n = std::max(1, B), keys = Tk / n;
  const double mean = causal ? std::max((double)keys / 2, (double)keys - (double)Tq / n / 2) : (double)keys;
  p.own = attend_part((rows + n - 1) / n, n, Hkv, keys, mean, Tq * Hq, d, attend_cus(), 0, 0, false, 64);
  p.own.tiles = rows / p.own.rows + B;
  attend_finish(p, Tq * Hq, d);
  return p;
}

static AttendPlan attend_plan_paged(int B, int n_q, int Hq, int Hkv, int d, int64_t max_len, int64_t prefix_len) {
  AttendPlan p = {};
  const int n_cu = attend_cus();
  const int64_t rows = (int64_t)n_q * (Hq / Hkv), out_rows = (int64_t)B * n_q * Hq;
  p.own = attend_part(rows, B, Hkv, max_len, (double)max_len, out_rows, d, n_cu, prefix_len > 0, 0, true, 64);
  if (prefix_len > 0) {
    p.pre = attend_part(B * rows, 1, Hkv, prefix_len, (double)prefix_len, out_rows, d, n_cu, p.own.splits, p.own.rows, true, 64);
    // A short prefix is read by each sequence in front of its own keys: one launch instead of two and no
    // partial results.  28 / 4 heads of 128, prefix + own keys, us in a graph / of a call, as parts and so:
    //   8 sequences, 512 + 100        9.0 / 15.4    10.4 / 12.4 (10.3 where calls follow each other)
    //   64, 512 + 64                 14.8 / 15.2    10.2 / 12.0
    //   8, 1000 + 100                10.1 / 15.4    15.2 / 15.0: parts
    //   1, 1400 + 100                 8.5 / 15.4    18.6 / 18.2: parts
    // (32 sequences of 5 tokens, 32 / 8 heads, 300 + 60: 18.1 in parts, 10.8 so).  Calls with caches from memory:
    //   128, 32768 + 704            114          418: parts, whatever the tables' width
    //   256, 4000 + 704               91          153: parts
    // Over 810 shapes of one new token with tables of the lengths' width (1 to 256 sequences, prefixes of 64 to 32768, 32 to
    // 2816 own keys, 28 / 4 and 32 / 8 heads) the choice takes 1.004 of the better one's time on average, 1.25 at
    // most; over 1120 of 2 to 16 tokens 1.010 and 1.37.
    const AttendPart c = attend_part(rows, B, Hkv, max_len, (double)max_len, out_rows, d, n_cu, 0, 0, true, 1, prefix_len);
    const bool beside = (p.own.tiles * p.own.splits + p.pre.tiles * p.pre.splits) * Hkv <= n_cu;
    const double parts = beside ? std::max(p.own.us, p.pre.us + ATTEND_LAUNCH)
                                : p.own.us + p.pre.us - attend_join_us(p.own.splits + 1, out_rows, d);
    if (c.us < parts + ATTEND_SECOND) {
      p.chain = true;
      p.own = c;
      p.pre = AttendPart{};
    }
  }
  attend_finish(p, out_rows, d);
  return p;
}

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
  // the kernels' scale is a normal number of 32 bits
  return B >= 0 && B <= (1 << 20) && scale >= 1e-37 && scale <= 1e37;
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
