// What the attention kernels share: element types, arguments, and which rows and keys a block
// works on.
#pragma once
#include "slh_device.h"
#include "slh_internal.h"

#include "slh.h"

namespace slh {

typedef __bf16 at_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_f16x4 __attribute__((ext_vector_type(4)));
typedef float at_f32x16 __attribute__((ext_vector_type(16)));
typedef float at_f32x4 __attribute__((ext_vector_type(4)));
typedef short at_s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t at_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t at_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) at_s16x4* at_tr_ptr;
typedef __attribute__((address_space(4))) const int* at_const_ints;
typedef __attribute__((address_space(1))) const void* at_gptr;
typedef __attribute__((address_space(3))) void* at_lptr;

struct AtBf16 {
  typedef at_bf16x8 vec;
  static constexpr uint32_t EXP = 0x7f807f80u;       // exponent bits of two elements
  static constexpr uint32_t CARRY = 0x00800080u;     // carries into the sign bit from a full exponent
  static constexpr float LIFT = 0.f;                 // the range is fp32's
  __device__ static at_f32x16 mfma(at_u32x4 a, at_u32x4 b, at_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  __device__ static at_f32x4 mfma16(at_u32x4 a, at_u32x4 b, at_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  __device__ static at_f32x4 mfma16k16(at_u32x2 a, at_u32x2 b, at_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(at_s16x4, a), __builtin_bit_cast(at_s16x4, b), c, 0, 0, 0);
  }
  __device__ static uint32_t pack(float lo, float hi) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (v2{(__bf16)lo, (__bf16)hi}));
  }
  __device__ static float value(uint16_t b) { return bf16_to_f32(b); }
};
struct AtF16 {
  typedef at_f16x8 vec;
  static constexpr uint32_t EXP = 0x7c007c00u;
  static constexpr uint32_t CARRY = 0x04000400u;
  static constexpr float LIFT = 7.f;                 // up to 2^15 with AT_LAG; full precision down to 2^-21 of the maximum
  __device__ static at_f32x16 mfma(at_u32x4 a, at_u32x4 b, at_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  __device__ static at_f32x4 mfma16(at_u32x4 a, at_u32x4 b, at_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  __device__ static at_f32x4 mfma16k16(at_u32x2 a, at_u32x2 b, at_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(at_f16x4, a), __builtin_bit_cast(at_f16x4, b), c, 0, 0, 0);
  }
  __device__ static uint32_t pack(float lo, float hi) {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (v2{(_Float16)lo, (_Float16)hi}));
  }
  __device__ static float value(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
};

struct AttendArgs {
  const uint16_t* q;      // element (token, head, e) at token q_st + head q_sh + e
  int64_t q_st, q_sh;
  const uint16_t* k;      // packed: element (token, head, e) by strides; paged: the cache
  const uint16_t* v;      //   [n_pages][Hkv][page][d]
  int64_t k_st, k_sh, v_st, v_sh;
  uint16_t* out;          // as q
  int64_t o_st, o_sh;
  float* lse;             // [tokens][Hq] or NULL
  int Hq, Hkv, g;         // g = Hq / Hkv
  float c;                // scale log2(e)
  float scale;
  int B, causal;
  // packed
  const int* cu_q;        // [B + 1]
  const int* cu_k;
  int64_t Tq, Tk;
  // paged
  const int* pages;       // [B][ld_pages]
  int64_t ld_pages;
  int max_pages;
  const int* lens;        // [B]
  const int* prefix_pages;
  int n_q, prefix_len, n_pages, lg_page;
  // keys split over blocks: partial results of each split, joined by k_attend_join
  int splits;             // of a packed sequence's or of a paged sequence's own keys
  int pre_splits;         // of the prefix, slots in front of the others
  int pre_tiles;          // row tiles of the prefix in this launch (0: not in it)
  int chain;              // the prefix's keys stand in front of each sequence's own (attend_rows.h)
  int64_t rows;           // tokens * Hq
  uint64_t by_heads, by_splits, by_pre_splits;   // at_divisor() of Hkv and the splits
  float* part_o;          // [slot][rows][d] sum p v, NULL: one split, results go to out
  float* part_ml;         // [slot][rows][2] maximum (of the unscaled scores) and sum p, AT_NO_KEY: the row sees none of its keys
};

// Transposing LDS read of 16 lanes: 4 rows of 16 elements, lane i gets column i.  `restrict` says
// (as it is inlined) that no load in flight to LDS writes what is read here; without it the
// compiler waits for all of them, the next tile's included.
__device__ __forceinline__ at_u32x2 at_tr_read(const uint16_t* __restrict__ p) {
  return __builtin_bit_cast(at_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_tr_ptr)p));
}

// The wait states between a matrix product and the first read of its result, which the compiler counts and
// fills.  Where two ways lead from the one to the other, of which the first that it follows is the longer and
// still shorter than the wait, it does not count the other (a short branch between them: scores that were read
// too early, here).  So they are spent in front of such branches: 8 states behind a 16 x 16 product, 12 behind a
// 32 x 32 x 16 one, as many as the compiler fills where nothing stands between.  The empty statements keep every
// product of x in front of the wait and every read of its results behind.
template <class T, int N>
__device__ __forceinline__ void at_products_done(T (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
  if constexpr (sizeof(T) == sizeof(at_f32x4))
    asm volatile("s_nop 7");
  else
    asm volatile("s_nop 7\n\ts_nop 3");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// A row's weights are taken relative to a maximum that may lag behind by up to 2^AT_LAG: the
// accumulated sums are rescaled only when some row of the wave passes it.  All weights (and so their sums, which
// the results are divided by) are raised by 2^LIFT of the type: those that are rounded to fp16, whose smallest step
// is 2^-24, would otherwise be lost below 2^-25 of the maximum, however many there are.
constexpr float AT_LAG = 8.f;

// Weights are 2^(s c - mu), mu the maximum times c, rounded: an error of 2^-24 mu that a row's weights share and the division
// takes out, unless it takes them past what holds them (fp16 from mu = 2^24 on, fp32 from 2^30).  Where a maximum of
// the wave times c is beyond AT_FAR, or c beyond 1 (products with the largest scores are past fp32), the maximum leaves the scores
// first.
constexpr float AT_FAR = 0x1p20f;
__device__ __forceinline__ bool at_far(float m, float c) { return __ballot(m != -INFINITY && fabsf(m) * c > AT_FAR) != 0; }

// A row that sees no key has the result 0 and no sums, which its limit says and not the sums: keys that it sees may all
// have the score -inf, and their 0 / 0 is to show.
constexpr float AT_NO_KEY = -1.f;
__device__ __forceinline__ float at_inverse(bool no_key, float l) {
  return no_key ? 0.f : l == 0.f ? __builtin_nanf("") : 1.0f / l;
}

// A tile's rows are reached by 32-bit offsets in bytes from its first.
constexpr int64_t AT_STRIDE = (int64_t)1 << 24;

// Blocks of a launch stay below.
constexpr int AT_BLOCKS = 1 << 23;
// x / n for a block number x < 2^23 and n < 2^16: x ceil(2^40 / n) / 2^40, whose error x n / 2^40 is less than
// the 1 / n by which it could reach the next whole number.
inline uint64_t at_divisor(int n) { return (((uint64_t)1 << 40) + n - 1) / (uint64_t)n; }
__device__ __forceinline__ int at_div(int x, uint64_t by) { return (int)(((uint64_t)(uint32_t)x * by) >> 40); }

// What one block works on: rows [r0, r1) of the n_tok * g of a run of tokens, against nk keys.
struct AtTask {
  int64_t tok0;           // first token in q and out
  int64_t key0;           // packed: first key's token
  int r0, r1;
  int nk;                 // keys that exist
  int base, floor;        // token i sees the keys below max(floor, base + i + 1)
  const int* list;        // paged: the pages
  int split, n_split, slot;
};

// The sequence and row tile of a packed batch's block `at`: sequence b has ceil(len_b g / ROWS)
// tiles, counted by 64 lanes at a time; the last rows of a causal sequence see the most keys and go
// first.  (Taking the tiles with the most keys of all sequences first costs more in each block than
// it saves at the end: 154 instead of 150 us for 23 sequences of 59 to 1458 tokens.)  False: no such
// tile.
template <int ROWS>
__device__ __forceinline__ bool at_find(const AttendArgs& a, int at, AtTask& t) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int lo = 0, n = 0, klo = 0, kn = 0;
    if (b < a.B) {
      const int q0 = a.cu_q[b], q1 = a.cu_q[b + 1], k0 = a.cu_k[b], k1 = a.cu_k[b + 1];
      lo = (int)min((int64_t)max(q0, 0), a.Tq);
      n = max(0, (int)min((int64_t)q1, a.Tq) - lo);
      klo = (int)min((int64_t)max(k0, 0), a.Tk);
      kn = max(0, (int)min((int64_t)k1, a.Tk) - klo);
    }
    int upto = (int)(((int64_t)n * a.g + ROWS - 1) / ROWS);
    // inclusive sums over the lanes: shifts by 1, 2, 4 and 8 within rows of 16, then the last of
    // each row, then of each half, added to the ones behind
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xA, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xC, 0xF, false);
    const unsigned long long hit = __ballot(upto > at);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int nb = __builtin_amdgcn_readlane(n, l);
      t.tok0 = __builtin_amdgcn_readlane(lo, l);
      t.key0 = __builtin_amdgcn_readlane(klo, l);
      t.nk = __builtin_amdgcn_readlane(kn, l);
      t.r0 = (__builtin_amdgcn_readlane(upto, l) - 1 - at) * ROWS;
      t.r1 = min(nb * a.g, t.r0 + ROWS);
      t.base = a.causal ? t.nk - nb : t.nk - 1;
      t.floor = a.causal ? 0 : t.nk;
      return true;
    }
    at -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// The task of a block.  Blocks are dealt to the XCDs in turn: the key/value head varies fastest,
// so that the blocks which read one head's keys meet in few of the XCDs' L2 caches.
template <bool PAGED, int ROWS>
__device__ __forceinline__ bool at_task(const AttendArgs& a, int x, AtTask& t, int& kvh) {
  const int all = x;
  x = at_div(x, a.by_heads);
  kvh = all - x * a.Hkv;
  if (PAGED) {
    if (x < a.pre_tiles * a.pre_splits) {    // every sequence's tokens against the prefix
      const int tile = at_div(x, a.by_pre_splits);
      t.split = x - tile * a.pre_splits;
      x = tile;
      t.n_split = a.pre_splits;
      t.slot = t.split;
      t.tok0 = 0;
      t.r0 = x * ROWS;
      t.r1 = min(a.B * a.n_q * a.g, t.r0 + ROWS);
      t.nk = t.floor = a.prefix_len;
      t.base = 0;
      t.list = a.prefix_pages;
    } else {                                 // one sequence's tokens against its own keys
      x -= a.pre_tiles * a.pre_splits;
      const int tile = at_div(x, a.by_splits);
      t.split = x - tile * a.splits;
      x = tile;
      t.n_split = a.splits;
      t.slot = a.pre_splits + t.split;
      const int tiles = (a.n_q * a.g + ROWS - 1) / ROWS;
      const int b = tiles == 1 ? x : x / tiles;
      t.tok0 = (int64_t)b * a.n_q;
      t.r0 = (x - b * tiles) * ROWS;
      t.r1 = min(a.n_q * a.g, t.r0 + ROWS);
      t.nk = min(max(a.lens[b], 0), a.max_pages << a.lg_page);
      t.base = t.nk - a.n_q;
      t.floor = 0;
      t.list = a.pages + b * a.ld_pages;
    }
    t.key0 = 0;
    return true;
  }
  const int tile = at_div(x, a.by_splits);
  t.split = x - tile * a.splits;
  t.n_split = a.splits;
  t.slot = t.split;
  return at_find<ROWS>(a, tile, t);
}

// limits of a task's tokens: token i sees the first at_sees() keys
__device__ __forceinline__ int at_sees(const AtTask& t, int i) {
  return min(t.nk, max(t.floor, t.base + i + 1));
}

// ---- attend_tiles.h: tiles of many rows; attend_rows.h: few rows, keys over the waves ----
constexpr int AT_WAVES = 4;                // waves of a block, of both
constexpr int AT_ROWS = 32 * AT_WAVES;     // rows of a block of the first
// Both in one launch: the prefix in tiles, `pre_blocks` of them, the sequences' own keys by rows.
// d, paged, bf16 and rows (16 or 32) pick the instantiation; `blocks` as the tasks need.
hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool bf16, int rows, int d, int64_t blocks, hipStream_t s);
hipError_t launch_attend_rows(const AttendArgs& a, bool paged, bool bf16, int rows, int d, int64_t blocks, hipStream_t s);
hipError_t launch_attend_both(const AttendArgs& a, bool bf16, int rows, int d, int64_t pre_blocks, int64_t blocks,
                              hipStream_t s);
hipError_t launch_attend_join(const AttendArgs& a, bool bf16, int d, int slots, hipStream_t s);

}  // namespace slh
