// The attention weight that each cached key received from a call's queries, added up by key and key/value head:
//   w[b][h][j] += sum over queries i and query heads of h that see key j of exp(scale q_i . k_j - lse_i)
//
// A key belongs to one wave, which goes through the rows ((token, query head) pairs) that see it: no atomics, the
// same bits every run.  S (rows x keys) = Q K^T, so that a lane holds several rows of one key and adds within its
// registers; the lanes of a key are added at the end.  Everything is fp32.
#include "attend8.h"
#include "weights_plan.h"

namespace slh {

struct WeightArgs {
  const uint16_t* q;       // element (token, head, e) at token q_st + head q_sh + e
  int64_t q_st, q_sh;
  const void* k;           // [n_pages][Hkv][page][d]
  const uint8_t* k_two;    // 8 bits: [n_pages][Hkv][page / block]
  int n_pages, lg_page, lg_block;
  const int* pages;        // [B][ld_pages]
  int64_t ld_pages;
  int max_rows;            // of a sequence
  const int *lens, *cu;    // [B], [B + 1] (NULL: n_each queries a sequence)
  int B, n_each, Hq, Hkv, g;
  int64_t Tq;
  const float* lse;        // [Tq][Hq]
  float scale;
  float* w;                // [B][Hkv][max_rows]
  int key_blocks;
  int runs;                // k_weights_tiles: blocks of a head
  int wide;                // its tiles may be 2^31 or more
  float* part;             // [runs][2][Hkv][256]
};

// exp(scale s - lse) is 2^(s c - l) with c = scale log2(e) and l = lse log2(e), each rounded once: an error of 2^-23 |lse| or so in the
// exponent, 2^-11 at WT_FAR.  From there on (past 1 at 2^23, and with an l that may be infinite) the scaled score is
// rounded as the attention rounds its maximum's for the lse, so that a key that has all of a query's weight gets 1.
constexpr float WT_FAR = 4096.f;
__device__ __forceinline__ bool weight_is_far(float lse) { return fabsf(lse) >= WT_FAR && lse != -INFINITY; }
__device__ __forceinline__ float weight_far(float s, float scale, float lse) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_exp2f((s * scale - lse) * 1.44269504f);
}

// ---- few rows: the new tokens of a batch ----
// A wave takes 64 keys and holds them while it goes through the rows, 16 at a time.  Bound by reading K once: everything that
// does not wait for the page table goes out in front of it, and the keys all at once.  Two tokens of 6 sequences of up to
// 49159 keys, 8 heads in 8 bits (262 MB): 54 us, 4.9 TB/s; with the same inputs again, part of which the last-level cache still
// holds, 44 (16 keys a wave: 71).
constexpr int WT_KEYS = 64;              // of a wave

template <class TY, int D, bool E8>
__global__ __launch_bounds__(256) void k_weights(WeightArgs a) {
  constexpr int KS = (D + 31) / 32, X = D / 64, R = D % 64, KT = WT_KEYS / 16;
  constexpr int KL = E8 ? X : KS;        // 16-byte loads of a key by a lane
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int x = blockIdx.x;
  const int kvh = x % a.Hkv;
  x /= a.Hkv;
  const int b = x / a.key_blocks, key0 = ((x - b * a.key_blocks) * 4 + wave) * WT_KEYS;
  const int n = min(max(a.lens[b], 0), a.max_rows);
  if (key0 >= n) return;
  const int64_t q0 = max((int64_t)0, min(a.cu ? (int64_t)a.cu[b] : (int64_t)b * a.n_each, a.Tq));
  const int64_t q1 = max((int64_t)0, min(a.cu ? (int64_t)a.cu[b + 1] : (int64_t)(b + 1) * a.n_each, a.Tq));
  const int nq = (int)max((int64_t)0, q1 - q0), rows = nq * a.g;
  int r0 = max(0, key0 - (n - nq)) * a.g;          // the first row that sees one of the keys
  if (r0 >= rows) return;

  // this lane's key of each 16
  int64_t line[KT];
  int page[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) page[t] = a.pages[b * a.ld_pages + (min(key0 + 16 * t + r16, n - 1) >> a.lg_page)];
  // and, in the first group of lanes, its sum so far
  float* const w = a.w + ((int64_t)b * a.Hkv + kvh) * a.max_rows + key0 + r16;
  float was[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) was[t] = grp == 0 && key0 + 16 * t + r16 < n ? w[16 * t] : 0.f;

  // first element of a row in step s: with codes, a lane's 16 bytes of a key are those of two steps
  auto d_of = [&](int s) {
    if (!E8) return 32 * s + 8 * grp;
    return !R || s < KS - 1 ? 64 * (s / 2) + 16 * grp + 8 * (s & 1) : 64 * X + 8 * grp;
  };
  at_u32x4 qf[KS];
  float lse[4];
  int limit[4];
  auto rows_of = [&] {
    const int rr = min(r0 + r16, rows - 1), i = rr / a.g, h = kvh * a.g + rr - i * a.g;
    const uint16_t* qp = a.q + (q0 + i) * a.q_st + h * a.q_sh;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = at_u32x4{0, 0, 0, 0};
      if (d_of(s) < D) qf[s] = *(const at_u32x4*)(qp + d_of(s));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = min(r0 + 4 * grp + e, rows - 1), tok = row / a.g;
      lse[e] = a.lse[(q0 + tok) * a.Hq + kvh * a.g + row - tok * a.g];
      limit[e] = r0 + 4 * grp + e < rows ? n - nq + tok + 1 : 0;
    }
  };
  rows_of();

  at_u32x4 k[KT][KL];
  at_u32x2 kr[KT];
  int two[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int j = min(key0 + 16 * t + r16, n - 1);
    line[t] = (((int64_t)((unsigned)page[t] < (unsigned)a.n_pages ? page[t] : 0) * a.Hkv + kvh) << a.lg_page) +
              (j & ((1 << a.lg_page) - 1));
    if constexpr (E8) {
      const uint8_t* kp = (const uint8_t*)a.k + line[t] * D;
#pragma unroll
      for (int s = 0; s < KL; ++s) k[t][s] = *(const at_u32x4*)(kp + 64 * s + 16 * grp);
      kr[t] = at_u32x2{0, 0};
      if (R && 8 * grp < R) kr[t] = *(const at_u32x2*)(kp + 64 * X + 8 * grp);
      two[t] = a.k_two[line[t] >> a.lg_block];
    } else {
      const uint16_t* kp = (const uint16_t*)a.k + line[t] * D;
#pragma unroll
      for (int s = 0; s < KL; ++s) {
        k[t][s] = at_u32x4{0, 0, 0, 0};
        if (32 * s + 8 * grp < D) k[t][s] = *(const at_u32x4*)(kp + 32 * s + 8 * grp);
      }
    }
  }

  float sum[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) sum[t] = 0.f;
  const float c = a.scale * 1.44269504f;
  auto work_by = [&](auto far) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      at_f32x4 sc[1] = {at_f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        at_u32x4 kf;
        if constexpr (E8) {
          const bool rest = R && s == KS - 1;
          const uint32_t c0 = rest ? kr[t][0] : k[t][s / 2 < KL ? s / 2 : 0][2 * (s & 1)];
          const uint32_t c1 = rest ? kr[t][1] : k[t][s / 2 < KL ? s / 2 : 0][2 * (s & 1) + 1];
          const float by = c8_two(two[t]);
          kf = at_u32x4{c8_pair<TY, false>(c0, by), c8_pair<TY, true>(c0, by), c8_pair<TY, false>(c1, by), c8_pair<TY, true>(c1, by)};
        } else {
          kf = k[t][s];
        }
        sc[0] = TY::mfma16(qf[s], kf, sc[0]);
      }
      at_products_done(sc);
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = decltype(far)::value ? weight_far(sc[0][e], a.scale, lse[e])
                                             : __builtin_amdgcn_exp2f(__builtin_fmaf(sc[0][e], c, -lse[e] * 1.44269504f));
        // a row without an lse has no weights to give
        part += key0 + 16 * t + r16 < limit[e] && lse[e] != -INFINITY ? p : 0.f;
      }
      sum[t] += part;
    }
  };
  // Whether an lse is far is asked for at the end, and the rows are gone through again: a branch in front of the products would
  // wait for the lse (56 rows of 8 x 32768 keys 68 instead of 64 us).
  bool far = false;
  auto look = [&] {
#pragma unroll
    for (int e = 0; e < 4; ++e) far |= weight_is_far(lse[e]);
  };
  const int r_first = r0;
  work_by(std::false_type{});
  look();
  while ((r0 += 16) < rows) {
    rows_of();
    work_by(std::false_type{});
    look();
  }
  if (__builtin_expect(__ballot(far) != 0, 0)) {
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] = 0.f;
    for (r0 = r_first; r0 < rows; r0 += 16) {
      rows_of();
      work_by(std::true_type{});
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[t]), __float_as_uint(sum[t]), false, false);
    sum[t] = __uint_as_float(w32[0]) + __uint_as_float(w32[1]);
    const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[t]), __float_as_uint(sum[t]), false, false);
    sum[t] = __uint_as_float(w16[0]) + __uint_as_float(w16[1]);
    if (grp == 0 && key0 + 16 * t + r16 < n) w[16 * t] = was[t] + sum[t];
  }
}

// ---- many rows: prompts, or their last queries ----
// The work is cut into tiles of 128 rows and 256 keys of one key/value head: those of a sequence by blocks of 256 keys, each with the
// rows from the first that sees one of them on.  All blocks of the grid take as many tiles, one behind the other, so that
// neither a long prompt's first keys, which every query sees, nor a batch of short prompts leaves a part of the card idle.  A
// run of tiles of one block of keys that is not the whole of it leaves its sums in the workspace, and k_weights_join adds
// those of each block of keys in order.
//
// A wave holds 64 of the 256 keys in registers and goes through the rows by v_mfma_f32_32x32x16; rows go straight to LDS a tile
// ahead and are read by all four waves.  For 32 x 32 scores stand 256 cycles of products beside 16 times (an addition to the product, an
// exponential, a sum).  Hence the exponent as one operation, log2(e) in the scale and in the lse that is prepared with the
// rows, and the next products between the exponentials.  Of the SIMDs' cycles the matrix units are busy for 43 % and vector instructions
// issue in 56 % with one prompt of 16384 tokens (1.13 ms; the power limit lowers the clock to 1.9 GHz), 22 % and 35 % with 23 prompts of 59 to
// 1458 tokens (88 us, 2.4 GHz): there a run of 14 tiles meets two blocks of keys, each of which begins with nothing in
// flight, 1.10 times the scores asked for are formed, a fifth of them masked, and waves wait for 41 % of their time.  At d = 128 23 registers and
// some scalars spill: they are stored and read back around the tiles of a block of keys, not within.

// Inclusive sums over the lanes of a wave; wide: of numbers below 2^45, past 31 bits in two parts.
__device__ __forceinline__ int64_t weight_scan(int64_t v, bool wide) {
  if (!wide) return c8_wave_scan((int)v);
  return c8_wave_scan((int)(v & 0xffffff)) + ((int64_t)c8_wave_scan((int)(v >> 24)) << 24);
}

// The value of lane l, for all (and known to be the same in all).
__device__ __forceinline__ int64_t weight_lane(int64_t v, int l) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32);
}

// A sequence's share of the work.
struct WeightSeq {
  int q0, nq, n;           // first query, queries, rows of the cache
  int row_tiles, key_blocks;
  // the first row tile that sees a key of block kb < key_blocks: key j is seen from row (j - (n - nq)) g on
  __device__ __forceinline__ int first(int g, int kb) const {
    const int key = kb * WT_BLOCK_KEYS - (n - nq);
    return key > 0 ? (int)((uint32_t)(key * g) / WT_ROWS) : 0;
  }
  // sum over the blocks of keys of row_tiles - first(): from block kb0 on first() is 2 g more for each
  __device__ __forceinline__ int64_t tiles(int g) const {
    if (!row_tiles || !key_blocks) return 0;
    const int kb0 = min(key_blocks, n < nq ? 0 : (n - nq) / WT_BLOCK_KEYS + 1), m = key_blocks - kb0;
    return (int64_t)key_blocks * row_tiles - (m ? (int64_t)m * first(g, kb0) + (int64_t)g * m * (m - 1) : 0);
  }
};
static_assert(2 * WT_ROWS == WT_BLOCK_KEYS, "first() rises by 2 g");
__device__ __forceinline__ WeightSeq weight_seq(const WeightArgs& a, int b) {
  WeightSeq s = {};
  if (b >= a.B) return s;
  const int64_t q0 = a.cu ? (int64_t)a.cu[b] : (int64_t)b * a.n_each, q1 = a.cu ? (int64_t)a.cu[b + 1] : q0 + a.n_each;
  s.q0 = (int)max((int64_t)0, min(q0, a.Tq));
  s.nq = max(0, (int)max((int64_t)0, min(q1, a.Tq)) - s.q0);
  s.n = min(max(a.lens[b], 0), a.max_rows);
  s.row_tiles = (int)(((int64_t)s.nq * a.g + WT_ROWS - 1) / WT_ROWS);
  s.key_blocks = (s.n + WT_BLOCK_KEYS - 1) / WT_BLOCK_KEYS;
  return s;
}

// the same of a sequence that is the same in all lanes
__device__ __forceinline__ WeightSeq weight_seq_of_all(const WeightArgs& a, int b) {
  WeightSeq s = weight_seq(a, b);
  s.q0 = __builtin_amdgcn_readfirstlane(s.q0), s.nq = __builtin_amdgcn_readfirstlane(s.nq), s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.row_tiles = __builtin_amdgcn_readfirstlane(s.row_tiles), s.key_blocks = __builtin_amdgcn_readfirstlane(s.key_blocks);
  return s;
}

// Where the run of block i of a head begins: tiles [i each, (i + 1) each) of `all`.
struct WeightPlace {
  int64_t all, each;
  int b, kb, tile;         // of the run's first tile
  WeightSeq s;
};
__device__ __forceinline__ bool weight_place(const WeightArgs& a, int i, WeightPlace& p) {
  const int lane = threadIdx.x & 63;
  const WeightSeq mine = weight_seq(a, lane);
  p.all = weight_lane(weight_scan(mine.tiles(a.g), a.wide), 63);
  for (int b0 = 64; b0 < a.B; b0 += 64) p.all += weight_lane(weight_scan(weight_seq(a, b0 + lane).tiles(a.g), a.wide), 63);
  p.each = a.wide ? (p.all + a.runs - 1) / a.runs : (int64_t)((uint32_t)(p.all + a.runs - 1) / (uint32_t)a.runs);
  int64_t at = i * p.each;
  if (at >= p.all) return false;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const WeightSeq s = b0 ? weight_seq(a, b0 + lane) : mine;
    const int64_t count = s.tiles(a.g), upto = weight_scan(count, a.wide);
    const unsigned long long hit = __ballot(upto > at);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      p.b = b0 + l;
      p.s = weight_seq_of_all(a, p.b);
      at -= weight_lane((upto - count), l);
      break;
    }
    at -= weight_lane(upto, 63);
  }
  for (int k0 = 0; k0 < p.s.key_blocks; k0 += 64) {
    const int kb = k0 + lane;
    const int64_t count = kb < p.s.key_blocks ? p.s.row_tiles - p.s.first(a.g, kb) : 0, upto = weight_scan(count, a.wide);
    const unsigned long long hit = __ballot(upto > at);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      p.kb = k0 + l;
      p.tile = p.s.first(a.g, p.kb) + (int)(at - weight_lane((upto - count), l));
      return true;
    }
    at -= weight_lane(upto, 63);
  }
  return false;
}

// Physical 16-byte chunk of logical chunk c of LDS row r: c ^ swizzle(r); 16 consecutive rows are read at one
// chunk and have to meet the 16 bank groups of 16 bytes.
template <int D> __device__ __forceinline__ int wt_swz(int r) {
  if (D == 128) return r & 15;
  if (D == 64) return (r & 7) ^ ((r >> 3) & 1);
  if (D == 96) return (r >> 2) & 3;
  return (r >> 3) & 1;                   // 80: 10 chunks a row
}

template <class TY, int D, bool E8>
__global__ __launch_bounds__(256, 2) void k_weights_tiles(WeightArgs a) {
  constexpr int CH = D / 8, KS = D / 16;
  constexpr int LDX = (WT_ROWS * CH / 64 + 3) / 4;              // 1 KB loads of a tile by a wave
  // One array: of several, the compiler takes every read for one of what loads to LDS write, and waits for them.
  // Of two tiles: the queries, the lse as they are and times log2(e), the limits, the ends of each 64 limits, and whether an lse is far.
  constexpr int TILE = WT_ROWS * D;
  __shared__ __attribute__((aligned(16))) uint16_t smem[2 * TILE + 12 * WT_ROWS + 20];
  float* const s_raw = (float*)(smem + 2 * TILE);
  float* const s_lse = s_raw + 2 * WT_ROWS;
  int* const s_limit = (int*)s_lse + 2 * WT_ROWS;
  int* const s_ends = s_limit + 2 * WT_ROWS;     // two least limits, two largest
  int* const s_far = s_ends + 8;                 // whether waves 2 and 3 have met a far lse
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, run = blockIdx.x / a.Hkv;
  WeightPlace at_run;
  if (!weight_place(a, run, at_run)) return;
  int64_t left = min(at_run.each, at_run.all - run * at_run.each);
  const float c = a.scale * 1.44269504f;
  if (wave >= 2) s_far[wave & 1] = 0;
  for (bool begin = true;; begin = false) {
    // the run's tiles of this block of keys
    const WeightSeq& t = at_run.s;
    const int n_tiles = (int)min(left, (int64_t)(t.row_tiles - at_run.tile));
    const bool whole = at_run.tile == t.first(a.g, at_run.kb) && at_run.tile + n_tiles == t.row_tiles;
    const int2 rows = make_int2(at_run.tile * WT_ROWS, min(t.nq * a.g, (at_run.tile + n_tiles) * WT_ROWS));
    const int block0 = at_run.kb * WT_BLOCK_KEYS, key0 = block0 + 64 * wave;

    // this wave's keys, one of each 32 a lane, in the type of the queries: d 16 s + 8 half
    at_u32x4 kf[2][KS];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = min(key0 + 32 * k + (lane & 31), t.n - 1);
      const int page = a.pages[at_run.b * a.ld_pages + (j >> a.lg_page)];
      const int64_t line = (((int64_t)((unsigned)page < (unsigned)a.n_pages ? page : 0) * a.Hkv + kvh) << a.lg_page) +
                           (j & ((1 << a.lg_page) - 1));
      if constexpr (E8) {
        const uint8_t* kp = (const uint8_t*)a.k + line * D + 8 * half;
        const float two = c8_two(a.k_two[line >> a.lg_block]);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const at_u32x2 w = *(const at_u32x2*)(kp + 16 * s);
          kf[k][s] = at_u32x4{c8_pair<TY, false>(w[0], two), c8_pair<TY, true>(w[0], two), c8_pair<TY, false>(w[1], two),
                              c8_pair<TY, true>(w[1], two)};
        }
      } else {
        const uint16_t* kp = (const uint16_t*)a.k + line * D + 8 * half;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[k][s] = *(const at_u32x4*)(kp + 16 * s);
      }
    }

    // Loads of a tile: load l of a wave fills 64 chunks of 16 bytes, this lane's at `from`, of row (tok, head) of the current
    // tile.  Rows past the last, in the last tile, repeat it.
    const int last = t.nq * a.g - 1, up_tok = WT_ROWS / a.g, up_head = WT_ROWS - up_tok * a.g;
    const uint16_t* const qbase = a.q + (int64_t)t.q0 * a.q_st + (int64_t)kvh * a.g * a.q_sh;
    const int64_t up = up_tok * a.q_st + up_head * a.q_sh, wrap = a.q_st - a.g * a.q_sh;
    const uint16_t* from[LDX];
    int head[LDX];
    auto place = [&](int l, int row) {
      const int n = (l * 4 + wave) * 64 + lane, r = n / CH, i = min(row + r, last) / a.g;
      head[l] = min(row + r, last) - i * a.g;
      from[l] = qbase + i * a.q_st + head[l] * a.q_sh + 8 * ((n - r * CH) ^ wt_swz<D>(r));
    };
#pragma unroll
    for (int l = 0; l < LDX; ++l) place(l, rows.x);
    auto load = [&](int buf) {
#pragma unroll
      for (int l = 0; l < LDX; ++l)
        if (WT_ROWS * CH / 64 % 4 == 0 || l * 4 + wave < WT_ROWS * CH / 64)
          __builtin_amdgcn_global_load_lds((at_gptr)from[l], (at_lptr)(smem + buf * TILE + (l * 4 + wave) * 512), 16, 0, 0);
    };
    // on to the tile of rows r0..
    auto move = [&](int r0) {
      if (r0 + WT_ROWS - 1 > last) {
#pragma unroll
        for (int l = 0; l < LDX; ++l) place(l, r0);
        return;
      }
      if (up_head == 0) {
#pragma unroll
        for (int l = 0; l < LDX; ++l) from[l] += up;
        return;
      }
#pragma unroll
      for (int l = 0; l < LDX; ++l) {
        from[l] += up, head[l] += up_head;
        if (head[l] >= a.g) head[l] -= a.g, from[l] += wrap;
      }
    };
    // Rows `lane` of a tile's first and second 64, by waves 0 and 1 (their lse on the way to LDS) and 2 and 3 (which prepare
    // them a tile later): row `at` is (at_tok, at_head).
    int at = rows.x + 64 * (wave & 1) + lane, at_tok = at / a.g, at_head = at - at_tok * a.g;
    auto next = [&] {
      at += WT_ROWS, at_tok += up_tok, at_head += up_head;
      if (at_head >= a.g) at_head -= a.g, ++at_tok;
    };
    const float* const lse0 = a.lse + (int64_t)t.q0 * a.Hq + kvh * a.g;
    auto lse_at = [&] { return lse0 + (at <= last ? (int64_t)at_tok * a.Hq + at_head : 0); };
    // lse times log2(e), and how many keys a row sees (0: it gives nothing, or its lse is far: these rows' turn comes behind the
    // tiles); limits do not fall from row to row
    auto row_out = [&](int buf, float lse) {
      const int sees = at >= rows.y || fabsf(lse) >= WT_FAR ? 0 : max(0, t.n - t.nq + at_tok + 1);
      const int to = buf * WT_ROWS + 64 * (wave & 1) + lane;
      s_lse[to] = lse * 1.44269504f;
      s_limit[to] = sees;
      int least = __builtin_amdgcn_readfirstlane(sees), most = (int)c8_wave_max(sees);
      if (__ballot(sees == 0)) {
        least = 0;
        if (__ballot(weight_is_far(lse))) s_far[wave & 1] = 1;
      }
      if (lane == 0) s_ends[4 * buf + (wave & 1)] = least, s_ends[4 * buf + 2 + (wave & 1)] = most;
    };
    // the loads of a tile, and of the lse of the next
    auto fetch = [&](int tile) {
      if (tile) move(rows.x + tile * WT_ROWS);
      load(tile & 1);
      if (wave < 2) {
        next();
        __builtin_amdgcn_global_load_lds((at_gptr)lse_at(), (at_lptr)(s_raw + ((tile + 1) & 1) * WT_ROWS + 64 * wave), 4, 0, 0);
      }
    };

    float sum[2] = {0.f, 0.f};
    const int tiles = (rows.y - rows.x + WT_ROWS - 1) / WT_ROWS;
    if (wave >= 2) row_out(0, *lse_at());
    fetch(0);
    // the keys are waited for here, and not, with every load in flight, in each tile
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(kf[k][s]));
    // A tile's rows, 32 at a time.  The products of the next 32 go out between the exponentials of these, in an order that is
    // kept: left to itself the compiler puts them one behind the other, and each waits for the other's unit.
    auto work = [&](auto masked, int buf) __attribute__((always_inline)) {
      constexpr int NB = WT_ROWS / 32;
      const uint16_t* const row = smem + buf * TILE + (lane & 31) * D;
      const float* const l_at = s_lse + buf * WT_ROWS + 4 * half;
      const int* const m_at = s_limit + buf * WT_ROWS + 4 * half;
      at_f32x16 sc[2][2];
      at_u32x4 qf[2];
      auto q_read = [&](int rb, int s) { return *(const at_u32x4*)(row + 32 * rb * D + 8 * ((2 * s + half) ^ wt_swz<D>(lane & 31))); };
      qf[0] = q_read(0, 0);
#pragma unroll
      for (int rb = -1; rb < NB; ++rb) {
        const bool more = rb + 1 < NB;
        at_f32x16(&nx)[2] = sc[(rb + 1) & 1];
        at_f32x16(&cu)[2] = sc[rb & 1];
        float part[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
        at_f32x4 l4[4];
        at_u32x4 m4[4];
        if (rb >= 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            l4[q] = *(const at_f32x4*)(l_at + 32 * rb + 8 * q);
            if (decltype(masked)::value) m4[q] = *(const at_u32x4*)(m_at + 32 * rb + 8 * q);
          }
        }
        if (more) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) nx[k][e] = 0.f;
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (more) {
            const int n = (rb + 1) * KS + s + 1;           // the next operand, of these rows or the next 32
            if (n < NB * KS) qf[n & 1] = q_read(n / KS, n % KS);
#pragma unroll
            for (int k = 0; k < 2; ++k) nx[k] = TY::mfma(qf[(n - 1) & 1], kf[k][s], nx[k]);
          }
          if (rb >= 0) {
#pragma unroll
            for (int x = s * 16 / KS; x < (s + 1) * 16 / KS; ++x)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                float add = __builtin_amdgcn_exp2f(__builtin_fmaf(cu[k][x], c, -l4[x / 4][x % 4]));
                if (decltype(masked)::value) add = key0 + 32 * k + (lane & 31) < (int)m4[x / 4][x % 4] ? add : 0.f;
                part[k][x & 1] += add;
              }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) sum[k] += part[k][0] + part[k][1];
      }
    };
    for (int tile = 0; tile < tiles; ++tile) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");    // this tile has landed; the other buffer is free
      if (tile + 1 < tiles) {
        fetch(tile + 1);
        if (wave >= 2) {
          next();
          row_out((tile + 1) & 1, s_raw[((tile + 1) & 1) * WT_ROWS + 64 * (wave & 1) + lane]);
        }
      }
      if (key0 >= t.n) continue;
      const at_u32x4 ends = *(const at_u32x4*)(s_ends + 4 * (tile & 1));
      if (__builtin_amdgcn_readfirstlane(max((int)ends[2], (int)ends[3])) <= key0) continue;   // none sees any
      if (__builtin_amdgcn_readfirstlane(min((int)ends[0], (int)ends[1])) >= key0 + 64)      // every row of the tile sees all of this wave's keys
        work(std::false_type{}, tile & 1);
      else
        work(std::true_type{}, tile & 1);
    }
    // Rows whose lse is far, rare and without haste: 32 rows at a time, of which the others give nothing.  In the tiles' loop this would
    // take registers from it (1 to 5 % of the time).
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(s_far[0] | s_far[1]), 0) && key0 < t.n) {
      int l32 = lane & 31, hf = half, q0 = t.q0, end = rows.y;
      asm volatile("" : "+v"(l32), "+v"(hf), "+s"(q0), "+s"(end));      // what follows from them is made here, and not held throughout
#pragma unroll 1
      for (int r0 = rows.x; r0 < end; r0 += 32) {
        const int row = min(r0 + l32, end - 1), i = row / a.g;
        const uint16_t* const qp = a.q + (q0 + i) * a.q_st + ((int64_t)kvh * a.g + row - i * a.g) * a.q_sh + 8 * hf;
        at_f32x16 sc[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[k][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const at_u32x4 qf = *(const at_u32x4*)(qp + 16 * s);
#pragma unroll
          for (int k = 0; k < 2; ++k) sc[k] = TY::mfma(qf, kf[k][s], sc[k]);
        }
        at_products_done(sc);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int r = r0 + 4 * hf + 8 * (x / 4) + x % 4, at_r = min(r, end - 1), tok = at_r / a.g;
          const float l = a.lse[((int64_t)q0 + tok) * a.Hq + kvh * a.g + at_r - tok * a.g];
          const int sees = r < end && weight_is_far(l) ? t.n - t.nq + tok + 1 : 0;
#pragma unroll
          for (int k = 0; k < 2; ++k) sum[k] += key0 + 32 * k + l32 < sees ? weight_far(sc[k][x], a.scale, l) : 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[k]), __float_as_uint(sum[k]), false, false);
      sum[k] = __uint_as_float(w32[0]) + __uint_as_float(w32[1]);
      const int j = key0 + 32 * k + (lane & 31);
      if (half == 0 && whole && j < t.n) a.w[((int64_t)at_run.b * a.Hkv + kvh) * a.max_rows + j] += sum[k];
      // a block has two such runs at most: one that goes on from the block before, one that the next goes on with
      if (half == 0 && !whole) a.part[((2 * (int64_t)run + !begin) * a.Hkv + kvh) * WT_BLOCK_KEYS + j - block0] = sum[k];
    }
    left -= n_tiles;
    if (left == 0) return;
    // on to the next block of keys, or the first of the next sequence that has tiles
    if (++at_run.kb == t.key_blocks) {
      at_run.kb = 0;
      do {
        if (++at_run.b >= a.B) return;               // never, as the counts are exact
        at_run.s = weight_seq_of_all(a, at_run.b);
      } while (!at_run.s.row_tiles || !at_run.s.key_blocks);
    }
    at_run.tile = at_run.s.first(a.g, at_run.kb);
    __syncthreads();                                 // every wave is done with the last tile
  }
}

// The sums of blocks of keys that several runs share: by the second of these, a thread a key.
__global__ __launch_bounds__(256) void k_weights_join(WeightArgs a) {
  const int kvh = blockIdx.x % a.Hkv, run = blockIdx.x / a.Hkv + 1, j = threadIdx.x;
  WeightPlace p;
  if (!weight_place(a, run, p)) return;
  const int first = p.s.first(a.g, p.kb);
  const int64_t from = run * p.each - (p.tile - first), to = from + p.s.row_tiles - first;
  const int64_t r0 = from / p.each, r1 = (to - 1) / p.each;
  if (p.tile == first || run != r0 + 1 || p.kb * WT_BLOCK_KEYS + j >= p.s.n) return;
  auto part = [&](int64_t r, int which) { return a.part[((2 * r + which) * a.Hkv + kvh) * WT_BLOCK_KEYS + j]; };
  // the first run's is its last one, unless that run lies in this block of keys as a whole
  float sum = part(r0, from > r0 * p.each);
  for (int64_t r = r0 + 1; r <= r1; ++r) sum += part(r, 0);
  a.w[((int64_t)p.b * a.Hkv + kvh) * a.max_rows + p.kb * WT_BLOCK_KEYS + j] += sum;
}

template <class TY, bool E8>
static void weights_launch(const WeightArgs& a, bool tiles, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  auto go = [&](auto D) {
    if (tiles)
      hipLaunchKernelGGL((k_weights_tiles<TY, decltype(D)::value, E8>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((k_weights<TY, decltype(D)::value, E8>), grid, block, 0, s, a);
  };
  switch (d) {
    case 64: go(std::integral_constant<int, 64>{}); break;
    case 80: go(std::integral_constant<int, 80>{}); break;
    case 96: go(std::integral_constant<int, 96>{}); break;
    default: go(std::integral_constant<int, 128>{}); break;
  }
}

static bool weights_sizes_ok(int64_t Tq, int B, int Hq, int Hkv, int d, int64_t max_len) {
  if (!attend_common_ok(SLH_BF16, B, Hq, Hkv, d, 1.0) || !attend_packed_ok(Tq, 0, Hq / Hkv)) return false;
  // blocks of a launch, and rows of the weights
  return max_len >= 0 && max_len <= INT32_MAX / 4 && (int64_t)B * Hkv * (max_len / 128 + 1) <= (1 << 23);
}

}  // namespace slh

extern "C" {

int64_t slh_attend_weights_workspace(int64_t Tq, int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int64_t max_len) {
  using namespace slh;
  if (!weights_sizes_ok(Tq, B, Hq, Hkv, d, max_len)) return SLH_EINVAL;
  return weights_plan(Tq, B, Hkv, Hq / Hkv, false).bytes;
}

int slh_attend_weights(const void* q, int64_t q_st, int64_t q_sh, const void* k_cache, const void* k_scale, int32_t dtype,
                       int64_t n_pages, int32_t page_size, int32_t block, int64_t Tq, int32_t B, int32_t Hq, int32_t Hkv,
                       int32_t d, const int32_t* page_table, int64_t ld_pages, int32_t max_pages, const int32_t* lens,
                       const int32_t* cu_q, const float* lse, double scale, float* weights, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  using namespace slh;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  if (page_size < 1 || page_size > 65536 || (page_size & (page_size - 1))) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * Hkv > INT32_MAX / page_size) return SLH_EINVAL;
  if (k_scale && !c8_sizes_ok(n_pages, page_size, Hkv, block)) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || !weights_sizes_ok(Tq, B, Hq, Hkv, d, (int64_t)max_pages * page_size))
    return SLH_EINVAL;
  if (!cu_q && (B ? Tq % B != 0 : Tq != 0)) return SLH_EINVAL;
  if (B == 0 || Tq == 0 || max_pages == 0) return SLH_OK;
  if (!attend_rows_ok(q, q_st, q_sh) || !attend_rows_ok(k_cache, 0, 0) || !page_table || !lens || !lse || !weights)
    return SLH_EINVAL;
  const WeightPlan p = weights_plan(Tq, B, Hkv, Hq / Hkv, !cu_q);
  if (p.bytes && (!workspace || ((uintptr_t)workspace) % 16 != 0 || workspace_bytes < p.bytes)) return SLH_EINVAL;
  WeightArgs a = {};
  a.q = (const uint16_t*)q, a.q_st = q_st, a.q_sh = q_sh;
  a.k = k_cache, a.k_two = (const uint8_t*)k_scale;
  a.n_pages = (int)n_pages, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.lg_block = k_scale ? __builtin_ctz((unsigned)block) : 0;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_rows = max_pages * page_size;
  a.lens = lens, a.cu = cu_q, a.B = B, a.n_each = cu_q ? 0 : (int)(Tq / B), a.Hq = Hq, a.Hkv = Hkv, a.g = Hq / Hkv;
  a.Tq = Tq, a.lse = lse, a.scale = (float)scale, a.w = weights;
  a.runs = p.runs, a.part = (float*)workspace;
  a.wide = weights_wide(Tq, B, a.g, a.max_rows, !cu_q, p.runs);
  a.key_blocks = (a.max_rows + 4 * WT_KEYS - 1) / (4 * WT_KEYS);
  const int64_t blocks = (p.tiles ? p.runs : (int64_t)B * a.key_blocks) * Hkv;
  (void)hipGetLastError();
  hipStream_t s = (hipStream_t)stream;
  if (dtype == SLH_BF16)
    k_scale ? weights_launch<AtBf16, true>(a, p.tiles, d, blocks, s) : weights_launch<AtBf16, false>(a, p.tiles, d, blocks, s);
  else
    k_scale ? weights_launch<AtF16, true>(a, p.tiles, d, blocks, s) : weights_launch<AtF16, false>(a, p.tiles, d, blocks, s);
  if (hipGetLastError() != hipSuccess) return SLH_EHIP;
  if (p.bytes) hipLaunchKernelGGL(k_weights_join, dim3((unsigned)((p.runs - 1) * Hkv)), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
