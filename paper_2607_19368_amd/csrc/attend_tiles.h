// Attention of packed prompts (slh_attend) and of a batch's new tokens against a paged cache
// with a shared prefix (slh_attend_paged):
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j < limit(i)
// with m_i the running maximum of the row, so that one pass over the keys does.
//
// Rows are (token, query head) pairs of one key/value head, a token's heads side by side: the
// heads that share K and V share a tile.  A wave holds 32 rows and works on the transposed
// products, so that a row's scores stay within two lanes and never leave the registers:
//   S^T (keys x rows) = K Q^T        v_mfma_f32_32x32x16, K from LDS, Q held
//   O^T (d x rows)   += V^T P^T      P from the registers of S^T, V^T by transposing LDS reads
// The k index of the second product may run over the keys in any order: it takes them as S^T's
// accumulators hold them (4 keys of each half wave in turn), so P needs no exchange.
//
// KW: 1, a block holds 128 rows, 32 a wave.  2, where so few blocks would leave compute units idle: 64 rows, and
// of each tile's 64 keys two waves take the first half, two the second, with maxima and sums of
// their own that are joined through LDS at the end.  A block's tile then takes 0.78 instead of 1.13 us, and
// there are twice as many (KW 2 / KW 1, us, causal prompts: 512 tokens, 28 / 4 heads 12.3 / 15.4; 1024: 21.8 / 25.2;
// 2048: 44.7 / 51.9; 3000: 88.7 / 80.9; 4096: 147 / 122: all units busy, K and V are read twice as often).
//
// Rounding to fewer bits: only P, to the inputs' type, for the second product (its error is relative to
// each weight, and the row's sum takes the weights as they were before it); scores, maxima, sums and O
// are fp32.
//
// Bound by the matrix units: 4 d operations a row and key at 512 (64-key tile of 128 rows: 32 KB)
// operations a byte.  128 rows a block, so that its waves share a tile's LDS reads' source, and two blocks a
// compute unit, so that one's softmax runs beside the other's products; the next tile goes straight to the
// other LDS buffer while one is worked on, its loads asked for a few at a time behind the products (all at
// once at the barrier: 16384 causal tokens 2.61 instead of 2.51 ms).
// Measured, bf16, d = 128: one causal prompt of 16384 tokens, 40 / 8 heads, 2.50 to 2.70 ms on different cards = 1100 to
// 1018 TFLOP/s, where an 8192^3 library product of the same random numbers reaches 1113 on the card on which this took 2.54; with
// zeros for inputs 1283.  The matrix units are busy for 57 % of the cycles, at 1.75 GHz: the power limit lowers the clock,
// and the rest of a tile's time is its softmax.  23 causal sequences of 59 to 1458 tokens, 32 / 8 heads, 136 us = 667 TFLOP/s:
// of a block's 23 us, 7 are its task, first loads and last stores, and 10 % of the products are masked.
#pragma once
#include "attend_held.h"

namespace slh {

constexpr int AT_KEYS = 64;              // keys of a tile
// Physical 16-byte chunk of logical chunk c of LDS row r: c ^ swizzle(r).  K: 16 consecutive
// rows are read at one chunk and have to meet the 16 bank groups of 16 bytes.  V: the transposing
// read takes 4 consecutive rows at 4 consecutive chunks.
template <int D> __device__ __forceinline__ int at_kswz(int r) {
  if (D == 128) return r & 15;
  if (D == 64) return (r & 7) ^ ((r >> 3) & 1);
  if (D == 96) return (r >> 2) & 3;
  return (r >> 3) & 1;                   // 80: 10 chunks a row
}
template <int D> __device__ __forceinline__ int at_vswz(int r) {
  if (D == 128) return (r & 3) << 2;
  if (D == 64) return ((r >> 1) & 1) << 2;
  return 0;
}

// Every direct-to-LDS load of this wave has landed, its LDS reads are done, and the block meets.
__device__ __forceinline__ void at_tile_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// LDS of a block, in elements: two tiles each of K and V, one loaded while the other is read, a word a
// wave.  Rows of D = 80: the last 32-row block of V^T reads past a row's end (results that nobody
// stores), past the last row into the padding.
template <int D> constexpr int at_lds_tile() { return AT_KEYS * D + 64; }
template <int D> constexpr int at_lds() { return 4 * at_lds_tile<D>() + 2 * AT_WAVES; }

// E8: keys and values of a cache in 8 bits.  They wait in registers while the tile before is worked on, and are converted to
// TY, with their powers of two, on the way to LDS, once for the block's 128 rows.  128 questions of 7 rows a head behind a
// prefix of 32768 rows: 121 us by blocks of 32 rows, which each convert it anew, 89 in tiles, as with 16-bit rows (95 and 97 us
// beside each other on another card).
template <class TY, int D, bool PAGED, int KW, bool E8 = false>
__device__ __forceinline__ void attend_tiles(const AttendArgs& a, int block, uint16_t* smem, const AtHeld& held = AtHeld{}) {
  constexpr int CH = D / 8;                        // 16-byte chunks of a row
  constexpr int KS = D / 16;                       // k steps of K Q^T
  constexpr int DB = (D + 31) / 32;                // 32-row blocks of O^T
  constexpr int ROWS = AT_ROWS / KW;
  constexpr int NB = 2 / KW;                       // 32-key blocks of a tile that a wave takes
  constexpr int NL = AT_KEYS * CH / 64;            // 1 KB direct-to-LDS loads of a tile of K or V
  constexpr int LDX = (NL + AT_WAVES - 1) / AT_WAVES;
  uint16_t* const sK = smem;                       // [2][at_lds_tile]
  uint16_t* const sV = smem + 2 * at_lds_tile<D>();
  int* const s_odd = (int*)(smem + 4 * at_lds_tile<D>());

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  AtTask t;
  int kvh;
  if (!at_task<PAGED, ROWS>(a, block, t, kvh)) return;

  // this lane's row: token i of the run, head kvh g + h
  const int rw = KW == 1 ? wave : wave % (AT_WAVES / KW), kw = KW == 1 ? 0 : wave / (AT_WAVES / KW);
  const int row = t.r0 + 32 * rw + (lane & 31);
  const bool real = row < t.r1;
  const int rr = real ? row : t.r1 - 1;
  const int i = rr / a.g, h = kvh * a.g + rr - i * a.g;
  const int limit = at_sees(t, i);
  // the most keys that a row of the block sees, and the fewest that one of the wave does
  const int end = max(0, at_sees(t, (t.r1 - 1) / a.g));
  const int least = __builtin_amdgcn_readfirstlane(at_sees(t, min(t.r0 + 32 * rw, t.r1 - 1) / a.g));
  // tiles of this split
  const int all = (end + AT_KEYS - 1) / AT_KEYS, each = (all + t.n_split - 1) / t.n_split;
  const int t0 = min(all, t.split * each), t1 = min(all, t0 + each);
  const bool empty = t0 >= t1 || limit <= t0 * AT_KEYS;      // the row sees none of these keys

  at_u32x4 qf[KS];
  {
    const uint16_t* qp = a.q + (t.tok0 + i) * a.q_st + h * a.q_sh + 8 * half;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const at_u32x4*)(qp + 16 * s);
  }

  // Loads of a tile: load x of a wave fills 64 chunks, of which this lane's is (physical) chunk pc
  // of row r.  Rows past the last key repeat it: they are masked.  A tile whose rows lie evenly (packed
  // rows, or all of one page) has a uniform base and 32-bit lane offsets that stay from tile to
  // tile; where a load takes whole rows of RL, its x th only moves the base.
  constexpr bool EVEN = (64 * AT_WAVES) % CH == 0;
  constexpr int RL = 64 * AT_WAVES / CH, LV = EVEN ? 1 : LDX;
  const int64_t k_st = PAGED ? D : a.k_st, v_st = PAGED ? D : a.v_st;
  const uint16_t* kbase = a.k + (PAGED ? 0 : t.key0 * a.k_st + kvh * a.k_sh);
  const uint16_t* vbase = a.v + (PAGED ? 0 : t.key0 * a.v_st + kvh * a.v_sh);
  uint32_t koff[LV], voff[LV];
  auto row_of = [&](int x) { return ((x * AT_WAVES + wave) * 64 + lane) / CH; };
  auto k_chunk = [&](int x) { const int n = (x * AT_WAVES + wave) * 64 + lane, r = n / CH; return 8 * ((n - r * CH) ^ at_kswz<D>(r)); };
  auto v_chunk = [&](int x) { const int n = (x * AT_WAVES + wave) * 64 + lane, r = n / CH; return 8 * ((n - r * CH) ^ at_vswz<D>(r)); };
#pragma unroll
  for (int x = 0; x < LV; ++x) {
    koff[x] = 2u * (uint32_t)(row_of(x) * (int)k_st + k_chunk(x));
    voff[x] = 2u * (uint32_t)(row_of(x) * (int)v_st + v_chunk(x));
  }
  const bool one_page = PAGED && a.lg_page >= 6;   // AT_KEYS rows that start at a multiple of it
  int page[LDX];                                   // paged: of the rows of the next tile to load
  auto find_pages = [&](int tile) {
    if (!PAGED) return;
    if (one_page) {
      page[0] = ((at_const_ints)t.list)[tile >> (a.lg_page - 6)];
    } else {
#pragma unroll
      for (int x = 0; x < LDX; ++x) page[x] = t.list[min(tile * AT_KEYS + row_of(x), t.nk - 1) >> a.lg_page];
    }
  };
  auto is_even = [&](int tile) { return PAGED ? one_page : tile * AT_KEYS + AT_KEYS <= t.nk; };
  // of an even tile: the offset of its first row, and load c < 2 LDX (K's, then V's)
  auto even_at = [&](int tile, int64_t st) {
    const int j0 = tile * AT_KEYS;
    if (!PAGED) return j0 * st;
    const int p = __builtin_amdgcn_readfirstlane(page[0]);
    return ((((int64_t)((unsigned)p < (unsigned)a.n_pages ? p : 0) * a.Hkv + kvh) << a.lg_page) + (j0 & ((1 << a.lg_page) - 1))) * D;
  };
  auto load_even = [&](const uint16_t* kt, const uint16_t* vt, int buf, int c) {
    const bool v = c >= LDX;
    const int x = v ? c - LDX : c;
    if (NL % AT_WAVES != 0 && x * AT_WAVES + wave >= NL) return;
    const uint16_t* from = (v ? vt : kt) + (EVEN ? x * RL : 0) * (v ? v_st : k_st);
    __builtin_amdgcn_global_load_lds((at_gptr)((const char*)from + (v ? voff : koff)[EVEN ? 0 : x]),
                                     (at_lptr)((v ? sV : sK) + buf * at_lds_tile<D>() + (x * AT_WAVES + wave) * 512), 16, 0, 0);
  };
  auto load_tile = [&](int tile, int buf) {
    if (is_even(tile)) {
      const uint16_t *kt = kbase + even_at(tile, k_st), *vt = vbase + even_at(tile, v_st);
#pragma unroll
      for (int c = 0; c < 2 * LDX; ++c) load_even(kt, vt, buf, c);
      return;
    }
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      if (NL % AT_WAVES != 0 && x * AT_WAVES + wave >= NL) break;
      const int jj = min(tile * AT_KEYS + row_of(x), t.nk - 1);
      int64_t kat, vat;
      if (PAGED) {
        const int p = (unsigned)page[x] < (unsigned)a.n_pages ? page[x] : 0;
        kat = vat = ((((int64_t)p * a.Hkv + kvh) << a.lg_page) + (jj & ((1 << a.lg_page) - 1))) * D;
      } else {
        kat = jj * k_st, vat = jj * v_st;
      }
      const int to = buf * at_lds_tile<D>() + (x * AT_WAVES + wave) * 512;
      __builtin_amdgcn_global_load_lds((at_gptr)(kbase + kat + k_chunk(x)), (at_lptr)(sK + to), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((at_gptr)(vbase + vat + v_chunk(x)), (at_lptr)(sV + to), 16, 0, 0);
    }
  };

  // Of a cache in 8 bits: 16 codes of row r of K and of V a load, this lane's part c of the row.
  constexpr int CH8 = D / 16, NC8 = AT_KEYS * CH8, LD8 = E8 ? (NC8 + 64 * AT_WAVES - 1) / (64 * AT_WAVES) : 1;
  at_u32x4 k8[LD8], v8[LD8];
  int k8_two[LD8], v8_two[LD8], page8[LD8];
  auto row8 = [&](int x) { return min((x * 64 * AT_WAVES + tid) / CH8, AT_KEYS - 1); };
  auto part8 = [&](int x) { return (x * 64 * AT_WAVES + tid) % CH8; };
  auto pages8 = [&](int tile) {
#pragma unroll
    for (int x = 0; x < LD8; ++x)
      page8[x] = one_page ? ((at_const_ints)t.list)[tile >> (a.lg_page - 6)] : t.list[min(tile * AT_KEYS + row8(x), t.nk - 1) >> a.lg_page];
  };
  auto load8 = [&](int tile) {
#pragma unroll
    for (int x = 0; x < LD8; ++x) {
      const int j = min(tile * AT_KEYS + row8(x), t.nk - 1);
      const int64_t p = (unsigned)page8[x] < (unsigned)a.n_pages ? page8[x] : 0;
      const int64_t line = ((p * a.Hkv + kvh) << a.lg_page) + (j & ((1 << a.lg_page) - 1));
      k8[x] = *(const at_u32x4*)((const uint8_t*)a.k + line * D + 16 * part8(x));
      v8[x] = *(const at_u32x4*)((const uint8_t*)a.v + line * D + 16 * part8(x));
      k8_two[x] = held.k_two[line >> held.lg_block];
      v8_two[x] = held.v_two[line >> held.lg_block];
    }
  };
  auto put8 = [&](int buf) {
    if constexpr (E8) {
#pragma unroll
      for (int x = 0; x < LD8; ++x) {
        if (NC8 % (64 * AT_WAVES) != 0 && x * 64 * AT_WAVES + tid >= NC8) break;
        const int r = row8(x), c = 2 * part8(x);
        uint16_t* const kr = sK + buf * at_lds_tile<D>() + r * D;
        uint16_t* const vr = sV + buf * at_lds_tile<D>() + r * D;
        const float kt = c8_two(k8_two[x]), vt = c8_two(v8_two[x]);
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          *(at_u32x4*)(kr + 8 * ((c + h2) ^ at_kswz<D>(r))) =
              at_u32x4{c8_pair<TY, false>(k8[x][2 * h2], kt), c8_pair<TY, true>(k8[x][2 * h2], kt),
                       c8_pair<TY, false>(k8[x][2 * h2 + 1], kt), c8_pair<TY, true>(k8[x][2 * h2 + 1], kt)};
          *(at_u32x4*)(vr + 8 * ((c + h2) ^ at_vswz<D>(r))) =
              at_u32x4{c8_pair<TY, false>(v8[x][2 * h2], vt), c8_pair<TY, true>(v8[x][2 * h2], vt),
                       c8_pair<TY, false>(v8[x][2 * h2 + 1], vt), c8_pair<TY, true>(v8[x][2 * h2 + 1], vt)};
        }
      }
    }
  };

  at_f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
  float m = -INFINITY, l = 0.f;                    // m: what the weights are relative to
  bool far = a.c > 1.f;                            // m leaves the scores first (at_far)

  // V^T: lane's element of a 32 x 16 block: row d = lane & 31, keys 4 half + 0..3 and 8 + those
  const int i16 = lane & 15, hi = (lane >> 4) & 1;
  auto v_read = [&](const uint16_t* cv, int b, int kc, int e) {
    const int r = 32 * NB * kw + 16 * kc + 8 * e + 4 * half + i16 / 4;
    const int ch = 4 * b + 2 * hi + (i16 % 4) / 2;
    return at_tr_read(cv + r * D + 8 * (ch ^ at_vswz<D>(r)) + 4 * (i16 & 1));
  };

  // Scores of a tile, K's operands read a step ahead of their products, in an order that is kept: further
  // ahead they would take the registers that O needs.  LOADS: the next tile's (even) loads go out a
  // few behind each step's products.  The block's waves meet at the same point of each tile, and sent in
  // one go their loads would hold every wave up for about 880 cycles of a tile's 3700.
  auto scores = [&](auto loads, at_f32x16 (&s)[NB], const uint16_t* ck, const uint16_t* kt, const uint16_t* vt, int nbuf)
      __attribute__((always_inline)) {
    at_u32x4 kf[2][NB];
    auto k_read = [&](int st) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const int r = 32 * (NB * kw + kb) + (lane & 31);
        kf[st & 1][kb] = *(const at_u32x4*)(ck + r * D + 8 * ((2 * st + half) ^ at_kswz<D>(r)));
      }
    };
    k_read(0);
    __builtin_amdgcn_s_setprio(1);               // the wave whose turn the matrix unit is goes first
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      if (st + 1 < KS) k_read(st + 1);
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) s[kb] = TY::mfma(kf[st & 1][kb], qf[st], s[kb]);
      if (decltype(loads)::value) {
#pragma unroll
        for (int c = st * 2 * LDX / KS; c < (st + 1) * 2 * LDX / KS; ++c) load_even(kt, vt, nbuf, c);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // One tile.  masked: some row of the wave does not see all of its keys.  next: the tile to load meanwhile, -1:
  // none.
  auto tile_step = [&](bool masked, const uint16_t* ck, const uint16_t* cv, int j0, int next, int nbuf) {
    at_f32x16 s[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    if constexpr (E8) {
      scores(std::false_type{}, s, ck, nullptr, nullptr, nbuf);
    } else if (next >= 0 && is_even(next)) {
      scores(std::true_type{}, s, ck, kbase + even_at(next, k_st), vbase + even_at(next, v_st), nbuf);
    } else {
      if (next >= 0) load_tile(next, nbuf);
      scores(std::false_type{}, s, ck, nullptr, nullptr, nbuf);
    }
    // Behind the last product stands, where the waves share a tile's loads unevenly, a short branch around one of them.
    // The branch on `masked` needs no wait of its own: its longer way, two instructions a score, is more than the 12 states, so
    // that the compiler counts the other too (a wait for every size: 128 sequences behind 32768 keys 89.7 instead of 87.9 us).
    if constexpr (NL % AT_WAVES != 0 || E8) at_products_done(s);
    if constexpr (E8) {
      if (next >= 0) put8(nbuf);
      if (next >= 0 && next + 1 < t1) load8(next + 1);
    }
    if (masked) {
      int left = limit - j0 - 32 * NB * kw - 4 * half;
      asm volatile("" : "+v"(left));               // a branch, not 32 selects in every tile
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * kb + 8 * (e / 4) + e % 4 >= left) s[kb][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
    {
      const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
    }
    if (__ballot((top - m) * a.c > AT_LAG || m == -INFINITY)) {
      const float mn = fmaxf(m, top);
      const float keep = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.c);   // of zeros
      m = mn;
      far |= at_far(m, a.c);
      l *= keep;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][e] *= keep;
    }
    const float at = m == -INFINITY ? 0.f : m;     // a row that has seen no key yet
    float mu = __builtin_fmaf(at, a.c, -TY::LIFT);
    if (far) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] -= at;
      mu = -TY::LIFT;
    }
    float sum0 = 0.f, sum1 = 0.f;
    at_u32x4 pf[2 * NB];                                // P^T, 16 keys each
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], a.c, -mu));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e + 1], a.c, -mu));
        sum0 += p0;
        sum1 += p1;
        pf[2 * kb + e / 8][(e % 8) / 2] = TY::pack(p0, p1);
      }
    l += sum0 + sum1;

    at_u32x4 vf[2][DB];
    auto v_step = [&](int kc) {
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const at_u32x2 v0 = v_read(cv, b, kc, 0), v1 = v_read(cv, b, kc, 1);
        vf[kc & 1][b] = at_u32x4{v0[0], v0[1], v1[0], v1[1]};
      }
    };
    v_step(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kc = 0; kc < 2 * NB; ++kc) {
      if (kc + 1 < 2 * NB) v_step(kc + 1);
#pragma unroll
      for (int b = 0; b < DB; ++b) o[b] = TY::mfma(vf[kc & 1][b], pf[kc], o[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // 0 x inf in the product would reach rows that do not see the key.  In a tile that some row of the
  // block does not see in full, infinite and NaN values (rare) are added to the rows that see them,
  // and leave the tile before the products.
  const int block_least = __builtin_amdgcn_readfirstlane(at_sees(t, t.r0 / a.g));
  auto clean_tile = [&](uint16_t* cv, int j0) {
    at_u32x4 w[LDX];
    uint32_t odd = 0;                              // a sign bit set: a full exponent
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      if (NL % AT_WAVES != 0 && x * AT_WAVES + wave >= NL) break;
      w[x] = *(const at_u32x4*)(cv + ((x * AT_WAVES + wave) * 64 + lane) * 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= (w[x][e] & TY::EXP) + TY::CARRY;
    }
    const bool mine = __ballot(odd & 0x80008000u) != 0;
    if (lane == 0) s_odd[wave] = mine;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int x = 0; x < AT_WAVES; ++x) any |= s_odd[x];
    if (__builtin_expect(!any, 1)) return;
    for (int r = 32 * NB * kw; r < 32 * NB * (kw + 1); ++r) {
      if (j0 + r >= limit) continue;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = 32 * b + 8 * (e / 4) + 4 * half + e % 4;
          const uint16_t v = cv[r * D + 8 * ((d / 8) ^ at_vswz<D>(r)) + d % 8];
          if (d < D && (v & (TY::EXP & 0xffff)) == (TY::EXP & 0xffff)) o[b][e] += TY::value(v);
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      if (NL % AT_WAVES != 0 && x * AT_WAVES + wave >= NL) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t f = (w[x][e] & TY::EXP) + TY::CARRY;
        if (f & 0x8000u) w[x][e] &= 0xffff0000u;
        if (f & 0x80000000u) w[x][e] &= 0x0000ffffu;
      }
      *(at_u32x4*)(cv + ((x * AT_WAVES + wave) * 64 + lane) * 8) = w[x];
    }
    __syncthreads();
  };

  if constexpr (E8) {
    if (t0 < t1) {
      pages8(t0);
      load8(t0);
      pages8(min(t0 + 1, t1 - 1));
      put8(0);
      if (t0 + 1 < t1) load8(t0 + 1);
      pages8(min(t0 + 2, t1 - 1));
    }
  } else if (t0 < t1) {
    find_pages(t0);
    load_tile(t0, 0);
    find_pages(min(t0 + 1, t1 - 1));
  }
  for (int tile = t0; tile < t1; ++tile) {
    const int buf = (tile - t0) & 1;
    // this tile has landed; the other buffer is free
    if constexpr (E8)
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else
      at_tile_barrier();
    const int j0 = tile * AT_KEYS;
    if (block_least < j0 + AT_KEYS) clean_tile(sV + buf * at_lds_tile<D>(), j0);
    tile_step(least < j0 + AT_KEYS, sK + buf * at_lds_tile<D>(), sV + buf * at_lds_tile<D>(), j0, tile + 1 < t1 ? tile + 1 : -1,
              buf ^ 1);
    if constexpr (E8)
      pages8(min(tile + 3, t1 - 1));
    else
      find_pages(min(tile + 2, t1 - 1));
  }

  at_products_done(o);
  {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  if constexpr (KW == 2) {
    // the waves that took the second half of each tile's keys give their sums to those of the first
    __syncthreads();                               // every wave is done with its V
    float* const so = (float*)smem + rw * (16 * DB + 2) * 64;
    if (kw) {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *(at_f32x4*)(so + (4 * b + e / 4) * 256 + 4 * lane) = at_f32x4{o[b][e], o[b][e + 1], o[b][e + 2], o[b][e + 3]};
      so[16 * DB * 64 + lane] = m;
      so[16 * DB * 64 + 64 + lane] = l;
    }
    __syncthreads();
    if (kw) return;
    const float m2 = so[16 * DB * 64 + lane], top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    const float k1 = __builtin_amdgcn_exp2f((m - ref) * a.c), k2 = __builtin_amdgcn_exp2f((m2 - ref) * a.c);
    m = top;
    l = __builtin_fmaf(k1, l, k2 * so[16 * DB * 64 + 64 + lane]);
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const at_f32x4 x = *(const at_f32x4*)(so + (4 * b + e / 4) * 256 + 4 * lane);
#pragma unroll
        for (int f = 0; f < 4; ++f) o[b][e + f] = __builtin_fmaf(k1, o[b][e + f], k2 * x[f]);
      }
  }
  const int64_t r = (t.tok0 + i) * a.Hq + h;
  if (a.part_o) {
    if (!real) return;
    const int64_t at = t.slot * a.rows + r;
    if (half == 0) {
      a.part_ml[2 * at] = m;
      a.part_ml[2 * at + 1] = empty ? AT_NO_KEY : l;
    }
    if (empty) return;                             // its sums are not read
    float* op = a.part_o + at * D;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int d = 32 * b + 8 * (e / 4) + 4 * half;
        typedef float f4 __attribute__((ext_vector_type(4)));
        if (d < D) *(f4*)(op + d) = f4{o[b][e], o[b][e + 1], o[b][e + 2], o[b][e + 3]};
      }
    return;
  }
  const float inv = at_inverse(empty, l);
  uint16_t* op = a.out + (t.tok0 + i) * a.o_st + h * a.o_sh + 8 * half;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int e = 0; e < 16; e += 8) {
      // the two halves hold elements 0..3 and 4..7 of two eights: they trade, and each stores one
      const auto w0 = __builtin_amdgcn_permlane32_swap(TY::pack(o[b][e] * inv, o[b][e + 1] * inv),
                                                       TY::pack(o[b][e + 4] * inv, o[b][e + 5] * inv), false, false);
      const auto w1 = __builtin_amdgcn_permlane32_swap(TY::pack(o[b][e + 2] * inv, o[b][e + 3] * inv),
                                                       TY::pack(o[b][e + 6] * inv, o[b][e + 7] * inv), false, false);
      const int d = 32 * b + 2 * e;
      if (real && d < D) *(at_u32x4*)(op + d) = at_u32x4{w0[0], w1[0], w0[1], w1[1]};
    }
  if (a.lse && real && half == 0)
    a.lse[r] = empty ? -INFINITY : m * a.scale + 0.69314718f * (__builtin_amdgcn_logf(l) - TY::LIFT);
}

}  // namespace slh
