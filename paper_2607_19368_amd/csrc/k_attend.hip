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
#include "slh_device.h"
#include "slh_internal.h"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "slh.h"

namespace slh {

typedef __bf16 at_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_f16x8 __attribute__((ext_vector_type(8)));
typedef float at_f32x16 __attribute__((ext_vector_type(16)));
typedef short at_s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t at_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t at_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) at_s16x4* at_tr_ptr;
typedef __attribute__((address_space(1))) const void* at_gptr;
typedef __attribute__((address_space(3))) void* at_lptr;

struct AtBf16 {
  typedef at_bf16x8 vec;
  static constexpr uint32_t EXP = 0x7f807f80u;       // exponent bits of two elements
  static constexpr uint32_t CARRY = 0x00800080u;     // carries into the sign bit from a full exponent
  __device__ static at_f32x16 mfma(at_u32x4 a, at_u32x4 b, at_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
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
  __device__ static at_f32x16 mfma(at_u32x4 a, at_u32x4 b, at_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
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
  int pre_blocks;         // blocks of the prefix
  int64_t rows;           // tokens * Hq
  float* part_o;          // [slot][rows][d] sum p v, NULL: one split, results go to out
  float* part_ml;         // [slot][rows][2] maximum (of the unscaled scores) and sum p
};

constexpr int AT_WAVES = 4;              // waves of a block
constexpr int AT_ROWS = 32 * AT_WAVES;   // rows of a block
constexpr int AT_KEYS = 64;              // keys of a tile
// A row's weights are taken relative to a maximum that may lag behind by up to 2^AT_LAG: the
// accumulated sums are rescaled only when some row of the wave passes it.  Weights up to 2^8
// lose nothing: their rounding is relative, and fp16 holds up to 2^15.
constexpr float AT_LAG = 8.f;

// A tile's rows are reached by 32-bit offsets in bytes from its first.
constexpr int64_t AT_STRIDE = (int64_t)1 << 24;

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

// The sequence and row tile of a packed batch's block `at`: sequence b has
// ceil(len_b g / AT_ROWS) tiles, counted by 64 lanes at a time.  False: no such tile.
__device__ __forceinline__ bool at_find(const AttendArgs& a, int at, AtTask& t) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int lo = 0, n = 0;
    if (b < a.B) {
      lo = min((int64_t)max(a.cu_q[b], 0), a.Tq);
      n = max(0, (int)min((int64_t)a.cu_q[b + 1], a.Tq) - lo);
    }
    const int tiles = (int)(((int64_t)n * a.g + AT_ROWS - 1) / AT_ROWS);
    int upto = tiles;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(upto, s);
      if (lane >= s) upto += o;
    }
    const unsigned long long hit = __ballot(upto > at);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int nb = __builtin_amdgcn_readlane(n, l);
      // the last rows of a causal sequence see the most keys: they go first
      const int tile = __builtin_amdgcn_readlane(upto, l) - 1 - at;
      t.tok0 = __builtin_amdgcn_readlane(lo, l);
      const int kb = b0 + l;
      const int64_t k0 = min((int64_t)max(a.cu_k[kb], 0), a.Tk);
      t.key0 = k0;
      t.nk = max(0, (int)(min((int64_t)a.cu_k[kb + 1], a.Tk) - k0));
      t.r0 = tile * AT_ROWS;
      t.r1 = min(nb * a.g, t.r0 + AT_ROWS);
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
template <bool PAGED>
__device__ __forceinline__ bool at_task(const AttendArgs& a, AtTask& t, int& kvh) {
  int x = blockIdx.x;
  kvh = x % a.Hkv;
  x /= a.Hkv;
  if (PAGED) {
    if (x < a.pre_blocks) {                  // every sequence's tokens against the prefix
      t.split = x % a.pre_splits;
      x /= a.pre_splits;
      t.n_split = a.pre_splits;
      t.slot = t.split;
      t.tok0 = 0;
      t.r0 = x * AT_ROWS;
      t.r1 = min(a.B * a.n_q * a.g, t.r0 + AT_ROWS);
      t.nk = t.floor = a.prefix_len;
      t.base = 0;
      t.list = a.prefix_pages;
    } else {                                 // one sequence's tokens against its own keys
      x -= a.pre_blocks;
      t.split = x % a.splits;
      x /= a.splits;
      t.n_split = a.splits;
      t.slot = a.pre_splits + t.split;
      const int tiles = (a.n_q * a.g + AT_ROWS - 1) / AT_ROWS;
      const int b = x / tiles;
      t.tok0 = (int64_t)b * a.n_q;
      t.r0 = (x - b * tiles) * AT_ROWS;
      t.r1 = min(a.n_q * a.g, t.r0 + AT_ROWS);
      t.nk = min(max(a.lens[b], 0), a.max_pages << a.lg_page);
      t.base = t.nk - a.n_q;
      t.floor = 0;
      t.list = a.pages + b * a.ld_pages;
    }
    t.key0 = 0;
    return true;
  }
  t.split = x % a.splits;
  t.n_split = a.splits;
  t.slot = t.split;
  return at_find(a, x / a.splits, t);
}

// Every direct-to-LDS load of this wave has landed, its LDS reads are done, and the block meets.
__device__ __forceinline__ void at_tile_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <class TY, int D, bool PAGED>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend(AttendArgs a) {
  constexpr int CH = D / 8;                        // 16-byte chunks of a row
  constexpr int KS = D / 16;                       // k steps of K Q^T
  constexpr int DB = (D + 31) / 32;                // 32-row blocks of O^T
  constexpr int NL = AT_KEYS * CH / 64;            // 1 KB direct-to-LDS loads of a tile of K or V
  constexpr int LDX = (NL + AT_WAVES - 1) / AT_WAVES;
  // two tiles each of K and V: one is loaded while the other is read.  Rows of D = 80: the last
  // 32-row block of V^T reads past a row's end (results that nobody stores), past the last row
  // into the padding
  __shared__ __attribute__((aligned(16))) uint16_t sK[2][AT_KEYS * D], sV[2][AT_KEYS * D + 64];
  __shared__ int s_odd[AT_WAVES];

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  AtTask t;
  int kvh;
  if (!at_task<PAGED>(a, t, kvh)) return;

  // this lane's row: token i of the run, head kvh g + h
  const int row = t.r0 + 32 * wave + (lane & 31);
  const bool real = row < t.r1;
  const int rr = real ? row : t.r1 - 1;
  const int i = rr / a.g, h = kvh * a.g + rr - i * a.g;
  auto sees = [&](int tok) { return min(t.nk, max(t.floor, t.base + tok + 1)); };
  const int limit = sees(i);
  // the most keys that a row of the block sees, and the fewest that one of the wave does
  const int end = max(0, sees((t.r1 - 1) / a.g));
  const int least = __builtin_amdgcn_readfirstlane(sees(min(t.r0 + 32 * wave, t.r1 - 1) / a.g));
  // tiles of this split
  const int all = (end + AT_KEYS - 1) / AT_KEYS, each = (all + t.n_split - 1) / t.n_split;
  const int t0 = min(all, t.split * each), t1 = min(all, t0 + each);

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
  auto load = [&](const uint16_t* kp, const uint16_t* vp, int buf, int x) {
    const int to = (x * AT_WAVES + wave) * 512;
    __builtin_amdgcn_global_load_lds((at_gptr)kp, (at_lptr)(&sK[buf][to]), 16, 0, 0);
    __builtin_amdgcn_global_load_lds((at_gptr)vp, (at_lptr)(&sV[buf][to]), 16, 0, 0);
  };
  const bool one_page = PAGED && a.lg_page >= 6;   // AT_KEYS rows that start at a multiple of it
  int page[LDX];                                   // paged: of the rows of the next tile to load
  auto find_pages = [&](int tile) {
    if (!PAGED) return;
    if (one_page) {
      page[0] = t.list[tile >> (a.lg_page - 6)];
    } else {
#pragma unroll
      for (int x = 0; x < LDX; ++x) page[x] = t.list[min(tile * AT_KEYS + row_of(x), t.nk - 1) >> a.lg_page];
    }
  };
  auto load_tile = [&](int tile, int buf) {
    const int j0 = tile * AT_KEYS;
    if ((!PAGED && j0 + AT_KEYS <= t.nk) || (PAGED && one_page)) {
      const uint16_t *kt = kbase, *vt = vbase;
      if (PAGED) {
        const int p = __builtin_amdgcn_readfirstlane(page[0]);
        const int64_t at = ((((int64_t)((unsigned)p < (unsigned)a.n_pages ? p : 0) * a.Hkv + kvh) << a.lg_page) +
                            (j0 & ((1 << a.lg_page) - 1))) * D;
        kt += at, vt += at;
      } else {
        kt += j0 * k_st, vt += j0 * v_st;
      }
#pragma unroll
      for (int x = 0; x < LDX; ++x) {
        if (x * AT_WAVES + wave >= NL) break;
        const int64_t more = EVEN ? x * RL : 0;
        load((const uint16_t*)((const char*)(kt + more * k_st) + koff[EVEN ? 0 : x]),
             (const uint16_t*)((const char*)(vt + more * v_st) + voff[EVEN ? 0 : x]), buf, x);
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      if (x * AT_WAVES + wave >= NL) break;
      const int jj = min(j0 + row_of(x), t.nk - 1);
      int64_t kat, vat;
      if (PAGED) {
        const int p = (unsigned)page[x] < (unsigned)a.n_pages ? page[x] : 0;
        kat = vat = ((((int64_t)p * a.Hkv + kvh) << a.lg_page) + (jj & ((1 << a.lg_page) - 1))) * D;
      } else {
        kat = jj * k_st, vat = jj * v_st;
      }
      load(kbase + kat + k_chunk(x), vbase + vat + v_chunk(x), buf, x);
    }
  };

  at_f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
  float m = -INFINITY, l = 0.f;                    // m: what the weights are relative to

  // V^T: lane's element of a 32 x 16 block: row d = lane & 31, keys 4 half + 0..3 and 8 + those
  const int i16 = lane & 15, hi = (lane >> 4) & 1;
  auto v_read = [&](const uint16_t* cv, int b, int kc, int e) {
    const int r = 16 * kc + 8 * e + 4 * half + i16 / 4;
    const int ch = 4 * b + 2 * hi + (i16 % 4) / 2;
    const at_s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (at_tr_ptr)(cv + r * D + 8 * (ch ^ at_vswz<D>(r)) + 4 * (i16 & 1)));
    return __builtin_bit_cast(at_u32x2, w);
  };

  // One tile.  masked: some row of the wave does not see all of its keys.
  auto tile_step = [&](bool masked, const uint16_t* ck, const uint16_t* cv, int j0) {
    at_f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    // K's operands are read a step ahead of their products, in an order that is kept: further
    // ahead they would take the registers that O needs
    at_u32x4 kf[2][2];
    auto k_read = [&](int st) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int r = 32 * kb + (lane & 31);
        kf[st & 1][kb] = *(const at_u32x4*)(ck + r * D + 8 * ((2 * st + half) ^ at_kswz<D>(r)));
      }
    };
    k_read(0);
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      if (st + 1 < KS) k_read(st + 1);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = TY::mfma(kf[st & 1][kb], qf[st], s[kb]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (masked) {
      int left = limit - j0 - 4 * half;
      asm volatile("" : "+v"(left));               // a branch, not 32 selects in every tile
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * kb + 8 * (e / 4) + e % 4 >= left) s[kb][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
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
      l *= keep;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][e] *= keep;
    }
    const float at = m == -INFINITY ? 0.f : m;     // a row that has seen no key yet
    float mu = at * a.c;
    if (a.c > 1.f) {
      // the largest scores times c are past fp32: the maximum leaves them first
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] -= at;
      mu = 0.f;
    }
    float sum0 = 0.f, sum1 = 0.f;
    at_u32x4 pf[4];                                // P^T, 16 keys each
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
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
#pragma unroll
    for (int kc = 0; kc < 4; ++kc) {
      if (kc < 3) v_step(kc + 1);
#pragma unroll
      for (int b = 0; b < DB; ++b) o[b] = TY::mfma(vf[kc & 1][b], pf[kc], o[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // 0 x inf in the product would reach rows that do not see the key.  In a tile that some row of the
  // block does not see in full, infinite and NaN values (rare) are added to the rows that see them,
  // and leave the tile before the products.
  const int block_least = __builtin_amdgcn_readfirstlane(sees(t.r0 / a.g));
  auto clean_tile = [&](uint16_t* cv, int j0) {
    at_u32x4 w[LDX];
    uint32_t odd = 0;                              // a sign bit set: a full exponent
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      if (x * AT_WAVES + wave >= NL) break;
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
    for (int r = 0; r < AT_KEYS; ++r) {
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
      if (x * AT_WAVES + wave >= NL) break;
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

  if (t0 < t1) {
    find_pages(t0);
    load_tile(t0, 0);
    find_pages(min(t0 + 1, t1 - 1));
  }
  for (int tile = t0; tile < t1; ++tile) {
    const int buf = (tile - t0) & 1;
    at_tile_barrier();                             // this tile has landed; the other buffer is free
    if (tile + 1 < t1) {
      load_tile(tile + 1, buf ^ 1);
      find_pages(min(tile + 2, t1 - 1));
    }
    const int j0 = tile * AT_KEYS;
    if (block_least < j0 + AT_KEYS) clean_tile(sV[buf], j0);
    tile_step(least < j0 + AT_KEYS, sK[buf], sV[buf], j0);
  }

  {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  if (!real) return;
  const bool empty = m == -INFINITY && l == 0.f;
  const int64_t r = (t.tok0 + i) * a.Hq + h;
  if (a.part_o) {
    const int64_t at = t.slot * a.rows + r;
    if (half == 0) {
      a.part_ml[2 * at] = m;
      a.part_ml[2 * at + 1] = l;
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
  const float inv = empty ? 0.f : 1.0f / l;
  uint16_t* op = a.out + (t.tok0 + i) * a.o_st + h * a.o_sh;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int d = 32 * b + 8 * (e / 4) + 4 * half;
      at_u32x2 w;
      w[0] = TY::pack(o[b][e] * inv, o[b][e + 1] * inv);
      w[1] = TY::pack(o[b][e + 2] * inv, o[b][e + 3] * inv);
      if (d < D) *(at_u32x2*)(op + d) = w;
    }
  if (a.lse && half == 0)
    a.lse[r] = empty ? -INFINITY : m * a.scale + 0.69314718f * __builtin_amdgcn_logf(l);
}

// Joins the splits of each row: out = sum_s w_s o_s / sum_s w_s l_s, w_s = exp2((m_s - max m) c).
// One wave a row, its lanes first over the splits, then over the elements.
template <class TY>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int d, int slots) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  float top = -INFINITY;
  bool any = false, nan = false;
  for (int s = lane; s < slots; s += 64) {
    const float ms = a.part_ml[2 * (s * a.rows + r)], ls = a.part_ml[2 * (s * a.rows + r) + 1];
    top = fmaxf(top, ms);
    any |= !(ms == -INFINITY && ls == 0.f);
    nan |= ls != ls;
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f, o0 = 0.f, o1 = 0.f;
  const int e = 2 * lane;
  if (__ballot(any)) {
    for (int s = 0; s < slots; ++s) {
      const int64_t at = s * a.rows + r;
      const float ms = a.part_ml[2 * at], ls = a.part_ml[2 * at + 1];
      if (ms == -INFINITY && ls == 0.f) continue;          // wave-uniform
      const float w = __builtin_amdgcn_exp2f((ms - ref) * a.c);
      l = __builtin_fmaf(w, ls, l);
      if (e < d) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 v = *(const f2*)(a.part_o + at * d + e);
        o0 = __builtin_fmaf(w, v[0], o0);
        o1 = __builtin_fmaf(w, v[1], o1);
      }
    }
  }
  const bool empty = !__ballot(any);
  const float inv = empty ? 0.f : 1.0f / l;
  const int64_t tok = r / a.Hq;
  const int h = (int)(r - tok * a.Hq);
  if (e < d) *(uint32_t*)(a.out + tok * a.o_st + h * a.o_sh + e) = TY::pack(o0 * inv, o1 * inv);
  if (a.lse && lane == 0) a.lse[r] = empty ? -INFINITY : top * a.scale + 0.69314718f * __builtin_amdgcn_logf(l);
}

template <class TY, bool PAGED>
static hipError_t attend_launch(const AttendArgs& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend<TY, 64, PAGED>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_attend<TY, 80, PAGED>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_attend<TY, 96, PAGED>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_attend<TY, 128, PAGED>), grid, block, 0, s, a); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part_o) return e;
  hipLaunchKernelGGL((k_attend_join<TY>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, s, a, d,
                     a.splits + a.pre_splits);
  return hipGetLastError();
}

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

// Splits of `tiles` key tiles so that `blocks` blocks become about two a compute unit, each with
// four tiles or more.
static int attend_splits(int64_t blocks, int64_t tiles, int n_cu) {
  return (int)std::max<int64_t>(1, std::min(std::min<int64_t>(2 * n_cu / std::max<int64_t>(1, blocks), tiles / 4), (int64_t)64));
}

// Workspace of `slots` partial results of `rows` rows: sums, then maxima and sums of weights.
static int64_t attend_ws_bytes(int64_t slots, int64_t rows, int d) { return slots * rows * (4 * d + 8); }
static void attend_ws_lay(AttendArgs& a, void* ws, int slots, int d) {
  a.part_o = (float*)ws;
  a.part_ml = a.part_o + slots * a.rows * d;
}

struct AttendPlan { int splits, pre_splits; int64_t blocks, pre_blocks; int64_t bytes; };

static AttendPlan attend_plan_packed(int64_t Tq, int64_t Tk, int B, int Hq, int Hkv, int d) {
  const int64_t tiles = Tq * (Hq / Hkv) / AT_ROWS + B;
  AttendPlan p = {};
  // of the average sequence: the tiles of rows that there are at least, its keys
  const int64_t sure = std::max<int64_t>(B, (Tq * (Hq / Hkv) + AT_ROWS - 1) / AT_ROWS) * Hkv;
  p.splits = attend_splits(sure, Tk / std::max(1, B) / AT_KEYS, attend_cus());
  p.blocks = tiles * Hkv * p.splits;
  p.bytes = p.splits > 1 ? attend_ws_bytes(p.splits, Tq * Hq, d) : 0;
  return p;
}

static AttendPlan attend_plan_paged(int B, int n_q, int Hq, int Hkv, int d, int64_t max_len, int64_t prefix_len) {
  const int n_cu = attend_cus(), g = Hq / Hkv;
  AttendPlan p = {};
  const int64_t own = (int64_t)B * (((int64_t)n_q * g + AT_ROWS - 1) / AT_ROWS);
  p.splits = attend_splits(own * Hkv, max_len / AT_KEYS, n_cu);
  if (prefix_len > 0) {
    const int64_t tiles = ((int64_t)B * n_q * g + AT_ROWS - 1) / AT_ROWS;
    p.pre_splits = attend_splits(tiles * Hkv, prefix_len / AT_KEYS, n_cu);
    p.pre_blocks = tiles * p.pre_splits;
  }
  p.blocks = (p.pre_blocks + own * p.splits) * Hkv;
  const int slots = p.splits + p.pre_splits;
  p.bytes = slots > 1 ? attend_ws_bytes(slots, (int64_t)B * n_q * Hq, d) : 0;
  return p;
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
static bool attend_ws_ok(const AttendPlan& p, const void* ws, int64_t bytes) {
  return p.bytes == 0 || (ws && ((uintptr_t)ws) % 16 == 0 && bytes >= p.bytes);
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
  const AttendPlan p = attend_plan_packed(Tq, Tk, B, Hq, Hkv, d);
  if (p.blocks > INT32_MAX / 256 || !attend_ws_ok(p, workspace, workspace_bytes)) return SLH_EINVAL;
  a.splits = p.splits, a.rows = Tq * Hq;
  if (p.bytes) attend_ws_lay(a, workspace, p.splits, d);
  (void)hipGetLastError();
  const hipError_t e = dtype == SLH_BF16 ? attend_launch<AtBf16, false>(a, d, p.blocks, (hipStream_t)stream)
                                         : attend_launch<AtF16, false>(a, d, p.blocks, (hipStream_t)stream);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
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
  if (n_pages < 1 || n_pages > INT32_MAX || page_size < 1 || page_size > 65536 || (page_size & (page_size - 1)))
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
  const AttendPlan p = attend_plan_paged(B, n_q, Hq, Hkv, d, (int64_t)max_pages * page_size, prefix_len);
  if (p.blocks > INT32_MAX / 256 || !attend_ws_ok(p, workspace, workspace_bytes)) return SLH_EINVAL;
  a.splits = p.splits, a.pre_splits = p.pre_splits, a.pre_blocks = (int)p.pre_blocks;
  a.rows = (int64_t)B * n_q * Hq;
  if (p.bytes) attend_ws_lay(a, workspace, p.splits + p.pre_splits, d);
  (void)hipGetLastError();
  const hipError_t e = dtype == SLH_BF16 ? attend_launch<AtBf16, true>(a, d, p.blocks, (hipStream_t)stream)
                                         : attend_launch<AtF16, true>(a, d, p.blocks, (hipStream_t)stream);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
