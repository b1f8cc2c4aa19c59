// Attention of few rows against many keys: decode steps, and prompts too short to fill the chip
// with tiles of 128 rows.  The same one-pass softmax as attend_tiles.h on the same transposed
// products, with 16 x 16 matrix instructions: a block holds 16 or 32 rows, and its four waves take
// the keys in turn, 16 at a time, each with a running maximum of its own; at the end they join
// through LDS.
//
// Bound by reading K and V once: nothing is shared between the waves while they run, so there
// is no barrier, only each wave's wait for its own loads, which go straight to LDS a step ahead.
// 16 keys a step: a wave's two stages of K and V are 16 KB (d = 128), so that two blocks fit a
// compute unit and one's start and end hide behind the other's steps; and pages of 16 rows or
// more hold whole steps, which makes their addresses uniform.  A short prefix (chain) is steps in front of
// a sequence's own.
//
// Measured, d = 128: two new tokens of 6 sequences of up to 49159 fp16 rows in pages of 32, 32 / 8 heads:
// 987 MB in 179 us = 5.5 TB/s, and 5 us of the join (a call 180.5; a pure read of large buffers reaches 6.55 TB/s, a copy 4.75).  512 causal
// bf16 tokens, 28 / 4 heads: 12.7 us, the dependent chain of 8 steps of 0.6 us behind the launch.  8 sequences of 97
// rows behind 512, 28 / 4 heads: 10.5 us, 10 such steps.
//
// Rounding to fewer bits: as in attend_tiles.h, the weights only, for the second product.
#pragma once
#include "attend.h"

namespace slh {

constexpr int RW_KEYS = 16;              // keys of a wave's step
constexpr int RW_STAGES = 2;

// Physical 16-byte chunk of logical chunk c of LDS row r: c ^ swizzle(r).  K: 16 rows at one chunk
// meet the 16 bank groups of 16 bytes.  V: the transposing read takes 8 consecutive rows at 2
// consecutive chunks a clock.
template <int D> __device__ __forceinline__ int rw_kswz(int r) {
  if (D == 128) return r;
  if (D == 64) return (r & 7) ^ (r >> 3);
  if (D == 96) return r >> 2;
  return r >> 3;                         // 80: 10 chunks a row
}
template <int D> __device__ __forceinline__ int rw_vswz(int r) {
  if (D == 128) return (r & 7) << 1;
  if (D == 64) return ((r >> 1) & 3) << 1;
  if (D == 96) return ((r >> 2) & 1) << 1;
  return 0;
}

// LDS of a block, in elements: the waves' stages of K and V, in the place of which their sums are joined, and
// maxima and sums of weights.
template <int D> constexpr int rw_lds_step() { return (RW_KEYS * D / 8 + 63) / 64 * 512; }
template <int D, int NR> constexpr int rw_lds_main() {
  const int stages = AT_WAVES * RW_STAGES * 2 * rw_lds_step<D>(), join = 2 * AT_WAVES * 16 * NR * (D + 4);
  return stages > join ? stages : join;
}
template <int D, int NR> constexpr int rw_lds() { return rw_lds_main<D, NR>() + 4 * AT_WAVES * 16 * NR; }

template <class TY, int D, int NR, bool PAGED>
__device__ __forceinline__ void attend_rows(const AttendArgs& a, int block, uint16_t* smem) {
  constexpr int ROWS = 16 * NR;
  constexpr int CH = D / 8;                        // 16-byte chunks of a row
  constexpr int KS = (D + 31) / 32;                // k steps of K Q^T
  constexpr int DB = D / 16;                       // 16-row blocks of O^T
  constexpr int NL = (RW_KEYS * CH + 63) / 64;     // 1 KB direct-to-LDS loads of a step of K or V
  constexpr int LB = rw_lds_step<D>();             // elements of a step's buffer (D = 80: 19 rows)
  constexpr int LDO = D + 4;                       // row of the waves' sums, when they join
  float* const s_m = (float*)(smem + rw_lds_main<D, NR>());   // [AT_WAVES][ROWS]
  float* const s_l = s_m + AT_WAVES * ROWS;

  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  AtTask t;
  int kvh;
  if (!at_task<PAGED, ROWS>(a, block, t, kvh)) return;

  const int end = max(0, at_sees(t, (t.r1 - 1) / a.g));
  const int least = __builtin_amdgcn_readfirstlane(at_sees(t, t.r0 / a.g));
  // steps of this split, in fours for the waves; steps [0, up) are those of a prefix in front
  const int up = PAGED && a.chain ? (a.prefix_len + RW_KEYS - 1) / RW_KEYS : 0;
  const int all = up + (end + RW_KEYS - 1) / RW_KEYS;
  const int each = ((all + t.n_split - 1) / t.n_split + AT_WAVES - 1) / AT_WAVES * AT_WAVES;
  const int u0 = min((int64_t)all, (int64_t)t.split * each), u1 = min(all, u0 + each);

  // Loads of a step: load x fills 64 chunks, of which this lane's is (physical) chunk pc of row r.
  // Rows past the last key repeat it: they are masked.  Packed rows, and those of pages of 16 or
  // more, lie evenly: a uniform base and lane offsets that stay from step to step.
  const int64_t k_st = PAGED ? D : a.k_st, v_st = PAGED ? D : a.v_st;
  const uint16_t* kbase = a.k + (PAGED ? 0 : t.key0 * a.k_st + kvh * a.k_sh);
  const uint16_t* vbase = a.v + (PAGED ? 0 : t.key0 * a.v_st + kvh * a.v_sh);
  uint16_t* const stage0 = smem + wave * RW_STAGES * 2 * LB;
  auto row_of = [&](int x) { return min((x * 64 + lane) / CH, RW_KEYS - 1); };
  auto k_chunk = [&](int x) { const int n = x * 64 + lane, r = n / CH; return 8 * ((n - r * CH) ^ rw_kswz<D>(r & 15)); };
  auto v_chunk = [&](int x) { const int n = x * 64 + lane, r = n / CH; return 8 * ((n - r * CH) ^ rw_vswz<D>(r & 15)); };
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int x = 0; x < NL; ++x) {
    koff[x] = 2u * (uint32_t)(row_of(x) * (int)k_st + k_chunk(x));
    voff[x] = 2u * (uint32_t)(row_of(x) * (int)v_st + v_chunk(x));
  }
  const bool even_pages = PAGED && a.lg_page >= 4;
  const int in_page = PAGED ? (1 << a.lg_page) - 1 : 0;
  // The page of step u where it has one: a scalar load, which is not waited for behind the steps' own
  // (pages are not written while the kernel runs, hence the constant address space).
  auto page_of = [&](int u) {
    if (!PAGED || !even_pages) return 0;
    return ((at_const_ints)(u < up ? a.prefix_pages : t.list))[((u < up ? u : u - up) * RW_KEYS) >> a.lg_page];
  };
  auto load = [&](int u, int page, uint16_t* to) {
    const int j0 = (u < up ? u : u - up) * RW_KEYS;
    if (PAGED ? even_pages : j0 + RW_KEYS <= t.nk) {
      const uint16_t *kt = kbase, *vt = vbase;
      if (PAGED) {
        const int64_t p = (unsigned)page < (unsigned)a.n_pages ? page : 0;
        const int64_t at = (((p * a.Hkv + kvh) << a.lg_page) + (j0 & in_page)) * D;
        kt += at, vt += at;
      } else {
        kt += j0 * k_st, vt += j0 * v_st;
      }
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        __builtin_amdgcn_global_load_lds((at_gptr)((const char*)kt + koff[x]), (at_lptr)(to + x * 512), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((at_gptr)((const char*)vt + voff[x]), (at_lptr)(to + LB + x * 512), 16, 0, 0);
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      int64_t r = min(j0 + row_of(x), (u < up ? a.prefix_len : t.nk) - 1);
      if (PAGED) {                                 // pages of fewer than 16 rows: one a row
        const int p = (u < up ? a.prefix_pages : t.list)[r >> a.lg_page];
        r = (((int64_t)((unsigned)p < (unsigned)a.n_pages ? p : 0) * a.Hkv + kvh) << a.lg_page) + (r & in_page);
      }
      __builtin_amdgcn_global_load_lds((at_gptr)(kbase + r * k_st + k_chunk(x)), (at_lptr)(to + x * 512), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((at_gptr)(vbase + r * v_st + v_chunk(x)), (at_lptr)(to + LB + x * 512), 16, 0, 0);
    }
  };

  // the first two steps' loads go out before the rows are looked at
  const int first = __builtin_amdgcn_readfirstlane(u0 + wave);
  int page = 0;                                    // of the next step to load
  if (first < u1) {
    load(first, page_of(first), stage0);
    if (first + AT_WAVES < u1) load(first + AT_WAVES, page_of(first + AT_WAVES), stage0 + 2 * LB);
    page = page_of(min(first + 2 * AT_WAVES, u1 - 1));
  }

  // this lane's rows (one of each 16): the first at_sees(token) keys
  int limit[NR];
  at_u32x4 qf[NR][KS];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int rr = min(t.r0 + 16 * n + r16, t.r1 - 1), i = rr / a.g, h = kvh * a.g + rr - i * a.g;
    limit[n] = at_sees(t, i);
    const uint16_t* qp = a.q + (t.tok0 + i) * a.q_st + h * a.q_sh + 8 * grp;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[n][s] = at_u32x4{0, 0, 0, 0};
      if (32 * s + 8 * grp < D) qf[n][s] = *(const at_u32x4*)(qp + 32 * s);
    }
  }
  // the queries are waited for here, and not, with every load in flight, in each step
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[n][s]));
  at_f32x4 o[NR][DB];
  float m[NR], l[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n] = -INFINITY, l[n] = 0.f;
#pragma unroll
    for (int b = 0; b < DB; ++b) o[n][b] = at_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  int buf = 0;
  for (int u = first; u < u1; u += AT_WAVES) {
    uint16_t* const ck = stage0 + buf * 2 * LB;
    uint16_t* const cv = ck + LB;
    buf ^= 1;
    if (u + AT_WAVES < u1)                         // this step's loads have landed
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    const bool pre = u < up;                       // every row sees the whole prefix
    const int j0 = (pre ? u : u - up) * RW_KEYS;
    const bool masked = (pre ? a.prefix_len : least) < j0 + RW_KEYS;
    if (masked) {
      // 0 x inf in the product would reach rows that do not see the key: infinite and NaN values
      // (rare) are added to the rows that see them, and leave the step before the products
      at_u32x4 w[NL];
      uint32_t odd = 0;                            // a sign bit set: a full exponent
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        w[x] = *(const at_u32x4*)(cv + (x * 64 + lane) * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= (w[x][e] & TY::EXP) + TY::CARRY;
      }
      if (__builtin_expect(__ballot(odd & 0x80008000u) != 0, 0)) {
#pragma unroll 1
        for (int r = 0; r < RW_KEYS; ++r)
#pragma unroll
          for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int d = 16 * b + 4 * grp + e;
              const uint16_t v = cv[r * D + 8 * ((d / 8) ^ rw_vswz<D>(r)) + d % 8];
              if ((v & (TY::EXP & 0xffff)) == (TY::EXP & 0xffff)) {
#pragma unroll
                for (int n = 0; n < NR; ++n)
                  if (j0 + r < (pre ? a.prefix_len : limit[n])) o[n][b][e] += TY::value(v);
              }
            }
#pragma unroll
        for (int x = 0; x < NL; ++x) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = (w[x][e] & TY::EXP) + TY::CARRY;
            if (f & 0x8000u) w[x][e] &= 0xffff0000u;
            if (f & 0x80000000u) w[x][e] &= 0x0000ffffu;
          }
          *(at_u32x4*)(cv + (x * 64 + lane) * 8) = w[x];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }

    at_f32x4 s[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) s[n] = at_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      at_u32x4 kf = *(const at_u32x4*)(ck + r16 * D + 8 * ((4 * st + grp) ^ rw_kswz<D>(r16)));
      if (D % 32 != 0 && 32 * st + 8 * grp >= D) kf = at_u32x4{0, 0, 0, 0};    // the next row's
#pragma unroll
      for (int n = 0; n < NR; ++n) s[n] = TY::mfma16(kf, qf[n][st], s[n]);
    }
    at_products_done(s);
    at_u32x2 pf[NR];                               // P^T: keys 4 grp + 0..3
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (masked) {
        int left = (pre ? a.prefix_len : limit[n]) - j0 - 4 * grp;
        asm volatile("" : "+v"(left));             // a branch, not selects in every step
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e >= left) s[n][e] = -INFINITY;
      }
      float top = fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3]));
      const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w32[0]), __uint_as_float(w32[1]));
      const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w16[0]), __uint_as_float(w16[1]));
      if (__ballot((top - m[n]) * a.c > AT_LAG || m[n] == -INFINITY)) {
        const float mn = fmaxf(m[n], top);
        const float keep = m[n] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[n] - mn) * a.c);   // of zeros
        m[n] = mn;
        l[n] *= keep;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][b][e] *= keep;
      }
      const float at = m[n] == -INFINITY ? 0.f : m[n];       // a row that has seen no key yet
      float mu = __builtin_fmaf(at, a.c, -TY::LIFT);
      if (a.c > 1.f) {
        // the largest scores times c are past fp32: the maximum leaves them first
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] -= at;
        mu = -TY::LIFT;
      }
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][e], a.c, -mu));
      l[n] += (p[0] + p[1]) + (p[2] + p[3]);
      pf[n] = at_u32x2{TY::pack(p[0], p[1]), TY::pack(p[2], p[3])};
    }
    const int vr = 4 * grp + r16 / 4, vs = rw_vswz<D>(vr);
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const at_u32x2 vf = at_tr_read(cv + vr * D + 8 * ((2 * b + (r16 % 4) / 2) ^ vs) + 4 * (r16 & 1));
#pragma unroll
      for (int n = 0; n < NR; ++n) o[n][b] = TY::mfma16k16(vf, pf[n], o[n][b]);
    }
    if (u + 2 * AT_WAVES < u1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // this step's buffer has been read
      load(u + 2 * AT_WAVES, page, ck);
      page = page_of(min(u + 3 * AT_WAVES, u1 - 1));
    }
  }

  // the waves join
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    at_products_done(o[n]);
    const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[n]), __float_as_uint(l[n]), false, false);
    l[n] = __uint_as_float(w32[0]) + __uint_as_float(w32[1]);
    const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(l[n]), __float_as_uint(l[n]), false, false);
    l[n] = __uint_as_float(w16[0]) + __uint_as_float(w16[1]);
  }
  __syncthreads();                                 // every wave is done with its V
  float* so = (float*)smem;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    if (grp == 0) s_m[wave * ROWS + 16 * n + r16] = m[n], s_l[wave * ROWS + 16 * n + r16] = l[n];
#pragma unroll
    for (int b = 0; b < DB; ++b)
      *(at_f32x4*)(so + (wave * ROWS + 16 * n + r16) * LDO + 16 * b + 4 * grp) = o[n][b];
  }
  __syncthreads();
  for (int x = tid; x < ROWS * CH; x += 64 * AT_WAVES) {
    const int r = x / CH, c = x - r * CH, row = t.r0 + r;
    if (row >= t.r1) break;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) top = fmaxf(top, s_m[w * ROWS + r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    at_f32x4 v0 = {0.f, 0.f, 0.f, 0.f}, v1 = v0;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
      const float k = __builtin_amdgcn_exp2f((s_m[w * ROWS + r] - ref) * a.c);
      const float* p = so + (w * ROWS + r) * LDO + 8 * c;
      sum = __builtin_fmaf(k, s_l[w * ROWS + r], sum);
      const at_f32x4 x0 = *(const at_f32x4*)p, x1 = *(const at_f32x4*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v0[e] = __builtin_fmaf(k, x0[e], v0[e]);
        v1[e] = __builtin_fmaf(k, x1[e], v1[e]);
      }
    }
    const int i = row / a.g, h = kvh * a.g + row - i * a.g;
    const int64_t out_row = (t.tok0 + i) * a.Hq + h;
    // sees none of this split's keys
    const bool empty = u0 >= u1 || (u0 >= up && at_sees(t, i) <= (u0 - up) * RW_KEYS);
    if (a.part_o) {
      const int64_t at = t.slot * a.rows + out_row;
      if (c == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = empty ? AT_NO_KEY : sum;
      if (empty) continue;                         // its sums are not read
      *(at_f32x4*)(a.part_o + at * D + 8 * c) = v0;
      *(at_f32x4*)(a.part_o + at * D + 8 * c + 4) = v1;
      continue;
    }
    const float inv = at_inverse(empty, sum);
    at_u32x4 w;
    w[0] = TY::pack(v0[0] * inv, v0[1] * inv);
    w[1] = TY::pack(v0[2] * inv, v0[3] * inv);
    w[2] = TY::pack(v1[0] * inv, v1[1] * inv);
    w[3] = TY::pack(v1[2] * inv, v1[3] * inv);
    *(at_u32x4*)(a.out + (t.tok0 + i) * a.o_st + h * a.o_sh + 8 * c) = w;
    if (a.lse && c == 0)
      a.lse[out_row] = empty ? -INFINITY : top * a.scale + 0.69314718f * (__builtin_amdgcn_logf(sum) - TY::LIFT);
  }
}

}  // namespace slh
