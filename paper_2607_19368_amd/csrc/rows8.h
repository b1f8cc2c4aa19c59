// Attention of few rows against many keys held in 8 bits: the one-pass softmax and the transposed products of
// attend_rows.h,
//   S^T (keys x rows) = K Q^T      v_mfma_f32_16x16x32
//   O^T (d x rows)   += V^T P^T    the same
// with keys that go from memory to registers and nowhere else.  A block holds 16 or 32 rows; its four waves take the
// keys in turn, 32 at a time, each with a running maximum of its own, and join through LDS at the end.
//
// A wave's step of 32 keys is two halves of 16, each within one block of the cache (so one power of two a half, which the
// conversion to the inputs' type takes along).  The operands' order of d and of the keys is free as long as both operands of
// a product have the same, and is chosen so that every byte arrives in the lane that needs it:
//   K: a lane's 16 bytes of a key are the eight d of two products, its queries are read to match;
//   V: a lane reads 8 bytes of each of its 8 keys (those whose weights it holds), an 8 x 8 transpose within the lane;
//      row 16 grp + e of product j's result is d = 8 (4 grp + e) + j, so that a lane holds whole eights of O.
//
// Rounding to fewer bits: the weights only, for the second product (codes times a power are exact in bf16 and fp16 within
// their range); scores, maxima, sums and O are fp32.
//
// Bound by reading the codes once: 6 sequences of up to 49159 keys, 8 heads, 494 MB in 95 us, 5.2 TB/s of the 6.5 that a pure read
// reaches.  Two steps' loads are in flight a wave; their addresses take one page a half, read a step ahead.
#pragma once
#include "attend8.h"

namespace slh {

constexpr int R8_KEYS = 32;              // keys of a wave's step

template <int D, int NR> constexpr int rows8_lds() { return AT_WAVES * 16 * NR * (D + 4) + 2 * AT_WAVES * 16 * NR; }   // floats

// What a wave has loaded of a step.
template <int D> struct Rows8Step {
  static constexpr int X = D / 64;       // whole 64-byte parts of a row, and the bytes behind them
  static constexpr int R = D % 64;
  at_u32x4 k[2][X];                      // [half][part]: 16 bytes at 64 part + 16 grp of key r16
  at_u32x2 kr[2];                        // 8 bytes at 64 X + 8 grp, where there are
  uint32_t v[8][X];                      // [key]: 4 X bytes at 4 X r16
  uint32_t vr[8];                        // R / 16 bytes at 64 X + R / 16 r16
  int k_two[2], v_two[2];                // bytes of the halves' powers
};

template <class TY, int D, int NR>
__device__ __forceinline__ void rows8(const Attend8Args& A, int block, float* smem) {
  typedef Rows8Step<D> Step;
  constexpr int X = Step::X, R = Step::R;
  constexpr int ROWS = 16 * NR;
  constexpr int KS = (D + 31) / 32;                // products of K Q^T for 16 keys
  constexpr int DB = D / 16;                       // products of V^T P^T
  constexpr int M = 4 * X, MR = R / 16;            // of those, of the whole parts and of the rest
  constexpr int LDO = D + 4;
  const AttendArgs& a = A.a;
  float* const s_m = smem + AT_WAVES * ROWS * LDO;            // [AT_WAVES][ROWS]
  float* const s_l = s_m + AT_WAVES * ROWS;

  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  AtTask t;
  int kvh;
  if (!at_task<true, ROWS>(a, block, t, kvh)) return;

  const int end = max(0, at_sees(t, (t.r1 - 1) / a.g));
  const int least = __builtin_amdgcn_readfirstlane(at_sees(t, t.r0 / a.g));
  // steps of this split, in fours for the waves; steps [0, up) are those of a prefix in front
  const int up = a.chain ? (a.prefix_len + R8_KEYS - 1) / R8_KEYS : 0;
  const int all = up + (end + R8_KEYS - 1) / R8_KEYS;
  const int each = ((all + t.n_split - 1) / t.n_split + AT_WAVES - 1) / AT_WAVES * AT_WAVES;
  const int u0 = min((int64_t)all, (int64_t)t.split * each), u1 = min(all, u0 + each);

  const uint8_t* const kbase = (const uint8_t*)a.k;
  const uint8_t* const vbase = (const uint8_t*)a.v;
  const uint32_t koff = (uint32_t)(r16 * D + 16 * grp), kroff = (uint32_t)(r16 * D + 64 * X + 8 * grp);
  const uint32_t voff = (uint32_t)(4 * grp * D + 4 * X * r16), vroff = (uint32_t)(4 * grp * D + 64 * X + MR * r16);
  const int in_page = (1 << a.lg_page) - 1;
  // Pages of a step's halves: scalar loads, which are not waited for behind the steps' own (pages are not written
  // while the kernel runs, hence the constant address space).  A half past the last key is the last key's again: its
  // rows are masked, and their power is one that was written.
  auto row_of = [&](int u, int half) {
    const bool pre = u < up;
    return min((pre ? u : u - up) * R8_KEYS + 16 * half, ((pre ? a.prefix_len : t.nk) - 1) & ~15);
  };
  auto page_of = [&](int u, int half) {
    return ((at_const_ints)(u < up ? a.prefix_pages : t.list))[row_of(u, half) >> a.lg_page];
  };
  auto load = [&](int u, const int (&page)[2], Step& s) {
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int64_t p = (unsigned)page[f] < (unsigned)a.n_pages ? page[f] : 0;
      const int64_t line = ((p * a.Hkv + kvh) << a.lg_page) + (row_of(u, f) & in_page);
      s.k_two[f] = A.held.k_two[line >> A.held.lg_block];
      s.v_two[f] = A.held.v_two[line >> A.held.lg_block];
      const uint8_t* const kt = kbase + line * D;
      const uint8_t* const vt = vbase + line * D;
#pragma unroll
      for (int x = 0; x < X; ++x) s.k[f][x] = *(const at_u32x4*)(kt + koff + 64 * x);
      if (R) {
        s.kr[f] = at_u32x2{0, 0};
        if (8 * grp < R) s.kr[f] = *(const at_u32x2*)(kt + kroff);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (X == 2) {
          const at_u32x2 w = *(const at_u32x2*)(vt + voff + i * D);
          s.v[4 * f + i][0] = w[0], s.v[4 * f + i][X - 1] = w[1];
        } else {
          s.v[4 * f + i][0] = *(const uint32_t*)(vt + voff + i * D);
        }
        if (MR == 2) s.vr[4 * f + i] = *(const uint16_t*)(vt + vroff + i * D);
        if (MR == 1) s.vr[4 * f + i] = *(const uint8_t*)(vt + vroff + i * D);
      }
    }
  };

  // this lane's rows (one of each 16): the first at_sees(token) keys
  int limit[NR];
  at_u32x4 qf[NR][KS];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int rr = min(t.r0 + 16 * n + r16, t.r1 - 1), i = rr / a.g, h = kvh * a.g + rr - i * a.g;
    limit[n] = at_sees(t, i);
    const uint16_t* qp = a.q + (t.tok0 + i) * a.q_st + h * a.q_sh;
#pragma unroll
    for (int x = 0; x < X; ++x) {
      qf[n][2 * x] = *(const at_u32x4*)(qp + 64 * x + 16 * grp);
      qf[n][2 * x + 1] = *(const at_u32x4*)(qp + 64 * x + 16 * grp + 8);
    }
    if (R) {
      qf[n][KS - 1] = at_u32x4{0, 0, 0, 0};
      if (8 * grp < R) qf[n][KS - 1] = *(const at_u32x4*)(qp + 64 * X + 8 * grp);
    }
  }
  at_f32x4 o[NR][DB];
  bool far = a.c > 1.f;                            // maxima leave the scores first (at_far)
  float m[NR], l[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n] = -INFINITY, l[n] = 0.f;
#pragma unroll
    for (int b = 0; b < DB; ++b) o[n][b] = at_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  auto step = [&](int u, Step& s) __attribute__((always_inline)) {
    const bool pre = u < up;                       // every row sees the whole prefix
    const int j0 = (pre ? u : u - up) * R8_KEYS;
    const bool masked = (pre ? a.prefix_len : least) < j0 + R8_KEYS;
    float k_two[2], v_two[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      k_two[f] = c8_two(__builtin_amdgcn_readfirstlane(s.k_two[f]));
      v_two[f] = c8_two(__builtin_amdgcn_readfirstlane(s.v_two[f]));
    }
    at_f32x4 sc[2 * NR];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
#pragma unroll
      for (int n = 0; n < NR; ++n) sc[2 * n + f] = at_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        uint32_t c0, c1;
        if (R && st == KS - 1)
          c0 = s.kr[f][0], c1 = s.kr[f][1];
        else
          c0 = s.k[f][st / 2][2 * (st & 1)], c1 = s.k[f][st / 2][2 * (st & 1) + 1];
        const at_u32x4 kf = {c8_pair<TY, false>(c0, k_two[f]), c8_pair<TY, true>(c0, k_two[f]),
                             c8_pair<TY, false>(c1, k_two[f]), c8_pair<TY, true>(c1, k_two[f])};
#pragma unroll
        for (int n = 0; n < NR; ++n) sc[2 * n + f] = TY::mfma16(kf, qf[n][st], sc[2 * n + f]);
      }
    }
    at_products_done(sc);
    at_u32x4 pf[NR];                               // P^T: keys 4 grp + 0..3 of each half
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (masked) {
        int left = (pre ? a.prefix_len : limit[n]) - j0 - 4 * grp;
        asm volatile("" : "+v"(left));             // a branch, not selects in every step
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * f + e >= left) sc[2 * n + f][e] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(sc[2 * n][0], sc[2 * n][1]), fmaxf(sc[2 * n][2], sc[2 * n][3])),
                        fmaxf(fmaxf(sc[2 * n + 1][0], sc[2 * n + 1][1]), fmaxf(sc[2 * n + 1][2], sc[2 * n + 1][3])));
      const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w32[0]), __uint_as_float(w32[1]));
      const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w16[0]), __uint_as_float(w16[1]));
      if (__ballot((top - m[n]) * a.c > AT_LAG || m[n] == -INFINITY)) {
        const float mn = fmaxf(m[n], top);
        const float keep = m[n] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[n] - mn) * a.c);   // of zeros
        m[n] = mn;
        far |= at_far(mn, a.c);
        l[n] *= keep;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][b][e] *= keep;
      }
      const float at = m[n] == -INFINITY ? 0.f : m[n];       // a row that has seen no key yet
      float mu = __builtin_fmaf(at, a.c, -TY::LIFT);
      if (far) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[2 * n + f][e] -= at;
        mu = -TY::LIFT;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * n + e / 4][e % 4], a.c, -mu));
      l[n] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      pf[n] = at_u32x4{TY::pack(p[0], p[1]), TY::pack(p[2], p[3]), TY::pack(p[4], p[5]), TY::pack(p[6], p[7])};
    }

    uint32_t odd = 0, past[2];
    if (masked) {
      past[0] = c8_past<TY>(__builtin_amdgcn_readfirstlane(s.v_two[0]));
      past[1] = c8_past<TY>(__builtin_amdgcn_readfirstlane(s.v_two[1]));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int x = 0; x < X; ++x) odd |= c8_odd(s.v[i][x], past[i / 4]);
        if (R) odd |= c8_odd(s.vr[i], past[i / 4]);
      }
    }
    // bytes of the keys 2 i and 2 i + 1 side by side, of the d pair q of part x (or of the rest)
    auto both = [&](const uint32_t c0, const uint32_t c1, int q) {
      return __builtin_amdgcn_perm(c1, c0, q ? 0x07030602u : 0x05010400u);
    };
    if (__builtin_expect(masked && __ballot(odd) != 0, 0)) {
      // 0 x NaN or infinity in the product would reach rows that do not see the key: products of where they are (NaN:
      // of both signs) with what each row sees say which results they reach, and they leave V
      const uint32_t one = std::is_same<TY, AtBf16>::value ? 0x3f80u : 0x3c00u;
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        at_u32x4 up_here, down_here;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t c0 = b < M ? s.v[2 * i][b / 4 < X ? b / 4 : 0] : s.vr[2 * i];
          const uint32_t c1 = b < M ? s.v[2 * i + 1][b / 4 < X ? b / 4 : 0] : s.vr[2 * i + 1];
          const int at = 8 * (b < M ? b % 4 : b - M) + 7;
          const uint32_t u0 = c8_odd(c0, past[i / 2]) & (c8_odd(c0, 0x01010101u) | ~c0);
          const uint32_t u1 = c8_odd(c1, past[i / 2]) & (c8_odd(c1, 0x01010101u) | ~c1);
          const uint32_t d0 = c8_odd(c0, past[i / 2]) & (c8_odd(c0, 0x01010101u) | c0);
          const uint32_t d1 = c8_odd(c1, past[i / 2]) & (c8_odd(c1, 0x01010101u) | c1);
          up_here[i] = ((u0 >> at) & 1u) * one | (((u1 >> at) & 1u) * one) << 16;
          down_here[i] = ((d0 >> at) & 1u) * one | (((d1 >> at) & 1u) * one) << 16;
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          at_u32x4 sees;
          const int left = (pre ? a.prefix_len : limit[n]) - j0 - 4 * grp;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = 16 * (i / 2) + 2 * (i % 2);
            sees[i] = (j < left ? one : 0u) | (j + 1 < left ? one : 0u) << 16;
          }
          at_f32x4 hit[2] = {at_f32x4{0.f, 0.f, 0.f, 0.f}, at_f32x4{0.f, 0.f, 0.f, 0.f}};
          hit[0] = TY::mfma16(up_here, sees, hit[0]);
          hit[1] = TY::mfma16(down_here, sees, hit[1]);
          at_products_done(hit);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (hit[0][e] > 0.f) o[n][b][e] += INFINITY;
            if (hit[1][e] > 0.f) o[n][b][e] -= INFINITY;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int x = 0; x < X; ++x) s.v[i][x] &= ~((c8_odd(s.v[i][x], past[i / 4]) >> 7) * 0xffu);
        if (R) s.vr[i] &= ~((c8_odd(s.vr[i], past[i / 4]) >> 7) * 0xffu);
      }
    }
#pragma unroll
    for (int b = 0; b < DB; b += 2) {
      // products b and b + 1: the two d of a byte pair
      at_u32x4 v0, v1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t c0 = b < M ? s.v[2 * i][b / 4 < X ? b / 4 : 0] : s.vr[2 * i];
        const uint32_t c1 = b < M ? s.v[2 * i + 1][b / 4 < X ? b / 4 : 0] : s.vr[2 * i + 1];
        const uint32_t w = both(c0, c1, b < M ? b % 4 / 2 : 0);
        v0[i] = c8_pair<TY, false>(w, v_two[i / 2]);
        v1[i] = c8_pair<TY, true>(w, v_two[i / 2]);
      }
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        o[n][b] = TY::mfma16(v0, pf[n], o[n][b]);
        if (b + 1 < DB) o[n][b + 1] = TY::mfma16(v1, pf[n], o[n][b + 1]);
      }
    }
  };

  // The next step's loads go out in front of a step's work, at the end of the keys the last step's again: a branch around
  // them would leave the compiler to wait for as many loads as the shorter way has in flight.
  Step s0, s1;
  const int first = __builtin_amdgcn_readfirstlane(u0 + wave);
  int page[2] = {0, 0};
  auto pages_of = [&](int u) { page[0] = page_of(min(u, u1 - 1), 0), page[1] = page_of(min(u, u1 - 1), 1); };
  if (first < u1) {
    pages_of(first);
    load(first, page, s0);
    pages_of(first + AT_WAVES);
  }
  for (int u = first; u < u1; u += 2 * AT_WAVES) {
    const int n1 = u + AT_WAVES, n2 = u + 2 * AT_WAVES;
    load(min(n1, u1 - 1), page, s1);
    pages_of(n2);
    step(u, s0);
    if (n1 >= u1) break;
    load(min(n2, u1 - 1), page, s0);
    pages_of(n2 + AT_WAVES);
    step(n1, s1);
  }

  // the waves join
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    at_products_done(o[n]);
    const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[n]), __float_as_uint(l[n]), false, false);
    l[n] = __uint_as_float(w32[0]) + __uint_as_float(w32[1]);
    const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(l[n]), __float_as_uint(l[n]), false, false);
    l[n] = __uint_as_float(w16[0]) + __uint_as_float(w16[1]);
    const int r = wave * ROWS + 16 * n + r16;
    if (grp == 0) s_m[r] = m[n], s_l[r] = l[n];
    // element e of product b: d = M (4 grp + e) + b, of the rest 64 X + MR (4 grp + e) + b - M
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float* const to = smem + r * LDO + M * (4 * grp + e);
#pragma unroll
      for (int b = 0; b < M; b += 4) *(at_f32x4*)(to + b) = at_f32x4{o[n][b][e], o[n][b + 1][e], o[n][b + 2][e], o[n][b + 3][e]};
#pragma unroll
      for (int b = M; b < DB; ++b) smem[r * LDO + 64 * X + MR * (4 * grp + e) + b - M] = o[n][b][e];
    }
  }
  __syncthreads();
  constexpr int CH = D / 8;
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
      const float* p = smem + (w * ROWS + r) * LDO + 8 * c;
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
    const bool empty = u0 >= u1 || (u0 >= up && at_sees(t, i) <= (u0 - up) * R8_KEYS);
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
