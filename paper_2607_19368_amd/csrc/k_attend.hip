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
};

constexpr int AT_WAVES = 4;              // waves of a block
constexpr int AT_ROWS = 32 * AT_WAVES;   // rows of a block
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

// What one block works on: rows [r0, r1) of a sequence's n_tok * g, keys [0, nk).
struct AtTask {
  int64_t tok0;           // first token of the sequence in q and out
  int64_t key0;           // packed: first key's token
  int r0, r1;
  int nk;                 // keys that exist
  int base, floor;        // token i sees the keys below max(floor, base + i + 1)
  const int* own;         // paged: the sequence's pages
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

template <class TY, int D, bool PAGED>
__global__ __launch_bounds__(64 * AT_WAVES) void k_attend(AttendArgs a) {
  constexpr int CH = D / 8;                        // 16-byte chunks of a row
  constexpr int KS = D / 16;                       // k steps of K Q^T
  constexpr int DB = (D + 31) / 32;                // 32-row blocks of O^T
  constexpr int LD = AT_KEYS * CH / 64 / AT_WAVES; // direct-to-LDS loads a wave per tile of K or V
  static_assert(LD * 64 * AT_WAVES == AT_KEYS * CH || CH == 10, "");
  constexpr int LDX = (AT_KEYS * CH / 64 + AT_WAVES - 1) / AT_WAVES;
  // rows of D = 80 and 96: the last 32-row block of V^T reads past a row's end (results that
  // nobody stores), past the last row into the padding
  __shared__ __attribute__((aligned(16))) uint16_t sK[AT_KEYS * D], sV[AT_KEYS * D + 64];

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.y;
  AtTask t;
  if (PAGED) {
    const int tiles = (a.n_q * a.g + AT_ROWS - 1) / AT_ROWS;
    const int b = blockIdx.x / tiles;
    const int len = min(max(a.lens[b], 0), (int)min((int64_t)a.max_pages << a.lg_page, (int64_t)INT32_MAX / 2));
    t.tok0 = (int64_t)b * a.n_q;
    t.key0 = 0;
    t.r0 = (blockIdx.x - b * tiles) * AT_ROWS;
    t.r1 = min(a.n_q * a.g, t.r0 + AT_ROWS);
    t.nk = a.prefix_len + len;
    t.base = a.prefix_len + len - a.n_q;
    t.floor = a.prefix_len;
    t.own = a.pages + b * a.ld_pages;
  } else if (!at_find(a, blockIdx.x, t)) {
    return;
  }

  // this lane's row: token i of the sequence, head kvh g + h
  const int row = t.r0 + 32 * wave + (lane & 31);
  const bool real = row < t.r1;
  const int rr = real ? row : t.r1 - 1;
  const int i = rr / a.g, h = kvh * a.g + rr - i * a.g;
  auto sees = [&](int tok) { return min(t.nk, max(t.floor, t.base + tok + 1)); };
  const int limit = sees(i);
  // of the block's rows, and the fewest of the wave's
  const int end = max(0, sees((t.r1 - 1) / a.g));
  const int least = sees(min(t.r0 + 32 * wave, t.r1 - 1) / a.g);

  at_u32x4 qf[KS];
  {
    const uint16_t* qp = a.q + (t.tok0 + i) * a.q_st + h * a.q_sh + 8 * half;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *(const at_u32x4*)(qp + 16 * s);
  }

  // address of key j's row; `known` false: its page entry is out of range
  auto key_row = [&](const uint16_t* base, int64_t st, int64_t sh, int j) -> const uint16_t* {
    if (!PAGED) return base + (t.key0 + j) * st + kvh * sh;
    const bool pre = j < a.prefix_len;
    const int o = pre ? j : j - a.prefix_len;
    int page = (pre ? a.prefix_pages : t.own)[o >> a.lg_page];
    if ((unsigned)page >= (unsigned)a.n_pages) page = 0;
    return base + ((((int64_t)page * a.Hkv + kvh) << a.lg_page) + (o & ((1 << a.lg_page) - 1))) * D;
  };

  at_f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
  float m = -INFINITY, l = 0.f;

  for (int j0 = 0; j0 < end; j0 += AT_KEYS) {
    // rows past the last key repeat it: they are masked
#pragma unroll
    for (int x = 0; x < LDX; ++x) {
      const int n = (x * AT_WAVES + wave) * 64 + lane;
      if (x < LD || (x * AT_WAVES + wave) * 64 < AT_KEYS * CH) {
        const int r = n / CH, pc = n - r * CH;
        const int j = min(j0 + r, t.nk - 1);
        __builtin_amdgcn_global_load_lds((at_gptr)(key_row(a.k, a.k_st, a.k_sh, j) + 8 * (pc ^ at_kswz<D>(r))),
                                         (at_lptr)(sK + (x * AT_WAVES + wave) * 512), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((at_gptr)(key_row(a.v, a.v_st, a.v_sh, j) + 8 * (pc ^ at_vswz<D>(r))),
                                         (at_lptr)(sV + (x * AT_WAVES + wave) * 512), 16, 0, 0);
      }
    }
    __syncthreads();

    at_f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
      const int r = 32 * kb + (lane & 31);
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const at_u32x4 kf = *(const at_u32x4*)(sK + r * D + 8 * ((2 * st + half) ^ at_kswz<D>(r)));
        s[kb] = TY::mfma(kf, qf[st], s[kb]);
      }
    }

    // a tile that some row of the wave sees in part
    const bool masked = least < j0 + AT_KEYS;
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + 32 * kb + 8 * (e / 4) + 4 * half + e % 4;
          if (j >= limit) s[kb][e] = -INFINITY;
        }
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
    const float mn = fmaxf(m, top);
    const float at = mn == -INFINITY ? 0.f : mn;             // a row that has seen no key yet
    const float keep = __builtin_amdgcn_exp2f((m - at) * a.c);
    m = mn;
    float mu = at * a.c;
    if (a.c > 1.f) {
      // the largest scores times c are past fp32: the maximum leaves them first
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] -= at;
      mu = 0.f;
    }
    float sum = 0.f;
    at_u32x4 pf[4];                                          // P^T, 16 keys each
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], a.c, -mu));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e + 1], a.c, -mu));
        sum += p0 + p1;
        pf[2 * kb + e / 8][(e % 8) / 2] = TY::pack(p0, p1);
      }
    l = l * keep + sum;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[b][e] *= keep;

    // V^T: lane's element of a 32 x 16 block: row d = lane & 31, keys 4 half + 0..3 and 8 + those
    const int i16 = lane & 15, hi = (lane >> 4) & 1;
    auto v_read = [&](int b, int kc, int e) {
      const int r = 16 * kc + 8 * e + 4 * half + i16 / 4;
      const int ch = 4 * b + 2 * hi + (i16 % 4) / 2;
      const at_s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (at_tr_ptr)(sV + r * D + 8 * (ch ^ at_vswz<D>(r)) + 4 * (i16 & 1)));
      return __builtin_bit_cast(at_u32x2, w);
    };
    uint32_t odd = 0;                       // a sign bit set: some element is infinite or NaN
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int kc = 0; kc < 4; ++kc) {
        const at_u32x2 v0 = v_read(b, kc, 0), v1 = v_read(b, kc, 1);
        at_u32x4 vf = {v0[0], v0[1], v1[0], v1[1]};
        if (masked) {
          // 0 x inf in the product would reach rows that do not see the key: such elements
          // leave the product and are added to the rows that see them
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = (vf[e] & TY::EXP) + TY::CARRY;
            odd |= f;
            if (f & 0x8000u) vf[e] &= 0xffff0000u;
            if (f & 0x80000000u) vf[e] &= 0x0000ffffu;
          }
        }
        o[b] = TY::mfma(vf, pf[kc], o[b]);
      }
    if (masked && __ballot(odd & 0x80008000u)) {
      for (int r = 0; r < AT_KEYS; ++r) {
        if (j0 + r >= limit) continue;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int d = 32 * b + 8 * (e / 4) + 4 * half + e % 4;
            const uint16_t w = sV[r * D + 8 * ((d / 8) ^ at_vswz<D>(r)) + d % 8];
            if (d < D && (w & (TY::EXP & 0xffff)) == (TY::EXP & 0xffff)) o[b][e] += TY::value(w);
          }
      }
    }
    __syncthreads();
  }

  {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  if (!real) return;
  const bool empty = m == -INFINITY && l == 0.f;
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
    a.lse[(t.tok0 + i) * a.Hq + h] = empty ? -INFINITY : m * a.scale + 0.69314718f * __builtin_amdgcn_logf(l);
}

template <class TY, bool PAGED>
static hipError_t attend_launch(const AttendArgs& a, int d, dim3 grid, hipStream_t s) {
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend<TY, 64, PAGED>), grid, dim3(64 * AT_WAVES), 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_attend<TY, 80, PAGED>), grid, dim3(64 * AT_WAVES), 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_attend<TY, 96, PAGED>), grid, dim3(64 * AT_WAVES), 0, s, a); break;
    default: hipLaunchKernelGGL((k_attend<TY, 128, PAGED>), grid, dim3(64 * AT_WAVES), 0, s, a); break;
  }
  return hipGetLastError();
}

static bool attend_rows_ok(const void* p, int64_t st, int64_t sh) {
  return p && ((uintptr_t)p) % 16 == 0 && st >= 0 && sh >= 0 && st % 8 == 0 && sh % 8 == 0;
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
  (void)Tq, (void)Tk, (void)B, (void)Hq, (void)Hkv, (void)d;
  return 0;
}

int slh_attend(const void* q, int64_t q_st, int64_t q_sh, const void* k, int64_t k_st, int64_t k_sh,
               const void* v, int64_t v_st, int64_t v_sh, int32_t dtype, int64_t Tq, int64_t Tk,
               int32_t B, int32_t Hq, int32_t Hkv, int32_t d, const int32_t* cu_q,
               const int32_t* cu_k, double scale, int32_t causal, void* out, int64_t o_st,
               int64_t o_sh, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  (void)workspace, (void)workspace_bytes;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  const int g = Hq / Hkv;
  if (Tq < 0 || Tk < 0 || Tk > INT32_MAX / 2 || Tq * g > INT32_MAX / 2) return SLH_EINVAL;
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
  const dim3 grid((unsigned)(Tq * g / AT_ROWS + B), (unsigned)Hkv);
  (void)hipGetLastError();
  const hipError_t e = dtype == SLH_BF16 ? attend_launch<AtBf16, false>(a, d, grid, (hipStream_t)stream)
                                         : attend_launch<AtF16, false>(a, d, grid, (hipStream_t)stream);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}

int64_t slh_attend_paged_workspace(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d,
                                   int64_t max_len, int64_t prefix_len) {
  (void)B, (void)n_q, (void)Hq, (void)Hkv, (void)d, (void)max_len, (void)prefix_len;
  return 0;
}

int slh_attend_paged(const void* q, int64_t q_st, int64_t q_sh, const void* k_cache,
                     const void* v_cache, int32_t dtype, int64_t n_pages, int32_t page_size,
                     int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d,
                     const int32_t* page_table, int64_t ld_pages, int32_t max_pages,
                     const int32_t* lens, const int32_t* prefix_pages, int64_t prefix_len,
                     double scale, void* out, int64_t o_st, int64_t o_sh, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  (void)workspace, (void)workspace_bytes;
  if (!attend_common_ok(dtype, B, Hq, Hkv, d, scale)) return SLH_EINVAL;
  const int g = Hq / Hkv;
  if (n_q < 0 || (int64_t)B * n_q * g > INT32_MAX / 2) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || page_size < 1 || page_size > 65536 || (page_size & (page_size - 1)))
    return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || (int64_t)max_pages * page_size > INT32_MAX / 4 || prefix_len < 0 ||
      prefix_len > INT32_MAX / 4)
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
  const int64_t tiles = ((int64_t)n_q * g + AT_ROWS - 1) / AT_ROWS;
  const dim3 grid((unsigned)(tiles * B), (unsigned)Hkv);
  (void)hipGetLastError();
  const hipError_t e = dtype == SLH_BF16 ? attend_launch<AtBf16, true>(a, d, grid, (hipStream_t)stream)
                                         : attend_launch<AtF16, true>(a, d, grid, (hipStream_t)stream);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
