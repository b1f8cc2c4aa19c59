// What happens to the rows of a projection before attention reads them: the RMS norm of
// each head, the rotation at the token's position, and, for keys and values, the way into
// a paged cache.
//
//   y = x / sqrt(mean(x^2) + eps) * w            (per head, where weights are given)
//   (a, b) -> (a cos - b sin, b cos + a sin)     pairs (i, i + rot/2), or (2i, 2i + 1)
//
// Arithmetic in fp32, one rounding at the end.  Bound by memory: each row is read once and
// written once, and a token's rot cosines and sines (fp32) are read from L1 or L2 by its heads.
// A row of d elements belongs to LPR lanes with two 8-element chunks each: a chunk of the
// rotation's first half and its partner, so that the half layout needs no exchange between
// lanes; the norm's sum of squares is the only one (DPP within at most 16 lanes).
//
// Measured, d = 128 (a copy of 4 GiB reaches 4.75 TB/s, reads and writes together): 32768 bf16 tokens of
// 28 + 4 heads, norms and rotation, 554 MB in 109 us = 5.1 TB/s; 5003 fp32 tokens of 12 + 12 heads of 80,
// 32 elements rotated, 77.5 MB in 18.4 us = 4.2 TB/s; 16384 fp16 tokens of 8 heads into a paged cache, 143 MB in 33 us =
// 4.3 TB/s; 24 tokens 3.7 us, which is the launch's.  The table of 65536 positions of 128 elements 18 us, of 2^20 213 us =
// 2.5 TB/s (a sine and a cosine in 64 bits for 8 bytes; a program makes it once).
#include "slh_device.h"
#include "slh_internal.h"

#include <cmath>

#include "slh.h"

namespace slh {

typedef __bf16 rp_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 rp_f16x8 __attribute__((ext_vector_type(8)));
typedef float rp_f32x4 __attribute__((ext_vector_type(4)));

template <int DT> struct RpType;
template <> struct RpType<SLH_BF16> { typedef uint16_t elem; typedef rp_bf16x8 vec; };
template <> struct RpType<SLH_F16> { typedef uint16_t elem; typedef rp_f16x8 vec; };
template <> struct RpType<SLH_F32> { typedef float elem; };

template <int DT>
__device__ __forceinline__ void rp_load8(const typename RpType<DT>::elem* p, float (&x)[8]) {
  if constexpr (DT == SLH_F32) {
    const rp_f32x4 a = *(const rp_f32x4*)p, b = *(const rp_f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    const auto v = *(const typename RpType<DT>::vec*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  }
}

template <int DT>
__device__ __forceinline__ void rp_store8(typename RpType<DT>::elem* p, const float (&x)[8]) {
  if constexpr (DT == SLH_F32) {
    *(rp_f32x4*)p = rp_f32x4{x[0], x[1], x[2], x[3]};
    *(rp_f32x4*)(p + 4) = rp_f32x4{x[4], x[5], x[6], x[7]};
  } else {
    typename RpType<DT>::vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
    *(typename RpType<DT>::vec*)p = v;
  }
}

// sum over aligned groups of LPR lanes (every lane active; the same bits in all of them)
template <int LPR>
__device__ __forceinline__ float rp_group_sum(float v) {
  if constexpr (LPR >= 2)
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP_XOR1, 0xF, 0xF, false));
  if constexpr (LPR >= 4)
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP_XOR2, 0xF, 0xF, false));
  if constexpr (LPR >= 8)
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP_HALF_MIRROR, 0xF, 0xF, false));
  if constexpr (LPR >= 16)
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP_ROR8, 0xF, 0xF, false));
  return v;
}

// One of the two row sets of a launch: `H` heads of every token.  Each set has blocks of
// its own, so that its fields are wave-uniform.
struct RopeSet {
  const void* x;          // element (t, h, e) at t st + h sh + e
  int64_t st, sh;
  int H;
  const void* w;          // [d] norm weights, NULL: no norm
  int turn;               // rotated
  void* out;              // as x; with slots: the cache [pages][H][page][d]
  int64_t ot, oh;
};
struct RopeArgs {
  RopeSet set[2];
  int T;
  int blocks0;            // blocks of set 0
  int d, rot, interleaved;
  float eps;
  const float* table;     // [n_pos][2][rot / 2]
  int64_t n_pos;
  const int* pos;         // [T]
  const int64_t* slots;   // [T] row of the paged cache per token (NULL: outputs by strides)
  int64_t n_slots;
  int lg_page;
};

template <int DT, int LPR>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a) {
  typedef typename RpType<DT>::elem elem;
  const bool second = (int)blockIdx.x >= a.blocks0;
  const RopeSet s = a.set[second];
  const int r = (((int)blockIdx.x - (second ? a.blocks0 : 0)) * 256 + (int)threadIdx.x) / LPR;
  const int p = threadIdx.x % LPR;
  // rows past the end take row 0's part in the sums and store nothing
  const bool real = r < a.T * s.H;
  const int row = real ? r : 0;
  const int t = (int)((unsigned)row / (unsigned)s.H);
  const int h = row - t * s.H;

  // chunks of this lane: a rotated pair, or two neighbours of what is not rotated
  const int nr = a.rot >> 4, nc = a.d >> 3;
  const bool pair = p < nr;
  const int c0 = pair ? p : 2 * p, c1 = pair ? p + nr : c0 + 1;
  const bool has0 = c0 < nc, has1 = c1 < nc;
  float x0[8] = {}, x1[8] = {};
  const elem* src = (const elem*)s.x + t * s.st + h * s.sh;
  if (has0) rp_load8<DT>(src + 8 * c0, x0);
  if (has1) rp_load8<DT>(src + 8 * c1, x1);

  if (s.w) {
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(x0[e], x0[e], __builtin_fmaf(x1[e], x1[e], sq));
    sq = rp_group_sum<LPR>(sq);
    const float inv = 1.0f / sqrtf(sq / (float)a.d + a.eps);
    float w[8];
    if (has0) {
      rp_load8<DT>((const elem*)s.w + 8 * c0, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x0[e] = x0[e] * inv * w[e];
    }
    if (has1) {
      rp_load8<DT>((const elem*)s.w + 8 * c1, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x1[e] = x1[e] * inv * w[e];
    }
  }
  if (s.turn && pair) {
    const int at = a.pos[t], half = a.rot >> 1;
    const bool known = at >= 0 && at < a.n_pos;
    const float* row_cos = a.table + (known ? (int64_t)at * a.rot : 0);
    const float bad = known ? 0.f : __builtin_nanf("");     // a position that the table lacks shows
    if (!a.interleaved) {
      float c[8], sn[8];
      rp_load8<SLH_F32>(row_cos + 8 * p, c);
      rp_load8<SLH_F32>(row_cos + half + 8 * p, sn);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = x0[e], v = x1[e];
        x0[e] = u * c[e] - v * sn[e] + bad;
        x1[e] = v * c[e] + u * sn[e] + bad;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float(&x)[8] = q ? x1 : x0;
        const int i0 = 4 * (q ? c1 : c0);
        const rp_f32x4 c = *(const rp_f32x4*)(row_cos + i0), sn = *(const rp_f32x4*)(row_cos + half + i0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[2 * e], v = x[2 * e + 1];
          x[2 * e] = u * c[e] - v * sn[e] + bad;
          x[2 * e + 1] = v * c[e] + u * sn[e] + bad;
        }
      }
    }
  }

  if (!real) return;
  elem* dst;
  if (a.slots) {
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const int64_t page = slot >> a.lg_page, in = slot & (((int64_t)1 << a.lg_page) - 1);
    dst = (elem*)s.out + ((((page * s.H + h) << a.lg_page) + in) * a.d);
  } else {
    dst = (elem*)s.out + t * s.ot + h * s.oh;
  }
  if (has0) rp_store8<DT>(dst + 8 * c0, x0);
  if (has1) rp_store8<DT>(dst + 8 * c1, x1);
}

template <int DT>
static hipError_t rope_launch(RopeArgs a, hipStream_t s) {
  // lanes a row: the rotated pairs and half of the other chunks, d / 16 rounded up
  const int need = (a.d / 8 + 1) / 2;
  auto go = [&](auto kernel, int lpr) {
    auto blocks = [&](int H) { return (int)(((int64_t)a.T * H * lpr + 255) / 256); };
    a.blocks0 = blocks(a.set[0].H);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.blocks0 + blocks(a.set[1].H))), dim3(256), 0, s, a);
  };
  if (need <= 1) go(k_rope<DT, 1>, 1);
  else if (need <= 2) go(k_rope<DT, 2>, 2);
  else if (need <= 4) go(k_rope<DT, 4>, 4);
  else if (need <= 8) go(k_rope<DT, 8>, 8);
  else go(k_rope<DT, 16>, 16);
  return hipGetLastError();
}

static int rope_run(const RopeArgs& a, int dtype, hipStream_t s) {
  (void)hipGetLastError();
  const hipError_t e = dtype == SLH_BF16  ? rope_launch<SLH_BF16>(a, s)
                       : dtype == SLH_F16 ? rope_launch<SLH_F16>(a, s)
                                          : rope_launch<SLH_F32>(a, s);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}

// Rows of `H` heads behind a pointer: aligned to 16 bytes, strides in whole chunks of 8.
static bool rope_rows_ok(const void* p, int64_t st, int64_t sh) {
  return p && ((uintptr_t)p) % 16 == 0 && st >= 0 && sh >= 0 && st % 8 == 0 && sh % 8 == 0;
}

static bool rope_common_ok(int dtype, int64_t T, int64_t heads, int d, const void* w0, const void* w1,
                           double eps, const float* table, int64_t n_pos, int rot, const int* pos) {
  if (dtype != SLH_BF16 && dtype != SLH_F32 && dtype != SLH_F16) return false;
  if (T < 0 || heads < 1 || d < 8 || d > 256 || d % 8 != 0) return false;
  if (T > 0 && T * heads > (int64_t)INT32_MAX / 16) return false;
  if (((uintptr_t)w0) % 16 != 0 || ((uintptr_t)w1) % 16 != 0) return false;
  if (!(eps >= 0.0) || std::isinf(eps)) return false;
  if (!table) return rot == 0;
  return ((uintptr_t)table) % 16 == 0 && (pos || T == 0) && n_pos >= 1 && rot >= 16 && rot <= d && rot % 16 == 0;
}

struct RopeFreqs { double f[128]; };

__global__ __launch_bounds__(256) void k_rope_table(float* table, int64_t n, int half, double mscale,
                                                    RopeFreqs fr) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t p = i / half;
  const int e = (int)(i - p * half);
  double sn, cs;
  sincos((double)p * fr.f[e], &sn, &cs);
  table[p * 2 * half + e] = (float)(mscale * cs);
  table[p * 2 * half + half + e] = (float)(mscale * sn);
}

}  // namespace slh

extern "C" {

int slh_rope_table(float* table, int64_t n_pos, int32_t rot_dim, double base, int32_t scaling,
                   double factor, int64_t orig_len, double beta_fast, double beta_slow,
                   void* stream) {
  using namespace slh;
  if (!table || ((uintptr_t)table) % 16 != 0 || n_pos < 1 || n_pos > ((int64_t)1 << 31)) return SLH_EINVAL;
  if (rot_dim < 16 || rot_dim > 256 || rot_dim % 16 != 0) return SLH_EINVAL;
  if (!(base > 1.0) || std::isinf(base)) return SLH_EINVAL;
  if (scaling < SLH_ROPE_PLAIN || scaling > SLH_ROPE_BANDS) return SLH_EINVAL;
  if (scaling != SLH_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return SLH_EINVAL;
  if (scaling == SLH_ROPE_BANDS &&
      (orig_len < 1 || !(beta_slow > 0.0) || !(beta_fast > beta_slow) || std::isinf(beta_fast)))
    return SLH_EINVAL;
  const int half = rot_dim / 2;
  const int64_t n = n_pos * half, blocks = (n + 255) / 256;
  if (blocks * 256 > (int64_t)UINT32_MAX) return SLH_EINVAL;      // threads of a launch
  RopeFreqs fr = {};
  double mscale = 1.0;
  if (scaling == SLH_ROPE_BASE) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  for (int i = 0; i < half; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == SLH_ROPE_LINEAR) f /= factor;
    if (scaling == SLH_ROPE_BANDS) {
      const double turns = (double)orig_len * f / (2.0 * M_PI);
      const double keep = std::fmin(1.0, std::fmax(0.0, (turns - beta_slow) / (beta_fast - beta_slow)));
      f = keep * f + (1.0 - keep) * f / factor;
    }
    fr.f[i] = f;
  }
  if (scaling == SLH_ROPE_BANDS) mscale = 0.1 * std::log(factor) + 1.0;
  (void)hipGetLastError();
  hipLaunchKernelGGL(k_rope_table, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, table, n, half,
                     mscale, fr);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

int slh_qk_norm_rope(const void* q, int64_t q_st, int64_t q_sh, int32_t Hq, void* q_out,
                     int64_t qo_st, int64_t qo_sh, const void* k, int64_t k_st, int64_t k_sh,
                     int32_t Hk, void* k_out, int64_t ko_st, int64_t ko_sh, int32_t dtype,
                     int64_t T, int32_t d, const void* q_weight, const void* k_weight, double eps,
                     const float* table, int64_t n_pos, int32_t rot_dim, const int32_t* pos,
                     int32_t interleaved, void* stream) {
  using namespace slh;
  if (Hq < 0 || Hk < 0 || Hq > 65536 || Hk > 65536) return SLH_EINVAL;
  if (!rope_common_ok(dtype, T, (int64_t)Hq + Hk, d, q_weight, k_weight, eps, table, n_pos, rot_dim, pos))
    return SLH_EINVAL;
  if (T == 0) return SLH_OK;
  if (Hq && !(rope_rows_ok(q, q_st, q_sh) && rope_rows_ok(q_out, qo_st, qo_sh))) return SLH_EINVAL;
  if (Hk && !(rope_rows_ok(k, k_st, k_sh) && rope_rows_ok(k_out, ko_st, ko_sh))) return SLH_EINVAL;
  const int turn = table != nullptr;
  RopeArgs a = {};
  a.set[0] = {q, q_st, q_sh, Hq, q_weight, turn, q_out, qo_st, qo_sh};
  a.set[1] = {k, k_st, k_sh, Hk, k_weight, turn, k_out, ko_st, ko_sh};
  a.T = (int)T;
  a.d = d, a.rot = rot_dim, a.interleaved = interleaved != 0, a.eps = (float)eps;
  a.table = table, a.n_pos = n_pos, a.pos = pos;
  return rope_run(a, dtype, (hipStream_t)stream);
}

int slh_kv_append(const void* k, int64_t k_st, int64_t k_sh, const void* v, int64_t v_st,
                  int64_t v_sh, int32_t dtype, int64_t T, int32_t H, int32_t d,
                  const void* k_weight, double eps, const float* table, int64_t n_pos,
                  int32_t rot_dim, const int32_t* pos, int32_t interleaved, void* k_cache,
                  void* v_cache, int64_t n_pages, int32_t page_size, const int64_t* slots,
                  void* stream) {
  using namespace slh;
  if (H < 1 || H > 65536) return SLH_EINVAL;
  if (!rope_common_ok(dtype, T, 2 * (int64_t)H, d, k_weight, nullptr, eps, table, n_pos, rot_dim, pos))
    return SLH_EINVAL;
  if (n_pages < 0 || n_pages > INT32_MAX || page_size < 1 || page_size > 65536 ||
      (page_size & (page_size - 1)))
    return SLH_EINVAL;
  if (T == 0) return SLH_OK;
  if (!rope_rows_ok(k, k_st, k_sh) || !rope_rows_ok(v, v_st, v_sh) || !rope_rows_ok(k_cache, 0, 0) ||
      !rope_rows_ok(v_cache, 0, 0) || !slots)
    return SLH_EINVAL;
  RopeArgs a = {};
  a.set[0] = {k, k_st, k_sh, H, k_weight, table != nullptr, k_cache, 0, 0};
  a.set[1] = {v, v_st, v_sh, H, nullptr, 0, v_cache, 0, 0};
  a.T = (int)T;
  a.d = d, a.rot = rot_dim, a.interleaved = interleaved != 0, a.eps = (float)eps;
  a.table = table, a.n_pos = n_pos, a.pos = pos;
  a.slots = slots, a.n_slots = n_pages * page_size, a.lg_page = __builtin_ctz((unsigned)page_size);
  return rope_run(a, dtype, (hipStream_t)stream);
}

}  // extern "C"
