// Rows of heads on their way to attention: loads and stores of eight elements, the RMS norm of a
// head and the rotation at its token's position.  A row of d elements belongs to LPR lanes with two
// 8-element chunks each: a chunk of the rotation's first half and its partner, so that the half
// layout needs no exchange between lanes; the norm's sum of squares is the only one (DPP within at
// most 16 lanes).
#pragma once
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

// Eight elements as they are loaded.
template <int DT> struct RpRaw {
  typename RpType<DT>::vec v;
  __device__ __forceinline__ void load(const typename RpType<DT>::elem* p) { v = *(const typename RpType<DT>::vec*)p; }
  __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
};
template <> struct RpRaw<SLH_F32> {
  rp_f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const rp_f32x4*)p, b = *(const rp_f32x4*)(p + 4); }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e] : b[e - 4]; }
};

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

// The chunks of lane p of a row: a rotated pair, or two neighbours of what is not rotated.
struct RopeLane { bool pair, has0, has1; int c0, c1; };
__device__ __forceinline__ RopeLane rp_lane(int p, int rot, int d) {
  const int nr = rot >> 4, nc = d >> 3;
  const bool pair = p < nr;
  const int c0 = pair ? p : 2 * p, c1 = pair ? p + nr : c0 + 1;
  return RopeLane{pair, c0 < nc, c1 < nc, c0, c1};
}

// What all rows of a call share.
struct RopeForm {
  int d, rot, interleaved;
  float eps;
  const float* table;     // [n_pos][2][rot / 2]
  int64_t n_pos;
};

// The table's cosines and sines for a lane's chunks at position `at`.
struct RopeTurn {
  rp_f32x4 c[2], s[2];
  float bad;              // NaN for a position that the table lacks, which shows
};
__device__ __forceinline__ RopeTurn rp_turn_of(const RopeForm& a, const RopeLane& l, int p, int at) {
  const int half = a.rot >> 1;
  const bool known = at >= 0 && at < a.n_pos;
  const float* row_cos = a.table + (known ? (int64_t)at * a.rot : 0);
  RopeTurn r;
  r.bad = known ? 0.f : __builtin_nanf("");
  // pairs (i, i + rot / 2): eights of both; pairs (2 i, 2 i + 1): four of each chunk
  const int i0 = a.interleaved ? 4 * l.c0 : 8 * p, i1 = a.interleaved ? 4 * l.c1 : 8 * p + 4;
  r.c[0] = *(const rp_f32x4*)(row_cos + i0), r.c[1] = *(const rp_f32x4*)(row_cos + i1);
  r.s[0] = *(const rp_f32x4*)(row_cos + half + i0), r.s[1] = *(const rp_f32x4*)(row_cos + half + i1);
  return r;
}
__device__ __forceinline__ void rp_turn(const RopeForm& a, const RopeTurn& r, float (&x0)[8], float (&x1)[8]) {
  if (!a.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = x0[e], v = x1[e], c = r.c[e / 4][e % 4], sn = r.s[e / 4][e % 4];
      x0[e] = u * c - v * sn + r.bad;
      x1[e] = v * c + u * sn + r.bad;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float(&x)[8] = q ? x1 : x0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = x[2 * e], v = x[2 * e + 1], c = r.c[q][e], sn = r.s[q][e];
        x[2 * e] = u * c - v * sn + r.bad;
        x[2 * e + 1] = v * c + u * sn + r.bad;
      }
    }
  }
}

// 1 / sqrt(mean of the squares + eps) of a row; every lane of it takes part.
template <int LPR>
__device__ __forceinline__ float rp_inverse(const RopeForm& a, const float (&x0)[8], const float (&x1)[8]) {
  float sq = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(x0[e], x0[e], __builtin_fmaf(x1[e], x1[e], sq));
  sq = rp_group_sum<LPR>(sq);
  return 1.0f / sqrtf(sq / (float)a.d + a.eps);
}

// Norm (where there are weights) and rotation (turn) of a row at position *pos; every lane of the
// row's LPR takes part.
template <int DT, int LPR>
__device__ __forceinline__ void rp_norm_turn(const RopeForm& a, const RopeLane& l, int p, const void* weights, bool turn,
                                             const int* pos, float (&x0)[8], float (&x1)[8]) {
  typedef typename RpType<DT>::elem elem;
  const bool pair = l.pair, has0 = l.has0, has1 = l.has1;
  const int c0 = l.c0, c1 = l.c1;
  if (weights) {
    const float inv = rp_inverse<LPR>(a, x0, x1);
    float w[8];
    if (has0) {
      rp_load8<DT>((const elem*)weights + 8 * c0, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x0[e] = x0[e] * inv * w[e];
    }
    if (has1) {
      rp_load8<DT>((const elem*)weights + 8 * c1, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x1[e] = x1[e] * inv * w[e];
    }
  }
  if (turn && pair) {
    const RopeTurn r = rp_turn_of(a, l, p, *pos);
    rp_turn(a, r, x0, x1);
  }
}

// Rows of `H` heads behind a pointer: aligned to 16 bytes, strides in whole chunks of 8.
inline bool rope_rows_ok(const void* p, int64_t st, int64_t sh) {
  return p && ((uintptr_t)p) % 16 == 0 && st >= 0 && sh >= 0 && st % 8 == 0 && sh % 8 == 0;
}

inline bool rope_common_ok(int dtype, int64_t T, int64_t heads, int d, const void* w0, const void* w1,
                           double eps, const float* table, int64_t n_pos, int rot, const int* pos) {
  if (dtype != SLH_BF16 && dtype != SLH_F32 && dtype != SLH_F16) return false;
  if (T < 0 || heads < 1 || d < 8 || d > 256 || d % 8 != 0) return false;
  if (T > 0 && T * heads > (int64_t)INT32_MAX / 16) return false;
  if (((uintptr_t)w0) % 16 != 0 || ((uintptr_t)w1) % 16 != 0) return false;
  if (!(eps >= 0.0) || std::isinf(eps)) return false;
  if (!table) return rot == 0;
  return ((uintptr_t)table) % 16 == 0 && (pos || T == 0) && n_pos >= 1 && rot >= 16 && rot <= d && rot % 16 == 0;
}

}  // namespace slh
