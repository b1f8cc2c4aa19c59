// The attention weight that each cached key received from a call's queries, added up by key and key/value head:
//   w[b][h][j] += sum over queries i and query heads of h that see key j of exp(scale q_i . k_j - lse_i)
//
// A key belongs to one wave, which goes through the rows ((token, query head) pairs) that see it: no atomics, the
// same bits every run.  S (rows x keys) = Q K^T by v_mfma_f32_16x16x32, so that a lane holds four rows of one
// key and adds within its registers; the four lane groups of a key are added at the end.
//
// The exponent is formed as scale s - lse, in that order, and multiplied by log2(e) after: both sides may be large, and
// only their difference has to be exact.  Everything is fp32.
#include "attend8.h"
#include "attend_plan.h"

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
};

constexpr int WT_KEYS = 32;              // of a wave

template <class TY, int D, bool E8>
__global__ __launch_bounds__(256) void k_weights(WeightArgs a) {
  constexpr int KS = (D + 31) / 32, X = D / 64, R = D % 64, KT = WT_KEYS / 16;
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

  // keys of this lane, one of each 16, in the type of the queries
  at_u32x4 kf[KT][KS];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int j = min(key0 + 16 * t + r16, n - 1);
    const int page = a.pages[b * a.ld_pages + (j >> a.lg_page)];
    const int64_t line = (((int64_t)((unsigned)page < (unsigned)a.n_pages ? page : 0) * a.Hkv + kvh) << a.lg_page) +
                         (j & ((1 << a.lg_page) - 1));
    if constexpr (E8) {
      const uint8_t* kp = (const uint8_t*)a.k + line * D;
      const float two = c8_two(a.k_two[line >> a.lg_block]);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        at_u32x2 c = {0, 0};
        if (!R || s < KS - 1)
          c = *(const at_u32x2*)(kp + 64 * (s / 2) + 16 * grp + 8 * (s & 1));
        else if (8 * grp < R)
          c = *(const at_u32x2*)(kp + 64 * X + 8 * grp);
        kf[t][s] = at_u32x4{c8_pair<TY, false>(c[0], two), c8_pair<TY, true>(c[0], two), c8_pair<TY, false>(c[1], two),
                            c8_pair<TY, true>(c[1], two)};
      }
    } else {
      const uint16_t* kp = (const uint16_t*)a.k + line * D;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        kf[t][s] = at_u32x4{0, 0, 0, 0};
        if (32 * s + 8 * grp < D) kf[t][s] = *(const at_u32x4*)(kp + 32 * s + 8 * grp);
      }
    }
  }
  // first element of a row in step s
  auto d_of = [&](int s) {
    if (!E8) return 32 * s + 8 * grp;
    return !R || s < KS - 1 ? 64 * (s / 2) + 16 * grp + 8 * (s & 1) : 64 * X + 8 * grp;
  };

  float sum[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) sum[t] = 0.f;
  // the first row that sees one of the keys
  for (int r0 = max(0, key0 - (n - nq)) * a.g; r0 < rows; r0 += 16) {
    const int rr = min(r0 + r16, rows - 1), i = rr / a.g, h = kvh * a.g + rr - i * a.g;
    const uint16_t* qp = a.q + (q0 + i) * a.q_st + h * a.q_sh;
    at_f32x4 sc[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) sc[t] = at_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      at_u32x4 qf = {0, 0, 0, 0};
      if (d_of(s) < D) qf = *(const at_u32x4*)(qp + d_of(s));
#pragma unroll
      for (int t = 0; t < KT; ++t) sc[t] = TY::mfma16(qf, kf[t][s], sc[t]);
    }
    at_products_done(sc);
    float part[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) part[t] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = r0 + 4 * grp + e, tok = row / a.g;
      const float lse = row < rows ? a.lse[(q0 + tok) * a.Hq + kvh * a.g + row - tok * a.g] : -INFINITY;
      const int limit = lse == -INFINITY ? 0 : n - nq + tok + 1;         // such a row has no weights to give
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][e], a.scale, -lse) * 1.44269504f);
        part[t] += key0 + 16 * t + r16 < limit ? p : 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] += part[t];
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[t]), __float_as_uint(sum[t]), false, false);
    sum[t] = __uint_as_float(w32[0]) + __uint_as_float(w32[1]);
    const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[t]), __float_as_uint(sum[t]), false, false);
    sum[t] = __uint_as_float(w16[0]) + __uint_as_float(w16[1]);
    const int j = key0 + 16 * t + r16;
    if (grp == 0 && j < n) a.w[((int64_t)b * a.Hkv + kvh) * a.max_rows + j] += sum[t];
  }
}

template <class TY, bool E8>
static void weights_launch(const WeightArgs& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_weights<TY, 64, E8>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_weights<TY, 80, E8>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_weights<TY, 96, E8>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_weights<TY, 128, E8>), grid, block, 0, s, a); break;
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
  return 0;
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
  (void)workspace, (void)workspace_bytes;
  WeightArgs a = {};
  a.q = (const uint16_t*)q, a.q_st = q_st, a.q_sh = q_sh;
  a.k = k_cache, a.k_two = (const uint8_t*)k_scale;
  a.n_pages = (int)n_pages, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.lg_block = k_scale ? __builtin_ctz((unsigned)block) : 0;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_rows = max_pages * page_size;
  a.lens = lens, a.cu = cu_q, a.B = B, a.n_each = cu_q ? 0 : (int)(Tq / B), a.Hq = Hq, a.Hkv = Hkv, a.g = Hq / Hkv;
  a.Tq = Tq, a.lse = lse, a.scale = (float)scale, a.w = weights;
  a.key_blocks = (a.max_rows + 4 * WT_KEYS - 1) / (4 * WT_KEYS);
  const int64_t blocks = (int64_t)B * Hkv * a.key_blocks;
  (void)hipGetLastError();
  hipStream_t s = (hipStream_t)stream;
  if (dtype == SLH_BF16)
    k_scale ? weights_launch<AtBf16, true>(a, d, blocks, s) : weights_launch<AtBf16, false>(a, d, blocks, s);
  else
    k_scale ? weights_launch<AtF16, true>(a, d, blocks, s) : weights_launch<AtF16, false>(a, d, blocks, s);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
