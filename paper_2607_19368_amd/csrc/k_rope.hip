// What happens to the rows of a projection before attention reads them: the RMS norm of
// each head, the rotation at the token's position, and, for keys and values, the way into
// a paged cache.
//
//   y = x / sqrt(mean(x^2) + eps) * w            (per head, where weights are given)
//   (a, b) -> (a cos - b sin, b cos + a sin)     pairs (i, i + rot/2), or (2i, 2i + 1)
//
// Arithmetic in fp32, one rounding at the end.  Bound by memory: each row is read once and
// written once, and a token's rot cosines and sines (fp32) are read from L1 or L2 by its heads.
//
// Measured, d = 128 (a copy of 4 GiB reaches 4.75 TB/s, reads and writes together): 32768 bf16 tokens of
// 28 + 4 heads, norms and rotation, 554 MB in 109 us = 5.1 TB/s; 5003 fp32 tokens of 12 + 12 heads of 80,
// 32 elements rotated, 77.5 MB in 18.4 us = 4.2 TB/s; 16384 fp16 tokens of 8 heads into a paged cache, 143 MB in 33 us =
// 4.3 TB/s; 24 tokens 3.7 us, which is the launch's.  The table of 65536 positions of 128 elements 18 us, of 2^20 213 us =
// 2.5 TB/s (a sine and a cosine in 64 bits for 8 bytes; a program makes it once).
#include "rope_rows.h"

namespace slh {

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
  RopeForm form;
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

  const RopeLane l = rp_lane(p, a.form.rot, a.form.d);
  float x0[8] = {}, x1[8] = {};
  const elem* src = (const elem*)s.x + t * s.st + h * s.sh;
  if (l.has0) rp_load8<DT>(src + 8 * l.c0, x0);
  if (l.has1) rp_load8<DT>(src + 8 * l.c1, x1);

  rp_norm_turn<DT, LPR>(a.form, l, p, s.w, s.turn, a.pos + t, x0, x1);

  if (!real) return;
  elem* dst;
  if (a.slots) {
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const int64_t page = slot >> a.lg_page, in = slot & (((int64_t)1 << a.lg_page) - 1);
    dst = (elem*)s.out + ((((page * s.H + h) << a.lg_page) + in) * a.form.d);
  } else {
    dst = (elem*)s.out + t * s.ot + h * s.oh;
  }
  if (l.has0) rp_store8<DT>(dst + 8 * l.c0, x0);
  if (l.has1) rp_store8<DT>(dst + 8 * l.c1, x1);
}

template <int DT>
static hipError_t rope_launch(RopeArgs a, hipStream_t s) {
  // lanes a row: the rotated pairs and half of the other chunks, d / 16 rounded up
  const int need = (a.form.d / 8 + 1) / 2;
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
  a.form = RopeForm{d, rot_dim, interleaved != 0, (float)eps, table, n_pos};
  a.pos = pos;
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
  a.form = RopeForm{d, rot_dim, interleaved != 0, (float)eps, table, n_pos};
  a.pos = pos;
  a.slots = slots, a.n_slots = n_pages * page_size, a.lg_page = __builtin_ctz((unsigned)page_size);
  return rope_run(a, dtype, (hipStream_t)stream);
}

}  // extern "C"
