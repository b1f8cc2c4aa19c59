// Kernels of attend_rows.h, and the one that joins the splits of a row.
#include "attend_rows.h"

namespace slh {

template <class TY, int D, int NR, bool PAGED>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend_rows(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t smem[rw_lds<D, NR>()];
  attend_rows<TY, D, NR, PAGED>(a, blockIdx.x, smem);
}

template <class TY, int NR, bool PAGED>
static void rows_launch(const AttendArgs& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend_rows<TY, 64, NR, PAGED>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_attend_rows<TY, 80, NR, PAGED>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_attend_rows<TY, 96, NR, PAGED>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_attend_rows<TY, 128, NR, PAGED>), grid, block, 0, s, a); break;
  }
}

template <class TY>
static void rows_pick(const AttendArgs& a, bool paged, int rows, int d, int64_t blocks, hipStream_t s) {
  if (paged)
    rows == 16 ? rows_launch<TY, 1, true>(a, d, blocks, s) : rows_launch<TY, 2, true>(a, d, blocks, s);
  else
    rows == 16 ? rows_launch<TY, 1, false>(a, d, blocks, s) : rows_launch<TY, 2, false>(a, d, blocks, s);
}

hipError_t launch_attend_rows(const AttendArgs& a, bool paged, bool bf16, int rows, int d, int64_t blocks,
                              hipStream_t s) {
  bf16 ? rows_pick<AtBf16>(a, paged, rows, d, blocks, s) : rows_pick<AtF16>(a, paged, rows, d, blocks, s);
  return hipGetLastError();
}

// Joins the splits of each row: out = sum_s w_s o_s / sum_s w_s l_s, w_s = exp2((m_s - max m) c).
// WAVES waves a row: their lanes find the weights of 64 splits at a time, then the half waves take
// the splits in turn, four elements a lane, four splits in flight.  One wave where there are many
// rows; four where few rows of many splits would leave it to the latency of 16 loads after another (a
// call with 28 rows, 64 splits: 18.2 instead of 21.8 us; 224 rows, 18 splits: 13.9, 15.4; 1280 rows: 26.9, 27.4;
// 2048 rows: 41.3, 40.9).  Bound by memory: partial results are fp32, 4 d + 8
// bytes a row and split, read once (128 tokens of 28 heads, up to 19 splits: 35 MB in 8.5 us;
// 387 tokens of 40 heads, 4 splits: 32 MB in 11 us).
template <class TY, int WAVES>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int d, int slots, int64_t row0) {
  constexpr int PARTS = 2 * WAVES;                 // half waves of a row
  __shared__ at_f32x4 s_o[WAVES == 1 ? 1 : WAVES * 32];
  const int lane = threadIdx.x & 63, half = lane >> 5, e = 4 * (lane & 31);
  const int wave = threadIdx.x >> 6, part = WAVES == 1 ? half : 2 * wave + half;
  const int64_t r = row0 + (WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x);
  if (r >= a.rows) return;
  const int64_t tok = r / a.Hq;
  const int h = (int)(r - tok * a.Hq);
  // packed rows in front of the first sequence or behind the last have no results
  if (a.cu_q && (tok < a.cu_q[0] || tok >= a.cu_q[a.B])) return;
  auto ml = [&](int s) { return *(const float2*)(a.part_ml + 2 * (s * a.rows + r)); };
  auto is_empty = [](float2 v) { return v.y == AT_NO_KEY; };
  const float2 none = make_float2(-INFINITY, AT_NO_KEY);
  const float2 first = lane < slots ? ml(lane) : none;
  float top = first.x;
  bool any = !is_empty(first);
  for (int s = lane + 64; s < slots; s += 64) {
    const float2 v = ml(s);
    top = fmaxf(top, v.x);
    any |= !is_empty(v);
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float ref = top == -INFINITY ? 0.f : top;
  const bool empty = __ballot(any) == 0;
  float l = 0.f;
  at_f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < slots; s0 += 64) {
    float2 v = first;
    if (s0) v = s0 + lane < slots ? ml(s0 + lane) : none;
    // an empty split has no sums: weight 0, and nothing of it is read
    const float w = is_empty(v) ? 0.f : __builtin_amdgcn_exp2f((v.x - ref) * a.c);
    l += is_empty(v) ? 0.f : w * v.y;
    const unsigned long long there = __ballot(!is_empty(v));
    const int n = min(64, slots - s0);
    for (int s1 = 0; s1 < n; s1 += 4 * PARTS) {
      at_f32x4 x[4];
      float ws[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = s1 + part + PARTS * q;
        x[q] = at_f32x4{0.f, 0.f, 0.f, 0.f};
        ws[q] = __shfl(w, at & 63);
        if (at < n && ((there >> at) & 1) && e < d) x[q] = *(const at_f32x4*)(a.part_o + ((s0 + at) * a.rows + r) * d + e);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (s1 + part + PARTS * q < n) {
#pragma unroll
          for (int c = 0; c < 4; ++c) o[c] = __builtin_fmaf(ws[q], x[q][c], o[c]);
        }
    }
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x);
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] += __shfl_xor(o[c], 32);
  if constexpr (WAVES > 1) {
    if (half == 0) s_o[32 * wave + lane] = o;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      const at_f32x4 x = s_o[32 * w + (lane & 31)];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += x[c];
    }
  }
  const float inv = at_inverse(empty, l);
  if (half == 0 && e < d)
    *(at_u32x2*)(a.out + tok * a.o_st + h * a.o_sh + e) =
        at_u32x2{TY::pack(o[0] * inv, o[1] * inv), TY::pack(o[2] * inv, o[3] * inv)};
  if (a.lse && lane == 0) a.lse[r] = empty ? -INFINITY : top * a.scale + 0.69314718f * (__builtin_amdgcn_logf(l) - TY::LIFT);
}

hipError_t launch_attend_join(const AttendArgs& a, bool bf16, int d, int slots, hipStream_t s) {
  const bool wide = slots > 8 && a.rows <= 1024;
  const dim3 block(256);
  // a launch has fewer than 2^32 threads: 2^25 rows, a wave each, at a time
  constexpr int64_t MOST = (int64_t)1 << 25;
  for (int64_t row0 = 0; row0 < a.rows; row0 += MOST) {
    const int64_t rows = a.rows - row0 < MOST ? a.rows - row0 : MOST;
    const dim3 grid((unsigned)(wide ? rows : (rows + 3) / 4));
    if (bf16 && wide)
      hipLaunchKernelGGL((k_attend_join<AtBf16, 4>), grid, block, 0, s, a, d, slots, row0);
    else if (bf16)
      hipLaunchKernelGGL((k_attend_join<AtBf16, 1>), grid, block, 0, s, a, d, slots, row0);
    else if (wide)
      hipLaunchKernelGGL((k_attend_join<AtF16, 4>), grid, block, 0, s, a, d, slots, row0);
    else
      hipLaunchKernelGGL((k_attend_join<AtF16, 1>), grid, block, 0, s, a, d, slots, row0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace slh
