// Kernels of attend_tiles.h for keys and values in 8 bits: tiles of 128 rows, and, behind a long prefix, the prefix in
// tiles and each sequence's own keys by rows (rows8.h) in one launch, the prefix's blocks first (as in
// k_attend_both.hip).
#include "attend_tiles.h"
#include "rows8.h"

namespace slh {

template <class TY, int D>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_tiles8(Attend8Args a) {
  __shared__ __attribute__((aligned(16))) uint16_t smem[at_lds<D>()];
  attend_tiles<TY, D, true, 1, true>(a.a, blockIdx.x, smem, a.held);
}

template <class TY, int D, int NR>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_both8(Attend8Args a, int pre_blocks, int blocks) {
  constexpr int LT = at_lds<D>(), LR = 2 * rows8_lds<D, NR>();
  __shared__ __attribute__((aligned(16))) uint16_t smem[LT > LR ? LT : LR];
  // the prefix's blocks are filled up to whole eights: block x of a kind stays on XCD x % 8
  const int before = (pre_blocks + 7) & ~7;
  if ((int)blockIdx.x < before) {
    if ((int)blockIdx.x < pre_blocks) attend_tiles<TY, D, true, 1, true>(a.a, blockIdx.x, smem, a.held);
  } else {
    const int x = (int)blockIdx.x - before;
    Attend8Args own = a;
    own.a.pre_tiles = 0;
    if (x < blocks - pre_blocks) rows8<TY, D, NR>(own, x, (float*)smem);
  }
}

template <class F>
static void sizes8(int d, F&& go) {
  switch (d) {
    case 64: go(std::integral_constant<int, 64>{}); break;
    case 80: go(std::integral_constant<int, 80>{}); break;
    case 96: go(std::integral_constant<int, 96>{}); break;
    default: go(std::integral_constant<int, 128>{}); break;
  }
}

hipError_t launch_tiles8(const Attend8Args& a, bool bf16, int d, int64_t blocks, hipStream_t s) {
  sizes8(d, [&](auto D) {
    if (bf16)
      hipLaunchKernelGGL((k_tiles8<AtBf16, decltype(D)::value>), dim3((unsigned)blocks), dim3(64 * AT_WAVES), 0, s, a);
    else
      hipLaunchKernelGGL((k_tiles8<AtF16, decltype(D)::value>), dim3((unsigned)blocks), dim3(64 * AT_WAVES), 0, s, a);
  });
  return hipGetLastError();
}

template <class TY, int NR>
static void both8_go(const Attend8Args& a, int d, int64_t pre, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)((pre + 7) / 8 * 8 + blocks - pre));
  sizes8(d, [&](auto D) {
    hipLaunchKernelGGL((k_both8<TY, decltype(D)::value, NR>), grid, dim3(64 * AT_WAVES), 0, s, a, (int)pre, (int)blocks);
  });
}

hipError_t launch_both8(const Attend8Args& a, bool bf16, int rows, int d, int64_t pre, int64_t blocks, hipStream_t s) {
  if (bf16)
    rows == 16 ? both8_go<AtBf16, 1>(a, d, pre, blocks, s) : both8_go<AtBf16, 2>(a, d, pre, blocks, s);
  else
    rows == 16 ? both8_go<AtF16, 1>(a, d, pre, blocks, s) : both8_go<AtF16, 2>(a, d, pre, blocks, s);
  return hipGetLastError();
}

}  // namespace slh
