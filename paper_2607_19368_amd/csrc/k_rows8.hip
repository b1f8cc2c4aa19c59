// Kernels of rows8.h.
#include "rows8.h"

namespace slh {

template <class TY, int D, int NR>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_rows8(Attend8Args a) {
  __shared__ __attribute__((aligned(16))) float smem[rows8_lds<D, NR>()];
  rows8<TY, D, NR>(a, blockIdx.x, smem);
}

template <class TY, int NR>
static void rows8_launch(const Attend8Args& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_rows8<TY, 64, NR>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_rows8<TY, 80, NR>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_rows8<TY, 96, NR>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_rows8<TY, 128, NR>), grid, block, 0, s, a); break;
  }
}

hipError_t launch_rows8(const Attend8Args& a, bool bf16, int rows, int d, int64_t blocks, hipStream_t s) {
  if (bf16)
    rows == 16 ? rows8_launch<AtBf16, 1>(a, d, blocks, s) : rows8_launch<AtBf16, 2>(a, d, blocks, s);
  else
    rows == 16 ? rows8_launch<AtF16, 1>(a, d, blocks, s) : rows8_launch<AtF16, 2>(a, d, blocks, s);
  return hipGetLastError();
}

}  // namespace slh
