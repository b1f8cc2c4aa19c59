// Kernels of attend_tiles.h: packed prompts, and a paged cache's prefix or many new tokens.
#include "attend_tiles.h"

namespace slh {

template <class TY, int D, bool PAGED>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t smem[at_lds<D>()];
  attend_tiles<TY, D, PAGED>(a, blockIdx.x, smem);
}

template <class TY, bool PAGED>
static void tiles_launch(const AttendArgs& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend<TY, 64, PAGED>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_attend<TY, 80, PAGED>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_attend<TY, 96, PAGED>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_attend<TY, 128, PAGED>), grid, block, 0, s, a); break;
  }
}

hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool bf16, int d, int64_t blocks, hipStream_t s) {
  if (paged)
    bf16 ? tiles_launch<AtBf16, true>(a, d, blocks, s) : tiles_launch<AtF16, true>(a, d, blocks, s);
  else
    bf16 ? tiles_launch<AtBf16, false>(a, d, blocks, s) : tiles_launch<AtF16, false>(a, d, blocks, s);
  return hipGetLastError();
}

}  // namespace slh
