// Kernels of attend_tiles.h: packed prompts, and a paged cache's prefix or many new tokens.
#include "attend_tiles.h"

namespace slh {

template <class TY, int D, bool PAGED, int KW>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t smem[at_lds<D>()];
  attend_tiles<TY, D, PAGED, KW>(a, blockIdx.x, smem);
}

template <class TY, bool PAGED, int KW>
static void tiles_launch(const AttendArgs& a, int d, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend<TY, 64, PAGED, KW>), grid, block, 0, s, a); break;
    case 80: hipLaunchKernelGGL((k_attend<TY, 80, PAGED, KW>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((k_attend<TY, 96, PAGED, KW>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_attend<TY, 128, PAGED, KW>), grid, block, 0, s, a); break;
  }
}

template <class TY>
static void tiles_pick(const AttendArgs& a, bool paged, int rows, int d, int64_t blocks, hipStream_t s) {
  if (paged)
    tiles_launch<TY, true, 1>(a, d, blocks, s);
  else if (rows == AT_ROWS)
    tiles_launch<TY, false, 1>(a, d, blocks, s);
  else
    tiles_launch<TY, false, 2>(a, d, blocks, s);
}

hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool bf16, int rows, int d, int64_t blocks,
                               hipStream_t s) {
  bf16 ? tiles_pick<AtBf16>(a, paged, rows, d, blocks, s) : tiles_pick<AtF16>(a, paged, rows, d, blocks, s);
  return hipGetLastError();
}

}  // namespace slh
