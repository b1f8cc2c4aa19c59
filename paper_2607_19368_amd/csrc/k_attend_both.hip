// A decode step behind a long prefix as one launch: the prefix for all sequences in tiles of 128 rows
// (attend_tiles.h: bound by the matrix units), each sequence's own keys by rows (attend_rows.h: bound by
// memory).  The prefix's blocks come first: the own keys' blocks fill the compute units as those end, so
// that the last prefix blocks do not run alone and one launch is saved.
//
// 128 sequences, 28 / 4 heads of 128, a prefix of 32768 rows and up to 641 own, bf16, us with the join: two
// launches 107, prefix first 101, own keys first 101, eights of both kinds alternating 144 (a unit that holds one
// of each has too few waves of either).  With the loads spread as in attend_tiles.h: 93, of which
// this kernel 84.3, the join 8.5.
#include "attend_rows.h"
#include "attend_tiles.h"

namespace slh {

template <class TY, int D, int NR>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend_both(AttendArgs a, int pre_blocks, int blocks) {
  constexpr int LT = at_lds<D>(), LR = rw_lds<D, NR>();
  __shared__ __attribute__((aligned(16))) uint16_t smem[LT > LR ? LT : LR];
  // The prefix's blocks are filled up to whole eights: block x of a kind stays on XCD x % 8, where the others
  // that read the same keys are.
  const int before = (pre_blocks + 7) & ~7;
  if ((int)blockIdx.x < before) {
    if ((int)blockIdx.x < pre_blocks) attend_tiles<TY, D, true, 1>(a, blockIdx.x, smem);
  } else {
    const int x = (int)blockIdx.x - before;
    AttendArgs own = a;
    own.pre_tiles = 0;
    if (x < blocks - pre_blocks) attend_rows<TY, D, NR, true>(own, x, smem);
  }
}

template <class TY, int NR>
static void both_launch(const AttendArgs& a, int d, int64_t pre, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)((pre + 7) / 8 * 8 + blocks - pre)), block(64 * AT_WAVES);
  switch (d) {
    case 64: hipLaunchKernelGGL((k_attend_both<TY, 64, NR>), grid, block, 0, s, a, (int)pre, (int)blocks); break;
    case 80: hipLaunchKernelGGL((k_attend_both<TY, 80, NR>), grid, block, 0, s, a, (int)pre, (int)blocks); break;
    case 96: hipLaunchKernelGGL((k_attend_both<TY, 96, NR>), grid, block, 0, s, a, (int)pre, (int)blocks); break;
    default: hipLaunchKernelGGL((k_attend_both<TY, 128, NR>), grid, block, 0, s, a, (int)pre, (int)blocks); break;
  }
}

hipError_t launch_attend_both(const AttendArgs& a, bool bf16, int rows, int d, int64_t pre, int64_t blocks,
                              hipStream_t s) {
  if (bf16)
    rows == 16 ? both_launch<AtBf16, 1>(a, d, pre, blocks, s) : both_launch<AtBf16, 2>(a, d, pre, blocks, s);
  else
    rows == 16 ? both_launch<AtF16, 1>(a, d, pre, blocks, s) : both_launch<AtF16, 2>(a, d, pre, blocks, s);
  return hipGetLastError();
}

}  // namespace slh
