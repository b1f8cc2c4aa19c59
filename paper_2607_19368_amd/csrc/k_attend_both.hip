// A decode step behind a long prefix as one launch: the prefix for all sequences in tiles of 128 rows
// (attend_tiles.h: bound by the matrix units), each sequence's own keys by rows (attend_rows.h: bound by
// memory).  Blocks of both kinds lie beside each other on a compute unit, so that the one's reads
// run under the other's products.
#include "attend_rows.h"
#include "attend_tiles.h"

namespace slh {

template <class TY, int D, int NR>
__global__ __launch_bounds__(64 * AT_WAVES, 2) void k_attend_both(AttendArgs a, int pre_blocks, int blocks) {
  constexpr int LT = at_lds<D>(), LR = rw_lds<D, NR>();
  __shared__ __attribute__((aligned(16))) uint16_t smem[LT > LR ? LT : LR];
  // Kinds alternate in proportion, by eights: block x of a kind stays on XCD x % 8, where the others that
  // read the same keys are.
  const int e = blockIdx.x >> 3, in = blockIdx.x & 7;
  const int pe = (pre_blocks + 7) >> 3, all = (int)gridDim.x >> 3;
  const int before = min(e, pe), upto = e < pe ? before + 1 : before;
  if (upto > before) {
    const int x = 8 * before + in;
    if (x < pre_blocks) attend_tiles<TY, D, true>(a, x, smem);
  } else {
    const int x = 8 * (e - before) + in;
    AttendArgs own = a;
    own.pre_tiles = 0;
    if (x < blocks - pre_blocks) attend_rows<TY, D, NR, true>(own, x, smem);
  }
}

template <class TY, int NR>
static void both_launch(const AttendArgs& a, int d, int64_t pre, int64_t blocks, hipStream_t s) {
  // an eight of a kind may be partly empty
  const dim3 grid((unsigned)(8 * ((pre + 7) / 8 + (blocks - pre + 7) / 8))), block(64 * AT_WAVES);
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
