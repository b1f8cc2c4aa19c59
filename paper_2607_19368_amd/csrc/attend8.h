// Attention of a batch's new tokens against a paged cache held in 8 bits (cache8.h), behind a shared
// prefix: what the kernels share.
#pragma once
#include "attend_held.h"

namespace slh {

struct Attend8Args {
  AttendArgs a;            // its k and v: the codes
  AtHeld held;             // powers of two [n_pages][Hkv][page / block]
};

// Bytes that are NaN codes (sign aside 0x7f): their sign bits set.
__device__ __forceinline__ uint32_t c8_nan(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// As the launches of attend.h: tiles of 128 rows, blocks of 16 or 32, and both in one launch.
hipError_t launch_tiles8(const Attend8Args& a, bool bf16, int d, int64_t blocks, hipStream_t s);
hipError_t launch_both8(const Attend8Args& a, bool bf16, int rows, int d, int64_t pre_blocks, int64_t blocks, hipStream_t s);
hipError_t launch_rows8(const Attend8Args& a, bool bf16, int rows, int d, int64_t blocks, hipStream_t s);

}  // namespace slh
