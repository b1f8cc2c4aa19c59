// Attention of a batch's new tokens against a paged cache held in 8 bits (cache8.h), behind a shared
// prefix: what the kernels share.
#pragma once
#include "attend_held.h"

namespace slh {

struct Attend8Args {
  AttendArgs a;            // its k and v: the codes
  AtHeld held;             // powers of two [n_pages][Hkv][page / block]
};

// For a block's byte (its power 2^k), what carries the magnitudes that are infinite in TY, and NaN, into a byte's sign: code
// 2^(T - k) and those above, T = 16 in fp16 (61440, the value of 240 2^8, is held, the next code's 65536 is not) and 128
// in bf16; at most 448 in use: k up to 7 and up to 119 leave NaN (0x7f) alone.
template <class TY>
__device__ __forceinline__ uint32_t c8_past(int byte) {
  const int e = (std::is_same<TY, AtBf16>::value ? 128 : 16) - (byte - 127);   // codes from 2^e
  const int least = e > 8 ? 0x7f : e >= -6 ? (e + 7) * 8 : e >= -9 ? 1 << (e + 9) : 1;
  return (uint32_t)(128 - least) * 0x01010101u;
}
// Bytes that are, by c8_past's word: their sign bits set.  0x01010101 is the word for NaN alone.
__device__ __forceinline__ uint32_t c8_odd(uint32_t x, uint32_t past) { return ((x & 0x7f7f7f7fu) + past) & 0x80808080u; }

// As the launches of attend.h: tiles of 128 rows, blocks of 16 or 32, and both in one launch.
hipError_t launch_tiles8(const Attend8Args& a, bool bf16, int d, int64_t blocks, hipStream_t s);
hipError_t launch_both8(const Attend8Args& a, bool bf16, int rows, int d, int64_t pre_blocks, int64_t blocks, hipStream_t s);
hipError_t launch_rows8(const Attend8Args& a, bool bf16, int rows, int d, int64_t blocks, hipStream_t s);

}  // namespace slh
