// Attention of a batch's new tokens against a paged cache held in 8 bits (cache8.h), behind a shared
// prefix: the arguments, and the conversions that the kernels share.
#pragma once
#include "attend.h"
#include "cache8.h"

#include <type_traits>

namespace slh {

struct Attend8Args {
  AttendArgs a;            // its k and v: the codes
  const uint8_t* k_two;    // [n_pages][Hkv][page / block]
  const uint8_t* v_two;
  int lg_block;
};

// Two elements of TY of two codes (of the lower or upper half of x) times 2^k, k the exponent of `two`.
template <class TY, bool HI>
__device__ __forceinline__ uint32_t c8_pair(uint32_t x, float two) {
  if constexpr (std::is_same<TY, AtBf16>::value)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, two, HI));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, two, HI));
}

// Bytes that are NaN codes (sign aside 0x7f): their sign bits set.
__device__ __forceinline__ uint32_t c8_nan(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

hipError_t launch_rows8(const Attend8Args& a, bool bf16, int rows, int d, int64_t blocks, hipStream_t s);

}  // namespace slh
