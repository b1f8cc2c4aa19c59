// Keys and values of a cache in 8 bits on their way into products.
#pragma once
#include "attend.h"
#include "cache8.h"

#include <type_traits>

namespace slh {

// The cache's powers of two, and rows of a block.  The codes are in AttendArgs.
struct AtHeld {
  const uint8_t* k_two;
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

}  // namespace slh
