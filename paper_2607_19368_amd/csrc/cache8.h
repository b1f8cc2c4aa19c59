// A paged cache held in 8 bits: e4m3 codes [pages][H][page][d], and for each block of rows of a page and
// head the power of two that its codes stand beside, [pages][H][page / block], as a byte: 127 + its
// exponent.  A code stands for code * 2^(byte - 127): a block that grows, or rows that move to another block,
// keep their values exactly (but for codes that fall among the subnormal ones, below 2^-6), and the conversion
// instructions take the power along.
#pragma once
#include "slh_device.h"
#include "slh_internal.h"

#include "slh.h"

namespace slh {

constexpr int C8_LEAST = 1;              // bytes of 2^-126 and, by type, of the largest power in use: 448-folds
constexpr int C8_MOST_F16 = 127 + 8;     // cover the type's largest value, and 240-folds are not past it
constexpr int C8_MOST = 127 + 120;
constexpr float C8_TOP = 448.f;          // largest e4m3 code
constexpr float C8_TOP_LAST = 240.f;     // largest that is used with the largest power
constexpr int C8_BLOCK = 16;             // fewest and most rows of a block
constexpr int C8_BLOCK_MOST = 256;

__device__ __forceinline__ float c8_two(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// Byte of the smallest power of two whose 448-fold (1.75 2^8) reaches a magnitude, by its bits.
__device__ __forceinline__ int c8_byte(uint32_t magnitude) {
  return (int)(magnitude >> 23) - 8 + ((magnitude & 0x7fffffu) > 0x600000u);
}

// Four codes of values that are at most 448.
__device__ __forceinline__ uint32_t c8_codes(float a, float b, float c, float d) {
  uint32_t v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// Four codes, times a power of two.
__device__ __forceinline__ uint32_t c8_rescaled(uint32_t codes, float two) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return c8_codes(lo[0] * two, lo[1] * two, hi[0] * two, hi[1] * two);
}

__device__ __forceinline__ uint32_t c8_wave_max(uint32_t v) {
  const auto t32 = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max((uint32_t)t32[0], (uint32_t)t32[1]);
  const auto t16 = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)t16[0], (uint32_t)t16[1]);
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_ROR8, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_HALF_MIRROR, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_XOR2, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_XOR1, 0xF, 0xF, false));
  return v;
}

// Inclusive sums over the lanes of a wave: shifts by 1, 2, 4 and 8 within rows of 16, then the last of
// each row, then of each half, added to the ones behind.
__device__ __forceinline__ int c8_wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

inline bool c8_sizes_ok(int64_t n_pages, int page_size, int H, int block) {
  return page_size >= C8_BLOCK && page_size <= 65536 && !(page_size & (page_size - 1)) && block >= C8_BLOCK &&
         block <= C8_BLOCK_MOST && block <= page_size && !(block & (block - 1)) && n_pages >= 1 && n_pages <= INT32_MAX &&
         H >= 1 && H <= 65535 && n_pages * H <= INT32_MAX / page_size;
}

}  // namespace slh
