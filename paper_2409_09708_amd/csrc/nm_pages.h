// A cache of keys and values in pages: where a token of a sequence lies, and rows in 8 bits.
//
// Token j of sequence b is slot j % page_size of page table[b][j / page_size].  A table's entry outside 0 .. pages - 1 is a page that
// is not there.  Rows in 8 bits are e4m3 codes times a power of two of their own: x = code 2^(byte - 127).  Dividing by a power of two
// is exact, so a row's codes follow from the definition alone, and what a code stands for is exact in bfloat16.
#ifndef NM_PAGES_H
#define NM_PAGES_H

#include "nm_launch.h"
#include "nm_mma.h"
#include "nm_rows.h"

namespace nm {

typedef u32x4_t u32x4_byte_t __attribute__((aligned(1)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// j / page_size for 0 <= j < 2^31: with L = ceil(log2 d) and m = floor(2^(31 + L) / d) + 1 < 2^32 + 1 the product j m / 2^(31 + L) is
// above j / d by less than j / 2^(31 + L) < 2^-L <= 1 / d, so its whole part is the quotient.
struct PageDivide {
  uint32_t by;
  int shift;  // -1: pages of one token
};
inline PageDivide page_divide(int d) {
  int L = 0;
  while (((int64_t)1 << L) < d) ++L;
  if (L == 0) return {0, -1};
  return {(uint32_t)(((uint64_t)1 << (31 + L)) / (uint64_t)d + 1), L - 1};
}
__device__ __forceinline__ int page_of(PageDivide p, int j) { return p.shift < 0 ? j : (int)(__umulhi((uint32_t)j, p.by) >> p.shift); }

// Sixteen codes to eight pairs of bfloat16; `exponent` is the row's byte.
__device__ __forceinline__ void decode16(u32x4_t codes, uint32_t exponent, u32x4_t (&out)[2]) {
  const float scale = __uint_as_float(exponent << 23);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    out[w / 2][w % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], scale, false));
    out[w / 2][w % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], scale, true));
  }
}

// The exponent byte of a row whose largest finite magnitude has these bits: the smallest power of two that leaves it at 448 = 1.75 2^8
// or below, between 2^-100 and 2^119 (a value rounded up stays finite in bfloat16, and the smallest is no subnormal of it).
constexpr int kLeastExponent = 27, kMostExponent = 246;
__device__ __forceinline__ uint32_t row_exponent(uint32_t top) {
  const int e = (int)(top >> 7) - 8 + ((top & 127) > 96 ? 1 : 0);
  return (uint32_t)(e < kLeastExponent ? kLeastExponent : e > kMostExponent ? kMostExponent : e);
}

// A pair of bfloat16 to codes: rounded to nearest even, infinities to NaN, which the format has.  (Finite values above 448 times the
// largest power of two are cut to that: 0x7F60 is 1.75 2^127.)
__device__ __forceinline__ uint32_t encode2(uint32_t pair, float scale) {
  auto cut = [](uint32_t v) { const uint32_t m = v & 0x7FFFu; return m > 0x7F60u && m < 0x7F80u ? (v & 0x8000u) | 0x7F60u : v; };
  typedef short i16x2_t __attribute__((ext_vector_type(2)));
  const uint32_t safe = cut(pair & 0xFFFFu) | cut(pair >> 16) << 16;
  const i16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(i16x2_t{0, 0}, __builtin_bit_cast(bf16x2_t, safe), scale, false);
  return (uint32_t)(uint16_t)r[0];
}

// Eight codes to four pairs.
__device__ __forceinline__ u32x4_t decode8(uint32_t lo, uint32_t hi, uint32_t exponent) {
  const float scale = __uint_as_float(exponent << 23);
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}

// Sixteen codes of a row, from `at` on, of which n are there (<= 0: none; zeros past them).  Any alignment.
__device__ __forceinline__ u32x4_t load_codes(const uint8_t* row, int at, int n) {
  u32x4_t v = {0, 0, 0, 0};
  if (n >= 16) return *reinterpret_cast<const u32x4_byte_t*>(row + at);
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (e < n) v[e / 4] |= (uint32_t)row[at + e] << (8 * (e % 4));
  return v;
}

}  // namespace nm

#endif  // NM_PAGES_H
