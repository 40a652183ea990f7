// Elements of rows that are bfloat16 or float, eight at a time, as 32-bit floats.  Accesses are 16 bytes wide at any element
// address: the hardware takes them unaligned.
#ifndef NM_ROWS_H
#define NM_ROWS_H

#include "nm_mma.h"

namespace nm {

typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(2)));

// Eight elements as they lie in memory; those from n (<= 8) on are not read and are zero.
template <bool F32>
struct Raw8 {
  u32x4_t v[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* base, int64_t at, int n) {
    if (n >= 8) {
      if constexpr (F32) {
        const u32x4_any_t* p = reinterpret_cast<const u32x4_any_t*>(static_cast<const float*>(base) + at);
        v[0] = p[0];
        v[1] = p[1];
      } else {
        v[0] = *reinterpret_cast<const u32x4_any_t*>(static_cast<const bf16_t*>(base) + at);
      }
      return;
    }
    v[0] = u32x4_t{0, 0, 0, 0};
    if constexpr (F32) v[1] = v[0];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) {
        if constexpr (F32) v[e / 4][e % 4] = static_cast<const uint32_t*>(base)[at + e];
        else v[0][e / 2] |= (uint32_t)static_cast<const bf16_t*>(base)[at + e] << (16 * (e & 1));
      }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (F32) return __uint_as_float(v[e / 4][e % 4]);
    else return __uint_as_float(e & 1 ? v[0][e / 2] & 0xFFFF0000u : v[0][e / 2] << 16);
  }
};

// The first n (<= 8) of eight elements, rounded to nearest even where the output is bfloat16.
__device__ __forceinline__ void store8(void* base, int64_t at, int n, const float (&v)[8], bool bf16) {
  if (bf16) {
    bf16_t* p = static_cast<bf16_t*>(base) + at;
    const u32x4_t u = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    if (n >= 8) {
      *reinterpret_cast<u32x4_any_t*>(p) = u;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = (bf16_t)(u[e / 2] >> (16 * (e & 1)));
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (n >= 8) {
      reinterpret_cast<u32x4_any_t*>(p)[0] = u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      reinterpret_cast<u32x4_any_t*>(p)[1] = u32x4_t{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = v[e];
    }
  }
}

// One element, and its way back.
template <bool F32>
__device__ __forceinline__ float load1(const void* base, int64_t at) {
  if constexpr (F32) return static_cast<const float*>(base)[at];
  else return bf16_to_f32(static_cast<const bf16_t*>(base)[at]);
}
__device__ __forceinline__ void store1(void* base, int64_t at, float v, bool bf16) {
  if (bf16) static_cast<bf16_t*>(base)[at] = (bf16_t)f32_to_bf16_rne(v);
  else static_cast<float*>(base)[at] = v;
}

}  // namespace nm

#endif  // NM_ROWS_H
