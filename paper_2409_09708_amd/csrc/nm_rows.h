// Elements of rows that are bfloat16 or float, as 32-bit floats: one, or eight consecutive ones by 16-byte accesses
// (aligned addresses).
#ifndef NM_ROWS_H
#define NM_ROWS_H

#include "nm_device.h"

namespace nm {

template <bool F32, int VEC>
__device__ __forceinline__ void load_vec(const void* base, int64_t at, float (&v)[VEC]) {
  if constexpr (F32) {
    const float* p = static_cast<const float*>(base) + at;
    if constexpr (VEC == 8) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = p[e];
    }
  } else {
    const bf16_t* p = static_cast<const bf16_t*>(base) + at;
    if constexpr (VEC == 8) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = bf16_to_f32(p[e]);
    }
  }
}

// (rounded to nearest even where the output is bfloat16)
template <int VEC>
__device__ __forceinline__ void store_vec(void* base, int64_t at, const float (&v)[VEC], bool bf16) {
  if (bf16) {
    bf16_t* p = static_cast<bf16_t*>(base) + at;
    if constexpr (VEC == 8) {
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = f32_to_bf16_rne(v[2 * e]) | (f32_to_bf16_rne(v[2 * e + 1]) << 16);
      *reinterpret_cast<uint4*>(p) = uint4{u[0], u[1], u[2], u[3]};
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) p[e] = (bf16_t)f32_to_bf16_rne(v[e]);
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if constexpr (VEC == 8) {
      *reinterpret_cast<float4*>(p) = float4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<float4*>(p + 4) = float4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) p[e] = v[e];
    }
  }
}

}  // namespace nm

#endif  // NM_ROWS_H
