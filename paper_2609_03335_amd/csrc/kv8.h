// The cell of a cache of 8-bit codes: key codes [B][D], value codes [B/4][D][4], two fp32 scales.
#pragma once

#include <type_traits>

#include "kv.h"

namespace wfkv {
namespace {

constexpr int kLeastPower = -100, kMostPower = 119;

typedef float f32x2_8 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float two_to(int e) { return __int_as_float((e + 127) << 23); }

// The least e for which a magnitude (its bits; finite) does not pass 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int least_power(uint32_t most) {
  const int e = (int)(most >> 23) - (127 + 8) + (int)((most & 0x7fffffu) > 0x600000u);
  return min(max(e, kLeastPower), kMostPower);
}

// The power that a scale of a cell stands for (whatever the cell holds, one that a scale can have).
__device__ __forceinline__ int power_of(float scale) {
  return min(max((int)(__float_as_uint(scale) >> 23) - 127, kLeastPower), kMostPower);
}

// Codes of four values (already divided by the scale), byte i that of x[i].  The instruction rounds to nearest even and
// would make NaN of what is above 448.
__device__ __forceinline__ uint32_t codes_of(const float* x) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -448.0f, 448.0f);
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], low, true);
}

// The same of four values that do not pass 448 times a power of two (above that the instruction gives no number).
typedef short i16x2_8 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t codes_under(const float* x, float scale) {
  const i16x2_8 low = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32((i16x2_8){0, 0}, x[0], x[1], scale, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(low, x[2], x[3], scale, true));
}
// ... of 16-bit values as they are, two in each word.
template <class T>
__device__ __forceinline__ uint32_t codes_under(uint32_t a, uint32_t b, float scale) {
  if constexpr (std::is_same_v<T, Bf16>) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    const i16x2_8 low = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16((i16x2_8){0, 0}, __builtin_bit_cast(v2, a), scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(low, __builtin_bit_cast(v2, b), scale, true));
  } else {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    const i16x2_8 low = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16((i16x2_8){0, 0}, __builtin_bit_cast(v2, a), scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(low, __builtin_bit_cast(v2, b), scale, true));
  }
}

// Values of the four codes of a word.
__device__ __forceinline__ void values_of(uint32_t w, float* x) {
  const f32x2_8 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
}

}  // namespace
}  // namespace wfkv
