// Vectors of one token's head, eight channels a lane of L lanes: 16-bit values to and from fp32, sums and
// maxima over a vector, norm and rotation.  Shared by the stores of both kinds of cache.
#pragma once

#include "kv.h"

namespace wfkv {
namespace {

template <class T>
__device__ __forceinline__ void unpack(const uint4& w, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = T::to(u[i] & 0xffffu);
    x[2 * i + 1] = T::to(u[i] >> 16);
  }
}

template <class T>
__device__ __forceinline__ uint4 pack(const float* x) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = T::from(x[2 * i]) | T::from(x[2 * i + 1]) << 16;
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// The value of the lane with the index bit X flipped, among lanes whose lower bits already
// agree in what they hold (sums and maxima over a vector): mirrors of 8 and 16 lanes
// serve as well as the flip, and stay out of LDS.
template <int X>
__device__ __forceinline__ int fold(int x) {
  if constexpr (X == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
  if constexpr (X == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true);   // lanes 2 3 0 1
  if constexpr (X == 4) return __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true);  // mirror of 8
  if constexpr (X == 8) return __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true);  // mirror of 16
  return __shfl_xor(x, X, 64);
}
template <int L>
__device__ __forceinline__ float vector_sum(float t) {
  t += __int_as_float(fold<1>(__float_as_int(t)));
  t += __int_as_float(fold<2>(__float_as_int(t)));
  t += __int_as_float(fold<4>(__float_as_int(t)));
  if constexpr (L > 8) t += __int_as_float(fold<8>(__float_as_int(t)));
  if constexpr (L > 16) t += __int_as_float(fold<16>(__float_as_int(t)));
  return t;
}
template <int L>
__device__ __forceinline__ uint32_t vector_max(uint32_t t) {
  t = max(t, (uint32_t)fold<1>((int)t));
  t = max(t, (uint32_t)fold<2>((int)t));
  t = max(t, (uint32_t)fold<4>((int)t));
  if constexpr (L > 8) t = max(t, (uint32_t)fold<8>((int)t));
  if constexpr (L > 16) t = max(t, (uint32_t)fold<16>((int)t));
  return t;
}
// The value of the lane half a vector away.
template <int L>
__device__ __forceinline__ int other_half(int x) {
  if constexpr (L == 16) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true);  // turned by 8 of 16
  if constexpr (L == 8) {  // mirror of 8, then of 4
    x = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true);
    return __builtin_amdgcn_update_dpp(0, x, 0x1B, 0xf, 0xf, true);
  }
  return __shfl_xor(x, L / 2, 64);
}

// 1 / sqrt(x) rounded to nearest: the instruction is within an ulp, one Newton
// step with the products' rounding errors carried along gives the rest.
__device__ __forceinline__ float inv_sqrt(float x) {
  const float r = rsqrtf(x), t = x * r;
  const float e = fmaf(-t, r, 1.0f) - fmaf(x, r, -t) * r;
  const float y = fmaf(0.5f * r, e, r);
  return fabsf(y) <= 3.4e38f ? y : r;  // x = 0 or infinite
}

// x * rsqrt(mean(x^2) + eps) * w over a vector of L lanes.
template <int L, class T>
__device__ __forceinline__ void norm(float* x, const uint4& weight, float eps) {
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = x[i] * x[i];
  const float t = vector_sum<L>(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
  const float r = inv_sqrt(t * (1.0f / (8 * L)) + eps);
  float w[8];
  unpack<T>(weight, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}

// A lane's cosines and sines of a position (cs: its cosines, then sines), taken once for all
// heads of a token: of its four pairs, or of its eight channels.
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ Turn turn_of(const float* cs, int rot, int interleaved, int lane) {
  const int half = rot >> 1, c0 = interleaved ? lane * 4 : lane * 8 - (lane * 8 < half ? 0 : half);
  float4 c[2], s[2];
  c[0] = c[1] = make_float4(1, 1, 1, 1);
  s[0] = s[1] = make_float4(0, 0, 0, 0);
  if (lane * 8 < rot) {
    c[0] = *reinterpret_cast<const float4*>(cs + c0);
    s[0] = *reinterpret_cast<const float4*>(cs + half + c0);
    if (!interleaved) {
      c[1] = *reinterpret_cast<const float4*>(cs + c0 + 4);
      s[1] = *reinterpret_cast<const float4*>(cs + half + c0 + 4);
    }
  }
  return Turn{{c[0].x, c[0].y, c[0].z, c[0].w, c[1].x, c[1].y, c[1].z, c[1].w},
              {s[0].x, s[0].y, s[0].z, s[0].w, s[1].x, s[1].y, s[1].z, s[1].w}};
}

// Rotation of the first rot channels.
template <int L>
__device__ __forceinline__ void rotate(float* x, const Turn& turn, int rot, int interleaved, int lane) {
  const int half = rot >> 1;
  if (interleaved) {
    if (lane * 8 >= rot) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * turn.c[i] - b * turn.s[i];
      x[2 * i + 1] = b * turn.c[i] + a * turn.s[i];
    }
    return;
  }
  // the partner channel is rot/2 away: half / 8 lanes, in the same vector
  const bool low = lane * 8 < half, in = lane * 8 < rot;
  float y[8];
  if (rot == 8 * L) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __int_as_float(other_half<L>(__float_as_int(x[i])));
  } else {
    const int at = (int)(threadIdx.x & 63) + (in ? (low ? half >> 3 : -(half >> 3)) : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], at, 64);
  }
  if (!in) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float own = x[i] * turn.c[i], other = y[i] * turn.s[i];
    x[i] = low ? own - other : own + other;
  }
}

template <class F>
hipError_t by_type(int d, int dtype, F&& f) {
  // (channels, type) -> f(std::integral_constant<int, D>, T)
  switch (d * 2 + dtype) {
    case 128: return f.template operator()<64, Bf16>();
    case 129: return f.template operator()<64, F16>();
    case 256: return f.template operator()<128, Bf16>();
    case 257: return f.template operator()<128, F16>();
    case 512: return f.template operator()<256, Bf16>();
    default: return f.template operator()<256, F16>();
  }
}

}  // namespace
}  // namespace wfkv
