// Norm and rotation of queries and keys, and the 4-bit store of keys and
// values (and its inverse).  A vector is one token's head: D channels, eight
// to a lane, so a wave holds 64 / (D / 8) vectors; everything between the one
// load and the one store of a vector stays in registers.
//
// The sum of squares adds neighbours first (channels 0+1, 2+3, ...; then those
// sums), every product and sum is rounded by itself, and codes come from exact
// comparisons with the scale's multiples (a scale has 8 bits, a threshold 3), so the
// stored codes are reproducible to the last bit by elementary operations.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;

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
__device__ __forceinline__ void norm(float* x, const void* weight, int lane, float eps) {
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = x[i] * x[i];
  float t = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
#pragma unroll
  for (int off = 1; off < L; off <<= 1) t += __shfl_xor(t, off, 64);
  const float r = inv_sqrt(t * (1.0f / (8 * L)) + eps);
  float w[8];
  unpack<T>(reinterpret_cast<const uint4*>(weight)[lane], w);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}

// Rotation of the first rot channels; cs: the position's cosines, then sines.
template <int L>
__device__ __forceinline__ void rotate(float* x, const float* cs, int rot, int interleaved, int lane) {
  const int half = rot >> 1;
  if (interleaved) {
    if (lane * 8 >= rot) return;
    const float4 c = *reinterpret_cast<const float4*>(cs + lane * 4);
    const float4 s = *reinterpret_cast<const float4*>(cs + half + lane * 4);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * cc[i] - b * ss[i];
      x[2 * i + 1] = b * cc[i] + a * ss[i];
    }
    return;
  }
  // the partner channel is rot/2 away: half / 8 lanes, in the same vector
  const bool low = lane * 8 < half, in = lane * 8 < rot;
  const int at = (int)(threadIdx.x & 63) + (in ? (low ? half >> 3 : -(half >> 3)) : 0);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], at, 64);
  if (!in) return;
  const int c0 = lane * 8 - (low ? 0 : half);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float4 c = *reinterpret_cast<const float4*>(cs + c0 + 4 * j);
    const float4 s = *reinterpret_cast<const float4*>(cs + half + c0 + 4 * j);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float own = x[4 * j + i] * cc[i], other = y[4 * j + i] * ss[i];
      x[4 * j + i] = low ? own - other : own + other;
    }
  }
}

// The eight codes of a lane (channel i in nibble i) and the vector's scale.
template <int L>
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t* scale) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int off = 1; off < L; off <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, 64));
  // infinities and NaN have the largest bit patterns
  const uint32_t s = most >= 0x7f800000u ? 0x7fc0u : Bf16::from(__uint_as_float(most) * (1.0f / 6.0f));
  const float f = Bf16::to(s);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    uint32_t c = (uint32_t)(a > 0.25f * f) + (uint32_t)(a >= 0.75f * f) + (uint32_t)(a > 1.25f * f) +
                 (uint32_t)(a >= 1.75f * f) + (uint32_t)(a > 2.5f * f) + (uint32_t)(a >= 3.5f * f) +
                 (uint32_t)(a > 5.0f * f);
    c |= (uint32_t)(x[i] < 0.0f) << 3;
    codes |= c << (4 * i);
  }
  *scale = s;
  return codes;
}

// One vector a group of L lanes: heads 0..hq-1 are queries, then hk keys, then
// hk values.
template <int D, class T>
__global__ __launch_bounds__(kThreads) void store(Geo g, StoreArgs a) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x % L;
  const int64_t v = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
  const int heads = g.hq + 2 * g.hk;
  const int64_t t = v / heads;
  if (t >= a.n_tokens) return;  // whole vectors leave
  const int h = (int)(v - t * heads);
  const bool is_q = h < g.hq, is_v = h >= g.hq + g.hk;
  const int kvh = h - g.hq - (is_v ? g.hk : 0);
  const uint16_t* src = is_q ? (const uint16_t*)a.q + t * a.q_stride + (int64_t)h * D
                       : is_v ? (const uint16_t*)a.v + t * a.v_stride + (int64_t)kvh * D
                              : (const uint16_t*)a.k + t * a.k_stride + (int64_t)kvh * D;
  const int64_t slot = a.slot[t];
  const int64_t block = slot >> g.b_log2;
  const bool stored = slot >= 0 && block < g.n_blocks;
  if (!is_q && !stored) return;
  float x[8];
  unpack<T>(reinterpret_cast<const uint4*>(src)[lane], x);
  if (!is_v) {
    const void* w = is_q ? a.how.q_weight : a.how.k_weight;
    if (w) norm<L, T>(x, w, lane, a.how.eps);
    if (a.how.rot_dim) {
      const int p = min(max(a.pos[t], 0), a.how.n_pos - 1);
      rotate<L>(x, a.how.cos_sin + (int64_t)p * a.how.rot_dim, a.how.rot_dim, a.how.interleaved, lane);
    }
  }
  if (is_q) {
    reinterpret_cast<uint4*>((uint16_t*)a.q_out + (t * g.hq + h) * D)[lane] = pack<T>(x);
    return;
  }
  uint32_t s;
  const uint32_t codes = quantise<L>(x, &s);
  const int off = (int)(slot & (g.b - 1));
  uint8_t* cell = a.cache + (block * g.hk + kvh) * (int64_t)g.cell;
  uint16_t* scales = reinterpret_cast<uint16_t*>(cell + g.b * D);
  if (!is_v) {
    reinterpret_cast<uint32_t*>(cell + off * (D / 2))[lane] = codes;
    if (lane == 0) scales[off] = (uint16_t)s;
    return;
  }
  // byte (r, off) holds channels r and r + D/2: the lane L/2 away has the other
  const uint32_t other = (uint32_t)__shfl_xor((int)codes, L / 2, 64);
  const bool low = lane < L / 2;
  const uint32_t lo = low ? codes : other >> 16, hi = low ? other : codes >> 16;
  uint8_t* row = cell + g.b * (D / 2) + (int64_t)((low ? lane : lane - L / 2) * 8 + (low ? 0 : 4)) * g.b + off;
#pragma unroll
  for (int i = 0; i < 4; ++i) row[i * g.b] = (uint8_t)(((lo >> (4 * i)) & 15u) | ((hi >> (4 * i)) & 15u) << 4);
  if (lane == 0) scales[g.b + off] = (uint16_t)s;
}

__device__ __forceinline__ float code_value(uint32_t c) {
  // 0, 0.5, 1, 1.5, 2, 3, 4, 6: halves below 1, else 1.m * 2^(e-1)
  const uint32_t e = (c >> 1) & 3u, m = c & 1u;
  const uint32_t bits = e ? (126u + e) << 23 | m << 22 : m ? 0x3f000000u : 0u;
  return __uint_as_float(bits | (c & 8u) << 28);
}

// One vector a group of L lanes: keys and values of each token and kv head.
template <int D, class T>
__global__ __launch_bounds__(kThreads) void load(Geo g, LoadArgs a) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x % L;
  const int64_t v = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
  const int64_t t = v / (2 * g.hk);
  if (t >= a.n_tokens) return;
  const int h = (int)(v - t * (2 * g.hk));
  const bool is_v = h >= g.hk;
  const int kvh = is_v ? h - g.hk : h;
  const int64_t slot = a.slot[t], block = slot >> g.b_log2;
  uint4* out = reinterpret_cast<uint4*>((uint16_t*)(is_v ? a.v : a.k) + (t * g.hk + kvh) * D) + lane;
  if (slot < 0 || block >= g.n_blocks) {
    *out = make_uint4(0, 0, 0, 0);
    return;
  }
  const int off = (int)(slot & (g.b - 1));
  const uint8_t* cell = a.cache + (block * g.hk + kvh) * (int64_t)g.cell;
  const float s = Bf16::to(reinterpret_cast<const uint16_t*>(cell + g.b * D)[(is_v ? g.b : 0) + off]);
  uint32_t codes;
  if (!is_v) {
    codes = reinterpret_cast<const uint32_t*>(cell + off * (D / 2))[lane];
  } else {
    const bool low = lane < L / 2;
    const uint8_t* row = cell + g.b * (D / 2) + (int64_t)(low ? lane : lane - L / 2) * 8 * g.b + off;
    codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes |= (uint32_t)((row[i * g.b] >> (low ? 0 : 4)) & 15) << (4 * i);
  }
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = code_value((codes >> (4 * i)) & 15u) * s;
    // the scale's rounding can take the largest code past the type's range
    if (fabsf(x[i]) > T::kMost) x[i] = copysignf(T::kMost, x[i]);
  }
  *out = pack<T>(x);
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

struct Store {
  const Geo& g;
  const StoreArgs& a;
  hipStream_t s;
  template <int D, class T>
  hipError_t operator()() {
    const int64_t threads = (int64_t)a.n_tokens * (g.hq + 2 * g.hk) * (D / 8);
    hipLaunchKernelGGL((store<D, T>), dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g, a);
    return hipGetLastError();
  }
};

struct Load {
  const Geo& g;
  const LoadArgs& a;
  hipStream_t s;
  template <int D, class T>
  hipError_t operator()() {
    const int64_t threads = (int64_t)a.n_tokens * 2 * g.hk * (D / 8);
    hipLaunchKernelGGL((load<D, T>), dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g, a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_store(const Geo& g, int dtype, const StoreArgs& a, hipStream_t s) {
  return by_type(g.d, dtype, Store{g, a, s});
}

hipError_t launch_load(const Geo& g, int dtype, const LoadArgs& a, hipStream_t s) {
  return by_type(g.d, dtype, Load{g, a, s});
}

}  // namespace wfkv
