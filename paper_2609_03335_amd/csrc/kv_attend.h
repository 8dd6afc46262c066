// What the attention kernels of both kinds of cache (kv_attend.hip, kv8_attend.hip) share: the 16-bit
// types' products, a row's blocks, and the joining of sums whose tokens were split over workgroups.
#pragma once

#include <cfloat>
#include <type_traits>

#include "kv.h"
#include "kv_sight.h"

namespace wfkv {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896341f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// What depends on the 16-bit type: the product, the codes as its operand, a pair of
// rounded values, and where the reference of the probabilities stands (in powers of two: p is
// 2^(score - reference)) and how far a score may pass it.
//
// bf16 has the range of fp32, so any p z keeps its bits and the reference is the largest score.
// f16 ends at 2^16 and has whole precision from 2^-14 on, so the reference goes by p z instead (kScaled):
// the largest is put high in that range, whatever the size of the values.  A p may then be large or small,
// in fp32.
struct MmaBf16 : Bf16 {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static constexpr float kSlack = 8.0f;
  static constexpr bool kScaled = false;
  static constexpr float kAimFixed = 0.0f;
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  template <int I>
  static __device__ __forceinline__ uint32_t codes(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, I));
  }
  // two 8-bit codes (I: the upper ones of the word) times a power of two
  template <int I>
  static __device__ __forceinline__ uint32_t codes8(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, I));
  }
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
  }
};
struct MmaF16 : F16 {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static constexpr float kSlack = 60.0f;
  static constexpr bool kScaled = true;
  // Running reference: the largest p z is from 2^12 to 2^15; one that is 2^-26 of it still has all its bits.
  // Fixed reference: the largest p z of some tokens that the query sees is 2^2 (a half step that f16 drops,
  // 2^-25, is 2^-27 of it), so that of all may be 14 powers of two above.  (600 normal queries over 9,000
  // keys: up to 10; at 2^6 a sixth of the workgroups had to run twice.)
  static constexpr float kAim = 12.0f, kAimFixed = 2.0f, kMostTerm = 0x1p15f, kMostLog = 15.0f;
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  template <int I>
  static __device__ __forceinline__ uint32_t codes(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, I));
  }
  template <int I>
  static __device__ __forceinline__ uint32_t codes8(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, by, I));
  }
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
  }
};

// The size of a value scale in powers of two: f16's largest at most, and so small that f16 has no place
// for the value at least (0, and what is not a number).
__device__ __forceinline__ float scale_log(float z) {
  return __builtin_amdgcn_logf(fminf(fmaxf(fabsf(z), 0x1p-40f), 0x1p16f));
}

// Over the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// A row's cells of one kv head.  id() is the block of a token (of the last cached
// token for one past it, so that it can be asked early and without a branch), cell() its address.
struct Pages {
  const int32_t* table;
  const uint8_t* base;
  uint32_t stride;
  unsigned most;
  int last, b_log2;
  __device__ Pages(const Geo& g, const AttendArgs& a, int row, int kvh, int len)
      : table(a.table + (int64_t)row * g.width), base(a.cache + (int64_t)kvh * g.cell),
        stride((uint32_t)g.hk * (uint32_t)g.cell), most((unsigned)g.n_blocks - 1u), last(max(len - 1, 0)),
        b_log2(g.b_log2) {}
  __device__ __forceinline__ unsigned id(int token) const { return (unsigned)table[(unsigned)min(token, last) >> b_log2]; }
  __device__ __forceinline__ const uint8_t* cell(unsigned id) const { return base + (uint64_t)min(id, most) * stride; }
};

struct Split {
  int tiles, splits;  // of the launch: column tiles of a row, shares of its tokens
  float* part;        // [splits][n_tokens][hq][D + 2] sums, reference, total
  int32_t* used;      // joined by a kernel: [n_tokens][hq] shares written; 1: the output is done
  int32_t* arrived;   // by the last workgroup: [n_rows][tiles][hk] shares done; 0 before and after a launch
                      // (all of a launch on one stream: another stream has other ones)
};

// Units of a row that a narrow workgroup takes without sharing: two a wave cost less than a
// join (one token over 500: 7.2 us against 8.1 for two shares).
constexpr int kAlone = 2 * kWaves;

// Partial sums go past the caches that the dies do not share, both ways: a release and an
// acquire that write those back and empty them for every workgroup cost more than the
// join (96 ragged rows 87 -> 150 us).
__device__ __forceinline__ void put(float* to, float a, float b) {
  const uint64_t w = (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(to), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get(const float* from) {
  const uint64_t w = __hip_atomic_load(reinterpret_cast<const uint64_t*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return (f32x2){__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32))};
}

// Whether this workgroup is the last of an item's `used` to get here.  The count goes back to 0 by the
// same operation that counts the last one.
__device__ __forceinline__ bool last_to_arrive(int32_t* arrived, int used, int* flag) {
  // Every wave's stores have reached the memory that all dies see before any of them counts, and the
  // sums are read after the last has counted: the clobber and the barriers keep the compiler to this order, and
  // the accesses are atomic, so that none of them is served from a cache of one die.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned most = (unsigned)used - 1u;
    *flag = atomicInc(reinterpret_cast<unsigned*>(arrived), most) == most;
  }
  __syncthreads();
  return *flag;
}

// Four channels of a head from its shares, in order.
template <int D, class M>
__device__ __forceinline__ void join_shares(const Geo& g, const AttendArgs& a, const Split& sp, int64_t head, int ch,
                                            int used) {
  const float* from = sp.part + head * (D + 2);
  const int64_t step = (int64_t)a.n_tokens * g.hq * (D + 2);
  float m = -INFINITY;
#pragma unroll 4
  for (int s = 0; s < used; ++s) m = fmaxf(m, get(from + s * step + D)[0]);
  const float r = m == -INFINITY ? 0.0f : m;
  float total = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = 0; s < used; ++s) {
    const float* at = from + s * step;
    const f32x2 t = get(at + D), v0 = get(at + ch), v1 = get(at + ch + 2);
    const float keep = __builtin_amdgcn_exp2f(t[0] - r);
    total += t[1] * keep;
    v[0] += v0[0] * keep, v[1] += v0[1] * keep, v[2] += v1[0] * keep, v[3] += v1[1] * keep;
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const u32x2 w = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
  *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + ch) = w;
}

// The shares of an item's columns, if this workgroup is the last that works on it.
template <int D, class M>
__device__ __forceinline__ void join_item(const Geo& g, const AttendArgs& a, const Split& sp, int row, int64_t tile,
                                          int kvh, int q0, int64_t col0, int64_t columns, int tile_columns, int used,
                                          int* flag) {
  if (!last_to_arrive(sp.arrived + ((int64_t)row * sp.tiles + tile) * g.hk + kvh, used, flag)) return;
  const int count = (int)min((int64_t)tile_columns, columns - col0);
  for (int x = threadIdx.x; x < count * (D / 4); x += blockDim.x) {
    const unsigned col = (unsigned)(col0 + x / (D / 4));
    const unsigned i = col / (unsigned)g.group, h = col - i * (unsigned)g.group;
    join_shares<D, M>(g, a, sp, (int64_t)(q0 + i) * g.hq + kvh * g.group + h, x % (D / 4) * 4, used);
  }
}

// The shares of each query's head, joined in a fixed order, four channels a thread.  Few
// shares (of prompts, P = 1): a group of D/4 threads a head.  Many (of single tokens): the
// workgroup's P groups take every P-th share of one head, then their sums in order.
template <int D, int P, class M>
__global__ __launch_bounds__(kThreads) void combine(Geo g, AttendArgs a, Split sp) {
  constexpr int L = D / 4, H = kThreads / (L * P);  // heads of a workgroup
  static_assert(P == 1 || H == 1, "all threads look for one head's largest reference");
  const int ch = threadIdx.x % L, part = threadIdx.x / L % P;
  const int64_t head = (int64_t)blockIdx.x * H + threadIdx.x / (L * P), heads = (int64_t)a.n_tokens * g.hq, t = head / g.hq;
  const bool mine = head < heads && t >= a.q_off[0] && t < a.q_off[a.n_rows];
  const int used = mine ? sp.used[head] : 0;
  if (used <= 1) return;  // (with P > 1, the whole workgroup)
  const float* from = sp.part + head * (D + 2);
  const int64_t step = heads * (D + 2);
  float m = -INFINITY;
  if constexpr (P > 1) {
    __shared__ float tops[kWaves];
    for (int s = threadIdx.x; s < used; s += kThreads) m = fmaxf(m, from[s * step + D]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, tops[w]);
  } else {
    for (int s = 0; s < used; ++s) m = fmaxf(m, from[s * step + D]);
  }
  const float r = m == -INFINITY ? 0.0f : m;
  float total = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = part; s < used; s += P) {
    const float* at = from + s * step;
    const float keep = __builtin_amdgcn_exp2f(at[D] - r);
    total += at[D + 1] * keep;
    const f32x2 v0 = *reinterpret_cast<const f32x2*>(at + 4 * ch), v1 = *reinterpret_cast<const f32x2*>(at + 4 * ch + 2);
    v[0] += v0[0] * keep, v[1] += v0[1] * keep, v[2] += v1[0] * keep, v[3] += v1[1] * keep;
  }
  if constexpr (P > 1) {
    __shared__ __attribute__((aligned(16))) f32x4 sums[P][L];
    __shared__ float totals[P];
    sums[part][ch] = v;
    if (ch == 0) totals[part] = total;
    __syncthreads();
    if (part) return;
    for (int k = 1; k < P; ++k) v += sums[k][ch], total += totals[k];
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const u32x2 w = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
  *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + 4 * ch) = w;
}

// Workgroups of a launch at most (a grid has fewer than 2^32 threads, 512 a workgroup here);
// batches of more rows take several.
constexpr int64_t kMostGrid = 1 << 22;

// Column tiles, shares and work area of a launch whose workgroups take `tile` columns;
// `want` workgroups fill the chip; rows of up to `alone` units are not shared.
template <int D>
Split split_of(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, int tile, int64_t want,
               int alone) {
  const int64_t most_kv = (int64_t)g.width * g.b;
  const int64_t max_kv = a.max_kv > 0 ? std::min((int64_t)a.max_kv, most_kv) : most_kv;
  Split sp;
  // (workgroups go on to the tiles past those launched: max_q may be unknown or too low)
  sp.tiles = (int)std::min<int64_t>((columns + tile - 1) / tile, std::max<int64_t>(1, kMostGrid / g.hk));
  const int64_t items = (int64_t)a.n_rows * g.hk * sp.tiles;
  // shares of at least a unit a wave, partial sums that fit the work area
  const int64_t heads = (int64_t)a.n_tokens * g.hq, units = (max_kv + 63) / 64;
  int64_t splits = std::min({want / items, (units + kWaves - 1) / kWaves,
                             (int64_t)(w.part_bytes / (heads * (D + 2) * 4))});
  if (units <= alone || std::max(heads, items) > (int64_t)(w.count_bytes / 4)) splits = 1;
  sp.splits = (int)std::max<int64_t>(1, splits);
  sp.part = w.part;
  sp.used = w.used;
  sp.arrived = w.arrived;
  return sp;
}

template <class K>
hipError_t launch(K kernel, const Geo& g, const AttendArgs& a, const Split& sp, int threads, hipStream_t s) {
  const int64_t row = (int64_t)g.hk * sp.tiles * sp.splits;  // workgroups
  const int rows = (int)std::max<int64_t>(1, std::min<int64_t>(a.n_rows, kMostGrid / row));
  for (int r = 0; r < a.n_rows; r += rows) {
    AttendArgs b = a;
    b.table += (int64_t)r * g.width, b.kv_len += r, b.q_off += r;
    b.n_rows = std::min(rows, a.n_rows - r);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(b.n_rows * row)), dim3(threads), 0, s, g, b, sp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace
}  // namespace wfkv
