// Norm and rotation of queries and keys, and the 4-bit store of keys and
// values (and its inverse).  A vector is one token's head: D channels, eight
// to a lane, so a wave holds 64 / (D / 8) vectors; everything between the one
// load and the one store of a vector stays in registers.
//
// The sum of squares adds neighbours first (channels 0+1, 2+3, ...; then those
// sums), every product and sum is rounded by itself, and codes come from exact
// comparisons with the scale's multiples (a scale has 8 bits, a threshold 3), so the
// stored codes are reproducible to the last bit by elementary operations.
//
// Bound by memory for prompts (q in and out is four fifths of the bytes): 16,384 tokens of
// 40 + 8 heads of 128 channels take 88 to 98 us, 4.3 to 4.8 TB/s of their 420 MB (a streaming
// kernel reaches 6.2); by the launch for single tokens (3.8 us).
#include "kv_vector.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;            // heads a lane group takes of a token, of many
constexpr int64_t kManyVectors = 32768;  // vectors of a call from which they are many

// The eight codes of a lane (channel i in nibble i) and the vector's scale.
template <int L>
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t* scale) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  most = vector_max<L>(most);
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

// A lane's four bytes of a value vector: channels r in the low, r + D/2 in the high nibbles of
// rows first_row(lane) .. + 3 of the cell's transposed codes.
template <int L>
__device__ __forceinline__ int first_row(int lane) {
  return lane < L / 2 ? lane * 8 : (lane - L / 2) * 8 + 4;
}
template <int L>
__device__ __forceinline__ uint32_t value_bytes(uint32_t codes, int lane) {
  const uint32_t other = (uint32_t)other_half<L>((int)codes);
  const bool low = lane < L / 2;
  const uint32_t lo = low ? codes : other >> 16, hi = low ? other : codes >> 16;
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) w |= (((lo >> (4 * i)) & 15u) | ((hi >> (4 * i)) & 15u) << 4) << (8 * i);
  return w;
}

// Values of kTile tokens of a kv head: codes go through LDS, so that four or sixteen tokens
// with consecutive slots (a prompt's) leave as one store.  LDS column a + i holds token i, a the
// first token's place among 16, which puts a run's stores on their alignment.
constexpr int kTile = 64, kPitch = kTile + 16;
template <int D, class T>
__device__ __forceinline__ void store_values(const Geo& g, const StoreArgs& a, unsigned tile, uint8_t* bytes,
                                             int64_t* slots, int64_t* runs) {
  constexpr int L = D / 8, V = kThreads / L;
  const int kvh = (int)(tile % (unsigned)g.hk), t0 = (int)(tile / (unsigned)g.hk) * kTile;
  const int lane = threadIdx.x % L;
  const int64_t first = a.slot[t0];
  const int shift = first >= 0 ? (int)(first & 15) : 0;
  // slots by column, -1: nothing stored
  for (int x = threadIdx.x; x < kPitch; x += kThreads) {
    const int i = x - shift;
    const int64_t s = i >= 0 && i < kTile && t0 + i < a.n_tokens ? a.slot[t0 + i] : -1;
    slots[x] = s >= 0 && s >> g.b_log2 < g.n_blocks ? s : -1;
  }
  uint4 raw[kTile / V];
#pragma unroll
  for (int j = 0; j < kTile / V; ++j) {
    const int t = min(t0 + j * V + (int)threadIdx.x / L, a.n_tokens - 1);
    raw[j] = reinterpret_cast<const uint4*>((const uint16_t*)a.v + t * a.v_stride + (int64_t)kvh * D)[lane];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kTile / V; ++j) {
    const int col = shift + j * V + (int)threadIdx.x / L;
    float x[8];
    unpack<T>(raw[j], x);
    uint32_t s;
    const uint32_t w = value_bytes<L>(quantise<L>(x, &s), lane);
    uint8_t* to = bytes + first_row<L>(lane) * kPitch + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i * kPitch] = (uint8_t)(w >> (8 * i));
    const int64_t slot = slots[col];
    if (lane == 0 && slot >= 0) {
      uint8_t* cell = a.cache + ((slot >> g.b_log2) * g.hk + kvh) * (int64_t)g.cell;
      reinterpret_cast<uint16_t*>(cell + g.b * D)[g.b + (int)(slot & (g.b - 1))] = (uint16_t)s;
    }
  }
  // four columns that are four tokens of a block in order, from a multiple of four: their first slot
  if (threadIdx.x < kPitch / 4) {
    const int64_t* s = slots + 4 * threadIdx.x;
    runs[threadIdx.x] = s[0] >= 0 && (s[0] & 3) == 0 && s[1] == s[0] + 1 && s[2] == s[0] + 2 && s[3] == s[0] + 3 ? s[0] : -1;
  }
  __syncthreads();
  constexpr int kChunks = kPitch / 16;
  for (int x = threadIdx.x; x < D / 2 * kChunks; x += kThreads) {
    const int r = x / kChunks, c = x % kChunks;
    const uint8_t* from = bytes + r * kPitch + c * 16;
    uint8_t* row = a.cache + (int64_t)kvh * g.cell + g.b * (D / 2) + r * g.b;
    auto at = [&](int64_t slot) { return row + (slot >> g.b_log2) * g.hk * (int64_t)g.cell + (slot & (g.b - 1)); };
    const int64_t* run = runs + 4 * c;
    const int64_t s = run[0];
    if (s >= 0 && (s & 15) == 0 && run[1] == s + 4 && run[2] == s + 8 && run[3] == s + 12) {
      *reinterpret_cast<uint4*>(at(s)) = *reinterpret_cast<const uint4*>(from);
      continue;
    }
    for (int k = 0; k < 4; ++k) {
      if (run[k] >= 0) {
        *reinterpret_cast<uint32_t*>(at(run[k])) = *reinterpret_cast<const uint32_t*>(from + 4 * k);
        continue;
      }
      for (int i = 0; i < 4; ++i) {
        const int64_t slot = slots[c * 16 + 4 * k + i];
        if (slot >= 0) *at(slot) = from[4 * k + i];
      }
    }
  }
}

// A group of L lanes takes a vector, or several of one token.
//   few (kMany = false): a vector a group, values written byte by byte;
//   many: heads h, h + n/kHeads, ... of one token a group (all loads on their way at once, position and
//   slot and norm weights taken once), values in tiles of tokens.
template <int D, class T, bool kMany>
__global__ __launch_bounds__(kThreads) void store(Geo g, StoreArgs a, unsigned groups, unsigned vector_blocks) {
  constexpr int L = D / 8, N = kMany ? kHeads : 1;
  if constexpr (kMany) {
    __shared__ __attribute__((aligned(16))) uint8_t bytes[D / 2 * kPitch];
    __shared__ int64_t slots[kPitch], runs[kPitch / 4];
    if (blockIdx.x >= vector_blocks) {
      store_values<D, T>(g, a, blockIdx.x - vector_blocks, bytes, slots, runs);
      return;
    }
  }
  const int lane = threadIdx.x % L;
  const unsigned v = blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const unsigned t = v / groups, h0 = v - t * groups;
  if (t >= (unsigned)a.n_tokens) return;  // whole vectors leave
  // heads 0..hq-1 are queries, then hk keys, then (few) hk values
  const int heads = g.hq + (kMany ? 1 : 2) * g.hk;
  const int64_t slot = a.slot[t], block = slot >> g.b_log2;
  const bool stored = slot >= 0 && block < g.n_blocks;
  const int off = (int)(slot & (g.b - 1));
  uint4 raw[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = min((int)(h0 + j * groups), heads - 1);
    const uint16_t* src = h < g.hq          ? (const uint16_t*)a.q + t * a.q_stride + (int64_t)h * D
                          : h < g.hq + g.hk ? (const uint16_t*)a.k + t * a.k_stride + (int64_t)(h - g.hq) * D
                                            : (const uint16_t*)a.v + t * a.v_stride + (int64_t)(h - g.hq - g.hk) * D;
    raw[j] = reinterpret_cast<const uint4*>(src)[lane];
  }
  const uint4 none = make_uint4(0, 0, 0, 0);
  const uint4 qw = a.how.q_weight ? reinterpret_cast<const uint4*>(a.how.q_weight)[lane] : none;
  const uint4 kw = a.how.k_weight ? reinterpret_cast<const uint4*>(a.how.k_weight)[lane] : none;
  const int rot = a.how.rot_dim;
  Turn turn = {};
  if (rot) turn = turn_of(a.how.cos_sin + (int64_t)min(max(a.pos[t], 0), a.how.n_pos - 1) * rot, rot, a.how.interleaved, lane);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = (int)(h0 + j * groups);
    if (h >= heads) break;
    const bool is_q = h < g.hq, is_v = h >= g.hq + g.hk;
    if (!is_q && !stored) break;
    float x[8];
    unpack<T>(raw[j], x);
    if (!is_v) {
      if (is_q ? a.how.q_weight : a.how.k_weight) norm<L, T>(x, is_q ? qw : kw, a.how.eps);
      if (rot) rotate<L>(x, turn, rot, a.how.interleaved, lane);
    }
    if (is_q) {
      reinterpret_cast<uint4*>((uint16_t*)a.q_out + ((int64_t)t * g.hq + h) * D)[lane] = pack<T>(x);
      continue;
    }
    uint32_t s;
    const uint32_t codes = quantise<L>(x, &s);
    uint8_t* cell = a.cache + (block * g.hk + (h - g.hq - (is_v ? g.hk : 0))) * (int64_t)g.cell;
    if (lane == 0) reinterpret_cast<uint16_t*>(cell + g.b * D)[(is_v ? g.b : 0) + off] = (uint16_t)s;
    if (!is_v) {
      reinterpret_cast<uint32_t*>(cell + off * (D / 2))[lane] = codes;
      continue;
    }
    const uint32_t w = value_bytes<L>(codes, lane);
    uint8_t* row = cell + g.b * (D / 2) + (int64_t)first_row<L>(lane) * g.b + off;
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i * g.b] = (uint8_t)(w >> (8 * i));
  }
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
  const unsigned v = blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const unsigned t = v / (2u * g.hk);
  if (t >= (unsigned)a.n_tokens) return;
  const int h = (int)(v - t * (2u * g.hk));
  const bool is_v = h >= g.hk;
  const int kvh = is_v ? h - g.hk : h;
  const int64_t slot = a.slot[t], block = slot >> g.b_log2;
  uint4* out = reinterpret_cast<uint4*>((uint16_t*)(is_v ? a.v : a.k) + ((int64_t)t * g.hk + kvh) * D) + lane;
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

// Tokens of one launch: a grid has fewer than 2^32 threads.
int most_tokens(int64_t threads_a_token) { return (int)std::max<int64_t>(1, ((int64_t)1 << 31) / threads_a_token / kTile * kTile); }

struct Store {
  const Geo& g;
  const StoreArgs& a;
  hipStream_t s;
  template <int D, class T>
  hipError_t operator()() {
    constexpr int L = D / 8;
    const int most = most_tokens((int64_t)(g.hq + 2 * g.hk) * L);
    for (int t0 = 0; t0 < a.n_tokens; t0 += most) {
      StoreArgs b = a;
      b.q = (const uint16_t*)a.q + t0 * a.q_stride;
      b.k = (const uint16_t*)a.k + t0 * a.k_stride;
      b.v = (const uint16_t*)a.v + t0 * a.v_stride;
      b.q_out = (uint16_t*)a.q_out + (int64_t)t0 * g.hq * D;
      b.slot = a.slot + t0;
      if (a.pos) b.pos = a.pos + t0;
      b.n_tokens = std::min(most, a.n_tokens - t0);
      const hipError_t e = one<D, T>(b);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  template <int D, class T>
  hipError_t one(const StoreArgs& b) {
    constexpr int64_t L = D / 8;
    // few and many, us: 40 + 8 heads of 128 channels 6.6 and 8.6 (256 tokens), 9.5 and 9.9 (512),
    // 16.7 and 13.8 (1,024), 175 and 93 (16,384); 14 + 2 heads of 64 4.1 and 5.6 (256), 5.4 and
    // 5.7 (1,024), 10.3 and 8.7 (4,096); 8 + 4 heads of 256 11.7 and 15.1 (1,024), 21 and 20 (2,048)
    if ((int64_t)b.n_tokens * (g.hq + 2 * g.hk) >= kManyVectors) {
      const unsigned groups = (unsigned)((g.hq + g.hk + kHeads - 1) / kHeads);
      const unsigned vectors = (unsigned)((b.n_tokens * groups * L + kThreads - 1) / kThreads);
      const unsigned tiles = (unsigned)((b.n_tokens + kTile - 1) / kTile) * (unsigned)g.hk;
      hipLaunchKernelGGL((store<D, T, true>), dim3(vectors + tiles), dim3(kThreads), 0, s, g, b, groups, vectors);
    } else {
      const unsigned groups = (unsigned)(g.hq + 2 * g.hk);
      const unsigned vectors = (unsigned)((b.n_tokens * groups * L + kThreads - 1) / kThreads);
      hipLaunchKernelGGL((store<D, T, false>), dim3(vectors), dim3(kThreads), 0, s, g, b, groups, vectors);
    }
    return hipGetLastError();
  }
};

struct Load {
  const Geo& g;
  const LoadArgs& a;
  hipStream_t s;
  template <int D, class T>
  hipError_t operator()() {
    const int64_t width = (int64_t)2 * g.hk * (D / 8);
    const int most = most_tokens(width);
    for (int t0 = 0; t0 < a.n_tokens; t0 += most) {
      LoadArgs b = a;
      b.slot = a.slot + t0;
      b.k = (uint16_t*)a.k + (int64_t)t0 * g.hk * D;
      b.v = (uint16_t*)a.v + (int64_t)t0 * g.hk * D;
      b.n_tokens = std::min(most, a.n_tokens - t0);
      hipLaunchKernelGGL((load<D, T>), dim3((unsigned)((b.n_tokens * width + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g, b);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
