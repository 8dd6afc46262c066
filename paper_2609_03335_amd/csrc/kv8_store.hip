// Norm and rotation of queries and keys and the store of keys and values as 8-bit codes with a scale for each
// block and head (and its inverse).
//
// The tokens of a call that lie in one block, one after the other, are a run; a workgroup takes the
// runs that begin among `tile` tokens of one kv head, from the first's first to the last's last token.  It goes over their keys and
// values twice: the largest magnitude of each run gives its block's scale, then the codes are written.  Where
// a run's block holds earlier tokens under a smaller scale, the block's codes are rounded to the new one in between.
// Sums of squares add neighbours first and every operation is rounded by itself, so that the codes are
// reproducible to the last bit by elementary operations.
#include "kv8.h"
#include "kv_vector.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTile = 64, kMostBlock = 256, kSpan = kMostTile + kMostBlock;
constexpr int kHeads = 4;                // query heads a lane group takes of a token, of many
constexpr int64_t kManyVectors = 32768;  // query vectors of a call from which they are many

// A launch's part of the work: queries of tokens [token, token + tokens), `groups` lane groups a token, by the first
// `vector_blocks` workgroups; `items` tiles of `tile` tokens of a kv head by the others.
struct Share {
  int token, tokens;
  unsigned groups, vector_blocks, items;
  int tile;
};

// A query's heads h0, h0 + groups, ...
template <int D, class T, int N>
__device__ __forceinline__ void queries(const Geo& g, const StoreArgs& a, const Share& part) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x % L;
  const unsigned v = blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const unsigned groups = part.groups, i = v / groups, h0 = v - i * groups;
  if (i >= (unsigned)part.tokens) return;  // whole vectors leave
  const int t = part.token + (int)i;
  uint4 raw[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = min((int)(h0 + j * groups), g.hq - 1);
    raw[j] = reinterpret_cast<const uint4*>((const uint16_t*)a.q + t * a.q_stride + (int64_t)h * D)[lane];
  }
  const uint4 w = a.how.q_weight ? reinterpret_cast<const uint4*>(a.how.q_weight)[lane] : make_uint4(0, 0, 0, 0);
  const int rot = a.how.rot_dim;
  Turn turn = {};
  if (rot) turn = turn_of(a.how.cos_sin + (int64_t)min(max(a.pos[t], 0), a.how.n_pos - 1) * rot, rot, a.how.interleaved, lane);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = (int)(h0 + j * groups);
    if (h >= g.hq) break;
    float x[8];
    unpack<T>(raw[j], x);
    if (a.how.q_weight) norm<L, T>(x, w, a.how.eps);
    if (rot) rotate<L>(x, turn, rot, a.how.interleaved, lane);
    reinterpret_cast<uint4*>((uint16_t*)a.q_out + ((int64_t)t * g.hq + h) * D)[lane] = pack<T>(x);
  }
}

// A token's key of a head, normed and rotated.
template <int D, class T>
__device__ __forceinline__ void key_of(const StoreArgs& a, int t, int kvh, int lane, const uint4& weight, float* x) {
  constexpr int L = D / 8;
  unpack<T>(reinterpret_cast<const uint4*>((const uint16_t*)a.k + t * a.k_stride + (int64_t)kvh * D)[lane], x);
  if (a.how.k_weight) norm<L, T>(x, weight, a.how.eps);
  const int rot = a.how.rot_dim;
  if (rot) {
    const Turn turn = turn_of(a.how.cos_sin + (int64_t)min(max(a.pos[t], 0), a.how.n_pos - 1) * rot, rot, a.how.interleaved, lane);
    rotate<L>(x, turn, rot, a.how.interleaved, lane);
  }
}

template <int L>
__device__ __forceinline__ uint32_t largest(const float* x) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  return vector_max<L>(most);
}

// What a workgroup knows of the tokens of its span.
struct Span {
  int64_t slot[kSpan];
  int lead[kSpan];            // first token of the token's run, -1: not this workgroup's
  uint32_t most[2][kSpan];    // of a run (at its first token): largest magnitudes of keys and values,
  int power[2][kSpan];        // then the powers of their scales;
  int begins[kSpan];          // whether it holds its block's first token
  uint32_t bad[kSpan];        // of a token: something in it is not finite
  int up[kSpan][3], ups;      // runs whose block is rounded anew: first token, powers to add
  int last_event[kSpan / 64];
  int first, end;             // this workgroup's tokens
};

template <int D, class T>
__device__ __forceinline__ void keys_values(const Geo& g, const StoreArgs& a, unsigned item, int tile, Span& sp) {
  constexpr int L = D / 8, V = kThreads / L;
  const int kvh = (int)(item % (unsigned)g.hk), t0 = (int)(item / (unsigned)g.hk) * tile;
  const int span = min(tile + g.b, a.n_tokens - t0);
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  if (threadIdx.x == 0) sp.ups = 0, sp.first = kSpan, sp.end = 0;
  // events: tokens that begin a run, or are not stored
  const int64_t none = -1;
  auto slot_at = [&](int i) {
    const int64_t s = a.slot[t0 + i];
    return s >= 0 && s >> g.b_log2 < g.n_blocks ? s : none;
  };
  uint64_t events[2], owned[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int i = p * kThreads + (int)threadIdx.x;
    events[p] = owned[p] = 0;
    if (i - (int)(threadIdx.x & 63) >= kSpan) continue;
    bool event = true, mine = false;
    if (i < span) {
      const int64_t s = slot_at(i), before = t0 + i > 0 ? slot_at(i - 1) : none;
      sp.slot[i] = s;
      event = s < 0 || before < 0 || before >> g.b_log2 != s >> g.b_log2;
      mine = event && s >= 0 && i < tile;
      sp.most[0][i] = sp.most[1][i] = sp.bad[i] = 0;
      sp.begins[i] = 0;
    }
    events[p] = __ballot(event);
    owned[p] = __ballot(mine);
    if ((threadIdx.x & 63) == 0) {
      const int at = 63 - __clzll((long long)events[p]);
      sp.last_event[i >> 6] = events[p] == 0 ? -2 : owned[p] >> at & 1 ? i + at : -1;
    }
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int i = p * kThreads + (int)threadIdx.x;
    if (i >= span) continue;
    const uint64_t upto = events[p] & (~0ull >> (63 - (threadIdx.x & 63)));
    int lead = -1;
    if (upto) {
      const int at = 63 - __clzll((long long)upto);
      if (owned[p] >> at & 1) lead = (i & ~63) + at;
    } else {
      int w = (i >> 6) - 1;
      while (w >= 0 && sp.last_event[w] == -2) --w;
      lead = w >= 0 ? sp.last_event[w] : -1;
    }
    sp.lead[i] = lead;
    if (lead >= 0) {
      atomicMin(&sp.first, i);
      atomicMax(&sp.end, i + 1);
      if ((sp.slot[i] & (g.b - 1)) == 0) sp.begins[lead] = 1;
    }
  }
  __syncthreads();
  const int first = sp.first, end = sp.end;
  const uint4 weight = a.how.k_weight ? reinterpret_cast<const uint4*>(a.how.k_weight)[lane] : make_uint4(0, 0, 0, 0);
  // (all lane groups take part in every pass, on the span's last token if on no other)
  for (int j = first; j < end; j += V) {
    const int i = min(j + group, end - 1);
    float x[8], y[8];
    key_of<D, T>(a, t0 + i, kvh, lane, weight, x);
    unpack<T>(reinterpret_cast<const uint4*>((const uint16_t*)a.v + (t0 + i) * a.v_stride + (int64_t)kvh * D)[lane], y);
    const uint32_t k = largest<L>(x), v = largest<L>(y);
    const int lead = sp.lead[i];
    if (lane || lead < 0) continue;
    // infinities and NaN have the largest bit patterns
    if (max(k, v) >= 0x7f800000u) {
      sp.bad[i] = 1;
    } else {
      atomicMax(&sp.most[0][lead], k);
      atomicMax(&sp.most[1][lead], v);
    }
  }
  __syncthreads();
  auto cell_of = [&](int i) { return a.cache + ((sp.slot[i] >> g.b_log2) * g.hk + kvh) * (int64_t)g.cell; };
  const int codes = 2 * g.b * D;  // bytes of them, then the scales
  for (int i = first + (int)threadIdx.x; i < end; i += kThreads) {
    if (sp.lead[i] != i) continue;
    float* scales = reinterpret_cast<float*>(cell_of(i) + codes);
    int rise[2] = {0, 0};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      int e = least_power(sp.most[p][i]);
      if (!sp.begins[i]) {
        const int old = power_of(scales[p]);
        e = max(e, old);
        rise[p] = old - e;
      }
      sp.power[p][i] = e;
      scales[p] = two_to(e);
    }
    if (rise[0] | rise[1]) {
      const int n = atomicAdd(&sp.ups, 1);
      sp.up[n][0] = i, sp.up[n][1] = rise[0], sp.up[n][2] = rise[1];
    }
  }
  __syncthreads();
  // codes under the old scale: 2^-40 of the largest is no code any more
  for (int n = 0; n < sp.ups; ++n) {
    uint4* at = reinterpret_cast<uint4*>(cell_of(sp.up[n][0]));
    for (int x = threadIdx.x; x < codes / 16; x += kThreads) {
      const int rise = sp.up[n][x < codes / 32 ? 1 : 2];
      if (rise == 0) continue;
      const float by = two_to(max(rise, -40));
      const uint4 w = at[x];
      uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[4];
        values_of(u[i], f);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] *= by;
        const uint32_t c = codes_of(f);
        // (what is not a number stays so: the clamp would make a number of it)
        uint32_t nan = (u[i] & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u;
        nan = (nan >> 7) * 0xffu;
        u[i] = (c & ~nan) | (u[i] & nan);
      }
      at[x] = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  if (sp.ups) __syncthreads();  // (the same for all: set before the last barrier)
  for (int j = first; j < end; j += V) {
    const int i = min(j + group, end - 1), lead = sp.lead[i];
    float x[8], y[8];
    key_of<D, T>(a, t0 + i, kvh, lane, weight, x);
    unpack<T>(reinterpret_cast<const uint4*>((const uint16_t*)a.v + (t0 + i) * a.v_stride + (int64_t)kvh * D)[lane], y);
    if (lead < 0 || j + group >= end) continue;
    const float ks = two_to(-sp.power[0][lead]), vs = two_to(-sp.power[1][lead]);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= ks, y[k] *= vs;
    uint32_t kc[2] = {codes_of(x), codes_of(x + 4)}, vc[2] = {codes_of(y), codes_of(y + 4)};
    if (sp.bad[i]) kc[0] = kc[1] = 0x7f7f7f7fu, vc[0] = vc[1] = 0;
    uint8_t* cell = cell_of(i);
    const int off = (int)(sp.slot[i] & (g.b - 1));
    reinterpret_cast<uint2*>(cell + off * D)[lane] = make_uint2(kc[0], kc[1]);
    uint8_t* to = cell + g.b * D + ((off >> 2) * D + lane * 8) * 4 + (off & 3);
#pragma unroll
    for (int k = 0; k < 8; ++k) to[4 * k] = (uint8_t)(vc[k / 4] >> (8 * (k % 4)));
  }
}

// Workgroups up to `vector_blocks` take queries, the others keys and values.
template <int D, class T, bool kMany>
__global__ __launch_bounds__(kThreads) void store8(Geo g, StoreArgs a, Share part) {
  __shared__ Span span;
  if (blockIdx.x < part.vector_blocks) {
    queries<D, T, kMany ? kHeads : 1>(g, a, part);
    return;
  }
  for (unsigned item = blockIdx.x - part.vector_blocks; item < part.items; item += gridDim.x - part.vector_blocks) {
    keys_values<D, T>(g, a, item, part.tile, span);
    __syncthreads();
  }
}

// One vector a group of L lanes: keys and values of each token and kv head.
template <int D, class T>
__global__ __launch_bounds__(kThreads) void load8(Geo g, LoadArgs a) {
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
  const float s = reinterpret_cast<const float*>(cell + 2 * g.b * D)[is_v];
  uint32_t codes[2];
  if (!is_v) {
    const uint2 w = reinterpret_cast<const uint2*>(cell + off * D)[lane];
    codes[0] = w.x, codes[1] = w.y;
  } else {
    const uint8_t* from = cell + g.b * D + ((off >> 2) * D + lane * 8) * 4 + (off & 3);
    codes[0] = codes[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes[i / 4] |= (uint32_t)from[4 * i] << (8 * (i % 4));
    // a token that is not a number says so in its key
    if ((cell[off * D] & 0x7f) == 0x7f) codes[0] = codes[1] = 0x7f7f7f7fu;
  }
  float x[8];
  values_of(codes[0], x);
  values_of(codes[1], x + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] *= s;
    // the code's rounding can pass the type's range
    if (fabsf(x[i]) > T::kMost) x[i] = copysignf(T::kMost, x[i]);
  }
  *out = pack<T>(x);
}

// Tokens of one launch: a grid has fewer than 2^32 threads.
int most_tokens(int64_t threads_a_token) { return (int)std::max<int64_t>(1, ((int64_t)1 << 31) / threads_a_token / kMostBlock * kMostBlock); }

struct Store8 {
  const Geo& g;
  const StoreArgs& a;
  hipStream_t s;
  template <int D, class T>
  hipError_t operator()() {
    constexpr int64_t L = D / 8;
    const bool many = (int64_t)a.n_tokens * g.hq >= kManyVectors;
    Share part;
    part.tile = a.n_tokens * (int64_t)g.hk >= kManyVectors / 4 ? kMostTile : 16;
    part.groups = (unsigned)(many ? (g.hq + kHeads - 1) / kHeads : g.hq);
    part.items = (unsigned)((a.n_tokens + part.tile - 1) / part.tile) * (unsigned)g.hk;
    // all keys and values in the first launch, so that no run is cut
    const int most = most_tokens(part.groups * L);
    for (part.token = 0; part.token < a.n_tokens; part.token += most, part.items = 0) {
      part.tokens = std::min(most, a.n_tokens - part.token);
      part.vector_blocks = (unsigned)((part.tokens * (int64_t)part.groups * L + kThreads - 1) / kThreads);
      const dim3 grid(part.vector_blocks + std::min(part.items, 1u << 22));
      if (many) hipLaunchKernelGGL((store8<D, T, true>), grid, dim3(kThreads), 0, s, g, a, part);
      else hipLaunchKernelGGL((store8<D, T, false>), grid, dim3(kThreads), 0, s, g, a, part);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
};

struct Load8 {
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
      hipLaunchKernelGGL((load8<D, T>), dim3((unsigned)((b.n_tokens * width + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, g, b);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
};

}  // namespace

hipError_t launch_store8(const Geo& g, int dtype, const StoreArgs& a, hipStream_t s) {
  return by_type(g.d, dtype, Store8{g, a, s});
}

hipError_t launch_load8(const Geo& g, int dtype, const LoadArgs& a, hipStream_t s) {
  return by_type(g.d, dtype, Load8{g, a, s});
}

}  // namespace wfkv
