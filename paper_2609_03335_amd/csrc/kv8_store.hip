// Norm and rotation of queries and keys and the store of keys and values as 8-bit codes with a scale for each
// block and head (and its inverse).
//
// The tokens of a call that lie in one block, one after the other, are a run; a workgroup takes the
// runs that begin among `tile` tokens of one kv head, from the first's first to the last's last token.  A scale is known
// when the last token of the run is, so normed keys and values stay in registers (two passes, 64 tokens of 128 channels; what a
// tile has beyond that is read again): largest magnitudes of the runs in LDS, scales, then codes.  Where a run's block
// holds earlier tokens under a smaller scale, the block's codes are rounded to the new one in between.  Value codes
// go through LDS once more, so that a thread stores two channels of four tokens, 8 bytes, instead of one byte four times.
// Sums of squares add neighbours first and every operation is rounded by itself, so that the codes are
// reproducible to the last bit by elementary operations.
//
// Large calls are bound by memory: 14,000 prompt tokens of 40 + 8 heads of 128 channels read 200 MB and write 172 (the counters
// say 265, rotations by each die, and 172: 5.1 TB/s), 85 us, of which the keys' and values' workgroups, three barriers and a chain of loads long, fill half
// while the queries' stream beside them; reading them back 19 us (4.4 TB/s).  Small ones are bound by the chain: 181 single
// tokens 6.4 us, most of them blocks that hold others, and 3.2 us back.
#include "kv8.h"
#include "kv_vector.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256, kManyThreads = 512, kPasses = 2, kManyWaves = 4;  // of a workgroup; where there are many tokens
// tokens of a tile, and that a workgroup looks at: up to a block's before the tile and behind it
constexpr int kMostTile = 256, kMostBlock = 256, kSpan = kMostTile + 2 * kMostBlock;
constexpr int kHeads = 4;                // query heads a lane group takes of a token, of many
// Vectors of a call from which they are many: more passes a workgroup, four heads a lane group.  Few against many (us), 40 + 8
// heads of 128 channels, prompts: 300 tokens (16,800) 15.5 and 15.1, 600 21.5 and 16.2, 2,000 30.5 and 26.4, 4,000 49 and 36;
// 32 + 8 heads, single tokens, a run each: 500 (24,000) 8.0 and 13.4, 2,000 (96,000) 23.9 and 23.4.
constexpr int64_t kManyVectors = 32768;

// A lane's part of a vector that is not read again here; of large calls past the caches (14,000 tokens of 40 + 8 heads
// stored and read back 115 -> 110 us).
template <bool kPast>
__device__ __forceinline__ void put(uint4* to, const uint4& x) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 w = {x.x, x.y, x.z, x.w};
  if constexpr (kPast) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to));
  else *reinterpret_cast<u32x4*>(to) = w;
}

// A launch's part of the work: `items` tiles of `tile` tokens of a kv head by workgroups 0, every, 2 every, ...
// (item_blocks of them; they wait for one load after the other, the others, which stream, use the time);
// queries of tokens [token, token + tokens), `groups` lane groups a token, by the others.
struct Share {
  int token, tokens;
  unsigned groups, item_blocks, items, every;
  int tile;
};

// A query's heads h0, h0 + groups, ...
template <int D, class T, int N, int W>
__device__ __forceinline__ void queries(const Geo& g, const StoreArgs& a, const Share& part, unsigned block) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x % L;
  const unsigned v = block * (W / L) + threadIdx.x / L;
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
    put<(N > 1)>(reinterpret_cast<uint4*>((uint16_t*)a.q_out + ((int64_t)t * g.hq + h) * D) + lane, pack<T>(x));
  }
}

// A key at a position, normed and rotated.
template <int D, class T>
__device__ __forceinline__ void key_of(const StoreArgs& a, int pos, const uint4& raw, int lane, const uint4& weight, float* x) {
  constexpr int L = D / 8;
  const int rot = a.how.rot_dim;
  Turn turn = {};
  if (rot) turn = turn_of(a.how.cos_sin + (int64_t)min(max(pos, 0), a.how.n_pos - 1) * rot, rot, a.how.interleaved, lane);
  unpack<T>(raw, x);
  if (a.how.k_weight) norm<L, T>(x, weight, a.how.eps);
  if (rot) rotate<L>(x, turn, rot, a.how.interleaved, lane);
}

// The bits of the largest magnitude of eight 16-bit values, as fp32's.
template <int L, class T>
__device__ __forceinline__ uint32_t largest(const uint4& raw) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto two = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(two(raw.x), two(raw.y)), __builtin_elementwise_max(two(raw.z), two(raw.w)));
  return __float_as_uint(T::to(vector_max<L>((uint32_t)max(m[0], m[1]))));
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
  int64_t cell[kSpan];        // its cell in the cache, and its place in it (-1: not this workgroup's)
  int16_t off[kSpan];
  uint8_t four[kSpan];        // whether it and the next three are the tokens of a word of values
  int lead[kSpan];            // first token of the token's run, -1: not this workgroup's
  uint32_t most[2][kSpan];    // of a run (at its first token): largest magnitudes of keys and values,
  int8_t power[2][kSpan];     // then the powers of their scales;
  uint8_t begins[kSpan];      // whether it holds its block's first token
  uint8_t bad[kSpan];         // of a token: something in it is not finite
  int16_t up[kSpan][3];       // runs whose block is rounded anew: first token, powers to add
  int ups;
  int last_event[kSpan / 64];
  int first, end;             // this workgroup's tokens
};

template <int D, class T, int P, int W>
__device__ __forceinline__ void keys_values(const Geo& g, const StoreArgs& a, unsigned item, int tile, Span& sp, uint8_t (&codes_of_pass)[P][8 * W]) {
  constexpr int L = D / 8, V = W / L, E = (kSpan + W - 1) / W;
  // (opaque, so that what follows from it is worked out here and not kept in registers, or scratch, across items: 110 -> 103 us)
  unsigned tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int kvh = (int)(item % (unsigned)g.hk), lane = (int)(tid % L), group = (int)(tid / L);
  if (tid == 0) sp.ups = 0, sp.first = kSpan, sp.end = 0;
  const int64_t none = -1;
  auto valid = [&](int64_t s) { return s >= 0 && s >> g.b_log2 < g.n_blocks ? s : none; };
  // A tile begins where the block of its first token begins, if that is in this call: runs of whole blocks
  // are whole in a tile then, and its passes of V tokens are theirs.
  auto aligned = [&](int x) {
    if (x <= 0 || x >= a.n_tokens) return min(max(x, 0), a.n_tokens);
    const auto* slot = (const __attribute__((address_space(4))) int64_t*)a.slot;
    const int64_t s = slot[x];
    const int k = (int)(s & (g.b - 1));
    return k <= x && slot[x - k] == s - k ? x - k : x;
  };
  const int x0 = (int)(item / (unsigned)g.hk) * tile, t0 = aligned(x0), own = max(aligned(x0 + tile) - t0, 0);
  const int span = min(own + g.b, a.n_tokens - t0);
  const uint4 weight = a.how.k_weight ? reinterpret_cast<const uint4*>(a.how.k_weight)[lane] : make_uint4(0, 0, 0, 0);
  auto slot_at = [&](int i) { return valid(a.slot[t0 + i]); };
  // (all lane groups take part in every pass, on some token of the span)
  auto at = [&](int p) __attribute__((always_inline)) { return min(p * V + group, span - 1); };
  auto load = [&](int p, uint4& x, uint4& y, int& pos) __attribute__((always_inline)) {
    const int t = t0 + at(p);
    x = reinterpret_cast<const uint4*>((const uint16_t*)a.k + t * a.k_stride + (int64_t)kvh * D)[lane];
    y = reinterpret_cast<const uint4*>((const uint16_t*)a.v + t * a.v_stride + (int64_t)kvh * D)[lane];
    pos = a.how.rot_dim ? a.pos[t] : 0;
  };
  // The first P stay in registers, and are done before it is known which tokens are this workgroup's: every load that
  // waits for another's result waits behind all that the CU has asked for.
  float keys[P][8];
  uint4 values[P];
  {
    uint4 raw[P];
    int pos[P];
#pragma unroll
    for (int p = 0; p < P; ++p) load(p, raw[p], values[p], pos[p]);
#pragma unroll
    for (int p = 0; p < P; ++p) key_of<D, T>(a, pos[p], raw[p], lane, weight, keys[p]);
  }
  // events: tokens that begin a run, or are not stored
  uint64_t events[E], owned[E];
#pragma unroll
  for (int p = 0; p < E; ++p) {
    const int i = p * W + (int)tid;
    events[p] = owned[p] = 0;
    if (i - (int)(tid & 63) >= kSpan) continue;
    bool event = true, mine = false;
    if (i < span) {
      const int64_t s = slot_at(i), before = t0 + i > 0 ? slot_at(i - 1) : none;
      sp.slot[i] = s;
      event = s < 0 || before < 0 || before >> g.b_log2 != s >> g.b_log2;
      mine = event && s >= 0 && i < own;
      sp.most[0][i] = sp.most[1][i] = sp.bad[i] = 0;
      sp.begins[i] = 0;
    }
    events[p] = __ballot(event);
    owned[p] = __ballot(mine);
    if ((tid & 63) == 0) {
      const int at = 63 - __clzll((long long)events[p]);
      sp.last_event[i >> 6] = events[p] == 0 ? -2 : owned[p] >> at & 1 ? i + at : -1;
    }
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < E; ++p) {
    const int i = p * W + (int)tid;
    if (i >= span) continue;
    const uint64_t upto = events[p] & (~0ull >> (63 - (tid & 63)));
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
    if (lead >= 0 && (sp.slot[i] & (g.b - 1)) == 0) sp.begins[lead] = 1;
    const uint64_t mine = __ballot(lead >= 0);
    if (mine && (tid & 63) == 0) {  // (lane 0 of a wave that has tokens of the span is in it)
      atomicMin(&sp.first, i + __ffsll((unsigned long long)mine) - 1);
      atomicMax(&sp.end, i + 64 - __clzll((long long)mine));
    }
  }
  __syncthreads();
  const int first = sp.first, end = sp.end;
  if (first >= end) return;
  const int passes = (end + V - 1) / V, begin = first / V;
  auto measure = [&](int p, const float* x, const uint4& y) __attribute__((always_inline)) {
    const uint32_t k = largest<L>(x), z = largest<L, T>(y);
    const int i = at(p), lead = sp.lead[i];
    if (lane || lead < 0) return;
    // infinities and NaN have the largest bit patterns
    if (max(k, z) >= 0x7f800000u) {
      sp.bad[i] = 1;
    } else {
      atomicMax(&sp.most[0][lead], k);
      atomicMax(&sp.most[1][lead], z);
    }
  };
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (p < passes) measure(p, keys[p], values[p]);
  for (int p = max(P, begin); p < passes; ++p) {
    float x[8];
    uint4 raw, y;
    int pos;
    load(p, raw, y, pos);
    key_of<D, T>(a, pos, raw, lane, weight, x);
    measure(p, x, y);
  }
  __syncthreads();
  // where tokens lie, and whether they and the next three are four of a word, by a thread each
  for (int i = first + (int)tid; i < end; i += W) {
    const int64_t s = sp.slot[i];
    const int lead = sp.lead[i];
    sp.cell[i] = ((s >> g.b_log2) * g.hk + kvh) * (int64_t)g.cell;
    sp.off[i] = lead < 0 ? -1 : (int)(s & (g.b - 1));
    sp.four[i] = lead >= 0 && (s & 3) == 0 && i + 3 < end && sp.lead[i + 3] == lead && sp.slot[i + 1] == s + 1 && sp.slot[i + 2] == s + 2 &&
                 sp.slot[i + 3] == s + 3;
  }
  auto cell_of = [&](int i) { return a.cache + sp.cell[i]; };
  const int codes = 2 * g.b * D;  // bytes of them, then the scales
  for (int i = first + (int)tid; i < end; i += W) {
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
      sp.power[p][i] = (int8_t)e;
      scales[p] = two_to(e);
    }
    if (rise[0] | rise[1]) {
      const int n = atomicAdd(&sp.ups, 1);
      sp.up[n][0] = (int16_t)i, sp.up[n][1] = (int16_t)rise[0], sp.up[n][2] = (int16_t)rise[1];
    }
  }
  __syncthreads();
  // codes under the old scale: 2^-40 of the largest is no code any more
  const int ups = sp.ups;
  for (int n = 0; n < ups; ++n) {
    uint4* cell = reinterpret_cast<uint4*>(cell_of(sp.up[n][0]));
    for (int x = (int)tid; x < codes / 16; x += W) {
      const int rise = sp.up[n][x < codes / 32 ? 1 : 2];
      if (rise == 0) continue;
      const float by = two_to(max(rise, -40));
      const uint4 w = cell[x];
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
      cell[x] = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  if (ups) __syncthreads();
  // Codes of a pass: its keys' in registers, its values' in LDS, as a thread stores two channels of four tokens.
  auto encode = [&](int p, float* x, const uint4& raw, uint8_t* bytes) __attribute__((always_inline)) -> uint2 {
    const int i = p * V + group, lead = i >= first && i < end ? sp.lead[i] : -1;
    uint32_t kc[2] = {0, 0}, vc[2] = {0, 0};
    if (lead >= 0) {
      const int ke = sp.power[0][lead], ve = sp.power[1][lead];
      const float ks = two_to(ke), vs = two_to(ve);
      kc[0] = codes_under(x, ks), kc[1] = codes_under(x + 4, ks);
      vc[0] = codes_under<T>(raw.x, raw.y, vs), vc[1] = codes_under<T>(raw.z, raw.w, vs);
      if (__builtin_expect(max(ke, ve) == kMostPower, 0)) {  // values may pass 448 times the largest scale
        float y[8];
        unpack<T>(raw, y);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= two_to(-ke), y[k] *= two_to(-ve);
        kc[0] = codes_of(x), kc[1] = codes_of(x + 4), vc[0] = codes_of(y), vc[1] = codes_of(y + 4);
      }
      if (sp.bad[i]) kc[0] = kc[1] = 0x7f7f7f7fu, vc[0] = vc[1] = 0;
    }
    reinterpret_cast<uint2*>(bytes + group * D)[lane] = make_uint2(vc[0], vc[1]);
    return make_uint2(kc[0], kc[1]);
  };
  auto store = [&](int p, const uint2& kc, const uint8_t* bytes) __attribute__((always_inline)) {
    const int i = p * V + group;
    const int off = i >= first && i < end ? sp.off[i] : -1;
    if (off >= 0) reinterpret_cast<uint2*>(cell_of(i) + off * D)[lane] = kc;
    const int q = (int)(tid / (D / 2)), ch = (int)(tid % (D / 2)) * 2, i0 = p * V + q * 4;
    uint32_t two[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) two[t] = *reinterpret_cast<const uint16_t*>(bytes + (q * 4 + t) * D + ch);
    if (i0 >= first && i0 < end && sp.four[i0]) {
      const uint32_t lo = (two[0] & 0xff) | (two[1] & 0xff) << 8 | (two[2] & 0xff) << 16 | two[3] << 24;
      const uint32_t hi = two[0] >> 8 | (two[1] & 0xff00) | (two[2] & 0xff00) << 8 | (two[3] & 0xff00) << 16;
      *reinterpret_cast<uint2*>(cell_of(i0) + g.b * D + sp.off[i0] * D + ch * 4) = make_uint2(lo, hi);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int k = i0 + t, off = k >= first && k < end ? sp.off[k] : -1;
        if (off < 0) continue;
        uint8_t* to = cell_of(k) + g.b * D + ((off >> 2) * D + ch) * 4 + (off & 3);
        to[0] = (uint8_t)two[t], to[4] = (uint8_t)(two[t] >> 8);
      }
    }
  };
  // (a barrier waits for the stores before it: all of the passes in registers go out behind one)
  uint2 kc[P];
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (p < passes) kc[p] = encode(p, keys[p], values[p], codes_of_pass[p]);
  __syncthreads();
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (p < passes) store(p, kc[p], codes_of_pass[p]);
  for (int p = max(P, begin); p < passes; ++p) {
    float x[8];
    uint4 raw, y;
    int pos;
    load(p, raw, y, pos);
    key_of<D, T>(a, pos, raw, lane, weight, x);
    __syncthreads();
    const uint2 c = encode(p, x, y, codes_of_pass[0]);
    __syncthreads();
    store(p, c, codes_of_pass[0]);
  }
}

template <int D, class T, bool kMany>
__global__ __launch_bounds__(kMany ? kManyThreads : kThreads, (kMany ? kManyWaves : 2)) void store8(Geo g, StoreArgs a, Share part) {
  constexpr int W = kMany ? kManyThreads : kThreads;
  __shared__ Span span;
  __shared__ __attribute__((aligned(16))) uint8_t codes_of_pass[kMany ? kPasses : 1][8 * W];
  const unsigned nth = blockIdx.x / part.every, before = min((blockIdx.x + part.every - 1) / part.every, part.item_blocks);
  if (nth * part.every != blockIdx.x || nth >= part.item_blocks) {
    queries<D, T, kMany ? kHeads : 1, W>(g, a, part, blockIdx.x - before);
    return;
  }
  for (unsigned item = nth; item < part.items; item += part.item_blocks) {
    keys_values<D, T, kMany ? kPasses : 1, W>(g, a, item, part.tile, span, codes_of_pass);
    __syncthreads();
  }
}

// A group of L lanes takes one of a token's 2 hk vectors (keys, then values), or N of them, `groups` apart.
template <int D, class T, int N>
__global__ __launch_bounds__(kThreads) void load8(Geo g, LoadArgs a, unsigned groups) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x % L, vectors = 2 * g.hk;
  const unsigned v = blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const unsigned t = v / groups, h0 = v - t * groups;
  if (t >= (unsigned)a.n_tokens) return;
  const int64_t slot = a.slot[t], block = slot >> g.b_log2;
  const bool held = slot >= 0 && block < g.n_blocks;
  const int off = (int)(slot & (g.b - 1)), by = 8 * (off & 3);
  const uint8_t* cells = a.cache + (held ? block : 0) * g.hk * (int64_t)g.cell;
  uint4 w[N][2];
  uint32_t first[N];
  float s[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = min((int)(h0 + j * groups), vectors - 1);
    const bool is_v = h >= g.hk;
    const uint8_t* cell = cells + (is_v ? h - g.hk : h) * (int64_t)g.cell;
    s[j] = reinterpret_cast<const float*>(cell + 2 * g.b * D)[is_v];
    if (is_v) {
      // the words of four tokens, as whole ones: one token's bytes would take as many lines
      const uint4* from = reinterpret_cast<const uint4*>(cell + g.b * D + ((off >> 2) * D + lane * 8) * 4);
      w[j][0] = from[0], w[j][1] = from[1];
      first[j] = cell[off * D];
    } else {
      const uint2 x = reinterpret_cast<const uint2*>(cell + off * D)[lane];
      w[j][0].x = x.x, w[j][0].y = x.y;
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int h = (int)(h0 + j * groups);
    if (h >= vectors) break;
    const bool is_v = h >= g.hk;
    uint4* out = reinterpret_cast<uint4*>((uint16_t*)(is_v ? a.v : a.k) + ((int64_t)t * g.hk + (is_v ? h - g.hk : h)) * D) + lane;
    if (!held) {
      *out = make_uint4(0, 0, 0, 0);
      continue;
    }
    uint32_t codes[2] = {w[j][0].x, w[j][0].y};
    if (is_v) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        codes[i] = (w[j][i].x >> by & 0xff) | (w[j][i].y >> by & 0xff) << 8 | (w[j][i].z >> by & 0xff) << 16 | (w[j][i].w >> by & 0xff) << 24;
      // a token that is not a number says so in its key
      if ((first[j] & 0x7f) == 0x7f) codes[0] = codes[1] = 0x7f7f7f7fu;
    }
    float x[8];
    values_of(codes[0], x);
    values_of(codes[1], x + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= s[j];
      // the code's rounding can pass the type's range
      if (fabsf(x[i]) > T::kMost) x[i] = copysignf(T::kMost, x[i]);
    }
    put<(N > 1)>(out, pack<T>(x));
  }
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
    const bool many = (int64_t)a.n_tokens * (g.hq + 2 * g.hk) >= kManyVectors;
    const int threads = many ? kManyThreads : kThreads;
    Share part;
    // two passes, or a block; one pass of a smaller workgroup
    part.tile = many ? std::max(kPasses * kManyThreads / (int)L, g.b) : kThreads / (int)L;
    part.groups = (unsigned)(many ? (g.hq + kHeads - 1) / kHeads : g.hq);
    part.items = (unsigned)((a.n_tokens + part.tile - 1) / part.tile) * (unsigned)g.hk;
    // all keys and values in the first launch, so that no run is cut
    const int most = most_tokens(part.groups * L);
    for (part.token = 0; part.token < a.n_tokens; part.token += most, part.items = 0) {
      part.tokens = std::min(most, a.n_tokens - part.token);
      part.item_blocks = std::min(part.items, 1u << 22);
      const unsigned streams = (unsigned)((part.tokens * (int64_t)part.groups * L + threads - 1) / threads);
      const dim3 grid(part.item_blocks + streams);
      // (items of more passes, which would be a tail, all first: blocks of 256 tokens 98 us against 153; of 64 100 against 96)
      const bool shared_out = many && part.tile == kPasses * kManyThreads / (int)L;
      // (an odd number: workgroups go to the eight dies in turn, and all are to have their share of these; 28 + 4 heads, every 3rd
      // for every 4th: 84 -> 65 us.  The heads of a tile on one die, where they find its rotations, read 220 MB for 265,
      // and took 104 us for 103.)
      part.every = part.item_blocks && shared_out ? (grid.x / part.item_blocks - 1) | 1 : 1;
      if (many) hipLaunchKernelGGL((store8<D, T, true>), grid, dim3(threads), 0, s, g, a, part);
      else hipLaunchKernelGGL((store8<D, T, false>), grid, dim3(threads), 0, s, g, a, part);
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
    const bool many = (int64_t)a.n_tokens * 2 * g.hk >= kManyVectors;
    const unsigned groups = many ? (2u * g.hk + kHeads - 1) / kHeads : 2u * g.hk;
    const int64_t width = (int64_t)groups * (D / 8);
    const int most = most_tokens(width);
    for (int t0 = 0; t0 < a.n_tokens; t0 += most) {
      LoadArgs b = a;
      b.slot = a.slot + t0;
      b.k = (uint16_t*)a.k + (int64_t)t0 * g.hk * D;
      b.v = (uint16_t*)a.v + (int64_t)t0 * g.hk * D;
      b.n_tokens = std::min(most, a.n_tokens - t0);
      const dim3 grid((unsigned)((b.n_tokens * width + kThreads - 1) / kThreads));
      if (many) hipLaunchKernelGGL((load8<D, T, kHeads>), grid, dim3(kThreads), 0, s, g, b, groups);
      else hipLaunchKernelGGL((load8<D, T, 1>), grid, dim3(kThreads), 0, s, g, b, groups);
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
