// Attention of a step's queries over the paged 8-bit cache.
//
//   o = sum_j p_j v_j,  p = softmax_j(scale q.k_j),  k_j = 2^e c_j,  v_j = 2^f d_j
//
// with codes c, d of 8 bits and one e and f for a block.  Codes are exact in bf16 and f16, and so are
// values in bf16: the conversion of the values' codes multiplies with their scale at no cost.  f16 could not hold
// them: there f is added to the exponent, p_j 2^f = 2^(score - reference + f) is rounded to f16 once, and a block's
// terms go into the softmax's total divided by 2^f (16 products of a lane and 64 tokens less than p_j times the scale:
// 7 chunks of up to 500 of 14 heads 54 -> 52 us, a prompt of 7,001 of 32 heads 440 -> 418).
// The scale of the keys goes to the score, in prompts of bf16 (attend8_wide) to the conversion.
//
// The split of the work is that of the 4-bit cache: a wave takes 16 C columns (a column is one query token's head, the heads
// that share a kv head side by side) and 64 cached tokens at a time, scores transposed (tokens down, columns across), token
// g*16 + t*4 + i of the 64 in row g*4 + i of score tile t, so that lane group g = lane/16 owns 16 consecutive
// tokens, of one block, and holds their probabilities where the product with the values wants them.  Of the values it loads
// four channels of four tokens at once: row n of output block r is channel 64 (r/4) + 4 n + r%4.
//
// Single tokens are bound by the reading of the cache: 80 rows of up to 5,000 tokens, 482 MB, 104 us (4.6 TB/s), with
// 400 such rows 405 us (5.7; a streaming kernel reaches 6.2, a probe that reads scattered cells 5.8), where the
// lengths' unevenness costs less; vector instructions are issued in 18% of the cycles of a busy CU, the matrix
// cores busy in 8%.  One row of 150,001 takes 62 us (4.9 TB/s, 5 of them the join), one of 1,000 9 us, launch and
// latency.  Prompts are bound by the matrix cores and the softmax's vector instructions together: 7,001 tokens of 32
// heads of 128 channels 377 to 390 us by card (1.03 to 1.06 PFLOP/s; a large product reaches 1.2 to 1.4) with the matrix cores busy for 47% of the
// cycles and other vector instructions issued in 33%.  Chunks of 64 channels are bound by vector instructions (a
// score of 64 products costs as much softmax as one of 128, and a code's conversion is used for 32 columns): 7
// chunks of up to 500 over 8,000 52 us (430 TFLOP/s), matrix cores 23%, others 66%.
#include "kv_attend.h"

namespace wfkv {
namespace {

// Eight codes as the operand of a product.
template <class M>
__device__ __forceinline__ u32x4 operand8(uint32_t lo, uint32_t hi, float by) {
  return (u32x4){M::template codes8<0>(lo, by), M::template codes8<1>(lo, by), M::template codes8<0>(hi, by), M::template codes8<1>(hi, by)};
}

// The bytes of tokens at .. at + 3 that are in [lo, hi).
__device__ __forceinline__ uint32_t seen_bytes(int at, int lo, int hi) {
  const int from = min(max(lo - at, 0), 4), left = min(max(hi - at, 0), 4);
  const uint32_t below = left == 4 ? ~0u : (1u << 8 * left) - 1u;
  return from == 4 ? 0u : below & (~0u << 8 * from);
}

// As Pages, for tokens that are the same for a whole wave.
struct UniformPages : Pages {
  using Pages::Pages;
  __device__ __forceinline__ unsigned id(int token) const {
    const auto* at = (const __attribute__((address_space(4))) int32_t*)table;
    return (unsigned)at[(unsigned)min(token, last) >> b_log2];
  }
};

// Waves a SIMD that the registers are held to: the two units in flight of single tokens take 149 (64 channels), 237
// and 490 of them, the one unit and two tiles of chunks 163 and 233.
template <int D>
constexpr int kOcc = D == 64 ? 3 : D == 128 ? 2 : 1;

// Up to this many shares of 16 columns are joined by the workgroup that is done last, more (or of
// more columns) by a kernel of their own, with a workgroup for each head: one token over 1,000 cached ones (4
// shares) takes 8.9 us against 10.2, over 4,000 (16) 15.2 against 11.5; 8 tokens (32 columns) over 1,000 18.6 against 13.4.
template <int C>
constexpr int kFused = C == 1 ? 4 : 1;

template <int D, int C, class M>
__global__ __launch_bounds__(kThreads, (kOcc<D>)) void attend8(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32;          // products of 32 channels per score tile
  constexpr int J = D / 64;           // runs of 64 channels
  constexpr int MT = D / 16;          // blocks of 16 channels of the output
  constexpr int JT = 4;               // channel blocks joined at once: a run of 64 channels
  constexpr int JP = JT * 16 + 4;     // and their padded row
  __shared__ __attribute__((aligned(16))) float join[kWaves][16 * C][JP];
  __shared__ float ref_of[kWaves][16 * C], sum_of[kWaves][16 * C];
  __shared__ int last;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // kv heads fastest (blocks of one head meet in one die's L2 where heads
  // divide the dies), then shares, then column tiles from the last (the longest under a
  // causal mask) to the first, then rows
  unsigned id = blockIdx.x;
  const int kvh = (int)(id % (unsigned)g.hk);
  id /= (unsigned)g.hk;
  const int split = (int)(id % (unsigned)sp.splits);
  id /= (unsigned)sp.splits;
  const int tile0 = sp.tiles - 1 - (int)(id % (unsigned)sp.tiles);
  const int row = (int)(id / (unsigned)sp.tiles);

  const int q0 = min(max(a.q_off[row], 0), a.n_tokens), q1 = min(max(a.q_off[row + 1], q0), a.n_tokens);
  const int64_t columns = (int64_t)(q1 - q0) * g.group;
  const int len = min(max(a.kv_len[row], 0), g.width << g.b_log2);
  const UniformPages rows(g, a, row, kvh, len);
  const float scale = a.scale * kLog2e;

  for (int64_t tile = tile0; tile * 16 * C < columns; tile += sp.tiles) {
    // (opaque, so that what follows from it is worked out here and not kept in registers across tiles)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int n = lane & 15, grp = lane >> 4;
    // this lane's columns: their query, and the tokens [lo, hi) they see
    u32x4 q[C][KS];
    int lo[C], hi[C];
    int lo_min = len, lo_max = 0, hi_min = INT32_MAX, hi_max = 0;
    auto note = [&](const Sight& see) __attribute__((always_inline)) {
      // (what is seen at all: queries that see nothing do not count)
      lo_min = min(lo_min, see.lo < see.hi ? see.lo : len);
      lo_max = max(lo_max, see.lo);
      hi_min = min(hi_min, see.hi);
      hi_max = max(hi_max, see.lo < see.hi ? see.hi : 0);
    };
    // (columns past the last repeat it and are not written)
    const unsigned col0 = (unsigned)(tile * 16 * C), col1 = (unsigned)min(tile * 16 * C + 16 * C, columns) - 1u;
    const unsigned i0 = col0 / (unsigned)g.group, i1 = col1 / (unsigned)g.group;
    unsigned own[C];  // the tokens of this lane's columns
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const unsigned col = min(col0 + c * 16 + n, col1);
      own[c] = col / (unsigned)g.group;
      const unsigned h = col - own[c] * (unsigned)g.group;
      const u32x4* src = reinterpret_cast<const u32x4*>((const uint16_t*)a.q + (int64_t)(q0 + own[c]) * a.q_stride +
                                                        (int64_t)(kvh * g.group + h) * D + grp * 16);
#pragma unroll
      for (int k = 0; k < KS; ++k) q[c][k] = src[k / 2 * 8 + k % 2];
    }
    // Up to two tokens (all columns of single tokens are one): positions by scalar loads, as the blocks below.
    if (i1 - i0 <= 1) {
      const auto* pos = (const __attribute__((address_space(4))) int32_t*)a.pos + q0;
      const Sight see0 = sight_of(pos[i0], len, a.window), see1 = sight_of(pos[i1], len, a.window);
      note(see0);
      note(see1);
#pragma unroll
      for (int c = 0; c < C; ++c) lo[c] = own[c] == i0 ? see0.lo : see1.lo, hi[c] = own[c] == i0 ? see0.hi : see1.hi;
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Sight see = sight_of(a.pos[q0 + own[c]], len, a.window);
        lo[c] = see.lo, hi[c] = see.hi;
        note(see);
      }
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) {
        lo_min = min(lo_min, __shfl_xor(lo_min, off, 64));
        lo_max = max(lo_max, __shfl_xor(lo_max, off, 64));
        hi_min = min(hi_min, __shfl_xor(hi_min, off, 64));
        hi_max = max(hi_max, __shfl_xor(hi_max, off, 64));
      }
      lo_min = __builtin_amdgcn_readfirstlane(lo_min);
      lo_max = __builtin_amdgcn_readfirstlane(lo_max);
      hi_min = __builtin_amdgcn_readfirstlane(hi_min);
      hi_max = __builtin_amdgcn_readfirstlane(hi_max);
    }
    // units of 64 tokens that any column sees, in equal shares of at least a unit a wave
    const int first = lo_min >> 6, units = max(0, ((hi_max + 63) >> 6) - first);
    // (a tile past those the launch knew of is not shared: its count would be another's)
    const int splits = tile < sp.tiles ? sp.splits : 1;
    const int share = units <= kAlone ? kAlone : max(kWaves, (units + splits - 1) / splits);
    const int used = max(1, (units + share - 1) / share);
    if (split >= used) continue;
    const int end = first + min(units, (split + 1) * share);

    f32x4 o[C][MT] = {};
    // (the reference before the first score is below any, and not infinite: hidden scores are)
    float ref[C], sum[C];
#pragma unroll
    for (int c = 0; c < C; ++c) ref[c] = -FLT_MAX, sum[c] = 0.0f;

    const int kgrp = n >> 2;  // the group whose keys this lane loads: row n of a score tile
    // A unit as it is loaded.  Keys: token t*4 + n%4 of group n/4, 16 channels of each run of 64; values: of four
    // tokens, four channels of each run of 64; the scales of the values' block.
    struct Unit {
      u32x4 kw[4][J], vw[J][4];
      f32x2 scales;
    };
    // (units past this share's last are that one again: their bytes are on their way anyway)
    const int u0 = first + split * share + wave, stop = max(end - 1, 0);
    // The blocks of a unit's four groups come by scalar loads: vector loads return in order, a wave's and to
    // a degree a CU's, so an id would arrive behind all the codes that were asked for before it.
    unsigned ids[4];
    auto ask = [&](int u) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 4; ++x) ids[x] = rows.id((min(u, stop) << 6) + x * 16);
    };
    auto id_of = [&](int x) __attribute__((always_inline)) {
      const unsigned lo = x & 1 ? ids[1] : ids[0], hi = x & 1 ? ids[3] : ids[2];
      return x & 2 ? hi : lo;
    };
    auto load_keys = [&](int u, Unit& w) __attribute__((always_inline)) {
      const int off = ((min(u, stop) << 6) + kgrp * 16) & (g.b - 1);
      const uint8_t* at = rows.cell(id_of(kgrp)) + (off + (n & 3)) * D + grp * 16;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) w.kw[t][j] = *reinterpret_cast<const u32x4*>(at + t * 4 * D + j * 64);
    };
    auto load_values = [&](int u, Unit& w) __attribute__((always_inline)) {
      const int off = ((min(u, stop) << 6) + grp * 16) & (g.b - 1);
      const uint8_t* cell = rows.cell(id_of(grp));
      w.scales = *reinterpret_cast<const f32x2*>(cell + 2 * g.b * D);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          w.vw[j][t] = *reinterpret_cast<const u32x4*>(cell + g.b * D + (off + 4 * t) * D + (j * 64 + n * 4) * 4);
    };
    // `more` is called once the keys are multiplied
    auto work = [&](int u, Unit& w, auto more) __attribute__((always_inline)) {
      const int base = u << 6;
      const float kz = w.scales[0] * scale;
      float vz = w.scales[1];
      const bool whole = base >= lo_max && base + 64 <= hi_min;
      // what no query sees may be anything, no number too, which a probability of 0 would not hide
      if (base < lo_min || base + 64 > hi_max) {
        const int j0 = base + grp * 16;
        if (j0 + 16 <= lo_min || j0 >= hi_max) vz = 1.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t mask = seen_bytes(j0 + t * 4, lo_min, hi_max);
#pragma unroll
          for (int j = 0; j < J; ++j) w.vw[j][t] &= mask;
        }
      }
      float vlog = 0.0f, unscale = 1.0f, limit = M::kSlack;
      if constexpr (M::kScaled) vlog = scale_log(vz), unscale = __builtin_amdgcn_exp2f(-vlog), limit = fminf(limit, M::kMostLog - vlog);
      // 32 tokens at a time: score tiles 2h and 2h + 1, one product with the values
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 s[C][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int c = 0; c < C; ++c) s[c][e] = (f32x4){0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const u32x4 kk = operand8<M>(w.kw[2 * h + e][k / 2][k % 2 * 2], w.kw[2 * h + e][k / 2][k % 2 * 2 + 1], 1.0f);
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][e] = M::mma(kk, q[c][k], s[c][e]);
          }
        }
        if (h) more();
        const int j0 = base + grp * 16 + h * 8;
        float most[C];
        bool up = false;
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[c][i / 4][i % 4] *= kz;
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i / 4][i % 4] = j0 + i >= lo[c] && j0 + i < hi[c] ? s[c][i / 4][i % 4] : -INFINITY;
          }
          float m = s[c][0][0];
#pragma unroll
          for (int i = 1; i < 8; ++i) m = fmaxf(m, s[c][i / 4][i % 4]);
          most[c] = m;
          up |= m > ref[c] + limit;
        }
        // the reference moves only when a score (kScaled: or its term) passes it by the limit
        if (__builtin_expect(__any(up), 0)) {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float r = most[c];
            // (values of next to nothing at the largest score: p stays far from fp32's end)
            if constexpr (M::kScaled) r = fmaxf(r - 40.0f, r + vlog - M::kAim);
            r = fmaxf(ref[c], column_max(r));
            const float keep = __builtin_amdgcn_exp2f(ref[c] - r);
            ref[c] = r;
            sum[c] *= keep;
#pragma unroll
            for (int k = 0; k < MT; ++k) o[c][k] *= keep;
          }
        }
        // probabilities (kScaled: times the value scale), in the order of the tokens
        u32x4 p[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float x[8], terms = 0.0f;
          const float by = M::kScaled ? ref[c] - vlog : ref[c];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] = __builtin_amdgcn_exp2f(s[c][i / 4][i % 4] - by);
            if constexpr (M::kScaled) terms = i ? terms + x[i] : x[i];
            else sum[c] += x[i];
          }
          if constexpr (M::kScaled) sum[c] = fmaf(terms, unscale, sum[c]);
#pragma unroll
          for (int b = 0; b < 4; ++b) p[c][b] = M::pair(x[2 * b], x[2 * b + 1]);
        }
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          const u32x4 vv = operand8<M>(w.vw[r / 4][2 * h][r % 4], w.vw[r / 4][2 * h + 1][r % 4], M::kScaled ? 1.0f : vz);
#pragma unroll
          for (int c = 0; c < C; ++c) o[c][r] = M::mma(vv, p[c], o[c][r]);
        }
      }
    };
    int u = u0;
    ask(u);
    if constexpr (C == 1) {
      // the next unit is on its way while one is worked on, its blocks one earlier still (with one unit's
      // registers and its blocks by vector loads 80 ragged rows of up to 5,000 127 us, so 104)
      Unit w0, w1;
      const auto none = [] {};
      load_keys(u, w0);
      load_values(u, w0);
      ask(u + kWaves);
      for (; u + kWaves < end; u += 2 * kWaves) {
        load_keys(u + kWaves, w1);
        load_values(u + kWaves, w1);
        ask(u + 2 * kWaves);
        work(u, w0, none);
        load_keys(u + 2 * kWaves, w0);
        load_values(u + 2 * kWaves, w0);
        ask(u + 3 * kWaves);
        work(u + kWaves, w1, none);
      }
      if (u < end) work(u, w0, none);
    } else {
      // (two units' registers would leave one wave a SIMD) the next keys alone
      Unit w;
      load_keys(u, w);
      for (; u < end; u += kWaves) {
        load_values(u, w);
        ask(u + kWaves);
        work(u, w, [&]() __attribute__((always_inline)) { load_keys(u + kWaves, w); });
      }
    }

    // join the waves
#pragma unroll
    for (int c = 0; c < C; ++c) {
      sum[c] = column_sum(sum[c]);
      if (grp == 0) {
        ref_of[wave][c * 16 + n] = ref[c];
        sum_of[wave][c * 16 + n] = sum[c];
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float m = ref[c];
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ref_of[w][c * 16 + n]);
      const float keep = __builtin_amdgcn_exp2f(ref[c] - m);
#pragma unroll
      for (int k = 0; k < MT; ++k) o[c][k] *= keep;
    }
#pragma unroll
    for (int j0 = 0; j0 < MT; j0 += JT) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)  // row grp*4 + i of block r is channel 4 (grp*4 + i) + r%4 of its run
          *reinterpret_cast<f32x4*>(&join[wave][c * 16 + n][(grp * 4 + i) * 4]) =
              (f32x4){o[c][j0][i], o[c][j0 + 1][i], o[c][j0 + 2][i], o[c][j0 + 3][i]};
      __syncthreads();
      // four channels a thread
      for (int x = threadIdx.x; x < 16 * C * JT * 4; x += kThreads) {
        const int cc = x / (JT * 4), ch = (x % (JT * 4)) * 4;
        const int64_t col = tile * 16 * C + cc;
        if (col >= columns) continue;
        f32x4 v = {0, 0, 0, 0};
        float m = -FLT_MAX, total = 0.0f;
        for (int w = 0; w < kWaves; ++w) {
          v += *reinterpret_cast<const f32x4*>(&join[w][cc][ch]);
          m = fmaxf(m, ref_of[w][cc]);
        }
        for (int w = 0; w < kWaves; ++w) total += sum_of[w][cc] * __builtin_amdgcn_exp2f(ref_of[w][cc] - m);
        const unsigned i = (unsigned)col / (unsigned)g.group, h = (unsigned)col - i * (unsigned)g.group;
        const int64_t head = (int64_t)(q0 + i) * g.hq + kvh * g.group + h;
        const int at = j0 * 16 + ch;
        if (used == 1) {
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
          const u32x2 w = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
          *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + at) = w;
        } else {
          float* to = sp.part + ((int64_t)split * a.n_tokens * g.hq + head) * (D + 2);
          put(to + at, v[0], v[1]);
          put(to + at + 2, v[2], v[3]);
          if (at == 0) put(to + D, m, total);
        }
        if (at == 0 && split == 0 && sp.splits > kFused<C>) sp.used[head] = used;
      }
      __syncthreads();
    }
    if (used > 1 && sp.splits <= kFused<C>)
      join_item<D, M>(g, a, sp, row, tile, kvh, q0, tile * 16 * C, columns, 16 * C, used, &last);
  }
}

// Many columns (prompts): the W waves of a workgroup take different columns, 16 C
// each, and the same tokens, whose codes they turn into operands once, in LDS.
//
// The tokens go by in steps of 32 (half h of a unit: tokens g*16 + h*8 .. +7 of its four
// groups).  Step n's probabilities are taken while the matrix cores multiply those of
// step n - 1 with their values and the queries with the keys of step n + 1.  LDS holds
// four steps of keys and of values; during the two steps of unit u the waves write keys
// 2u + 3 and 2u + 4 and values 2u + 2 and 2u + 3, whose codes they loaded a unit earlier.
// A chunk of operands is read from LDS while the one before it is multiplied.
//
// There is no running maximum: probabilities are taken against a reference that stands
// from the start, the largest score (f16: with the value's scale) among the last tokens that all of a
// wave's columns see.  A softmax does not depend on it as long as nothing overflows or vanishes.  For
// bf16, whose range is that of fp32, the total tells at the end whether it did: then the true maximum is found and
// the workgroup runs once more, so that the loop itself has no branch and touches the sums with
// matrix instructions alone.  f16 has 13 powers of two above the reference, which scales that differ from block
// to block pass often (8,000 tokens with scales of two powers either way: most workgroups), so there the
// loop looks at each step's largest term and moves the reference where it has to.
template <int D, int C, int W, class M>
__global__ __launch_bounds__(64 * W, (D == 256 ? 1 : 2)) void attend8_wide(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32, MT = D / 16;
  constexpr int kFrag = 64;  // 16-byte lanes of an operand
  // Chunks of CH operands, NC of them to a step's values or keys.  With several, the next
  // step's values may not replace the last one's: eight steps of LDS, or where that is too
  // much (VS = 4) a barrier between.
  constexpr int CH = D == 256 ? 8 : D == 128 ? 2 : 4, NC = D / 16 / CH, VS = NC > 1 && D < 256 ? 8 : 4;
  constexpr bool kMid = NC > 1 && VS == 4;
  __shared__ u32x4 kbuf[4][2 * KS][kFrag], vbuf[VS][MT][kFrag];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned id = blockIdx.x;
  const int kvh = (int)(id % (unsigned)g.hk);
  id /= (unsigned)g.hk;
  const int split = (int)(id % (unsigned)sp.splits);
  id /= (unsigned)sp.splits;
  const int tile0 = sp.tiles - 1 - (int)(id % (unsigned)sp.tiles);
  const int row = (int)(id / (unsigned)sp.tiles);

  const int q0 = min(max(a.q_off[row], 0), a.n_tokens), q1 = min(max(a.q_off[row + 1], q0), a.n_tokens);
  const int64_t columns = (int64_t)(q1 - q0) * g.group;
  const int len = min(max(a.kv_len[row], 0), g.width << g.b_log2);
  const Pages pages(g, a, row, kvh, len);
  const float scale = a.scale * kLog2e;
  __shared__ int range[2];

  for (int64_t tile = tile0; tile * 16 * C * W < columns; tile += sp.tiles) {
    // (opaque, so that what follows from it is worked out here and not kept in registers
    // across tiles)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int n = lane & 15, grp = lane >> 4;
    const int64_t col0 = (tile * W + wave) * 16 * C;
    u32x4 q[C][KS];
    int lo[C], hi[C];
    int lo_min = len, lo_max = 0, hi_min = INT32_MAX, hi_max = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const unsigned col = (unsigned)min(col0 + c * 16 + n, columns - 1);
      const unsigned i = col / (unsigned)g.group, h = col - i * (unsigned)g.group;
      const u32x4* src = reinterpret_cast<const u32x4*>((const uint16_t*)a.q + (int64_t)(q0 + i) * a.q_stride +
                                                        (int64_t)(kvh * g.group + h) * D + grp * 16);
#pragma unroll
      for (int k = 0; k < KS; ++k) q[c][k] = src[k / 2 * 8 + k % 2];
      const Sight see = sight_of(a.pos[q0 + i], len, a.window);
      lo[c] = see.lo, hi[c] = see.hi;
      // (what is seen at all: queries that see nothing do not count)
      lo_min = min(lo_min, lo[c] < hi[c] ? lo[c] : len);
      lo_max = max(lo_max, lo[c]);
      hi_min = min(hi_min, hi[c]);
      hi_max = max(hi_max, lo[c] < hi[c] ? hi[c] : 0);
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
      lo_min = min(lo_min, __shfl_xor(lo_min, off, 64));
      lo_max = max(lo_max, __shfl_xor(lo_max, off, 64));
      hi_min = min(hi_min, __shfl_xor(hi_min, off, 64));
      hi_max = max(hi_max, __shfl_xor(hi_max, off, 64));
    }
    lo_min = __builtin_amdgcn_readfirstlane(lo_min);
    lo_max = __builtin_amdgcn_readfirstlane(lo_max);
    hi_min = __builtin_amdgcn_readfirstlane(hi_min);
    hi_max = __builtin_amdgcn_readfirstlane(hi_max);
    // the tokens that any column of the workgroup sees
    if (threadIdx.x == 0) range[0] = len, range[1] = 0;
    __syncthreads();
    if (lane == 0) {
      atomicMin(&range[0], lo_min);
      atomicMax(&range[1], hi_max);
    }
    __syncthreads();
    const int seen_lo = __builtin_amdgcn_readfirstlane(range[0]), seen_hi = __builtin_amdgcn_readfirstlane(range[1]);
    const int first = seen_lo >> 6, units = max(0, ((seen_hi + 63) >> 6) - first);
    const int share = max(kWaves, (units + sp.splits - 1) / sp.splits);
    const int used = max(1, (units + share - 1) / share);
    if (split >= used) {
      __syncthreads();  // range is read by all before it is set again
      continue;
    }
    const int begin = first + split * share, count = min(units - split * share, share);

    // What a wave turns into operands in a unit: of the keys, KP of the KS operands of one
    // score tile of one of two steps; of the values, VP times VC of the 2 MT operands of two
    // steps, VC channels side by side: row n of operand r is channel 16 VC (r / VC) + VC n + r % VC.
    constexpr int KP = KS * 4 / W, KG = KS / KP, VT = 2 * MT / W, VC = VT < 4 ? VT : 4, VP = VT / VC, VJ = MT / VC;
    static_assert(KP >= 1 && KG * KP == KS && KG * 4 == W && VC * VP * W == 2 * MT, "waves divide the operands");
    const int kstep = wave / (2 * KG), ktile = wave / KG % 2, kpart = wave % KG;
    struct Codes {
      u32x2 k[KP];
      uint32_t v[VP][2][VC];
      float ks, vs[VP];  // scales of the keys' and the values' blocks (not kScaled)
      f32x2 z;           // those of this lane's own tokens (kScaled)
    };
    // ... and the blocks they are in, asked for a unit earlier still
    struct Ids {
      unsigned k, v[VP], z;
    };
    auto ask = [&](int kat, int vat, int zat, Ids& d) __attribute__((always_inline)) {
      d.k = pages.id(((begin + ((kat + kstep) >> 1)) << 6) + (n >> 2) * 16);
#pragma unroll
      for (int x = 0; x < VP; ++x) d.v[x] = pages.id(((begin + ((vat + (wave + x * W) / VJ) >> 1)) << 6) + grp * 16);
      if constexpr (M::kScaled) d.z = pages.id(((begin + (zat >> 1)) << 6) + grp * 16);
    };
    auto load_keys = [&](int step, unsigned id, Codes& w) __attribute__((always_inline)) {
      const int s = step + kstep, t = (s & 1) * 2 + ktile;
      const int off = (((begin + (s >> 1)) << 6) + (n >> 2) * 16) & (g.b - 1);
      const uint8_t* cell = pages.cell(id);
      const uint8_t* at = cell + (off + t * 4 + (n & 3)) * D + grp * 16;
      if constexpr (KP == 1) {
        w.k[0] = *reinterpret_cast<const u32x2*>(at + kpart / 2 * 64 + kpart % 2 * 8);
      } else {
#pragma unroll
        for (int k = 0; k < KP / 2; ++k) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(at + (kpart * KP / 2 + k) * 64);
          w.k[2 * k] = (u32x2){x[0], x[1]}, w.k[2 * k + 1] = (u32x2){x[2], x[3]};
        }
      }
      if constexpr (!M::kScaled) w.ks = *reinterpret_cast<const float*>(cell + 2 * g.b * D);
    };
    auto store_keys = [&](int step, const Codes& w) {
      const int s = step + kstep;
#pragma unroll
      for (int k = 0; k < KP; ++k)
        kbuf[s & 3][ktile * KS + kpart * KP + k][lane] = operand8<M>(w.k[k][0], w.k[k][1], M::kScaled ? 1.0f : w.ks);
    };
    auto load_values = [&](int step, const unsigned (&id)[VP], Codes& w) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < VP; ++x) {
        const int job = wave + x * W, s = step + job / VJ, r = job % VJ;
        const int off = ((((begin + (s >> 1)) << 6) + grp * 16) & (g.b - 1)) + (s & 1) * 8;
        const uint8_t* cell = pages.cell(id[x]);
        const uint8_t* at = cell + g.b * D + off * D + (r * 16 + n) * (4 * VC);
#pragma unroll
        for (int t = 0; t < 2; ++t) __builtin_memcpy(w.v[x][t], __builtin_assume_aligned(at + t * 4 * D, 4 * VC), 4 * VC);
        if constexpr (!M::kScaled) w.vs[x] = reinterpret_cast<const float*>(cell + 2 * g.b * D)[1];
      }
    };
    auto store_values = [&](int step, Codes& w) {
#pragma unroll
      for (int x = 0; x < VP; ++x) {
        const int job = wave + x * W, s = step + job / VJ, r = job % VJ;
        // what no query of the workgroup sees may be anything, no number too, which a probability of 0 would not hide
        const int base = (begin + (s >> 1)) << 6, j0 = base + grp * 16;
        if (base < seen_lo || base + 64 > seen_hi) {
          if (j0 + 16 <= seen_lo || j0 >= seen_hi) w.vs[x] = 1.0f;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const uint32_t mask = seen_bytes(j0 + (s & 1) * 8 + t * 4, seen_lo, seen_hi);
#pragma unroll
            for (int c = 0; c < VC; ++c) w.v[x][t][c] &= mask;
          }
        }
#pragma unroll
        for (int c = 0; c < VC; ++c)
          vbuf[s & (VS - 1)][r * VC + c][lane] = operand8<M>(w.v[x][0][c], w.v[x][1][c], M::kScaled ? 1.0f : w.vs[x]);
      }
    };
    // scales of this lane's tokens in the unit of a step
    auto load_scales = [&](unsigned id) __attribute__((always_inline)) -> f32x2 {
      if constexpr (M::kScaled) return *reinterpret_cast<const f32x2*>(pages.cell(id) + 2 * g.b * D);
      return (f32x2){1.0f, 1.0f};
    };
    // ... the keys' times that of the scores, the values' only of what is seen
    auto scales_of = [&](int u, f32x2 z) __attribute__((always_inline)) -> f32x2 {
      const int j0 = ((begin + u) << 6) + grp * 16;
      return (f32x2){z[0] * scale, j0 + 16 <= seen_lo || j0 >= seen_hi ? 1.0f : z[1]};
    };

    f32x4 o[C][MT];
    float ref[C], sum[C];
    u32x4 p[C];
    f32x4 s[C][2];
    // a step's operands: of the values RB of the lower, RB of the upper half of the
    // channels; of the keys KS of each score tile
    u32x4 op[2][CH];
    auto read_values = [&](int step, int part, u32x4 (&to)[CH]) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < CH; ++x) to[x] = vbuf[step & (VS - 1)][part * CH + x][lane];
    };
    auto read_keys = [&](int step, int part, u32x4 (&to)[CH]) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < CH; ++x) to[x] = kbuf[step & 3][part * CH + x][lane];
    };
    auto outputs = [&](int part, const u32x4 (&from)[CH]) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < CH; ++x)
#pragma unroll
        for (int c = 0; c < C; ++c) o[c][part * CH + x] = M::mma(from[x], p[c], o[c][part * CH + x]);
    };
    auto scores = [&](int part, const u32x4 (&from)[CH]) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < CH; ++x) {
        const int e = (part * CH + x) / KS, k = (part * CH + x) % KS;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (k == 0) s[c][e] = (f32x4){0, 0, 0, 0};
          s[c][e] = M::mma(from[x], q[c][k], s[c][e]);
        }
      }
    };
    // the largest score (kScaled: with the scale of its value) of each column among the tokens of units [u0, u1)
    // that it sees, straight from the cache
    auto largest = [&](int u0, int u1, float (&m)[C]) {
#pragma unroll
      for (int c = 0; c < C; ++c) m[c] = -INFINITY;
      for (int u = u0; u < u1; ++u) {
        const int ktoken = (u << 6) + (n >> 2) * 16, ztoken = (u << 6) + grp * 16;
        const unsigned kid = pages.id(ktoken), zid = pages.id(ztoken);
        const uint8_t* kcell = pages.cell(kid);
        const uint8_t* kat = kcell + ((ktoken & (g.b - 1)) + (n & 3)) * D + grp * 16;
        const f32x2 z = *reinterpret_cast<const f32x2*>(pages.cell(zid) + 2 * g.b * D);
        const float kz = z[0] * scale;
        float vl = 0.0f;
        if constexpr (M::kScaled) vl = scale_log(z[1]);
        // (all loads on their way at once)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          f32x4 x[C] = {};
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(kat + t * 4 * D + k / 2 * 64 + k % 2 * 8);
            const u32x4 kk = operand8<M>(w[0], w[1], 1.0f);
#pragma unroll
            for (int c = 0; c < C; ++c) x[c] = M::mma(kk, q[c][k], x[c]);
          }
          const int j0 = ztoken + t * 4;
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) m[c] = fmaxf(m[c], j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] * kz + vl : -INFINITY);
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c) m[c] = column_max(m[c]);
    };

    auto whole = [&](int u) {
      const int base = (begin + u) << 6;
      return base >= lo_max && base + 64 <= hi_min;
    };
   for (int pass = 0;; ++pass) {
    // pass 0 takes the reference from the last unit that all of the wave's columns see
    // whole, or at all, unless they see the first one whole (below); pass 1 from all.  (A window may hide
    // that unit from the wave's last queries: they see the next one.)
    const int near = hi_min >= 64 && ((hi_min >> 6) - 1) << 6 >= lo_max ? (hi_min >> 6) - 1 : max(hi_min - 1, 0) >> 6;
    if (pass) largest(begin, begin + count, ref);
    else largest(near, near + (hi_min == 0 || whole(0) ? 0 : M::kScaled && near << 6 < lo_max && (near + 1) << 6 < hi_max ? 2 : 1), ref);
    // keys of steps 0 to 3, values and scales of steps 0 and 1; all on their way at once
    Codes w, w0, w2;
    Ids d, d0, d2, d3;
    ask(0, 0, 0, d0);
    ask(2, 2, 2, d2);
    ask(3, 4, 4, d3);
    ask(5, 4, 4, d);
    load_keys(0, d0.k, w0);
    load_values(0, d0.v, w0);
    w0.z = load_scales(d0.z);
    load_keys(2, d2.k, w2);
    load_values(2, d2.v, w);
    w.z = load_scales(d2.z);
    load_keys(3, d3.k, w);
    store_keys(0, w0);
    store_values(0, w0);
    f32x2 now = scales_of(0, w0.z);  // of the unit worked on
    store_keys(2, w2);  // step 3's come again in unit 0, the same
    __syncthreads();
#pragma unroll
    for (int part = 0; part < NC; ++part) {
      read_keys(0, part, op[0]);
      scores(part, op[0]);
    }
    if (pass == 0 && whole(0)) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = s[c][i / 4][i % 4] * (M::kScaled ? now[0] : scale);
          ref[c] = fmaxf(ref[c], M::kScaled ? x + scale_log(now[1]) : x);
        }
        ref[c] = column_max(ref[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // (f16, none of those tokens in sight: below any score, so that the first one in sight sets it)
      ref[c] = fabsf(ref[c]) < INFINITY ? ref[c] - M::kAimFixed : M::kScaled ? -FLT_MAX : 0.0f;
      sum[c] = 0.0f, p[c] = (u32x4){0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < MT; ++k) o[c][k] = (f32x4){0, 0, 0, 0};
    }
    // there are no values before step 0's: any finite ones do, the probabilities are 0
    read_values(0, 0, op[0]);
    __syncthreads();  // unit 0 writes step 4's keys over step 0's

    auto unit = [&](int u, auto masked) __attribute__((always_inline)) {
      constexpr bool kMask = decltype(masked)::value;
      // codes loaded a unit ago into LDS, the next ones on their way
      store_keys(2 * u + 3, w);
      if (!kMid) store_values(2 * u + 2, w);
      const f32x2 next = scales_of(u + 1, w.z);
      float vlog = 0.0f, unscale = 1.0f;
      if constexpr (M::kScaled) vlog = scale_log(now[1]), unscale = __builtin_amdgcn_exp2f(-vlog);
      load_keys(2 * u + 5, d.k, w);
      if (!kMid) load_values(2 * u + 4, d.v, w);
      w.z = load_scales(d.z);
      if (!kMid) ask(2 * u + 7, 2 * u + 6, 2 * u + 6, d);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int step = 2 * u + h;
        const int j0 = ((begin + u) << 6) + grp * 16 + h * 8;
        float x[C][8];
        // values of the step before; op[part % 2] holds chunk `part`
#pragma unroll
        for (int part = 0; part < NC; ++part) {
          if (part + 1 < NC) read_values(max(step - 1, 0), part + 1, op[(part + 1) % 2]);
          else read_keys(step + 1, 0, op[(part + 1) % 2]);
          __builtin_amdgcn_sched_barrier(0);
          outputs(part, op[part % 2]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[c][i] = fmaf(s[c][i / 4][i % 4], M::kScaled ? now[0] : scale, M::kScaled ? vlog - ref[c] : -ref[c]);
            if (kMask) x[c][i] = j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] : -INFINITY;
          }
        // f16 ends at 2^16: a term above 2^15 moves the reference
        if constexpr (M::kScaled) {
          bool up = false;
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float m = x[c][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) m = fmaxf(m, x[c][i]);
            up |= m > M::kMostLog;
          }
          if (__builtin_expect(__any(up), 0)) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
              float m = -INFINITY;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                x[c][i] = s[c][i / 4][i % 4] * now[0];
                if (kMask) x[c][i] = j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] : -INFINITY;
                m = fmaxf(m, x[c][i]);
              }
              const float r = fmaxf(ref[c], column_max(m + vlog) - M::kAimFixed), keep = __builtin_amdgcn_exp2f(ref[c] - r);
              ref[c] = r;
              sum[c] *= keep;
#pragma unroll
              for (int k = 0; k < MT; ++k) o[c][k] *= keep;
#pragma unroll
              for (int i = 0; i < 8; ++i) x[c][i] += vlog - r;
            }
          }
        }
        // keys of the step after
#pragma unroll
        for (int part = 0; part < NC; ++part) {
          if (part + 1 < NC) read_keys(step + 1, part + 1, op[(NC + part + 1) % 2]);
          else read_values(step, 0, op[(NC + part + 1) % 2]);
          __builtin_amdgcn_sched_barrier(0);
          scores(part, op[(NC + part) % 2]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float terms = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[c][i] = __builtin_amdgcn_exp2f(x[c][i]);
            if constexpr (M::kScaled) terms = i ? terms + x[c][i] : x[c][i];
            else sum[c] += x[c][i];
          }
          if constexpr (M::kScaled) sum[c] = fmaf(terms, unscale, sum[c]);
#pragma unroll
          for (int b = 0; b < 4; ++b) p[c][b] = M::pair(x[c][2 * b], x[c][2 * b + 1]);
        }
        if (kMid && h == 0) {
          // step 2u read the later chunks of step 2u - 1's values, which 2u + 3's replace
          __syncthreads();
          store_values(2 * u + 2, w);
          load_values(2 * u + 4, d.v, w);
          ask(2 * u + 7, 2 * u + 6, 2 * u + 6, d);
        }
      }
      now = next;
      __syncthreads();
    };
    // (waves may be in different ones of the two loops: each unit has the same barriers in both)
    for (int u = 0; u < count;) {
      while (u < count && !whole(u)) unit(u++, std::true_type());
      while (u < count && whole(u)) unit(u++, std::false_type());
    }
#pragma unroll
    for (int part = 0; part < NC; ++part) {
      if (part) read_values(max(2 * count - 1, 0), part, op[0]);
      outputs(part, op[0]);
    }
    // was the reference near enough?
    bool bad = false;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      sum[c] = column_sum(sum[c]);
      const bool sees = max(lo[c], begin << 6) < min(hi[c], (begin + count) << 6);
      bool fine = sum[c] >= 0x1p-60f && sum[c] <= 0x1p60f;
#pragma unroll
      for (int k = 0; k < MT; ++k) fine &= fabsf(o[c][k][0] + o[c][k][1] + o[c][k][2] + o[c][k][3]) < INFINITY;
      bad |= !M::kScaled && sees && !fine;
    }
    // (also: all have read LDS before the next tile or pass writes it)
    if (!__syncthreads_or(bad) || pass) break;
   }

#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = col0 + c * 16 + n;
      if (col >= columns) continue;
      const unsigned i = (unsigned)col / (unsigned)g.group, h = (unsigned)col - i * (unsigned)g.group;
      const int64_t head = (int64_t)(q0 + i) * g.hq + kvh * g.group + h;
      const float inv = sum[c] == 0.0f ? 0.0f : 1.0f / sum[c];
      float* to = sp.part + ((int64_t)split * a.n_tokens * g.hq + head) * (D + 2);
#pragma unroll
      for (int r = 0; r < MT; r += VC) {
        // rows grp*4 + i of operands r .. r + VC - 1: VC channels from 16 r + VC (grp*4 + i) on
        float v[4 * VC];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < VC; ++x) v[i * VC + x] = o[c][r + x][i];
        const int at = r * 16 + grp * 4 * VC;
#pragma unroll
        for (int x = 0; x < VC; ++x) {
          if (used == 1) {
            const u32x2 b = {M::pair(v[4 * x] * inv, v[4 * x + 1] * inv), M::pair(v[4 * x + 2] * inv, v[4 * x + 3] * inv)};
            *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + at + 4 * x) = b;
          } else {
            *reinterpret_cast<f32x2*>(to + at + 4 * x) = (f32x2){v[4 * x], v[4 * x + 1]};
            *reinterpret_cast<f32x2*>(to + at + 4 * x + 2) = (f32x2){v[4 * x + 2], v[4 * x + 3]};
          }
        }
      }
      if (grp == 0) {
        if (used > 1) to[D] = sum[c] == 0.0f ? -INFINITY : ref[c], to[D + 1] = sum[c];
        if (split == 0 && sp.splits > 1) sp.used[head] = used;
      }
    }
  }
}

// Few columns (1 or 2 tiles of 16 a workgroup); the tokens are split so that all
// workgroups run at once.
template <int D, int C, class M>
hipError_t narrow(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, hipStream_t s) {
  // Of long rows with few columns the shares are the nearest number to what fills the chip, of others the next below: 40 rows of
  // up to 5,000 tokens of 8 kv heads of 128 channels 61 us in two shares against 72, of 30,000 296 and 363; but of 1,500 25 and 22, and 2
  // chunks of 500 over 8,000 33 and 26.
  const int64_t items = (int64_t)a.n_rows * g.hk * ((columns + 16 * C - 1) / (16 * C)), seen = a.window > 0 ? std::min(a.max_kv, a.window) : a.max_kv;
  const int64_t spare = seen >= 2048 && columns <= 128 ? items / 2 : 0;
  const Split sp = split_of<D>(g, a, w, columns, 16 * C, w.n_cu * kOcc<D> + spare, kAlone);
  const hipError_t e = launch(attend8<D, C, M>, g, a, sp, kThreads, s);
  if (e != hipSuccess || sp.splits <= kFused<C>) return e;
  // (heads x 256 threads: shares are only taken of up to kCountBytes / 4 heads)
  hipLaunchKernelGGL((combine<D, kThreads / (D / 4), M>), dim3((unsigned)(a.n_tokens * g.hq)), dim3(kThreads), 0, s, g, a, sp);
  return hipGetLastError();
}

// (256 channels: four waves, a SIMD each, of two tiles of columns: a prompt of 7,001 of 32 heads 900 us, 892 TFLOP/s, against
// 1,328 with one; f16 1,007 against 1,380, though 79 of its registers go to scratch.  Of 128 channels in f16 2 do.)
template <int D, class M>
hipError_t wide(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, hipStream_t s) {
  constexpr int C = 2, W = D == 256 ? 4 : 8, H = kThreads / (D / 4);
  // A CU holds one workgroup of 128 or 256 channels.  The shares of one row are alike and are to run all at once (200 tokens of 32
  // heads of 128 over 16,000 79 us, with twice the shares 113; 400 127 and 195); of several rows, which are not, twice as many
  // even out (8 rows of 100 tokens over up to 5,000 65 us against 83, 4 of 300 94 against 142; several rows of one length,
  // which would be alike too, were not measured).
  const Split sp = split_of<D>(g, a, w, columns, 16 * C * W, w.n_cu * (D > 64 && a.n_rows == 1 ? 1 : 2), kWaves);
  const hipError_t e = launch(attend8_wide<D, C, W, M>, g, a, sp, 64 * W, s);
  if (e != hipSuccess || sp.splits == 1) return e;
  const int64_t heads = (int64_t)a.n_tokens * g.hq;
  hipLaunchKernelGGL((combine<D, 1, M>), dim3((unsigned)((heads + H - 1) / H)), dim3(kThreads), 0, s, g, a, sp);
  return hipGetLastError();
}

template <int D, class M>
hipError_t by_columns(const Geo& g, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  const int64_t columns = (int64_t)(a.max_q > 0 ? std::min(a.max_q, a.n_tokens) : a.n_tokens) * g.group;
  if (columns <= 16) return narrow<D, 1, M>(g, a, w, columns, s);
  // (of 256 channels one tile fits the registers with two units in flight, and two need scratch: 80 rows of 8 tokens over
  // up to 5,000 278 us with one tile against 348, f16 281 against 412.  A code is then converted for 16 columns, for 128 by
  // wide workgroups: 80 rows of 40 columns 265 us narrow and 349 wide, of 64 425 and 405, of 96 442 and 368.)
  constexpr int C = D == 256 ? 1 : 2;
  if (columns <= (D == 256 ? 48 : 128)) return narrow<D, C, M>(g, a, w, columns, s);
  // Narrow workgroups convert the codes for 32 columns, wide ones for 128 or 256, but take 10 us and more to fill
  // their pipeline, and ragged rows leave CUs without one.  (The tokens of the call tell how many columns there are in all.)
  // At 64 channels, where the softmax costs more than the products, wide ones win only where there are several for
  // each CU: a prompt of 7,001 of 32 heads 280 us narrow against 256 wide, of 12 heads 110 against 132, of 2,000 of 32 heads
  // 37 against 45; 7 and 30 chunks of up to 500 over 8,000 of 14 heads (f16) 56 against 62, 171 against 226.
  // At 128 channels, narrow against wide: a prompt of 1,000 of 32 heads 29 and 38, of 2,000 70 and 65, of 4,000 199 and 136; 128
  // tokens over 4,000 29 and 37, 256 over 4,000 43 and 42, over 16,000 102 and 84; 16 prompts of 400 119 and 74.  At 256: 40 tokens of 32 heads over
  // up to 5,000 36 and 55, 8 rows of them 83 and 79; 100 tokens 56 and 68, over 16,000 151 and 137; 300 over 1,000 50 and 42; a
  // prompt of 400 41 and 30, of 1,000 108 and 49.
  const int64_t all = (int64_t)a.n_tokens * g.hq;
  if constexpr (D == 64) {
    if (all < 256 * 3 * w.n_cu) return narrow<D, C, M>(g, a, w, columns, s);
  } else {
    const int64_t at_once = w.n_cu * kOcc<D>, wgs = (all + 31) / 32;
    if (a.max_kv > 0 && wgs * 2 <= at_once * (D == 256 ? 2 : 5) && wgs * a.max_kv <= at_once * 3500) return narrow<D, C, M>(g, a, w, columns, s);
  }
  return wide<D, M>(g, a, w, columns, s);
}

}  // namespace

hipError_t launch_attend8(const Geo& g, int dtype, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  switch (g.d * 2 + dtype) {
    case 128: return by_columns<64, MmaBf16>(g, a, w, s);
    case 129: return by_columns<64, MmaF16>(g, a, w, s);
    case 256: return by_columns<128, MmaBf16>(g, a, w, s);
    case 257: return by_columns<128, MmaF16>(g, a, w, s);
    case 512: return by_columns<256, MmaBf16>(g, a, w, s);
    default: return by_columns<256, MmaF16>(g, a, w, s);
  }
}

}  // namespace wfkv
