// Attention of a step's queries over the paged 4-bit cache.
//
//   o = sum_j p_j v_j,  p = softmax_j(scale q.k_j),  k_j = s_j c_j,  v_j = z_j d_j
//
// with 4-bit codes c, d and one scale s, z a token.  Codes are exact in bf16 and
// f16, so the matrix instructions multiply codes and the scales stay outside:
// the score is (scale s_j) (q.c_j), the output sum_j (p_j z_j) d_j.  p_j z_j is
// rounded to 16 bits once; sums, maxima and exponentials are fp32.
//
// A wave takes 16 C columns -- a column is one query token's head, the heads
// that share a kv head side by side -- and 64 cached tokens at a time.  The scores
// are taken transposed (tokens down, columns across), so that a lane ends up with
// 16 tokens of one column, and those are, in the order chosen below, the very
// operand that the product with the values wants: nothing moves between lanes but
// the running maximum.  Token g*16 + t*4 + i of the 64 is row g*4 + i of score tile
// t, so lane group g = lane/16 owns 16 consecutive tokens: 16 bytes of a row of the
// transposed value codes, 32 of the scales, one block of the cache.
//
// The four waves of a workgroup take every fourth 64 tokens of the same columns and
// join their sums through LDS; with few columns the tokens are also split over
// workgroups, whose partial sums are joined in order, by the last workgroup or a second kernel.
//
// Single tokens are bound by the reading of the cache: 64 f16 rows of up to 24,000 tokens, 1.03 GB,
// 214 us (4.8 TB/s; a streaming kernel reaches 6.2, torch's copy 5.1) with vector instructions issued in
// 55% of the cycles of a busy CU, one row of 200,001 50 us (4.2 TB/s), one of 1,000
// by its launch and latency, 8.4 us.  Prompts are bound by the matrix cores and the vector
// instructions of the softmax together: 8,191 tokens of 32 heads of 128 channels take 553 us, 1.0
// PFLOP/s (a large product reaches 1.2), with the matrix cores busy for 42% of the cycles of a
// busy CU and vector instructions issued in 38%; at 64 channels, where a score costs half the
// product and the same softmax, it is 27% and 50%.
#include "kv_attend.h"

namespace wfkv {
namespace {

// Eight codes as the operand of a product: byte i holds elements 2i and 2i + 1.
template <class M>
__device__ __forceinline__ u32x4 operand(uint32_t w) {
  return (u32x4){M::template codes<0>(w), M::template codes<1>(w), M::template codes<2>(w), M::template codes<3>(w)};
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Waves a SIMD that the registers are held to.
template <int D, int C>
constexpr int kOcc = D * C <= 64 ? 4 : D * C <= 128 ? 3 : D * C <= 256 ? 2 : 1;

// Up to this many shares of 16 columns are joined by the workgroup that is done last, more (or of
// more columns, which it would take one after the other) by a kernel of their own, with a
// workgroup for each head: one token over 1,000 cached ones (4 shares) takes 8.4 us against 9.5, over
// 2,000 (8) 10.8 against 9.5; 24 tokens (48 columns) over 1,000 18.7 against 12.8, over 2,000 26 against 13.
template <int C>
constexpr int kFused = C == 1 ? 4 : 1;

template <int D, int C, class M>
__global__ __launch_bounds__(kThreads, (kOcc<D, C>)) void attend(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32;          // products of 32 channels per score tile
  constexpr int RB = D / 32;          // blocks of 16 rows of value codes
  constexpr int MT = D / 16;          // blocks of 16 channels of the output
  constexpr int KW = D / 32;          // dwords of a lane's key codes of a token
  constexpr int JT = C >= 4 ? 2 : 4;  // channel blocks joined at once
  constexpr int JP = JT * 16 + 4;     // and their padded row
  __shared__ __attribute__((aligned(16))) float join[kWaves][16 * C][JP];
  __shared__ float ref_of[kWaves][16 * C], sum_of[kWaves][16 * C];
  __shared__ int last;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, grp = lane >> 4;
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
  const Pages pages(g, a, row, kvh, len);
  const float scale = a.scale * kLog2e;

  for (int64_t tile = tile0; tile * 16 * C < columns; tile += sp.tiles) {
    // this lane's columns: their query, and the tokens [lo, hi) they see
    u32x4 q[C][KS];
    int lo[C], hi[C];
    int lo_min = INT32_MAX, lo_max = 0, hi_min = INT32_MAX, hi_max = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // columns past the last repeat it and are not written
      const unsigned col = (unsigned)min(tile * 16 * C + c * 16 + n, columns - 1);
      const unsigned i = col / (unsigned)g.group, h = col - i * (unsigned)g.group;
      const u32x4* src = reinterpret_cast<const u32x4*>((const uint16_t*)a.q + (int64_t)(q0 + i) * a.q_stride +
                                                        (int64_t)(kvh * g.group + h) * D + grp * (D / 4));
#pragma unroll
      for (int k = 0; k < KS; ++k) q[c][k] = src[k];
      const Sight see = sight_of(a.pos[q0 + i], len, a.window);
      lo[c] = see.lo, hi[c] = see.hi;
      lo_min = min(lo_min, lo[c]);
      lo_max = max(lo_max, lo[c]);
      hi_min = min(hi_min, hi[c]);
      hi_max = max(hi_max, hi[c]);
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
    // keys of a unit: token t*4 + n%4 of group n/4, this lane's quarter of the channels
    uint32_t kw[4][KW];
    auto load_keys = [&](int u, unsigned id) __attribute__((always_inline)) {
      const int off = ((u << 6) + kgrp * 16) & (g.b - 1);
      const uint8_t* at = pages.cell(id) + (off + (n & 3)) * (D / 2) + grp * (D / 8);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (KW == 2) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(at + t * 4 * (D / 2));
          kw[t][0] = w[0], kw[t][1] = w[1];
        } else {
#pragma unroll
          for (int k = 0; k < KW / 4; ++k) {
            const u32x4 w = reinterpret_cast<const u32x4*>(at + t * 4 * (D / 2))[k];
#pragma unroll
            for (int j = 0; j < 4; ++j) kw[t][4 * k + j] = w[j];
          }
        }
      }
    };

    // a unit's keys are loaded while the one before is worked on, its blocks one earlier still
    const int u0 = first + split * share + wave;
    unsigned kid = pages.id((u0 << 6) + kgrp * 16), vid = pages.id((u0 << 6) + grp * 16);
    load_keys(u0, kid);
    kid = pages.id(((u0 + kWaves) << 6) + kgrp * 16);
    for (int u = u0; u < end; u += kWaves) {
      const int base = u << 6;
      const uint8_t* vcell = pages.cell(vid);
      const int voff = (base + grp * 16) & (g.b - 1);
      vid = pages.id(base + (kWaves << 6) + grp * 16);
      const uint8_t* scales = vcell + g.b * D + voff * 2;
      const u32x4 ks0 = reinterpret_cast<const u32x4*>(scales)[0], ks1 = reinterpret_cast<const u32x4*>(scales)[1];
      const u32x4 vs0 = reinterpret_cast<const u32x4*>(scales + g.b * 2)[0];
      const u32x4 vs1 = reinterpret_cast<const u32x4*>(scales + g.b * 2)[1];
      u32x4 vw[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r)
        vw[r] = *reinterpret_cast<const u32x4*>(vcell + g.b * (D / 2) + (r * 16 + n) * g.b + voff);

      const bool whole = base >= lo_max && base + 64 <= hi_min;
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
            const u32x4 kk = operand<M>(kw[2 * h + e][k]);
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][e] = M::mma(kk, q[c][k], s[c][e]);
          }
        }
        if (h) {
          load_keys(u + kWaves, kid);
          kid = pages.id(base + (2 * kWaves << 6) + kgrp * 16);
        }
        const u32x4 ks = h ? ks1 : ks0, vs = h ? vs1 : vs0;
        float kz[8], vz[8];  // of tokens e*4 + i
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          kz[2 * w] = bf_lo(ks[w]) * scale, kz[2 * w + 1] = bf_hi(ks[w]) * scale;
          vz[2 * w] = bf_lo(vs[w]), vz[2 * w + 1] = bf_hi(vs[w]);
        }
        const int j0 = base + grp * 16 + h * 8;
        float most[C];
        bool up = false;
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[c][i / 4][i % 4] *= kz[i];
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i / 4][i % 4] = j0 + i >= lo[c] && j0 + i < hi[c] ? s[c][i / 4][i % 4] : -INFINITY;
          }
          float m = s[c][0][0];
#pragma unroll
          for (int i = 1; i < 8; ++i) m = fmaxf(m, s[c][i / 4][i % 4]);
          most[c] = m;
          up |= m > ref[c] + M::kSlack;
        }
        // the reference moves only when a score passes it by the slack
        if (__builtin_expect(__any(up), 0)) {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            float r = most[c];
            if constexpr (M::kScaled) {
              r -= 40.0f;  // (values of next to nothing at the largest score: p stays far from fp32's end)
#pragma unroll
              for (int i = 0; i < 8; ++i) r = fmaxf(r, s[c][i / 4][i % 4] + scale_log(vz[i]) - M::kAim);
            }
            r = fmaxf(ref[c], column_max(r));
            const float keep = __builtin_amdgcn_exp2f(ref[c] - r);
            ref[c] = r;
            sum[c] *= keep;
#pragma unroll
            for (int k = 0; k < MT; ++k) o[c][k] *= keep;
          }
        }
        // probabilities times value scales, in the order of the value operand:
        // element 2b + e is token e*4 + b
        u32x4 p[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(s[c][i / 4][i % 4] - ref[c]);
            sum[c] += e;
            x[i] = e * vz[i];
            // a hidden token's scale may be anything
            if (!whole) x[i] = j0 + i >= lo[c] && j0 + i < hi[c] ? x[i] : 0.0f;
          }
          if constexpr (M::kScaled) {  // ... or when a term passes what its type holds
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
            if (__builtin_expect(__any(m > M::kMostTerm), 0)) {
              m = column_max(m);
              const float up = m > M::kMostTerm && m < INFINITY ? __builtin_amdgcn_logf(m) - M::kAim : 0.0f;
              const float keep = __builtin_amdgcn_exp2f(-up);
              ref[c] += up;
              sum[c] *= keep;
#pragma unroll
              for (int k = 0; k < MT; ++k) o[c][k] *= keep;
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] *= keep;
            }
          }
#pragma unroll
          for (int b = 0; b < 4; ++b) p[c][b] = M::pair(x[b], x[4 + b]);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          // bytes of four tokens of score tiles 2h and 2h + 1: low nibbles are
          // channel r*16 + n, high ones that + D/2
          const uint32_t w0 = vw[r][2 * h], w1 = vw[r][2 * h + 1], mask = 0x0f0f0f0fu;
          const u32x4 vlo = operand<M>((w0 & mask) | (w1 << 4 & ~mask));
          const u32x4 vhi = operand<M>((w0 >> 4 & mask) | (w1 & ~mask));
#pragma unroll
          for (int c = 0; c < C; ++c) {
            o[c][r] = M::mma(vlo, p[c], o[c][r]);
            o[c][r + RB] = M::mma(vhi, p[c], o[c][r + RB]);
          }
        }
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
        for (int k = 0; k < JT; ++k)
          *reinterpret_cast<f32x4*>(&join[wave][c * 16 + n][k * 16 + grp * 4]) = o[c][j0 + k];
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
// bf16, whose range is that of fp32, the total tells at the end whether it did; f16 cannot lose
// what matters beside those tokens, and what passes its range makes sums that are not finite.  Where the
// reference was too far off, or those tokens are hidden from a query, the true maximum is found and
// the workgroup runs once more, so that the loop itself has no branch and touches the sums with
// matrix instructions alone.
template <int D, int C, int W, class M>
__global__ __launch_bounds__(64 * W, (D == 256 ? 1 : 2)) void attend_wide(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32, RB = D / 32, MT = D / 16;
  constexpr int kFrag = 64;  // 16-byte lanes of an operand
  // Chunks of CH operands, NC of them to a step's values or keys.  With several, the next
  // step's values may not replace the last one's: eight steps of LDS, or where that is too
  // much (VS = 4) a barrier between.
  constexpr int CH = D == 256 ? 8 : D == 128 ? 2 : 4, NC = D / 16 / CH, VS = NC > 1 && D < 256 ? 8 : 4;
  constexpr bool kMid = NC > 1 && VS == 4;
  __shared__ u32x4 kbuf[4][2 * KS][kFrag], vbuf[VS][2 * RB][kFrag];
  __shared__ __attribute__((aligned(16))) float kzbuf[4][32], vzbuf[4][32];

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
    int lo_min = INT32_MAX, lo_max = 0, hi_min = INT32_MAX, hi_max = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const unsigned col = (unsigned)min(col0 + c * 16 + n, columns - 1);
      const unsigned i = col / (unsigned)g.group, h = col - i * (unsigned)g.group;
      const u32x4* src = reinterpret_cast<const u32x4*>((const uint16_t*)a.q + (int64_t)(q0 + i) * a.q_stride +
                                                        (int64_t)(kvh * g.group + h) * D + grp * (D / 4));
#pragma unroll
      for (int k = 0; k < KS; ++k) q[c][k] = src[k];
      const Sight see = sight_of(a.pos[q0 + i], len, a.window);
      lo[c] = see.lo, hi[c] = see.hi;
      lo_min = min(lo_min, lo[c]);
      lo_max = max(lo_max, lo[c]);
      hi_min = min(hi_min, hi[c]);
      hi_max = max(hi_max, hi[c]);
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
    if (threadIdx.x == 0) range[0] = INT32_MAX, range[1] = 0;
    __syncthreads();
    if (lane == 0) {
      atomicMin(&range[0], lo_min);
      atomicMax(&range[1], hi_max);
    }
    __syncthreads();
    const int first = __builtin_amdgcn_readfirstlane(range[0]) >> 6;
    const int units = max(0, ((__builtin_amdgcn_readfirstlane(range[1]) + 63) >> 6) - first);
    const int share = max(kWaves, (units + sp.splits - 1) / sp.splits);
    const int used = max(1, (units + share - 1) / share);
    if (split >= used) {
      __syncthreads();  // range is read by all before it is set again
      continue;
    }
    const int begin = first + split * share, count = min(units - split * share, share);

    // What a wave turns into operands in a unit: of the keys, KP of the KS operands of one
    // score tile of one of two steps; of the values, VP of the 2 RB row blocks of two
    // steps.
    constexpr int KP = KS * 4 / W, KG = KS / KP, VP = (2 * RB + W - 1) / W;
    static_assert(KP >= 1 && KG * KP == KS && KG * 4 == W, "waves divide the keys' operands");
    const int kstep = wave / (2 * KG), ktile = wave / KG % 2, kpart = wave % KG;
    struct Codes {
      uint32_t k[KP];
      u32x2 v[VP];
      uint32_t z;
    };
    // ... and the blocks they are in, asked for a unit earlier still
    struct Ids {
      unsigned k, v[VP], z;
    };
    auto ask = [&](int kat, int vat, int zat, Ids& d) __attribute__((always_inline)) {
      d.k = pages.id(((begin + ((kat + kstep) >> 1)) << 6) + (n >> 2) * 16);
#pragma unroll
      for (int x = 0; x < VP; ++x) d.v[x] = pages.id(((begin + ((vat + (wave + x * W) / RB) >> 1)) << 6) + grp * 16);
      d.z = pages.id(((begin + (zat >> 1)) << 6) + grp * 16);
    };
    auto load_keys = [&](int step, unsigned id, Codes& w) __attribute__((always_inline)) {
      const int s = step + kstep, t = (s & 1) * 2 + ktile;
      const int off = (((begin + (s >> 1)) << 6) + (n >> 2) * 16) & (g.b - 1);
      const uint8_t* at = pages.cell(id) + (off + t * 4 + (n & 3)) * (D / 2) + grp * (D / 8) + kpart * (KP * 4);
      if constexpr (KP == 1) {
        w.k[0] = *reinterpret_cast<const uint32_t*>(at);
      } else if constexpr (KP == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(at);
        w.k[0] = x[0], w.k[1] = x[1];
      } else {
#pragma unroll
        for (int k = 0; k < KP / 4; ++k) {
          const u32x4 x = reinterpret_cast<const u32x4*>(at)[k];
#pragma unroll
          for (int j = 0; j < 4; ++j) w.k[4 * k + j] = x[j];
        }
      }
    };
    auto store_keys = [&](int step, const Codes& w) {
      const int s = step + kstep;
#pragma unroll
      for (int k = 0; k < KP; ++k) kbuf[s & 3][ktile * KS + kpart * KP + k][lane] = operand<M>(w.k[k]);
    };
    auto load_values = [&](int step, const unsigned (&id)[VP], Codes& w) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < VP; ++x) {
        // (waves beyond the last row block load the same as others, and store nothing)
        const int job = wave + x * W, s = step + job / RB, r = job % RB;
        const int off = (((begin + (s >> 1)) << 6) + grp * 16) & (g.b - 1);
        w.v[x] = *reinterpret_cast<const u32x2*>(pages.cell(id[x]) + g.b * (D / 2) + (r * 16 + n) * g.b + off + (s & 1) * 8);
      }
    };
    auto store_values = [&](int step, const Codes& w) {
#pragma unroll
      for (int x = 0; x < VP; ++x) {
        const int job = wave + x * W, s = step + job / RB, r = job % RB;
        if (job >= 2 * RB) continue;
        const uint32_t w0 = w.v[x][0], w1 = w.v[x][1], mask = 0x0f0f0f0fu;
        vbuf[s & (VS - 1)][r][lane] = operand<M>((w0 & mask) | (w1 << 4 & ~mask));
        vbuf[s & (VS - 1)][r + RB][lane] = operand<M>((w0 >> 4 & mask) | (w1 & ~mask));
      }
    };
    // scales of the two steps of a unit, a token a lane: wave 0 the keys', wave 1 the values'
    auto load_scales = [&](int step, unsigned id) __attribute__((always_inline)) -> uint32_t {
      const int off = (((begin + (step >> 1)) << 6) + lane) & (g.b - 1);
      return reinterpret_cast<const uint16_t*>(pages.cell(id) + g.b * D)[(wave & 1 ? g.b : 0) + off];
    };
    auto store_scales = [&](int step, uint32_t z) {
      if (wave > 1) return;
      // token grp*16 + x of the unit: step x/8, place grp*8 + x%8
      float* to = wave ? &vzbuf[0][0] : &kzbuf[0][0];
      to[((step + (n >> 3)) & 3) * 32 + grp * 8 + (n & 7)] = __uint_as_float(z << 16) * (wave ? 1.0f : scale);
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
        const uint8_t* kat = pages.cell(kid) + ((ktoken & (g.b - 1)) + (n & 3)) * (D / 2) + grp * (D / 8);
        const uint8_t* zat = pages.cell(zid) + g.b * D + (ztoken & (g.b - 1)) * 2;
        // (all loads on their way at once: 256 f16 prompts of 64 tokens 179 -> 161 us)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t* at = reinterpret_cast<const uint32_t*>(kat + t * 4 * (D / 2));
          const u32x2 z = *reinterpret_cast<const u32x2*>(zat + t * 8);
          u32x2 v = {};
          if constexpr (M::kScaled) v = *reinterpret_cast<const u32x2*>(zat + g.b * 2 + t * 8);
          f32x4 x[C] = {};
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const u32x4 kk = operand<M>(at[k]);
#pragma unroll
            for (int c = 0; c < C; ++c) x[c] = M::mma(kk, q[c][k], x[c]);
          }
          const int j0 = ztoken + t * 4;
          const float kz[4] = {bf_lo(z[0]) * scale, bf_hi(z[0]) * scale, bf_lo(z[1]) * scale, bf_hi(z[1]) * scale};
          float vl[4] = {};
          if constexpr (M::kScaled) {
            vl[0] = scale_log(bf_lo(v[0])), vl[1] = scale_log(bf_hi(v[0]));
            vl[2] = scale_log(bf_lo(v[1])), vl[3] = scale_log(bf_hi(v[1]));
          }
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              m[c] = fmaxf(m[c], j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] * kz[i] + vl[i] : -INFINITY);
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
    w0.z = load_scales(0, d0.z);
    load_keys(2, d2.k, w2);
    load_values(2, d2.v, w);
    w.z = load_scales(2, d2.z);
    load_keys(3, d3.k, w);
    store_keys(0, w0);
    store_values(0, w0);
    store_scales(0, w0.z);
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
          const float x = s[c][i / 4][i % 4] * kzbuf[0][grp * 8 + i];
          ref[c] = fmaxf(ref[c], M::kScaled ? x + scale_log(vzbuf[0][grp * 8 + i]) : x);
        }
        ref[c] = column_max(ref[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      ref[c] = fabsf(ref[c]) < INFINITY ? ref[c] - M::kAimFixed : 0.0f;
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
      store_scales(2 * u + 2, w.z);
      load_keys(2 * u + 5, d.k, w);
      if (!kMid) load_values(2 * u + 4, d.v, w);
      w.z = load_scales(2 * u + 4, d.z);
      if (!kMid) ask(2 * u + 7, 2 * u + 6, 2 * u + 6, d);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int step = 2 * u + h;
        float kz[8], vz[8];
        *reinterpret_cast<f32x4*>(kz) = *reinterpret_cast<const f32x4*>(&kzbuf[step & 3][grp * 8]);
        *reinterpret_cast<f32x4*>(kz + 4) = *reinterpret_cast<const f32x4*>(&kzbuf[step & 3][grp * 8 + 4]);
        *reinterpret_cast<f32x4*>(vz) = *reinterpret_cast<const f32x4*>(&vzbuf[step & 3][grp * 8]);
        *reinterpret_cast<f32x4*>(vz + 4) = *reinterpret_cast<const f32x4*>(&vzbuf[step & 3][grp * 8 + 4]);
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
            x[c][i] = fmaf(s[c][i / 4][i % 4], kz[i], -ref[c]);
            if (kMask) x[c][i] = j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] : -INFINITY;
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
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[c][i] = __builtin_amdgcn_exp2f(x[c][i]);
            sum[c] += x[c][i];
            x[c][i] *= vz[i];
            // a hidden token's scale may be anything
            if (kMask) x[c][i] = j0 + i >= lo[c] && j0 + i < hi[c] ? x[c][i] : 0.0f;
          }
#pragma unroll
          for (int b = 0; b < 4; ++b) p[c][b] = M::pair(x[c][b], x[c][4 + b]);
        }
        if (kMid && h == 0) {
          // step 2u read the later chunks of step 2u - 1's values, which 2u + 3's replace
          __syncthreads();
          store_values(2 * u + 2, w);
          load_values(2 * u + 4, d.v, w);
          ask(2 * u + 7, 2 * u + 6, 2 * u + 6, d);
        }
      }
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
      // (kScaled: 0 is the reference of a query that saw none of the tokens it was to come from)
      bool fine = M::kScaled ? ref[c] != 0.0f : sum[c] >= 0x1p-60f && sum[c] <= 0x1p60f;
#pragma unroll
      for (int k = 0; k < MT; ++k) fine &= fabsf(o[c][k][0] + o[c][k][1] + o[c][k][2] + o[c][k][3]) < INFINITY;
      bad |= sees && !fine;
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
      for (int k = 0; k < MT; ++k) {
        // block k of 16 channels, k >= RB: of the upper half
        const int at = k * 16 + grp * 4;
        const f32x4 v = o[c][k];
        if (used == 1) {
          const u32x2 b = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
          *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + at) = b;
        } else {
          *reinterpret_cast<f32x2*>(to + at) = (f32x2){v[0], v[1]};
          *reinterpret_cast<f32x2*>(to + at + 2) = (f32x2){v[2], v[3]};
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
// workgroups run at once.  Shares above that cost more than the balance that they bring (one
// token over 200,001 cached: 53 us at 3 workgroups a CU, 61 at 6, 77 at 12).
template <int D, int C, class M>
hipError_t narrow(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, hipStream_t s) {
  const Split sp = split_of<D>(g, a, w, columns, 16 * C, w.n_cu * kOcc<D, C>, kAlone);
  const hipError_t e = launch(attend<D, C, M>, g, a, sp, kThreads, s);
  if (e != hipSuccess || sp.splits <= kFused<C>) return e;
  // (heads x 256 threads: shares are only taken of up to kCountBytes / 4 heads)
  hipLaunchKernelGGL((combine<D, kThreads / (D / 4), M>), dim3((unsigned)(a.n_tokens * g.hq)), dim3(kThreads), 0, s, g, a, sp);
  return hipGetLastError();
}

template <int D, class M>
hipError_t wide(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, hipStream_t s) {
  constexpr int C = D == 256 ? 1 : 2, W = D == 256 ? 4 : 8, H = kThreads / (D / 4);
  const Split sp = split_of<D>(g, a, w, columns, 16 * C * W, w.n_cu * 2, kWaves);
  const hipError_t e = launch(attend_wide<D, C, W, M>, g, a, sp, 64 * W, s);
  if (e != hipSuccess || sp.splits == 1) return e;
  const int64_t heads = (int64_t)a.n_tokens * g.hq;
  hipLaunchKernelGGL((combine<D, 1, M>), dim3((unsigned)((heads + H - 1) / H)), dim3(kThreads), 0, s, g, a, sp);
  return hipGetLastError();
}

template <int D, class M>
hipError_t by_columns(const Geo& g, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  const int64_t columns = (int64_t)(a.max_q > 0 ? std::min(a.max_q, a.n_tokens) : a.n_tokens) * g.group;
  // 32 rows over up to 6,000 tokens: 49 us narrow against 178 wide for 5 tokens each (20
  // columns), 133 against 190 for 32 (128 columns); one such row 20 against 36
  if (columns <= 16) return narrow<D, 1, M>(g, a, w, columns, s);
  // More columns too where narrow workgroups run all at once and their tokens are not many: a wide one's
  // pipeline and LDS take 10 us and more to fill.  32 heads of 128 channels, narrow against wide:
  // a prompt of 256 9.0 and 21 us, of 400 12 and 27, 128 tokens over 4,000 28 and 40, 256 over 4,000
  // 44 and 46, over 16,000 109 and 92; 16 prompts of 400 (more than at once) 52 and 43.
  const int64_t at_once = w.n_cu * kOcc<D, 2>, narrow_wgs = (int64_t)a.n_rows * g.hk * ((columns + 31) / 32);
  const bool few = a.max_kv > 0 && narrow_wgs <= at_once && narrow_wgs * a.max_kv <= at_once * 3500;
  if (columns <= 128 || few) return narrow<D, 2, M>(g, a, w, columns, s);
  return wide<D, M>(g, a, w, columns, s);
}

}  // namespace

hipError_t launch_attend(const Geo& g, int dtype, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
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
