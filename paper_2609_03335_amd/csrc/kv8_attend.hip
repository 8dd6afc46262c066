// Attention of a step's queries over the paged 8-bit cache.
//
//   o = sum_j p_j v_j,  p = softmax_j(scale q.k_j),  k_j = 2^e c_j,  v_j = 2^f d_j
//
// with codes c, d of 8 bits and one e and f for a block.  Codes are exact in bf16 and f16, and
// so are bf16 values: the conversion of the values' codes multiplies with their scale.  f16 could not hold them:
// there the scale goes to the probabilities.  Keys are multiplied as codes, their scale goes to the score.
//
// The split of the work is that of the 4-bit cache: a wave takes 16 C columns (a column is one query token's head, the heads
// that share a kv head side by side) and 64 cached tokens at a time, scores transposed (tokens down, columns across), token
// g*16 + t*4 + i of the 64 in row g*4 + i of score tile t, so that lane group g = lane/16 owns 16 consecutive
// tokens, of one block, and holds their probabilities where the product with the values wants them.  Of the values it loads
// four channels of four tokens at once: row n of output block r is channel 64 (r/4) + 4 n + r%4.
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

// Waves a SIMD that the registers are held to.
template <int D, int C>
constexpr int kOcc = D * C <= 64 ? 4 : D * C <= 128 ? 3 : D * C <= 256 ? 2 : 1;

// Up to this many shares of 16 columns are joined by the workgroup that is done last, more (or of
// more columns) by a kernel of their own, with a workgroup for each head.
template <int C>
constexpr int kFused = C == 1 ? 4 : 1;

template <int D, int C, class M>
__global__ __launch_bounds__(kThreads, (kOcc<D, C>)) void attend8(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32;          // products of 32 channels per score tile
  constexpr int J = D / 64;           // runs of 64 channels
  constexpr int MT = D / 16;          // blocks of 16 channels of the output
  constexpr int JT = 4;               // channel blocks joined at once: a run of 64 channels
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
    int lo_min = len, lo_max = 0, hi_min = INT32_MAX, hi_max = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // columns past the last repeat it and are not written
      const unsigned col = (unsigned)min(tile * 16 * C + c * 16 + n, columns - 1);
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
    // keys of a unit: token t*4 + n%4 of group n/4, 16 channels of each run of 64
    u32x4 kw[4][J];
    auto load_keys = [&](int u, unsigned id) __attribute__((always_inline)) {
      const int off = ((u << 6) + kgrp * 16) & (g.b - 1);
      const uint8_t* at = pages.cell(id) + (off + (n & 3)) * D + grp * 16;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) kw[t][j] = *reinterpret_cast<const u32x4*>(at + t * 4 * D + j * 64);
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
      const f32x2 scales = *reinterpret_cast<const f32x2*>(vcell + 2 * g.b * D);
      const float kz = scales[0] * scale;
      float vz = scales[1];
      // values: of four tokens, four channels of each run of 64
      u32x4 vw[J][4];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          vw[j][t] = *reinterpret_cast<const u32x4*>(vcell + g.b * D + (voff + 4 * t) * D + (j * 64 + n * 4) * 4);

      const bool whole = base >= lo_max && base + 64 <= hi_min;
      // what no query sees may be anything, no number too, which a probability of 0 would not hide
      if (base < lo_min || base + 64 > hi_max) {
        const int j0 = base + grp * 16;
        if (j0 + 16 <= lo_min || j0 >= hi_max) vz = 1.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t mask = seen_bytes(j0 + t * 4, lo_min, hi_max);
#pragma unroll
          for (int j = 0; j < J; ++j) vw[j][t] &= mask;
        }
      }
      float vlog = 0.0f;
      if constexpr (M::kScaled) vlog = scale_log(vz) - M::kAim;
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
            const u32x4 kk = operand8<M>(kw[2 * h + e][k / 2][k % 2 * 2], kw[2 * h + e][k / 2][k % 2 * 2 + 1], 1.0f);
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][e] = M::mma(kk, q[c][k], s[c][e]);
          }
        }
        if (h) {
          load_keys(u + kWaves, kid);
          kid = pages.id(base + (2 * kWaves << 6) + kgrp * 16);
        }
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
              for (int i = 0; i < 8; ++i) r = fmaxf(r, s[c][i / 4][i % 4] + vlog);
            }
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
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(s[c][i / 4][i % 4] - ref[c]);
            sum[c] += e;
            x[i] = M::kScaled ? e * vz : e;
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
          for (int b = 0; b < 4; ++b) p[c][b] = M::pair(x[2 * b], x[2 * b + 1]);
        }
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          const u32x4 vv = operand8<M>(vw[r / 4][2 * h][r % 4], vw[r / 4][2 * h + 1][r % 4], M::kScaled ? 1.0f : vz);
#pragma unroll
          for (int c = 0; c < C; ++c) o[c][r] = M::mma(vv, p[c], o[c][r]);
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

// Few columns (1 or 2 tiles of 16 a workgroup); the tokens are split so that all
// workgroups run at once.
template <int D, int C, class M>
hipError_t narrow(const Geo& g, const AttendArgs& a, const AttendWork& w, int64_t columns, hipStream_t s) {
  const Split sp = split_of<D>(g, a, w, columns, 16 * C, w.n_cu * kOcc<D, C>, kAlone);
  const hipError_t e = launch(attend8<D, C, M>, g, a, sp, kThreads, s);
  if (e != hipSuccess || sp.splits <= kFused<C>) return e;
  // (heads x 256 threads: shares are only taken of up to kCountBytes / 4 heads)
  hipLaunchKernelGGL((combine<D, kThreads / (D / 4), M>), dim3((unsigned)(a.n_tokens * g.hq)), dim3(kThreads), 0, s, g, a, sp);
  return hipGetLastError();
}

template <int D, class M>
hipError_t by_columns(const Geo& g, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  const int64_t columns = (int64_t)(a.max_q > 0 ? std::min(a.max_q, a.n_tokens) : a.n_tokens) * g.group;
  if (columns <= 16) return narrow<D, 1, M>(g, a, w, columns, s);
  return narrow<D, 2, M>(g, a, w, columns, s);
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
