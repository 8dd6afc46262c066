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
// workgroups, whose partial sums a second kernel joins in order.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896341f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// What depends on the 16-bit type: the product, the codes as its operand, a pair of
// rounded values, and how far a score may pass the running maximum (in powers of
// two) before the sums are rescaled: p z must stay below the type's largest
// value, z of f16 values is at most 10,917.
struct MmaBf16 : Bf16 {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static constexpr float kSlack = 8.0f;
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  template <int I>
  static __device__ __forceinline__ uint32_t codes(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, I));
  }
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
  }
};
struct MmaF16 : F16 {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static constexpr float kSlack = 2.0f;
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  template <int I>
  static __device__ __forceinline__ uint32_t codes(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, I));
  }
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
  }
};

// Eight codes as the operand of a product: byte i holds elements 2i and 2i + 1.
template <class M>
__device__ __forceinline__ u32x4 operand(uint32_t w) {
  return (u32x4){M::template codes<0>(w), M::template codes<1>(w), M::template codes<2>(w), M::template codes<3>(w)};
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Over the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// Waves a SIMD that the registers are held to.
template <int D, int C>
constexpr int kOcc = D * C <= 64 ? 4 : D * C <= 128 ? 3 : D * C <= 256 ? 2 : 1;

struct Split {
  int tiles, splits;  // of the launch: column tiles of a row, shares of its tokens
  float* part;        // [splits][n_tokens][hq][D + 2] sums, maximum, total
  int32_t* used;      // [n_tokens][hq] shares written; 1: the output is done
};

template <int D, int C, class M>
__global__ __launch_bounds__(kThreads, (kOcc<D, C>)) void attend(Geo g, AttendArgs a, Split sp) {
  constexpr int KS = D / 32;          // products of 32 channels per score tile
  constexpr int RB = D / 32;          // blocks of 16 rows of value codes
  constexpr int MT = D / 16;          // blocks of 16 channels of the output
  constexpr int KW = D / 32;          // dwords of a lane's key codes of a token
  constexpr int JT = C >= 4 ? 2 : 4;  // channel blocks joined at once
  constexpr int JP = JT * 16 + 4;     // and their padded row
  __shared__ __attribute__((aligned(16))) float join[kWaves][16 * C][JP];
  __shared__ float top_of[kWaves][16 * C], sum_of[kWaves][16 * C];

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
  const int32_t* table = a.table + (int64_t)row * g.width;
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
      const int p = a.pos[q0 + i];
      hi[c] = p < 0 ? 0 : min(len, p < INT32_MAX ? p + 1 : p);
      lo[c] = a.window && p >= a.window ? p - a.window + 1 : 0;
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
    const int share = max(kWaves, (units + sp.splits - 1) / sp.splits);
    const int used = max(1, (units + share - 1) / share);
    if (split >= used) continue;
    const int end = first + min(units, (split + 1) * share);

    f32x4 o[C][MT] = {};
    float top[C], ref[C], sum[C];
#pragma unroll
    for (int c = 0; c < C; ++c) top[c] = -INFINITY, ref[c] = 0.0f, sum[c] = 0.0f;

    // cell and offset of a group's 16 tokens
    auto cell_at = [&](int token, int& off) {
      off = token & (g.b - 1);
      const unsigned id = token < len ? (unsigned)table[token >> g.b_log2] : 0u;
      return a.cache + ((int64_t)min(id, (unsigned)g.n_blocks - 1u) * g.hk + kvh) * (int64_t)g.cell;
    };
    const int kgrp = n >> 2;  // the group whose keys this lane loads: row n of a score tile

    for (int u = first + split * share + wave; u < end; u += kWaves) {
      const int base = u << 6;
      int koff, voff;
      const uint8_t* kcell = cell_at(base + kgrp * 16, koff);
      const uint8_t* vcell = cell_at(base + grp * 16, voff);
      // keys: token t*4 + n%4 of group n/4, this lane's quarter of the channels
      uint32_t kw[4][KW];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint8_t* at = kcell + (koff + t * 4 + (n & 3)) * (D / 2) + grp * (D / 8);
        if constexpr (KW == 2) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(at);
          kw[t][0] = w[0], kw[t][1] = w[1];
        } else {
#pragma unroll
          for (int k = 0; k < KW / 4; ++k) {
            const u32x4 w = reinterpret_cast<const u32x4*>(at)[k];
#pragma unroll
            for (int j = 0; j < 4; ++j) kw[t][4 * k + j] = w[j];
          }
        }
      }
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
          up |= m > top[c] + M::kSlack;
        }
        // the running maximum moves only when a score passes it by the slack
        if (__any(up)) {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const float m = fmaxf(top[c], column_max(most[c]));
            const float r = m == -INFINITY ? 0.0f : m;
            const float keep = __builtin_amdgcn_exp2f(top[c] - r);
            top[c] = m;
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
        top_of[wave][c * 16 + n] = top[c];
        sum_of[wave][c * 16 + n] = sum[c];
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float m = -INFINITY;
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, top_of[w][c * 16 + n]);
      const float keep = __builtin_amdgcn_exp2f(top[c] - (m == -INFINITY ? 0.0f : m));
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
        float m = -INFINITY, total = 0.0f;
        for (int w = 0; w < kWaves; ++w) {
          v += *reinterpret_cast<const f32x4*>(&join[w][cc][ch]);
          m = fmaxf(m, top_of[w][cc]);
        }
        const float r = m == -INFINITY ? 0.0f : m;
        for (int w = 0; w < kWaves; ++w) total += sum_of[w][cc] * __builtin_amdgcn_exp2f(top_of[w][cc] - r);
        const unsigned i = (unsigned)col / (unsigned)g.group, h = (unsigned)col - i * (unsigned)g.group;
        const int64_t head = (int64_t)(q0 + i) * g.hq + kvh * g.group + h;
        const int at = j0 * 16 + ch;
        if (used == 1) {
          const float inv = total == 0.0f ? 0.0f : 1.0f / total;
          const u32x2 w = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
          *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + at) = w;
        } else {
          float* to = sp.part + ((int64_t)split * a.n_tokens * g.hq + head) * (D + 2);
          *reinterpret_cast<f32x2*>(to + at) = (f32x2){v[0], v[1]};
          *reinterpret_cast<f32x2*>(to + at + 2) = (f32x2){v[2], v[3]};
          if (at == 0) to[D] = m, to[D + 1] = total;
        }
        if (at == 0 && split == 0 && sp.splits > 1) sp.used[head] = used;
      }
      __syncthreads();
    }
  }
}

// The shares of one query's head, joined in a fixed order: four channels a thread,
// every kParts-th share a group of threads, then the groups.
template <int D, class M>
__global__ __launch_bounds__(kThreads) void combine(Geo g, AttendArgs a, Split sp) {
  constexpr int kParts = kThreads / (D / 4);
  __shared__ float tops[kWaves], totals[kParts];
  __shared__ __attribute__((aligned(16))) f32x4 sums[kParts][D / 4];
  const int64_t head = blockIdx.x, heads = (int64_t)a.n_tokens * g.hq;
  const int64_t t = head / g.hq;
  if (t < a.q_off[0] || t >= a.q_off[a.n_rows]) return;
  const int used = sp.used[head];
  if (used <= 1) return;
  const int ch = threadIdx.x % (D / 4), part = threadIdx.x / (D / 4);
  const float* from = sp.part + head * (D + 2);
  const int64_t step = heads * (D + 2);
  float m = -INFINITY;
  for (int s = threadIdx.x; s < used; s += kThreads) m = fmaxf(m, from[s * step + D]);
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, tops[w]);
  const float r = m == -INFINITY ? 0.0f : m;
  float total = 0.0f;
  f32x4 v = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = part; s < used; s += kParts) {
    const float* at = from + s * step;
    const float keep = __builtin_amdgcn_exp2f(at[D] - r);
    total += at[D + 1] * keep;
    const f32x2 v0 = *reinterpret_cast<const f32x2*>(at + 4 * ch), v1 = *reinterpret_cast<const f32x2*>(at + 4 * ch + 2);
    v[0] += v0[0] * keep, v[1] += v0[1] * keep, v[2] += v1[0] * keep, v[3] += v1[1] * keep;
  }
  sums[part][ch] = v;
  if (ch == 0) totals[part] = total;
  __syncthreads();
  if (part) return;
  for (int k = 1; k < kParts; ++k) v += sums[k][ch], total += totals[k];
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const u32x2 w = {M::pair(v[0] * inv, v[1] * inv), M::pair(v[2] * inv, v[3] * inv)};
  *reinterpret_cast<u32x2*>((uint16_t*)a.out + head * D + 4 * ch) = w;
}

template <int D, int C, class M>
hipError_t go(const Geo& g, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  const int max_q = a.max_q > 0 ? std::min(a.max_q, a.n_tokens) : a.n_tokens;
  const int64_t most_kv = (int64_t)g.width * g.b;
  const int64_t max_kv = a.max_kv > 0 ? std::min((int64_t)a.max_kv, most_kv) : most_kv;
  Split sp;
  sp.tiles = (int)(((int64_t)max_q * g.group + 16 * C - 1) / (16 * C));
  const int64_t items = (int64_t)a.n_rows * g.hk * sp.tiles;
  const int64_t units = (max_kv + 63) / 64;
  // enough workgroups to fill the chip several times, shares of at least a unit a
  // wave, partial sums that fit the work area
  const int64_t heads = (int64_t)a.n_tokens * g.hq;
  int64_t splits = std::min({(int64_t)w.n_cu * 6 / items, (units + kWaves - 1) / kWaves,
                             (int64_t)(w.part_bytes / (heads * (D + 2) * 4)), (int64_t)(w.used_bytes / 4 / heads ? 1 << 20 : 1)});
  sp.splits = (int)std::max<int64_t>(1, splits);
  sp.part = w.part;
  sp.used = w.used;
  const int64_t grid = items * sp.splits;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((attend<D, C, M>), dim3((unsigned)grid), dim3(kThreads), 0, s, g, a, sp);
  if (sp.splits > 1) {
    hipLaunchKernelGGL((combine<D, M>), dim3((unsigned)heads), dim3(kThreads), 0, s, g, a, sp);
  }
  return hipGetLastError();
}

template <int D, class M>
hipError_t by_columns(const Geo& g, const AttendArgs& a, const AttendWork& w, hipStream_t s) {
  const int64_t columns = (int64_t)(a.max_q > 0 ? std::min(a.max_q, a.n_tokens) : a.n_tokens) * g.group;
  if (columns <= 16) return go<D, 1, M>(g, a, w, s);
  if (columns <= 32 || D == 256) return go<D, 2, M>(g, a, w, s);
  if constexpr (D < 256) return go<D, 4, M>(g, a, w, s);
  return hipErrorInvalidValue;
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
