// Attention of a step's queries over the paged 4-bit cache.
//
// A wave takes one query: 64 cached tokens at a time, one a lane, with the
// running maximum and sum of a softmax; then each lane sums its channels of the
// values over the 64 tokens.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float code_value(uint32_t c) {
  const uint32_t e = (c >> 1) & 3u, m = c & 1u;
  const uint32_t bits = e ? (126u + e) << 23 | m << 22 : m ? 0x3f000000u : 0u;
  return __uint_as_float(bits | (c & 8u) << 28);
}

template <int D, class T>
__global__ __launch_bounds__(kThreads) void attend(Geo g, AttendArgs a) {
  __shared__ float qs[kThreads / 64][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + wave;
  const int64_t t = item / g.hq;
  const int h = (int)(item - t * g.hq), kvh = h / g.group;
  int row = -1;
  if (t < a.n_tokens && t >= a.q_off[0] && t < a.q_off[a.n_rows]) {
    int lo = 0, hi = a.n_rows;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.q_off[mid] <= t) lo = mid; else hi = mid;
    }
    row = lo;
  }
  if (row >= 0)
    for (int c = lane; c < D; c += 64)
      qs[wave][c] = T::to(((const uint16_t*)a.q)[t * a.q_stride + (int64_t)h * D + c]) * a.scale;
  __syncthreads();
  if (row < 0) return;
  const int64_t most = (int64_t)g.width * g.b;
  const int len = (int)min(max((int64_t)a.kv_len[row], (int64_t)0), most);
  const int64_t p = a.pos[t];
  const int end = (int)min((int64_t)len, p + 1);
  const int begin = a.window ? (int)max((int64_t)0, p - a.window + 1) : 0;
  float m = -INFINITY, sum = 0.0f, o[D / 64] = {};
  for (int base = begin & ~63; base < end; base += 64) {
    const int j = base + lane;
    const bool see = j >= begin && j < end;
    float s = -INFINITY, vs = 0.0f;
    const uint8_t* cell = nullptr;
    if (see) {
      const unsigned id = (unsigned)a.table[(int64_t)row * g.width + (j >> g.b_log2)];
      const int64_t block = min(id, (unsigned)g.n_blocks - 1);
      cell = a.cache + (block * g.hk + kvh) * (int64_t)g.cell;
      const int off = j & (g.b - 1);
      const uint32_t* codes = reinterpret_cast<const uint32_t*>(cell + off * (D / 2));
      float dot = 0.0f;
      for (int w = 0; w < D / 8; ++w) {
        const uint32_t u = codes[w];
        for (int i = 0; i < 8; ++i) dot += qs[wave][w * 8 + i] * code_value((u >> (4 * i)) & 15u);
      }
      const uint16_t* scales = reinterpret_cast<const uint16_t*>(cell + g.b * D);
      s = dot * Bf16::to(scales[off]);
      vs = Bf16::to(scales[g.b + off]);
    }
    float top = s;
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    top = fmaxf(top, m);
    const float ref = top == -INFINITY ? 0.0f : top;
    const float keep = expf(m - ref), e = see ? expf(s - ref) : 0.0f;
    m = top;
    float all = e;
    for (int off = 32; off > 0; off >>= 1) all += __shfl_xor(all, off, 64);
    sum = sum * keep + all;
    for (int i = 0; i < D / 64; ++i) o[i] *= keep;
    const float pv = see ? e * vs : 0.0f;
    for (int k = 0; k < 64; ++k) {
      const int jj = base + k;
      if (jj < begin || jj >= end) continue;
      const unsigned long long at = __shfl((unsigned long long)(uintptr_t)cell, k, 64);
      const uint8_t* values = reinterpret_cast<const uint8_t*>((uintptr_t)at) + g.b * (D / 2);
      const float w = __shfl(pv, k, 64);
      for (int i = 0; i < D / 64; ++i) {
        const int c = i * 64 + lane, r = c & (D / 2 - 1);
        const uint32_t byte = values[(int64_t)r * g.b + (jj & (g.b - 1))];
        o[i] += w * code_value(c < D / 2 ? byte & 15u : byte >> 4);
      }
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  for (int i = 0; i < D / 64; ++i)
    ((uint16_t*)a.out)[(t * g.hq + h) * D + i * 64 + lane] = (uint16_t)T::from(o[i] * inv);
}

template <int D, class T>
hipError_t go(const Geo& g, const AttendArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.n_tokens * g.hq;
  hipLaunchKernelGGL((attend<D, T>), dim3((unsigned)((items + 3) / 4)), dim3(kThreads), 0, s, g, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const Geo& g, int dtype, const AttendArgs& a, hipStream_t s) {
  switch (g.d * 2 + dtype) {
    case 128: return go<64, Bf16>(g, a, s);
    case 129: return go<64, F16>(g, a, s);
    case 256: return go<128, Bf16>(g, a, s);
    case 257: return go<128, F16>(g, a, s);
    case 512: return go<256, Bf16>(g, a, s);
    default: return go<256, F16>(g, a, s);
  }
}

}  // namespace wfkv
