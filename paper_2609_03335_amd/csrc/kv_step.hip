// Block tables and slots of one step from the rows' lengths: an inclusive sum
// of the rows' needs decides who is granted and where in the ring of free
// blocks each row takes or gives back its blocks; an exclusive sum of the new
// tokens places the rows' tokens.  One workgroup; integer arithmetic only.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Inclusive sum over the workgroup; *total gets the sum of all threads.
__device__ int64_t block_sum(int64_t x, int64_t* total, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  __syncthreads();
  *total = all;
  return before + x;
}

__global__ __launch_bounds__(kThreads) void step(Geo g, StepArgs a) {
  __shared__ int64_t part[kWaves];
  const unsigned n = (unsigned)g.n_blocks;
  const unsigned head = (unsigned)a.pool_in[0] % n;
  const int64_t room = min(max(a.pool_in[1], 0), g.n_blocks);
  const int64_t most = (int64_t)g.width * g.b;
  const int lane = threadIdx.x & 63;
  int64_t need_base = 0, token_base = 0, back_base = 0, got = 0;
  for (int base = 0; base < a.n_rows; base += kThreads) {
    const int r = base + (int)threadIdx.x;
    const bool in = r < a.n_rows;
    const int64_t fresh = in ? a.fresh[r] : 0;
    const int64_t len = in ? min(max((int64_t)a.len_in[r], (int64_t)0), most) : 0;
    const bool ended = fresh < 0;
    const int64_t grow = ended ? 0 : fresh;
    const int64_t have = (len + g.b - 1) >> g.b_log2;
    const bool fits = len + grow <= most;
    const int64_t need = fits && !ended ? ((len + grow + g.b - 1) >> g.b_log2) - have : 0;
    int64_t need_all, token_all, back_all;
    const int64_t upto = need_base + block_sum(need, &need_all, part);
    const int64_t token = token_base + block_sum(grow, &token_all, part) - grow;
    const int64_t back = ended ? have : 0;
    const int64_t give = back_base + block_sum(back, &back_all, part) - back;
    const bool ok = in && !ended && fits && (need == 0 || upto <= room);
    if (in) {
      a.granted[r] = ok;
      a.len_out[r] = (int32_t)(ended ? 0 : ok ? len + grow : len);
      a.q_off[r] = (int32_t)min(token, (int64_t)INT32_MAX);
    }
    if (ok && need) got = max(got, upto);
    // each row's blocks, by the whole wave
    uint64_t todo = __ballot(in && ((ok && need) || back));
    while (todo) {
      const int src = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      const int64_t row = base + (int)(threadIdx.x & ~63u) + src;
      const int64_t h = __shfl(have, src, 64), m = __shfl(need, src, 64), u = __shfl(upto, src, 64);
      const int64_t b = __shfl(back, src, 64), to = __shfl(give, src, 64);
      int32_t* mine = a.table + row * g.width;
      for (int64_t i = lane; i < m; i += 64)
        mine[h + i] = a.ring[(head + (uint64_t)(u - m + i)) % n];
      for (int64_t i = lane; i < b; i += 64)
        a.ring[(head + (uint64_t)(room + to + i)) % n] = mine[i];
    }
    need_base += need_all;
    token_base += token_all;
    back_base += back_all;
  }
  // the sum of the granted needs is the largest prefix among them
  for (int off = 32; off > 0; off >>= 1) got = max(got, (int64_t)__shfl_xor(got, off, 64));
  __syncthreads();
  if (lane == 0) part[threadIdx.x >> 6] = got;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) got = max(got, part[w]);
  const int64_t tokens = min(token_base, (int64_t)INT32_MAX);
  if (threadIdx.x == 0) {
    a.q_off[a.n_rows] = (int32_t)tokens;
    a.pool_out[0] = (int32_t)((head + (uint64_t)got) % n);
    a.pool_out[1] = (int32_t)(room - got + back_base);
  }
  __threadfence_block();
  __syncthreads();
  for (int t = threadIdx.x; t < a.n_tokens; t += kThreads) {
    int64_t slot = -1;
    int pos = 0;
    if (t < tokens) {
      int lo = 0, hi = a.n_rows;  // the last row that starts at or before t
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_off[mid] <= t) lo = mid; else hi = mid;
      }
      const int64_t p = min(max((int64_t)a.len_in[lo], (int64_t)0), most) + t - a.q_off[lo];
      pos = (int)p;
      if (a.granted[lo])
        slot = (int64_t)a.table[(int64_t)lo * g.width + (p >> g.b_log2)] * g.b + (p & (g.b - 1));
    }
    a.slot[t] = slot;
    a.pos[t] = pos;
  }
}

}  // namespace

hipError_t launch_step(const Geo& g, const StepArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(step, dim3(1), dim3(kThreads), 0, s, g, a);
  return hipGetLastError();
}

}  // namespace wfkv
