// Block tables and slots of one step from the rows' lengths: an inclusive sum
// of the rows' needs decides who is granted and where in the ring of free
// blocks each row takes or gives back its blocks; an exclusive sum of the new
// tokens places the rows' tokens.  Integer arithmetic only; bound by the latency
// of a launch and of one scan, then by the stores of the tokens.
//
// Up to kLdsRows rows every workgroup does the whole scan (48 KB from L2 at most),
// so that one launch suffices: it then serves its share of the rows and of the
// tokens, and takes a token's new block from the ring itself, as another workgroup may
// not have written the table yet.  More rows: one workgroup scans, a second
// launch places the tokens.  4,096 rows, 134,000 tokens: 16 us (one workgroup
// for everything took 420 us, nearly all in the tokens); 64 rows 8 us.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kPer = 4;  // rows a thread
constexpr int kLdsRows = kThreads * kPer;

// A row's part of the step.
struct Row {
  int64_t grow, need, back;  // tokens, blocks taken, blocks given back
  int64_t have;              // blocks held
  int len;                   // tokens held, within the table
  bool ended, fits;
};

__device__ __forceinline__ Row row_of(const Geo& g, int fresh, int len) {
  Row r;
  const int64_t most = (int64_t)g.width << g.b_log2;
  r.len = (int)min(max((int64_t)len, (int64_t)0), most);
  r.ended = fresh < 0;
  r.grow = r.ended ? 0 : fresh;
  r.have = ((int64_t)r.len + g.b - 1) >> g.b_log2;
  r.fits = r.len + r.grow <= most;
  r.need = r.fits && !r.ended ? ((r.len + r.grow + g.b - 1) >> g.b_log2) - r.have : 0;
  r.back = r.ended ? r.have : 0;
  return r;
}

// Three sums over the workgroup at once: in[] becomes the sum of the threads
// before this one, total[] that of all.
__device__ __forceinline__ void block_sums(int64_t (&in)[3], int64_t (&total)[3], int64_t (*part)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) x[k] = in[k];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int64_t y = __shfl_up(x[k], off, 64);
      if (lane >= off) x[k] += y;
    }
  if (lane == 63)
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][wave] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    int64_t before = 0, all = 0;
    for (int w = 0; w < kWaves; ++w) {
      const int64_t p = part[k][w];
      before += w < wave ? p : 0;
      all += p;
    }
    in[k] = before + x[k] - in[k];
    total[k] = all;
  }
  __syncthreads();
}

__device__ __forceinline__ int clip(int64_t x) { return (int)min(x, (int64_t)INT32_MAX); }

// A row's blocks from (need > 0) or to (need < 0) the ring, from index `start` of the
// taken or the given ones on; blocks first, first + step, ... of them.
__device__ __forceinline__ void move_blocks(const Geo& g, const StepArgs& a, unsigned head, unsigned room,
                                            int64_t row, int have, int need, unsigned start, int first, int step) {
  const unsigned n = (unsigned)g.n_blocks;
  int32_t* mine = a.table + row * g.width;
  for (int i = first; i < need; i += step) mine[have + i] = a.ring[(head + start + (unsigned)i) % n];
  for (int i = first; i < -need; i += step) a.ring[(head + room + start + (unsigned)i) % n] = mine[i];
}

__global__ __launch_bounds__(kThreads) void step_one(Geo g, StepArgs a, int slice) {
  __shared__ int64_t part[3][kWaves];
  __shared__ int top[kWaves];
  // per row: tokens before it, tokens held, start in the ring (-1: refused), blocks
  __shared__ int off_of[kLdsRows + 1], len_of[kLdsRows], start_of[kLdsRows], need_of[kLdsRows];
  const unsigned n = (unsigned)g.n_blocks;
  const unsigned head = (unsigned)a.pool_in[0] % n;
  const int room = min(max(a.pool_in[1], 0), g.n_blocks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r0 = threadIdx.x * kPer;
  int fresh[kPer], len[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const bool in = r0 + k < a.n_rows;
    fresh[k] = in ? a.fresh[r0 + k] : 0;
    len[k] = in ? a.len_in[r0 + k] : 0;
  }
  int64_t at[3] = {0, 0, 0}, total[3];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const Row r = row_of(g, fresh[k], len[k]);
    at[0] += r.need, at[1] += r.grow, at[2] += r.back;
  }
  block_sums(at, total, part);
  int64_t got = 0;
  const int s0 = blockIdx.x * slice, s1 = min(s0 + slice, a.n_rows);  // the rows this workgroup serves
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = r0 + k;
    const Row x = row_of(g, fresh[k], len[k]);
    const bool in = r < a.n_rows;
    const bool ok = in && !x.ended && x.fits && (x.need == 0 || at[0] + x.need <= room);
    if (ok && x.need) got = at[0] + x.need;
    off_of[r] = clip(at[1]);
    len_of[r] = x.len;
    start_of[r] = ok ? (int)min(at[0], (int64_t)room) : x.ended ? (int)at[2] : -1;
    need_of[r] = ok ? (int)x.need : -(int)x.back;
    if (in && r >= s0 && r < s1) {
      a.granted[r] = ok;
      a.len_out[r] = x.ended ? 0 : ok ? (int)(x.len + x.grow) : x.len;
      a.q_off[r] = clip(at[1]);
    }
    at[0] += x.need, at[1] += x.grow, at[2] += x.back;
  }
  const int tokens = clip(total[1]);
  // the sum of the granted needs is the largest prefix among them
  int most = (int)got;
  for (int off = 32; off > 0; off >>= 1) most = max(most, __shfl_xor(most, off, 64));
  if (lane == 0) top[wave] = most;
  if (threadIdx.x == 0) off_of[kLdsRows] = tokens;
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    for (int w = 0; w < kWaves; ++w) most = max(most, top[w]);
    a.q_off[a.n_rows] = tokens;
    a.pool_out[0] = (int)((head + (unsigned)most) % n);
    a.pool_out[1] = (int)(room - most + total[2]);
  }
  // blocks: a lane a row for one block, the wave for the rest of longer ones
  for (int base = s0 + wave * 64; base < s1; base += kThreads) {
    const int r = base + lane;
    const int need = r < s1 ? need_of[r] : 0;
    const int have = r < s1 ? (int)(((int64_t)len_of[r] + g.b - 1) >> g.b_log2) : 0;
    const int start = r < s1 ? start_of[r] : 0;
    const int one = min(max(need, -1), 1);
    if (need) move_blocks(g, a, head, (unsigned)room, r, have, one, (unsigned)start, 0, 1);
    uint64_t more = __ballot(need > 1 || need < -1);
    while (more) {
      const int src = __ffsll((unsigned long long)more) - 1;
      more &= more - 1;
      move_blocks(g, a, head, (unsigned)room, base + src, __shfl(have, src, 64), __shfl(need, src, 64),
                  (unsigned)__shfl(start, src, 64), 1 + lane, 64);
    }
  }
  for (int t = blockIdx.x * kThreads + threadIdx.x; t < a.n_tokens; t += gridDim.x * kThreads) {
    int64_t slot = -1;
    int pos = 0;
    if (t < tokens) {
      int lo = 0, hi = a.n_rows;  // the last row that starts at or before t
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off_of[mid] <= t) lo = mid; else hi = mid;
      }
      pos = len_of[lo] + (t - off_of[lo]);
      if (start_of[lo] >= 0 && need_of[lo] >= 0) {  // granted: a released row has no tokens
        const int block = pos >> g.b_log2, have = (int)(((int64_t)len_of[lo] + g.b - 1) >> g.b_log2);
        const int id = block < have ? a.table[(int64_t)lo * g.width + block]
                                    : a.ring[(head + (unsigned)start_of[lo] + (unsigned)(block - have)) % n];
        slot = (int64_t)id * g.b + (pos & (g.b - 1));
      }
    }
    a.slot[t] = slot;
    a.pos[t] = pos;
  }
}

// Any number of rows: one workgroup, kThreads rows at a time.
__global__ __launch_bounds__(kThreads) void step_rows(Geo g, StepArgs a) {
  __shared__ int64_t part[3][kWaves];
  __shared__ int top[kWaves];
  const unsigned n = (unsigned)g.n_blocks;
  const unsigned head = (unsigned)a.pool_in[0] % n;
  const int room = min(max(a.pool_in[1], 0), g.n_blocks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t base[3] = {0, 0, 0};
  int most = 0;
  for (int r0 = 0; r0 < a.n_rows; r0 += kThreads) {
    const int r = r0 + (int)threadIdx.x;
    const bool in = r < a.n_rows;
    const Row x = row_of(g, in ? a.fresh[r] : 0, in ? a.len_in[r] : 0);
    int64_t at[3] = {x.need, x.grow, x.back}, total[3];
    block_sums(at, total, part);
#pragma unroll
    for (int k = 0; k < 3; ++k) at[k] += base[k], base[k] += total[k];
    const bool ok = in && !x.ended && x.fits && (x.need == 0 || at[0] + x.need <= room);
    if (ok && x.need) most = max(most, (int)(at[0] + x.need));
    if (in) {
      a.granted[r] = ok;
      a.len_out[r] = x.ended ? 0 : ok ? (int)(x.len + x.grow) : x.len;
      a.q_off[r] = clip(at[1]);
    }
    const int need = ok ? (int)x.need : -(int)x.back, have = (int)x.have;
    const int start = ok ? (int)min(at[0], (int64_t)room) : (int)at[2];
    uint64_t todo = __ballot(need != 0);
    while (todo) {
      const int src = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      move_blocks(g, a, head, (unsigned)room, r0 + wave * 64 + src, __shfl(have, src, 64), __shfl(need, src, 64),
                  (unsigned)__shfl(start, src, 64), lane, 64);
    }
  }
  for (int off = 32; off > 0; off >>= 1) most = max(most, __shfl_xor(most, off, 64));
  if (lane == 0) top[wave] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 0; w < kWaves; ++w) most = max(most, top[w]);
    a.q_off[a.n_rows] = clip(base[1]);
    a.pool_out[0] = (int)((head + (unsigned)most) % n);
    a.pool_out[1] = (int)(room - most + base[2]);
  }
}

__global__ __launch_bounds__(256) void step_tokens(Geo g, StepArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= a.n_tokens) return;
  int64_t slot = -1;
  int pos = 0;
  if (t < a.q_off[a.n_rows]) {
    int lo = 0, hi = a.n_rows;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.q_off[mid] <= t) lo = mid; else hi = mid;
    }
    pos = row_of(g, 0, a.len_in[lo]).len + (t - a.q_off[lo]);
    if (a.granted[lo])
      slot = (int64_t)a.table[(int64_t)lo * g.width + (pos >> g.b_log2)] * g.b + (pos & (g.b - 1));
  }
  a.slot[t] = slot;
  a.pos[t] = pos;
}

}  // namespace

hipError_t launch_step(const Geo& g, const StepArgs& a, hipStream_t s) {
  if (a.n_rows <= kLdsRows) {
    // a workgroup for every 1,024 tokens, and for every 256 rows
    const int wgs = std::max(1, std::min(256, std::max((a.n_tokens + kThreads - 1) / kThreads, a.n_rows / 256)));
    const int slice = ((a.n_rows + wgs - 1) / wgs + 63) / 64 * 64;
    hipLaunchKernelGGL(step_one, dim3(wgs), dim3(kThreads), 0, s, g, a, slice);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(step_rows, dim3(1), dim3(kThreads), 0, s, g, a);
  if (a.n_tokens) hipLaunchKernelGGL(step_tokens, dim3((a.n_tokens + 255) / 256), dim3(256), 0, s, g, a);
  return hipGetLastError();
}

}  // namespace wfkv
