// Block tables and slots of one step from the rows' lengths: an inclusive sum
// of the rows' needs decides who is granted and where in the ring of free
// blocks each row takes or gives back its blocks; an exclusive sum of the new
// tokens places the rows' tokens.  Integer arithmetic only; bound by the latency
// of a launch and of one scan, then by the stores of the tokens.
//
// Up to kLdsRows rows every workgroup does the whole scan (32 KB from L2 at most),
// so that one launch suffices: it then serves its share of the rows and of the
// tokens, and takes a token's new block from the ring itself, as another workgroup may
// not have written the table yet.  More rows: one workgroup scans, a second
// launch places the tokens.  64 rows take 4.1 us, 4,096 rows with 134,000 tokens 11.9 (one
// workgroup for everything took 420); with 64-bit sums through LDS it was 8.0 and 15.8.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kPer = 4;  // rows a thread
constexpr int kLdsRows = kThreads * kPer;

// A row's part of the step.
struct Row {
  uint32_t grow, need, back;  // tokens, blocks taken, blocks given back
  uint32_t have;              // blocks held
  uint32_t len;               // tokens held, within the table: at most 2^30
  bool ended, fits;
};

__device__ __forceinline__ Row row_of(const Geo& g, int fresh, int len) {
  Row r;
  const uint32_t most = (uint32_t)g.width << g.b_log2;
  r.len = min((uint32_t)max(len, 0), most);
  r.ended = fresh < 0;
  r.grow = r.ended ? 0u : (uint32_t)fresh;
  r.have = (r.len + g.b - 1) >> g.b_log2;
  r.fits = r.len + r.grow <= most;
  r.need = r.fits && !r.ended ? ((r.len + r.grow + g.b - 1) >> g.b_log2) - r.have : 0;
  r.back = r.ended ? r.have : 0;
  return r;
}

// Sums stop at 2^32 - 1, which compares as the true sum does with anything that fits.
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sum of this lane's and the lower lanes' values of a wave, or (kRow) of its 16 lanes.
template <bool kRow>
__device__ __forceinline__ uint32_t scan(uint32_t x) {
  x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));  // from 1, 2, 4, 8 lanes below
  x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  if constexpr (!kRow) {
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));  // lane 15 of rows 0 and 2
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));  // lane 31
  }
  return x;
}

// Three sums over the workgroup at once: in[] becomes the sum of the threads
// before this one, total[] that of all.
__device__ __forceinline__ void block_sums(uint32_t (&in)[3], uint32_t (&total)[3], uint32_t (*part)[kWaves]) {
  static_assert(kWaves == 16, "a row of lanes holds the waves' sums");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t x = scan<false>(in[k]);
    if (lane == 63) part[k][wave] = x;
    // (from the lane below: a difference would be wrong where a sum stopped)
    in[k] = (uint32_t)__shfl_up((int)x, 1, 64);
    if (lane == 0) in[k] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t p = scan<true>(part[k][lane & 15]);
    total[k] = (uint32_t)__builtin_amdgcn_readlane((int)p, 15);
    if (wave) in[k] = add(in[k], (uint32_t)__builtin_amdgcn_readlane((int)p, wave - 1));
  }
  __syncthreads();
}

__device__ __forceinline__ int clip(uint32_t x) { return (int)min(x, (uint32_t)INT32_MAX); }

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
  __shared__ uint32_t part[3][kWaves];
  __shared__ int top[kWaves];
  // per row: tokens before it, tokens held, start in the ring (-1: refused), blocks
  __shared__ int off_of[kLdsRows], len_of[kLdsRows], start_of[kLdsRows], need_of[kLdsRows];
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
  uint32_t at[3] = {0, 0, 0}, total[3];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const Row r = row_of(g, fresh[k], len[k]);
    at[0] = add(at[0], r.need), at[1] = add(at[1], r.grow), at[2] = add(at[2], r.back);
  }
  block_sums(at, total, part);
  int most = 0;
  const int s0 = blockIdx.x * slice, s1 = min(s0 + slice, a.n_rows);  // the rows this workgroup serves
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = r0 + k;
    if (r >= a.n_rows) break;
    const Row x = row_of(g, fresh[k], len[k]);
    const uint32_t upto = add(at[0], x.need);
    const bool ok = !x.ended && x.fits && (x.need == 0 || upto <= (uint32_t)room);
    if (ok && x.need) most = (int)upto;
    off_of[r] = clip(at[1]);
    len_of[r] = (int)x.len;
    start_of[r] = ok ? (int)min(at[0], (uint32_t)room) : x.ended ? (int)at[2] : -1;
    need_of[r] = ok ? (int)x.need : -(int)x.back;
    if (r >= s0 && r < s1) {
      a.granted[r] = ok;
      a.len_out[r] = (int)(x.ended ? 0u : ok ? x.len + x.grow : x.len);
      a.q_off[r] = clip(at[1]);
    }
    at[0] = upto, at[1] = add(at[1], x.grow), at[2] = add(at[2], x.back);
  }
  const int tokens = clip(total[1]);
  // the sum of the granted needs is the largest prefix among them
  if (blockIdx.x == 0) {
    for (int off = 32; off > 0; off >>= 1) most = max(most, __shfl_xor(most, off, 64));
    if (lane == 0) top[wave] = most;
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    for (int w = 0; w < kWaves; ++w) most = max(most, top[w]);
    a.q_off[a.n_rows] = tokens;
    a.pool_out[0] = (int)((head + (unsigned)most) % n);
    a.pool_out[1] = (int)((unsigned)room - (unsigned)most + total[2]);
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
  // tokens from the last wave on: the first ones may still wait for their blocks
  const int mine = kThreads - 64 - wave * 64 + lane;
  for (int64_t at = (int64_t)blockIdx.x * kThreads + mine; at < a.n_tokens; at += gridDim.x * kThreads) {
    const int t = (int)at;
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
  __shared__ uint32_t part[3][kWaves];
  __shared__ int top[kWaves];
  const unsigned n = (unsigned)g.n_blocks;
  const unsigned head = (unsigned)a.pool_in[0] % n;
  const int room = min(max(a.pool_in[1], 0), g.n_blocks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t base[3] = {0, 0, 0};
  int most = 0;
  for (int r0 = 0; r0 < a.n_rows; r0 += kThreads) {
    const int r = r0 + (int)threadIdx.x;
    const bool in = r < a.n_rows;
    const Row x = row_of(g, in ? a.fresh[r] : 0, in ? a.len_in[r] : 0);
    uint32_t at[3] = {x.need, x.grow, x.back}, total[3];
    block_sums(at, total, part);
#pragma unroll
    for (int k = 0; k < 3; ++k) at[k] = add(at[k], base[k]), base[k] = add(base[k], total[k]);
    const uint32_t upto = add(at[0], x.need);
    const bool ok = in && !x.ended && x.fits && (x.need == 0 || upto <= (uint32_t)room);
    if (ok && x.need) most = max(most, (int)upto);
    if (in) {
      a.granted[r] = ok;
      a.len_out[r] = (int)(x.ended ? 0u : ok ? x.len + x.grow : x.len);
      a.q_off[r] = clip(at[1]);
    }
    const int need = ok ? (int)x.need : -(int)x.back, have = (int)x.have;
    const int start = ok ? (int)min(at[0], (uint32_t)room) : (int)at[2];
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
    a.pool_out[1] = (int)((unsigned)room - (unsigned)most + base[2]);
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
    pos = (int)row_of(g, 0, a.len_in[lo]).len + (t - a.q_off[lo]);
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
