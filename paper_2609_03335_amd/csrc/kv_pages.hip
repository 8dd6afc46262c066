// Blocks that several rows hold: forks, releases, compaction, and the copies they ask for.
//
// Integer arithmetic only, but for the copies.  What has to be in order -- which fork gets which block
// of the ring, the ring's new entries, the k-th block that moves and the k-th place for it -- comes from prefix
// sums over lists or block ids; atomics only count, so that their order does not matter.
//
// Each phase needs all of the one before.  Caches of up to kOneBlocks blocks are the work of one workgroup, with what
// it knows of every block in LDS: one launch (from Python 8 us, of which the kernel is ...).  Larger ones take a
// kernel a phase, 2 to 3 us and a place in the queue each.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;
constexpr int kScan = 1024;              // threads of a workgroup that scans
constexpr int kOneBlocks = 32768, kOneEntries = 32768;  // blocks and table entries of one workgroup
constexpr int kSteps = kOneBlocks / kScan;
constexpr int kChunks = WF_KV_PAGES_WORK / 4;  // parts of the block ids that are counted by themselves

// Sum of the threads' values before this one in a workgroup of kScan, and of all.
__device__ __forceinline__ uint32_t before(uint32_t x, uint32_t* total, uint32_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)sum, off, 64);
    if (lane >= off) sum += y;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint32_t base = 0, all = 0;
  for (int w = 0; w < kScan / 64; ++w) {
    const uint32_t p = part[w];
    if (w < wave) base += p;
    all += p;
  }
  __syncthreads();
  *total = all;
  return base + sum - x;
}

struct Pool {
  uint32_t n, head, room;
  __device__ Pool(const Geo& g, const int32_t* in)
      : n((uint32_t)g.n_blocks), head((uint32_t)in[0] % n), room((uint32_t)min(max(in[1], 0), g.n_blocks)) {}
};

__device__ __forceinline__ int length(const Geo& g, int len) { return min(max(len, 0), g.width << g.b_log2); }
__device__ __forceinline__ int held(const Geo& g, int len) { return (int)(((int64_t)length(g, len) + g.b - 1) >> g.b_log2); }

__device__ __forceinline__ void copy_ints(const int32_t* from, int32_t* to, int64_t n, int64_t at, int64_t step) {
  for (; at < n; at += step) to[at] = from[at];
}

// A fork as the rows' lengths allow it: its tokens, below 0 where it is refused.
__device__ __forceinline__ int fork_tokens(const Geo& g, const ForkArgs& a, int i) {
  const int src = a.src[i], dst = a.dst[i], want = a.tokens[i];
  if ((unsigned)src >= (unsigned)a.n_rows || (unsigned)dst >= (unsigned)a.n_rows || src == dst || want < 0) return -1;
  return a.len_in[dst] > 0 ? -1 : min(want, length(g, a.len_in[src]));
}

// Workgroup 0 goes through the forks; the others copy lengths and counts.
__global__ __launch_bounds__(kScan) void fork_grant(Geo g, ForkArgs a) {
  if (blockIdx.x) {
    const int64_t at = (int64_t)(blockIdx.x - 1) * kScan + threadIdx.x, step = (int64_t)(gridDim.x - 1) * kScan;
    copy_ints(a.shared_in, a.shared_out, g.n_blocks, at, step);
    copy_ints(a.len_in, a.len_out, a.n_rows, at, step);
    return;
  }
  __shared__ uint32_t part[kScan / 64];
  const Pool pool(g, a.pool_in);
  uint32_t base = 0, taken = 0;
  for (int i0 = 0; i0 < a.n_forks; i0 += kScan) {
    const int i = i0 + (int)threadIdx.x;
    const int k = i < a.n_forks ? fork_tokens(g, a, i) : -1;
    const uint32_t need = k > 0 && (k & (g.b - 1)) != 0;
    uint32_t total;
    const uint32_t at = base + before(need, &total, part);  // (at most n_forks)
    if (i < a.n_forks) {
      const bool ok = k >= 0 && (!need || at < pool.room);
      a.granted[i] = ok;
      a.from[i] = ok && need ? a.table[(int64_t)a.src[i] * g.width + (k >> g.b_log2)] : -1;
      a.to[i] = ok && need ? a.ring[(pool.head + at) % pool.n] : -1;
    }
    base += total;
  }
  taken = min(base, pool.room);  // needs are of one block each: the granted ones are the first
  if (threadIdx.x == 0) {
    a.pool_out[0] = (int)((pool.head + taken) % pool.n);
    a.pool_out[1] = (int)(pool.room - taken);
  }
}

// `parts` workgroups a fork share its entries.
__global__ __launch_bounds__(kThreads) void fork_rows(Geo g, ForkArgs a, int parts) {
  const int i = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x % (unsigned)parts);
  if (!a.granted[i]) return;
  const int k = fork_tokens(g, a, i), full = k >> g.b_log2;
  const int32_t* theirs = a.table + (int64_t)a.src[i] * g.width;
  int32_t* mine = a.table + (int64_t)a.dst[i] * g.width;
  for (int j = part * kThreads + (int)threadIdx.x; j < full; j += parts * kThreads) {
    const int id = theirs[j];
    mine[j] = id;
    if ((unsigned)id < (unsigned)g.n_blocks) atomicAdd(a.shared_out + id, 1);
  }
  if (part == 0 && threadIdx.x == 0) {
    if (k & (g.b - 1)) mine[full] = a.to[i];
    a.len_out[a.dst[i]] = k;
  }
}

__global__ __launch_bounds__(kThreads) void release_begin(Geo g, ReleaseArgs a) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
  copy_ints(a.shared_in, a.shared_out, g.n_blocks, at, step);
  for (int64_t r = at; r < a.n_rows; r += step) a.len_out[r] = a.release[r] ? 0 : a.len_in[r];
}

__global__ __launch_bounds__(kThreads) void release_rows(Geo g, ReleaseArgs a, int parts) {
  const int r = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x % (unsigned)parts);
  if (!a.release[r]) return;
  const int32_t* mine = a.table + (int64_t)r * g.width;
  const int have = held(g, a.len_in[r]);
  for (int j = part * kThreads + (int)threadIdx.x; j < have; j += parts * kThreads) {
    const int id = mine[j];
    if ((unsigned)id < (unsigned)g.n_blocks) atomicSub(a.shared_out + id, 1);
  }
}

// The ids of chunk `c` of `chunks`: [first, last).
struct Chunk {
  int first, last;
  __device__ Chunk(const Geo& g, int c, int chunks) {
    const int size = (int)(((int64_t)g.n_blocks + chunks - 1) / chunks);
    first = (int)min((int64_t)c * size, (int64_t)g.n_blocks);
    last = (int)min((int64_t)first + size, (int64_t)g.n_blocks);
  }
};

__device__ __forceinline__ uint32_t sum_of(uint32_t x, uint32_t* part) {
  uint32_t total;
  before(x, &total, part);
  return total;
}

__global__ __launch_bounds__(kScan) void release_count(Geo g, ReleaseArgs a) {
  __shared__ uint32_t part[kScan / 64];
  const Chunk c(g, blockIdx.x, gridDim.x);
  uint32_t n = 0;
  for (int b = c.first + (int)threadIdx.x; b < c.last; b += kScan) n += a.shared_out[b] < 0;
  n = sum_of(n, part);
  if (threadIdx.x == 0) a.work[blockIdx.x] = (int)n;
}

__global__ __launch_bounds__(kScan) void release_write(Geo g, ReleaseArgs a) {
  __shared__ uint32_t part[kScan / 64];
  const Pool pool(g, a.pool_in);
  const Chunk c(g, blockIdx.x, gridDim.x);
  const uint32_t mine = threadIdx.x < gridDim.x ? (uint32_t)a.work[threadIdx.x] : 0;
  const uint32_t all = sum_of(mine, part);
  uint32_t base = sum_of(threadIdx.x < blockIdx.x ? mine : 0, part);
  for (int b0 = c.first; b0 < c.last; b0 += kScan) {
    const int b = b0 + (int)threadIdx.x;
    const uint32_t over = b < c.last && a.shared_out[b] < 0;
    uint32_t total;
    const uint32_t at = base + before(over, &total, part);
    if (over) {
      a.ring[(pool.head + pool.room + at) % pool.n] = b;
      a.shared_out[b] = 0;
    }
    base += total;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.pool_out[0] = (int)pool.head;
    a.pool_out[1] = (int)min(pool.room + all, pool.n);
  }
}

// For one workgroup: entries of a list of up to kOneBlocks that a test picks, in order.  count() takes the
// test of one's entries in steps of kScan, first() then gives the place of a step's first one in this wave.
struct Picked {
  uint16_t (*of)[kScan / 64];  // [kSteps][waves]: picked, then picked before
  uint32_t* part;
  __device__ __forceinline__ void count(int step, bool pick) {
    const uint64_t mask = __ballot(pick);
    if ((threadIdx.x & 63) == 0) of[step][threadIdx.x >> 6] = (uint16_t)__popcll(mask);
  }
  __device__ __forceinline__ uint32_t scan(int steps) {
    __syncthreads();
    uint16_t* at = &of[0][0] + threadIdx.x;
    const bool in = (int)threadIdx.x < steps * (kScan / 64);
    uint32_t total;
    const uint32_t n = in ? *at : 0, x = before(n, &total, part);
    if (in) *at = (uint16_t)x;
    __syncthreads();
    return total;
  }
  __device__ __forceinline__ uint32_t place(int step, bool pick) const {
    return of[step][threadIdx.x >> 6] + (uint32_t)__popcll(__ballot(pick) & ((1ull << (threadIdx.x & 63)) - 1ull));
  }
};
static_assert(kSteps * (kScan / 64) <= kScan, "a thread for every count");

// The rows that `pick` names, each the work of a wave's 64 lanes (`act`); neighbours go to different waves.
template <class P, class A>
__device__ __forceinline__ void each_row(int n_rows, P pick, A act) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int r0 = 0; r0 < n_rows; r0 += kScan) {
    const int r = r0 + lane * (kScan / 64) + wave;
    uint64_t todo = __ballot(r < n_rows && pick(r));
    while (todo) {
      const int src = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      act(r0 + src * (kScan / 64) + wave, lane);
    }
  }
}

__global__ __launch_bounds__(kScan) void release_one(Geo g, ReleaseArgs a) {
  __shared__ int left[kOneBlocks];
  __shared__ uint16_t counts[kSteps][kScan / 64];
  __shared__ uint32_t part[kScan / 64];
  const Pool pool(g, a.pool_in);
#pragma unroll 8
  for (int b = threadIdx.x; b < g.n_blocks; b += kScan) left[b] = a.shared_in[b];
  __syncthreads();
  each_row(
      a.n_rows,
      [&](int r) {
        const bool ends = a.release[r] != 0;
        a.len_out[r] = ends ? 0 : a.len_in[r];
        return ends;
      },
      [&](int r, int lane) {
        const int32_t* mine = a.table + (int64_t)r * g.width;
        const int have = held(g, a.len_in[r]);
#pragma unroll 4
        for (int j = lane; j < have; j += 64) {
          const int id = mine[j];
          if ((unsigned)id < (unsigned)g.n_blocks) atomicSub(left + id, 1);
        }
      });
  __syncthreads();
  Picked over{counts, part};
  const int steps = (g.n_blocks + kScan - 1) / kScan;
  for (int k = 0; k < steps; ++k) {
    const int b = k * kScan + (int)threadIdx.x;
    over.count(k, b < g.n_blocks && left[b] < 0);
  }
  const uint32_t all = over.scan(steps);
  for (int k = 0; k < steps; ++k) {
    const int b = k * kScan + (int)threadIdx.x;
    const int n = b < g.n_blocks ? left[b] : 0;
    const uint32_t at = over.place(k, n < 0);
    if (n < 0) a.ring[(pool.head + pool.room + at) % pool.n] = b;
    if (b < g.n_blocks) a.shared_out[b] = max(n, 0);
  }
  if (threadIdx.x == 0) {
    a.pool_out[0] = (int)pool.head;
    a.pool_out[1] = (int)min(pool.room + all, pool.n);
  }
}

__global__ __launch_bounds__(kScan) void fork_one(Geo g, ForkArgs a) {
  __shared__ int count[kOneBlocks];
  __shared__ uint32_t part[kScan / 64];
  const Pool pool(g, a.pool_in);
#pragma unroll 8
  for (int b = threadIdx.x; b < g.n_blocks; b += kScan) count[b] = a.shared_in[b];
  const int i = (int)threadIdx.x;  // a fork a thread
  const int k = i < a.n_forks ? fork_tokens(g, a, i) : -1;
  const uint32_t need = k > 0 && (k & (g.b - 1)) != 0;
  uint32_t total;
  const uint32_t at = before(need, &total, part);
  const bool ok = k >= 0 && (!need || at < pool.room);
  const int full = ok ? k >> g.b_log2 : 0, src = ok ? a.src[i] : 0, dst = ok ? a.dst[i] : 0;
  // lengths of the rows that no fork fills, then of those
  copy_ints(a.len_in, a.len_out, a.n_rows, threadIdx.x, kScan);
  if (i < a.n_forks) {
    a.granted[i] = ok;
    const int old = ok && need ? a.table[(int64_t)src * g.width + full] : -1, fresh = ok && need ? a.ring[(pool.head + at) % pool.n] : -1;
    a.from[i] = old;
    a.to[i] = fresh;
    if (ok && need) a.table[(int64_t)dst * g.width + full] = fresh;
  }
  __syncthreads();
  if (ok) a.len_out[dst] = k;
  const int lane = threadIdx.x & 63;
  uint64_t todo = __ballot(full > 0);
  while (todo) {
    const int who = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    const int n = __shfl(full, who, 64);
    const int32_t* theirs = a.table + (int64_t)__shfl(src, who, 64) * g.width;
    int32_t* mine = a.table + (int64_t)__shfl(dst, who, 64) * g.width;
#pragma unroll 4
    for (int j = lane; j < n; j += 64) {
      const int id = theirs[j];
      mine[j] = id;
      if ((unsigned)id < (unsigned)g.n_blocks) atomicAdd(count + id, 1);
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < g.n_blocks; b += kScan) a.shared_out[b] = count[b];
  if (threadIdx.x == 0) {
    const uint32_t taken = min(total, pool.room);
    a.pool_out[0] = (int)((pool.head + taken) % pool.n);
    a.pool_out[1] = (int)(pool.room - taken);
  }
}

// What ids[] of a block says: in use, free; below `keep` and free, kTaken - k: it becomes the place of the
// k-th block that moves; from `keep` on and in use, k: it is that block.
constexpr int kUsed = 0, kFree = -1, kTaken = -2;

__global__ __launch_bounds__(kThreads) void compact_begin(Geo g, CompactArgs a) {
  for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < g.n_blocks; b += (int64_t)gridDim.x * kThreads) a.ids[b] = kUsed;
}

__global__ __launch_bounds__(kThreads) void compact_free(Geo g, CompactArgs a) {
  const Pool pool(g, a.pool_in);
  for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < pool.room; i += gridDim.x * kThreads) {
    const int id = a.ring_in[(pool.head + i) % pool.n];
    if ((unsigned)id < (unsigned)g.n_blocks) a.ids[id] = kFree;
  }
}

__global__ __launch_bounds__(kScan) void compact_count(Geo g, CompactArgs a) {
  __shared__ uint32_t part[kScan / 64];
  const Chunk c(g, blockIdx.x, gridDim.x);
  uint32_t goes = 0, hole = 0;
  for (int b = c.first + (int)threadIdx.x; b < c.last; b += kScan) {
    const bool used = a.ids[b] == kUsed;
    goes += used && b >= a.keep;
    hole += !used && b < a.keep;
  }
  goes = sum_of(goes, part);
  hole = sum_of(hole, part);
  if (threadIdx.x == 0) a.work[2 * blockIdx.x] = (int)goes, a.work[2 * blockIdx.x + 1] = (int)hole;
}

__global__ __launch_bounds__(kScan) void compact_place(Geo g, CompactArgs a) {
  __shared__ uint32_t part[kScan / 64];
  const Chunk c(g, blockIdx.x, gridDim.x);
  const bool in = threadIdx.x < gridDim.x, lower = threadIdx.x < blockIdx.x;
  const uint32_t my_goes = in ? (uint32_t)a.work[2 * threadIdx.x] : 0, my_holes = in ? (uint32_t)a.work[2 * threadIdx.x + 1] : 0;
  const uint32_t goes = sum_of(my_goes, part), holes = sum_of(my_holes, part);
  uint32_t g0 = sum_of(lower ? my_goes : 0, part), h0 = sum_of(lower ? my_holes : 0, part);
  const bool done = goes <= holes;
  const int most = min(a.keep, g.n_blocks - a.keep);
  // what is left of the outputs
  const int at = (int)(blockIdx.x * kScan + threadIdx.x), step = (int)(gridDim.x * kScan);
  for (int64_t i = (int64_t)(done ? goes : 0) + at; i < most; i += step) a.from[i] = a.to[i] = -1;
  for (int64_t i = (int64_t)(done ? holes - goes : 0) + at; i < a.keep; i += step) a.ring_out[i] = -1;
  if (at == 0) {
    a.done[0] = done;
    a.pool_out[0] = 0;
    a.pool_out[1] = done ? (int)(holes - goes) : 0;
  }
  if (!done) return;
  for (int b0 = c.first; b0 < c.last; b0 += kScan) {
    const int b = b0 + (int)threadIdx.x;
    const bool used = b < c.last && a.ids[b] == kUsed, idle = b < c.last && !used;
    const uint32_t go = used && b >= a.keep, hole = idle && b < a.keep;
    uint32_t total;
    const uint32_t i = g0 + before(go, &total, part);
    g0 += total;
    const uint32_t j = h0 + before(hole, &total, part);
    h0 += total;
    if (go) a.from[i] = b, a.ids[b] = (int)i;
    if (hole && j < goes) a.to[j] = b, a.ids[b] = kTaken - (int)j;
    if (hole && j >= goes) a.ring_out[j - goes] = b;
  }
}

// Workgroups up to `tables` rewrite the rows' entries, `parts` of them a row; the others write the counts by new id.
__global__ __launch_bounds__(kThreads) void compact_rows(Geo g, CompactArgs a, unsigned tables, int parts) {
  if (!a.done[0]) return;
  if (blockIdx.x >= tables) {
    const int64_t step = (int64_t)(gridDim.x - tables) * kThreads;
    for (int64_t b = (int64_t)(blockIdx.x - tables) * kThreads + threadIdx.x; b < a.keep; b += step) {
      const int v = a.ids[b];
      a.shared_out[b] = v == kUsed ? a.shared_in[b] : v == kFree ? 0 : a.shared_in[a.from[kTaken - v]];
    }
    return;
  }
  const int r = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x % (unsigned)parts);
  int32_t* mine = a.table + (int64_t)r * g.width;
  const int have = held(g, a.len[r]);
  for (int j = part * kThreads + (int)threadIdx.x; j < have; j += parts * kThreads) {
    const int id = mine[j];
    if (id < a.keep || id >= g.n_blocks) continue;
    const int k = a.ids[id];
    if (k >= 0) mine[j] = a.to[k];  // (below 0: a free block, which no row should hold)
  }
}

__global__ __launch_bounds__(kScan) void compact_one(Geo g, CompactArgs a) {
  // of a block: in use, free, or the place among those that move (`goes`); the k-th free one of the front
  constexpr uint16_t kIn = 0xffff, kOut = 0xfffe;
  __shared__ uint16_t state[kOneBlocks], hole_id[kOneBlocks];
  __shared__ uint16_t counts[2][kSteps][kScan / 64];
  __shared__ uint32_t part[kScan / 64];
  const Pool pool(g, a.pool_in);
  for (int b = threadIdx.x; b < g.n_blocks; b += kScan) state[b] = kIn;
  __syncthreads();
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < pool.room; i += kScan) {
    const int id = a.ring_in[(pool.head + i) % pool.n];
    if ((unsigned)id < (unsigned)g.n_blocks) state[id] = kOut;
  }
  __syncthreads();
  const int steps = (g.n_blocks + kScan - 1) / kScan;
  Picked goes{counts[0], part}, holes{counts[1], part};
  for (int k = 0; k < steps; ++k) {
    const int b = k * kScan + (int)threadIdx.x;
    const bool in = b < g.n_blocks, used = in && state[b] == kIn;
    goes.count(k, used && b >= a.keep);
    holes.count(k, in && !used && b < a.keep);
  }
  const uint32_t n_goes = goes.scan(steps), n_holes = holes.scan(steps);
  const bool done = n_goes <= n_holes;
  const int most = min(a.keep, g.n_blocks - a.keep);
  for (int i = (int)(done ? n_goes : 0u) + (int)threadIdx.x; i < most; i += kScan) a.from[i] = a.to[i] = -1;
  for (int i = (int)(done ? n_holes - n_goes : 0u) + (int)threadIdx.x; i < a.keep; i += kScan) a.ring_out[i] = -1;
  if (threadIdx.x == 0) {
    a.done[0] = done;
    a.pool_out[0] = 0;
    a.pool_out[1] = done ? (int)(n_holes - n_goes) : 0;
  }
  if (!done) return;  // (all threads)
  for (int k = 0; k < steps; ++k) {
    const int b = k * kScan + (int)threadIdx.x;
    const bool in = b < g.n_blocks, used = in && state[b] == kIn;
    const bool go = used && b >= a.keep, hole = in && !used && b < a.keep;
    const uint32_t i = goes.place(k, go), j = holes.place(k, hole);
    if (go) a.from[i] = b, state[b] = (uint16_t)i;  // (i < n_blocks / 2)
    if (hole) hole_id[j] = (uint16_t)b;
    if (hole && j < n_goes) a.to[j] = b;
    if (hole && j >= n_goes) a.ring_out[j - n_goes] = b;
  }
  __syncthreads();
  // counts by new id: those that stay, those that come, 0 for what is free
  for (int b = threadIdx.x; b < a.keep; b += kScan)
    if (state[b] == kIn) a.shared_out[b] = a.shared_in[b];
  for (int b = a.keep + (int)threadIdx.x; b < g.n_blocks; b += kScan)
    if (state[b] < kOut) a.shared_out[hole_id[state[b]]] = a.shared_in[b];
  for (uint32_t j = n_goes + threadIdx.x; j < n_holes; j += kScan) a.shared_out[hole_id[j]] = 0;
  each_row(
      a.n_rows, [&](int r) { return a.len[r] > 0; },
      [&](int r, int lane) {
        int32_t* mine = a.table + (int64_t)r * g.width;
        const int have = held(g, a.len[r]);
#pragma unroll 4
        for (int j = lane; j < have; j += 64) {
          const int id = mine[j];
          // (a free block, which no row should hold, stays as it is)
          if (id >= a.keep && id < g.n_blocks && state[id] < kOut) mine[j] = hole_id[state[id]];
        }
      });
}

// A workgroup's step: 16 KiB of a pair of blocks in one layer, four loads of a thread on their way at once (its
// registers are plain vectors and filled without a condition: what may be missing would go through LDS, one by one).
// Stores past the caches: 900 blocks of 131 KB 51 -> 47 us (5.1 TB/s), 800 of 66 KB in two layers 47 -> 40; eight loads 52 us.
constexpr int kPiece = 4 * kThreads;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// grid: pieces x pairs (those after come in turns), layers
__global__ __launch_bounds__(kThreads) void copy(CopyArgs a, int n_blocks, int vectors, unsigned pieces) {
  const unsigned piece = blockIdx.x % pieces, step = gridDim.x / pieces;
  u32x4* base = reinterpret_cast<u32x4*>(a.cache + blockIdx.y * a.layer_stride);
  const auto* froms = (const __attribute__((address_space(4))) int32_t*)a.from;
  const auto* tos = (const __attribute__((address_space(4))) int32_t*)a.to;
  const int v0 = (int)(piece * kPiece + threadIdx.x);
  for (unsigned i = blockIdx.x / pieces; i < (unsigned)a.n; i += step) {
    const int from = froms[i], to = tos[i];
    if (from == to || (unsigned)from >= (unsigned)n_blocks || (unsigned)to >= (unsigned)n_blocks) continue;
    const u32x4* src = base + (int64_t)from * vectors;
    u32x4* dst = base + (int64_t)to * vectors;
    u32x4 w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = src[min(v0 + k * kThreads, vectors - 1)];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (v0 + k * kThreads < vectors) __builtin_nontemporal_store(w[k], dst + v0 + k * kThreads);
  }
}

// Workgroups that share a row's entries: one for every 1,024, fewer where there are many rows.
int parts_of(const Geo& g, int rows) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({(g.width + 1023) / 1024, 65536 / std::max(1, rows), 64}));
}
int chunks_of(const Geo& g) { return (int)std::min<int64_t>(kChunks, ((int64_t)g.n_blocks + 4 * kScan - 1) / (4 * kScan)); }
unsigned groups_of(int64_t n, int threads) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(1024, (n + 4 * threads - 1) / (4 * threads))); }

}  // namespace

hipError_t launch_fork(const Geo& g, const ForkArgs& a, hipStream_t s) {
  // (a workgroup goes through the forks' entries in steps of 1,024)
  if (g.n_blocks <= kOneBlocks && a.n_forks <= kScan && (int64_t)a.n_forks * g.width <= kOneEntries / 2) {
    hipLaunchKernelGGL(fork_one, dim3(1), dim3(kScan), 0, s, g, a);
    return hipGetLastError();
  }
  const unsigned copies = groups_of(std::max(g.n_blocks, a.n_rows), kScan);
  hipLaunchKernelGGL(fork_grant, dim3(1 + copies), dim3(kScan), 0, s, g, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_forks == 0) return e;
  const int parts = parts_of(g, a.n_forks);
  hipLaunchKernelGGL(fork_rows, dim3((unsigned)a.n_forks * parts), dim3(kThreads), 0, s, g, a, parts);
  return hipGetLastError();
}

hipError_t launch_release(const Geo& g, const ReleaseArgs& a, hipStream_t s) {
  if (g.n_blocks <= kOneBlocks && (int64_t)a.n_rows * g.width <= 2 * kOneEntries) {
    hipLaunchKernelGGL(release_one, dim3(1), dim3(kScan), 0, s, g, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(release_begin, dim3(groups_of(std::max(g.n_blocks, a.n_rows), kThreads)), dim3(kThreads), 0, s, g, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.n_rows) {
    const int parts = parts_of(g, a.n_rows);
    hipLaunchKernelGGL(release_rows, dim3((unsigned)a.n_rows * parts), dim3(kThreads), 0, s, g, a, parts);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(release_count, dim3(chunks_of(g)), dim3(kScan), 0, s, g, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(release_write, dim3(chunks_of(g)), dim3(kScan), 0, s, g, a);
  return hipGetLastError();
}

hipError_t launch_compact(const Geo& g, const CompactArgs& a, hipStream_t s) {
  if (g.n_blocks <= kOneBlocks && (int64_t)a.n_rows * g.width <= kOneEntries) {
    hipLaunchKernelGGL(compact_one, dim3(1), dim3(kScan), 0, s, g, a);
    return hipGetLastError();
  }
  const unsigned over = groups_of(g.n_blocks, kThreads);
  hipLaunchKernelGGL(compact_begin, dim3(over), dim3(kThreads), 0, s, g, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_free, dim3(over), dim3(kThreads), 0, s, g, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_count, dim3(chunks_of(g)), dim3(kScan), 0, s, g, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_place, dim3(chunks_of(g)), dim3(kScan), 0, s, g, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int parts = parts_of(g, a.n_rows);
  const unsigned tables = (unsigned)a.n_rows * parts;
  hipLaunchKernelGGL(compact_rows, dim3(tables + groups_of(a.keep, kThreads)), dim3(kThreads), 0, s, g, a, tables, parts);
  return hipGetLastError();
}

hipError_t launch_copy(const Geo& g, const CopyArgs& a, int n_cu, hipStream_t s) {
  const int vectors = (int)((int64_t)g.hk * g.cell / 16);
  const unsigned pieces = (unsigned)((vectors + kPiece - 1) / kPiece);
  const int64_t pairs = std::max<int64_t>(1, std::min<int64_t>(a.n, (int64_t)n_cu * 16 / ((int64_t)pieces * a.n_layers)));
  hipLaunchKernelGGL(copy, dim3((unsigned)(pairs * pieces), (unsigned)a.n_layers), dim3(kThreads), 0, s, a, g.n_blocks, vectors, pieces);
  return hipGetLastError();
}

}  // namespace wfkv
