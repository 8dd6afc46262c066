// Blocks that several rows hold: forks, releases, compaction, and the copies they ask for.
//
// Integer arithmetic only, but for the copies.  What has to be in order -- which fork gets which block
// of the ring, the ring's new entries, the k-th block that moves and the k-th place for it -- comes from prefix
// sums over lists or block ids; atomics only count, so that their order does not matter.
//
// Each phase needs all of the one before, so what bounds a call is the number of phases and each one's round trips to
// memory (2 to 3 us a kernel), not the bytes: a few hundred KB.  Caches of up to kOneBlocks blocks are the work of one
// workgroup, with what it knows of every block in LDS (4 bytes of it or 2, what 160 KB hold), barriers between the
// phases and eight loads of a thread on their way at once: one launch.  4 forks among 16 rows and 100 blocks 4.3 us, the copies
// 3.0 (9 to 10 us a call of both from Python); 4 of 64 rows of 7,984 blocks released 7.2 us (as kernels of a phase each 15 from Python,
// so 8); a compaction of 767 blocks and 24 rows 6.0 us, of 6,263 and 96 rows 14.2.
// Larger ones take a kernel a phase, ids and entries over all CUs: 1,500 rows of up to 377 entries and 249,669 blocks released
// 3.0 + 6.8 + 3.2 + 4.9 us, of which the walk over the rows' entries (atomics in L2) is the longest; 250 forks of rows of 236
// entries 3.7 + 6.6.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;
constexpr int kScan = 1024;              // threads of a workgroup that scans
constexpr int kOneBlocks = 32768, kOneEntries = 32768;  // blocks and table entries of one workgroup
constexpr int kSteps = kOneBlocks / kScan;
constexpr int kAtOnce = 4;               // ids of a thread that are looked at at once
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

// For one workgroup: entries of a list of up to kOneBlocks that a test picks, in order.  count() takes the
// test of one's entries in steps of kScan, place() after scan() gives where a picked one comes.
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

__global__ __launch_bounds__(kScan) void release_count(Geo g, ReleaseArgs a) {
  __shared__ uint32_t part[kScan / 64];
  const Chunk c(g, blockIdx.x, gridDim.x);
  uint32_t n = 0;
#pragma unroll 4
  for (int b = c.first + (int)threadIdx.x; b < c.last; b += kScan) n += a.shared_out[b] < 0;
  n = sum_of(n, part);
  if (threadIdx.x == 0) a.work[blockIdx.x] = (int)n;
}

// The sum of the chunks' counts before this one (of every `stride`-th entry of work, from `at` on), and of all.
__device__ __forceinline__ uint32_t chunks_before(const int32_t* work, int stride, int at, uint32_t* all, uint32_t* part) {
  __shared__ uint32_t mine;
  const uint32_t n = threadIdx.x < gridDim.x ? (uint32_t)work[stride * threadIdx.x + at] : 0;
  const uint32_t x = before(n, all, part);
  if (threadIdx.x == blockIdx.x) mine = x;
  __syncthreads();
  const uint32_t out = mine;
  __syncthreads();
  return out;
}

__global__ __launch_bounds__(kScan) void release_write(Geo g, ReleaseArgs a) {
  __shared__ uint32_t part[kScan / 64];
  __shared__ uint16_t counts[kAtOnce][kScan / 64];
  const Pool pool(g, a.pool_in);
  const Chunk c(g, blockIdx.x, gridDim.x);
  uint32_t all;
  uint32_t base = chunks_before(a.work, 1, 0, &all, part);
  Picked over{counts, part};
  for (int b0 = c.first; b0 < c.last; b0 += kAtOnce * kScan) {
    bool mine[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int b = b0 + k * kScan + (int)threadIdx.x;
      mine[k] = a.shared_out[min(b, c.last - 1)] < 0 && b < c.last;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) over.count(k, mine[k]);
    const uint32_t total = over.scan(kAtOnce);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int b = b0 + k * kScan + (int)threadIdx.x;
      const uint32_t at = base + over.place(k, mine[k]);
      if (mine[k]) {
        a.ring[(pool.head + pool.room + at) % pool.n] = b;
        a.shared_out[b] = 0;
      }
    }
    base += total;
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.pool_out[0] = (int)pool.head;
    a.pool_out[1] = (int)min(pool.room + all, pool.n);
  }
}

// The table entries of the rows' blocks, have(r) of row r: act(its index in the table, its id), for ids of the cache.  Eight
// a thread are on their way at once.
template <class H, class A>
__device__ __forceinline__ void each_entry(const Geo& g, const int32_t* table, int n_rows, H have, A act) {
  constexpr int N = 8;
  const unsigned width = (unsigned)g.width, all = (unsigned)n_rows * width;
  for (unsigned x0 = threadIdx.x; x0 < all; x0 += N * kScan) {
    int id[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const unsigned x = min(x0 + u * kScan, all - 1), r = x / width;
      id[u] = (int)(x - r * width) < have((int)r) ? (int)x : -1;
    }
#pragma unroll
    for (int u = 0; u < N; ++u) id[u] = id[u] >= 0 ? table[id[u]] : -1;
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (x0 + u * kScan < all && (unsigned)id[u] < (unsigned)g.n_blocks) act(x0 + u * kScan, id[u]);
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
  // (a wave takes one after the other of the rows that end, neighbours go to different waves: right for few or long ones, 4
  // of 64 rows of up to 250 entries 8 us from Python and all 64 11.  Each costs a round trip to memory however short it
  // is: all of 1,500 rows of up to 4 entries 73 us, 40 of them 9; the kernels of a phase each take 9,000 such rows in 16.)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int r0 = 0; r0 < a.n_rows; r0 += kScan) {
    const int r = r0 + lane * (kScan / 64) + wave, len = r < a.n_rows ? a.len_in[r] : 0;
    const bool ends = r < a.n_rows && a.release[r] != 0;
    if (r < a.n_rows) a.len_out[r] = ends ? 0 : len;
    uint64_t todo = __ballot(ends);
    while (todo) {
      const int who = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      const int32_t* mine = a.table + (int64_t)(r0 + who * (kScan / 64) + wave) * g.width;
      const int have = held(g, __shfl(len, who, 64));
      for (int j0 = lane; j0 < have; j0 += 8 * 64) {
        int id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = mine[min(j0 + u * 64, have - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (j0 + u * 64 < have && (unsigned)id[u] < (unsigned)g.n_blocks) atomicSub(left + id[u], 1);
      }
    }
  }
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
  // the whole blocks, eight entries of a thread at once, of all forks together
  __shared__ int of_fork[3][kScan];
  of_fork[0][i] = full, of_fork[1][i] = src, of_fork[2][i] = dst;
  __syncthreads();
  constexpr int N = 8;
  const unsigned width = (unsigned)g.width, all = (unsigned)a.n_forks * width;
  for (unsigned x0 = threadIdx.x; x0 < all; x0 += N * kScan) {
    int id[N];
    int64_t to[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const unsigned x = min(x0 + u * kScan, all - 1), f = x / width, j = x - f * width;
      const bool in = x0 + u * kScan < all && (int)j < of_fork[0][f];
      to[u] = in ? (int64_t)of_fork[2][f] * g.width + j : -1;
      id[u] = in ? a.table[(int64_t)of_fork[1][f] * g.width + j] : -1;
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (to[u] < 0) continue;
      a.table[to[u]] = id[u];
      if ((unsigned)id[u] < (unsigned)g.n_blocks) atomicAdd(count + id[u], 1);
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
#pragma unroll 4
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
  __shared__ uint16_t counts[2][kAtOnce][kScan / 64];
  uint32_t goes, holes;
  uint32_t g0 = chunks_before(a.work, 2, 0, &goes, part), h0 = chunks_before(a.work, 2, 1, &holes, part);
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
  Picked go{counts[0], part}, hole{counts[1], part};
  for (int b0 = c.first; b0 < c.last; b0 += kAtOnce * kScan) {
    bool goes_b[kAtOnce], hole_b[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int b = b0 + k * kScan + (int)threadIdx.x;
      const bool used = a.ids[min(b, c.last - 1)] == kUsed;
      goes_b[k] = used && b < c.last && b >= a.keep;
      hole_b[k] = !used && b < c.last && b < a.keep;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) go.count(k, goes_b[k]), hole.count(k, hole_b[k]);
    const uint32_t n_go = go.scan(kAtOnce), n_hole = hole.scan(kAtOnce);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int b = b0 + k * kScan + (int)threadIdx.x;
      const uint32_t i = g0 + go.place(k, goes_b[k]), j = h0 + hole.place(k, hole_b[k]);
      if (goes_b[k]) a.from[i] = b, a.ids[b] = (int)i;
      if (hole_b[k] && j < goes) a.to[j] = b, a.ids[b] = kTaken - (int)j;
      if (hole_b[k] && j >= goes) a.ring_out[j - goes] = b;
    }
    g0 += n_go, h0 += n_hole;
    __syncthreads();
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
  // counts by new id: of what stays, and of what comes; 0 for what is free
  for (int b0 = threadIdx.x; b0 < g.n_blocks; b0 += 8 * kScan) {
    int n[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) n[u] = a.shared_in[min(b0 + u * kScan, g.n_blocks - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int b = b0 + u * kScan;
      if (b >= g.n_blocks) break;
      if (b < a.keep ? state[b] == kIn : state[b] < kOut) a.shared_out[b < a.keep ? b : hole_id[state[b]]] = n[u];
    }
  }
  for (uint32_t j = n_goes + threadIdx.x; j < n_holes; j += kScan) a.shared_out[hole_id[j]] = 0;
  each_entry(
      g, a.table, a.n_rows, [&](int r) { return held(g, a.len[r]); },
      [&](unsigned at, int id) {
        // (a free block, which no row should hold, stays as it is)
        if (id >= a.keep && state[id] < kOut) a.table[at] = hole_id[state[id]];
      });
}

// A workgroup's step: 16 KiB of a pair of blocks in one layer, four loads of a thread on their way at once (its
// registers are plain vectors and filled without a condition: what may be missing would go through LDS, one by one).
// Stores past the caches: 900 blocks of 131 KB 51 -> 47 us (5.1 TB/s), 800 of 66 KB in two layers 47 -> 40; eight loads 52 us.
// (A streaming kernel reaches 6.2 TB/s.  An 8-bit block is 16 bytes a head longer than whole steps, so its last step copies next to
// nothing: 8 heads of 16 tokens of 128 channels are 2,056 vectors, two steps and 8 vectors.)  Pairs that are left out are read and
// passed over one by one: a list of 524,288 for 5 layers with 20 pairs takes 314 us, one of 32,768 22, the 20 alone 3.5 (from Python).
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
  if (g.n_blocks <= kOneBlocks && a.n_forks <= kScan && (int64_t)a.n_forks * g.width <= kOneEntries) {
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
  if (g.n_blocks <= kOneBlocks && (int64_t)a.n_rows * g.width <= kOneEntries) {
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
