// Blocks that several rows hold: forks, releases, compaction, and the copies they ask for.
//
// Integer arithmetic only, but for the copies.  What has to be in order -- which fork gets which block
// of the ring, the ring's new entries, the k-th block that moves and the k-th place for it -- comes from prefix
// sums over lists or block ids; atomics only count, so that their order does not matter.  A kernel a phase,
// as each needs all of the one before: bound by the launches' latency (2 to 3 us each), then by the arrays of
// n_blocks entries.
#include "kv.h"

namespace wfkv {
namespace {

constexpr int kThreads = 256;
constexpr int kScan = 1024;              // threads of a workgroup that scans
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

// 16 KiB of a pair of blocks in one layer a step of a workgroup.
constexpr int kPiece = 4 * kThreads;

__global__ __launch_bounds__(kThreads) void copy(CopyArgs a, int n_blocks, int vectors, unsigned pieces) {
  const uint64_t all = (uint64_t)pieces * a.n * a.n_layers;
  for (uint64_t x = blockIdx.x; x < all; x += gridDim.x) {
    const unsigned piece = (unsigned)(x % pieces);
    const uint64_t y = x / pieces;
    const int i = (int)(y % (unsigned)a.n), layer = (int)(y / (unsigned)a.n);
    const int from = a.from[i], to = a.to[i];
    if (from == to || (unsigned)from >= (unsigned)n_blocks || (unsigned)to >= (unsigned)n_blocks) continue;
    uint4* base = reinterpret_cast<uint4*>(a.cache + layer * a.layer_stride);
    const uint4* src = base + (int64_t)from * vectors;
    uint4* dst = base + (int64_t)to * vectors;
    const int v0 = (int)(piece * kPiece + threadIdx.x);
    uint4 w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (v0 + k * kThreads < vectors) w[k] = src[v0 + k * kThreads];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (v0 + k * kThreads < vectors) dst[v0 + k * kThreads] = w[k];
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
  const unsigned copies = groups_of(std::max(g.n_blocks, a.n_rows), kScan);
  hipLaunchKernelGGL(fork_grant, dim3(1 + copies), dim3(kScan), 0, s, g, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_forks == 0) return e;
  const int parts = parts_of(g, a.n_forks);
  hipLaunchKernelGGL(fork_rows, dim3((unsigned)a.n_forks * parts), dim3(kThreads), 0, s, g, a, parts);
  return hipGetLastError();
}

hipError_t launch_release(const Geo& g, const ReleaseArgs& a, hipStream_t s) {
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
  const uint64_t all = (uint64_t)pieces * a.n * a.n_layers;
  hipLaunchKernelGGL(copy, dim3((unsigned)std::min<uint64_t>(all, (uint64_t)n_cu * 16)), dim3(kThreads), 0, s, a, g.n_blocks, vectors, pieces);
  return hipGetLastError();
}

}  // namespace wfkv
