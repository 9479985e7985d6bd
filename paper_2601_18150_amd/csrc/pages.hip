// Pages of the KV cache: copying them, giving a sequence's pages to the sequences forked from it,
// freeing a sequence's, and moving the pages in use together.  One call covers the caches of many
// layers: their base pointers travel in the kernel arguments, kCachesPerLaunch at a time, so that
// the copies of one layer's few pages and of all layers' are one launch.  A cache is `num_blocks`
// blocks of `block_bytes`; what the bytes are does not matter here.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "launch.hpp"

namespace fp8rl {
namespace {

constexpr int kThreads = 256;
constexpr int kPageTokens = 16;

struct Caches {
  uint8_t* base[kCachesPerLaunch];
  int64_t block_bytes, num_blocks;
};

__device__ __forceinline__ bool in_cache(const Caches& c, int blk) { return blk >= 0 && (int64_t)blk < c.num_blocks; }

// A workgroup copies one block of several caches, kSlices slices of 4 KiB all told: every load is on its way
// before the first is stored, which with fewer bytes in flight a CU are two latencies in a row.  Bound by
// HBM: 112 tails of 16 KiB in 72 caches, 132 MB written, the seven parents' read once: 37.2 us for a cache at a time, 26.8
// so (5.2 TB/s); compaction that moves half of 12 layers' pages, 801 MB read and written: 170 / 167 us, the rate of a
// large copy.
constexpr int kSlices = 8;
constexpr int kSliceBytes = 16 * kThreads;

__host__ __device__ inline int64_t slices_of(int64_t block_bytes) { return (block_bytes + kSliceBytes - 1) / kSliceBytes; }
// caches whose blocks a workgroup copies together
__host__ __device__ inline int caches_per_group(int64_t block_bytes) {
  const int64_t s = slices_of(block_bytes);
  return s >= kSlices ? 1 : s < 1 ? kSlices : (int)(kSlices / s);
}

// Block dst = block src of the caches of column x.
__device__ __forceinline__ void copy_block(const Caches& c, int x, int count, int src, int dst) {
  const int per = caches_per_group(c.block_bytes), spb = (int)slices_of(c.block_bytes);
  const int first = x * per, total = min(per, count - first) * spb;
  const int64_t lane = threadIdx.x * 16;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  for (int s0 = 0; s0 < total; s0 += kSlices) {
    u32x4 v[kSlices];
#pragma unroll
    for (int u = 0; u < kSlices; ++u) {                    // (past the end: the last slice, the last bytes again)
      const int s = min(s0 + u, total - 1), i = s / spb;   // (uniform)
      const int64_t off = min((int64_t)(s - i * spb) * kSliceBytes + lane, c.block_bytes - 16);
      v[u] = *reinterpret_cast<const u32x4*>(c.base[first + i] + src * c.block_bytes + off);
    }
#pragma unroll
    for (int u = 0; u < kSlices; ++u) {
      const int s = s0 + u, i = s / spb;
      const int64_t off = (int64_t)(s - i * spb) * kSliceBytes + lane;
      if (s < total && off < c.block_bytes)
        *reinterpret_cast<u32x4*>(c.base[first + i] + dst * c.block_bytes + off) = v[u];
    }
  }
}

// Workgroup (column of caches, pair).
__global__ __launch_bounds__(kThreads) void copy_blocks_kernel(const Caches c, int caches, const int32_t* __restrict__ src,
                                                              const int32_t* __restrict__ dst, int64_t count) {
  for (int64_t i = blockIdx.y; i < count; i += gridDim.y) {
    const int s = src[i], d = dst[i];
    if (in_cache(c, s) && in_cache(c, d) && s != d) copy_block(c, blockIdx.x, caches, s, d);
  }
}

struct ForkArgs {
  int32_t* table;
  int64_t rows;
  int max_blocks;
  int32_t* seq_lens;
  int32_t* refs;
  const int32_t* parents;
  const int32_t* children;
  const int32_t* new_blocks;
  int64_t count;
};

// Workgroup (column of caches, fork): the parent's last page, where it is partly filled, copied to the child's
// own; column 0's also writes the child's row, length and the counts (sums of whole numbers: the
// order in which forks of one parent add to them does not show).
__global__ __launch_bounds__(kThreads) void fork_kernel(const Caches c, int caches, const ForkArgs p, bool tables) {
  for (int64_t i = blockIdx.y; i < p.count; i += gridDim.y) {
    const int parent = p.parents[i], child = p.children[i];
    if (parent < 0 || parent >= p.rows || child < 0 || child >= p.rows || parent == child) continue;
    const int len = (int)min((int64_t)max(p.seq_lens[parent], 0), (int64_t)p.max_blocks * kPageTokens);
    const int whole = len / kPageTokens;
    const int32_t* from = p.table + parent * (int64_t)p.max_blocks;
    const bool tail = len % kPageTokens != 0;
    int src = 0, dst = 0;
    if (tail) {
      src = from[whole];
      dst = p.new_blocks[i];
      if (!in_cache(c, src) || !in_cache(c, dst)) continue;            // no page for it: no fork
      if (src != dst) copy_block(c, blockIdx.x, caches, src, dst);
    }
    if (!tables || blockIdx.x != 0) continue;
    int32_t* to = p.table + child * (int64_t)p.max_blocks;
    for (int e = threadIdx.x; e < whole; e += kThreads) {
      const int blk = from[e];
      to[e] = blk;
      if (in_cache(c, blk)) atomicAdd(p.refs + blk, 1);
    }
    if (threadIdx.x == 0) {
      if (tail) {
        to[whole] = dst;
        atomicAdd(p.refs + dst, 1);
      }
      p.seq_lens[child] = len;
    }
  }
}

// One workgroup per sequence; its length is taken (and made 0) once, so that a sequence named
// twice is freed once.
__global__ __launch_bounds__(kThreads) void free_kernel(const int32_t* __restrict__ table, int64_t rows, int max_blocks,
                                                       int32_t* seq_lens, int32_t* refs, int64_t num_blocks,
                                                       const int32_t* __restrict__ sequences) {
  __shared__ int len;
  const int s = sequences[blockIdx.x];
  if (s < 0 || s >= rows) return;
  if (threadIdx.x == 0) len = atomicExch(seq_lens + s, 0);
  __syncthreads();
  const int used = (int)min(((int64_t)max(len, 0) + kPageTokens - 1) / kPageTokens, (int64_t)max_blocks);
  for (int e = threadIdx.x; e < used; e += kThreads) {
    const int blk = table[s * (int64_t)max_blocks + e];
    if (blk >= 0 && blk < num_blocks) atomicSub(refs + blk, 1);
  }
}

// Compaction.  With L blocks in use, the k-th free block below L (from the bottom) takes the k-th
// block in use from the top: as many as there are blocks in use from L on, and no block moves that
// need not.  Three launches: blocks in use per chunk; each chunk's ranks from those; the moves.
constexpr int kChunkPerThread = 8;
constexpr int kChunk = kThreads * kChunkPerThread;

__device__ __forceinline__ int block_sum(int v, int* red) {              // of 256 threads, to all of them
  v = wave_inclusive_sum(v);
  if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = v;
  __syncthreads();
  const int s = red[0] + red[1] + red[2] + red[3];
  __syncthreads();
  return s;
}

__global__ __launch_bounds__(kThreads) void count_kernel(const int32_t* __restrict__ refs, int64_t num_blocks,
                                                        int32_t* __restrict__ chunk_live) {
  __shared__ int red[4];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kChunkPerThread; ++i) {
    const int64_t b = (int64_t)blockIdx.x * kChunk + i * kThreads + threadIdx.x;
    n += b < num_blocks && refs[b] > 0;
  }
  n = block_sum(n, red);
  if (threadIdx.x == 0) chunk_live[blockIdx.x] = n;
}

struct CompactPlan {
  int32_t* chunk_live;     // blocks in use of each chunk
  int32_t* moves;          // [1]
  int32_t* holes;          // k-th free block below L, from the bottom
  int32_t* movers;         // k-th block in use from the top
  int32_t* rank;           // of blocks from L on: their k, or -1 where free
};

__global__ __launch_bounds__(kThreads) void plan_kernel(const int32_t* __restrict__ refs, int64_t num_blocks, int chunks,
                                                       const CompactPlan p, int32_t* __restrict__ live) {
  __shared__ int red[4];
  __shared__ int wave_sum[4];
  int all = 0, before = 0;
  for (int i = threadIdx.x; i < chunks; i += kThreads) {
    const int n = p.chunk_live[i];
    all += n;
    before += i < (int)blockIdx.x ? n : 0;
  }
  all = block_sum(all, red);
  before = block_sum(before, red);
  // (thread t has blocks t * 8 .. of the chunk, so that ranks run along the threads)
  const int64_t b0 = (int64_t)blockIdx.x * kChunk + threadIdx.x * kChunkPerThread;
  int used[kChunkPerThread], mine = 0;
#pragma unroll
  for (int i = 0; i < kChunkPerThread; ++i) {
    used[i] = b0 + i < num_blocks && refs[b0 + i] > 0;
    mine += used[i];
  }
  const int upto = wave_inclusive_sum(mine);
  if ((threadIdx.x & 63) == 63) wave_sum[threadIdx.x >> 6] = upto;
  __syncthreads();
  int rank = before + upto - mine;                       // blocks in use in front of b0
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) rank += wave_sum[w];
#pragma unroll
  for (int i = 0; i < kChunkPerThread; ++i) {
    const int64_t b = b0 + i;
    if (b < num_blocks) {
      if (b == all) *p.moves = all - rank;               // blocks in use from L on
      if (b < all) {
        if (!used[i]) p.holes[b - rank] = (int32_t)b;
      } else {
        const int k = all - 1 - rank;
        p.rank[b] = used[i] ? k : -1;
        if (used[i]) p.movers[k] = (int32_t)b;
      }
    }
    rank += used[i];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *live = all;
    if (all == num_blocks) *p.moves = 0;                 // (no block L)
  }
}

struct CompactArgs {
  int32_t* table;
  int64_t rows;
  int max_blocks;
  const int32_t* seq_lens;
  int32_t* refs;
  const int32_t* live;
  CompactPlan plan;
};

// Workgroup (column of caches, k), k + gridDim.y, ..: a move; the column behind them (`tables`): the
// counts of the blocks that moved, and the rows that name them.
__global__ __launch_bounds__(kThreads) void move_kernel(const Caches c, int caches, int columns, const CompactArgs p) {
  const int moves = *p.plan.moves;
  if ((int)blockIdx.x < columns) {
    for (int k = blockIdx.y; k < moves; k += gridDim.y)
      copy_block(c, blockIdx.x, caches, p.plan.movers[k], p.plan.holes[k]);
    return;
  }
  for (int64_t k = (int64_t)blockIdx.y * kThreads + threadIdx.x; k < moves; k += (int64_t)gridDim.y * kThreads) {
    const int from = p.plan.movers[k];
    p.refs[p.plan.holes[k]] = p.refs[from];
    p.refs[from] = 0;
  }
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const int64_t used = min(((int64_t)max(p.seq_lens[row], 0) + kPageTokens - 1) / kPageTokens, (int64_t)p.max_blocks);
    for (int e = threadIdx.x; e < used; e += kThreads) {
      int32_t* at = p.table + row * p.max_blocks + e;
      const int blk = *at;
      // a block from L on that is in use moves to the hole of its rank; all others stay
      if (moves > 0 && in_cache(c, blk) && blk >= *p.live) {
        const int k = p.plan.rank[blk];
        if (k >= 0) *at = p.plan.holes[k];
      }
    }
  }
}

Caches caches_of(void* const* caches, int64_t first, int64_t count, int64_t block_bytes, int64_t num_blocks) {
  Caches c{};
  for (int64_t i = 0; i < count; ++i) c.base[i] = static_cast<uint8_t*>(caches[first + i]);
  c.block_bytes = block_bytes;
  c.num_blocks = num_blocks;
  return c;
}

// Runs f(caches, how many, first launch?) for every kCachesPerLaunch of them.
template <class F>
hipError_t each_launch(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks, F f) {
  for (int64_t at = 0; at < num_caches; at += kCachesPerLaunch) {
    const int64_t n = num_caches - at < kCachesPerLaunch ? num_caches - at : kCachesPerLaunch;
    f(caches_of(caches, at, n, block_bytes, num_blocks), (unsigned)n, at == 0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

unsigned columns_of(unsigned caches, int64_t block_bytes) {
  const unsigned per = (unsigned)caches_per_group(block_bytes);
  return (caches + per - 1) / per;
}

unsigned grid_y(int64_t n) { return (unsigned)(n < 32768 ? n : 32768); }

}  // namespace

hipError_t launch_kv_copy_blocks(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks,
                                 const int32_t* src, const int32_t* dst, int64_t count, hipStream_t stream) {
  return each_launch(caches, num_caches, block_bytes, num_blocks, [&](const Caches& c, unsigned n, bool) {
    hipLaunchKernelGGL(copy_blocks_kernel, dim3(columns_of(n, block_bytes), grid_y(count)), dim3(kThreads), 0, stream, c,
                       (int)n, src, dst, count);
  });
}

hipError_t launch_kv_fork(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks, int32_t* table,
                          int64_t rows, int64_t max_blocks, int32_t* seq_lens, int32_t* refs, const int32_t* parents,
                          const int32_t* children, const int32_t* new_blocks, int64_t count, hipStream_t stream) {
  const ForkArgs p{table, rows, (int)max_blocks, seq_lens, refs, parents, children, new_blocks, count};
  return each_launch(caches, num_caches, block_bytes, num_blocks, [&](const Caches& c, unsigned n, bool first) {
    hipLaunchKernelGGL(fork_kernel, dim3(block_bytes > 0 ? columns_of(n, block_bytes) : 1, grid_y(count)), dim3(kThreads), 0,
                       stream, c, (int)n, p, first);
  });
}

hipError_t launch_kv_free(const int32_t* table, int64_t rows, int64_t max_blocks, int32_t* seq_lens, int32_t* refs,
                          int64_t num_blocks, const int32_t* sequences, int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)count), dim3(kThreads), 0, stream, table, rows, (int)max_blocks, seq_lens,
                     refs, num_blocks, sequences);
  return hipGetLastError();
}

static int64_t chunks_of(int64_t num_blocks) { return (num_blocks + kChunk - 1) / kChunk; }

int64_t kv_compact_workspace_words(int64_t num_blocks) { return chunks_of(num_blocks) + 1 + 3 * num_blocks; }

hipError_t launch_kv_compact(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks,
                             int32_t* table, int64_t rows, int64_t max_blocks, const int32_t* seq_lens, int32_t* refs,
                             int32_t* live, int32_t* workspace, hipStream_t stream) {
  const int64_t chunks = chunks_of(num_blocks);
  CompactPlan plan;
  plan.chunk_live = workspace;
  plan.moves = workspace + chunks;
  plan.holes = plan.moves + 1;
  plan.movers = plan.holes + num_blocks;
  plan.rank = plan.movers + num_blocks;
  hipLaunchKernelGGL(count_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, stream, refs, num_blocks, plan.chunk_live);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(plan_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, stream, refs, num_blocks, (int)chunks, plan,
                     live);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const CompactArgs p{table, rows, (int)max_blocks, seq_lens, refs, live, plan};
  // enough workgroups for every move that a half-free cache can need, and for the rows
  const int64_t most = num_blocks / 2 > rows ? num_blocks / 2 : rows;
  const unsigned y = (unsigned)(most < 1 ? 1 : most < 1024 ? most : 1024);
  return each_launch(caches, num_caches, block_bytes, num_blocks, [&](const Caches& c, unsigned n, bool first) {
    const unsigned columns = block_bytes > 0 ? columns_of(n, block_bytes) : 0;
    if (columns + first == 0) return;
    hipLaunchKernelGGL(move_kernel, dim3(columns + (first ? 1 : 0), y), dim3(kThreads), 0, stream, c, (int)n, (int)columns,
                       p);
  });
}

}  // namespace fp8rl
