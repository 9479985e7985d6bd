// Decode attention for a batch whose sequences share long prefixes (the samples drawn from one
// prompt).  The queries of a group's members, every head that reads a kv head, are the rows of one
// product against the prefix, whose pages are read once for all of them: in tiles of 128 rows
// (attn_core.hpp), of 32 where they are few (attn_stream.hpp).  What a member has behind the prefix is
// read for its own heads alone, by the same stream.  One launch does both, the prefixes' workgroups first:
// they are bound by arithmetic where groups are large, the others by reading the cache.  A second joins
// the records (attn_merge.hpp).  The grid holds every tile that there may be, and every part of a sequence; what has
// nothing to do lies together at the end of its kind: workgroups go to the XCDs and to the shader engines
// in turn, and a regular pattern of empty ones left half of those idle (4 prefixes of 18000 tokens, 16 members each: 70
// us, 50 so).  16 groups of 16 sequences, 1808 shared tokens and up to 2500 of their own, 32 heads over 8: 719 MB in
// 161 us, 4.5 TB/s, near the rate of a large copy; 4 of 32 with 18000 + up to 1500: 187 MB, 39 GFLOP in 80 us,
// the prefixes' products on 256 workgroups, one a CU, that share no tile.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_core.hpp"
#include "attn_merge.hpp"
#include "attn_stream.hpp"
#include "launch.hpp"

namespace fp8rl {
namespace {

struct SharedArgs {
  const uint16_t* q;
  const uint8_t* k;
  const uint8_t* v;
  int64_t num_blocks;
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_lens;
  int max_seq_len, batch;
  const int32_t* group_offsets;
  const int32_t* prefix_lens;
  int groups, max_prefix_len;
  int kv_heads, group_log2;
  const float* k_scale;
  const float* v_scale;
  float sm_scale;
  uint16_t* out;
  int prefix_tiles, prefix_records, split_keys, record_count;
  float* records;          // (sequence, kv head, record): the prefix's first
  int32_t* prefix;         // of each sequence: tokens of it that are read with its group's
};

// Pages per record of a sequence's own `pages`, divided over `records`; at least 256 tokens.
constexpr int kOwnMinPages = 16;
__device__ __forceinline__ int own_split_pages(int pages, int records) {
  return max((max(pages, 0) + records - 1) / records, kOwnMinPages);
}

__device__ __forceinline__ int clamped_len(const SharedArgs& p, int b) {
  return min(max(p.seq_lens[b], 0), p.max_seq_len);
}

// Smallest over the wave.
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// Rows of a group up to which it takes tiles of 32 (8 groups of 12 / 16 / 24 / 32 with 4 rows each over 4000 tokens, us
// with 32: 56.5 / 61.7 / 72.0 / 96.8, 64: 50.6 / 53.9 / 73.1 / 97.2, 96: 50.6 / 53.0 / 69.9 / 98.1, 128: 50.7 / 53.2 /
// 69.7 / 99.2).
constexpr int kSharedSmall = 96;

// The part of group g that is shared: whole pages of its first member's.
__device__ __forceinline__ int shared_prefix(const SharedArgs& p, int g, int first) {
  return min(min(max(p.prefix_lens[g], 0), p.max_prefix_len), clamped_len(p, first)) / kPageTokens * kPageTokens;
}

// The group of sequence b, or -1: the last offset that is not above b, by 64 probes at a time.
__device__ __forceinline__ int group_of(const SharedArgs& p, int b) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = p.groups + 1;
  for (;;) {
    const int stride = (n + 63) / 64;
    const int i = lo + lane * stride;
    const int below = __popcll(__ballot(i < lo + n && p.group_offsets[min(i, p.groups)] <= b));
    if (below == 0) return -1;
    lo += (below - 1) * stride;
    n = min(stride, p.groups + 1 - lo);
    if (stride == 1) break;
  }
  return lo == p.groups ? -1 : __builtin_amdgcn_readfirstlane(lo);
}

// At most 32 rows (row0 ..) of the `rows` queries of sequences first .. against keys begin .. end - 1: record
// `index` of each.
__device__ __forceinline__ void stream_record(const SharedArgs& p, const AttnRow& row, int begin, int end, int len,
                                              const PagedKv& pages, int first, int row0, int rows, int index, float sscale,
                                              const TileLds& lds, StreamStats& stats) {
  const int group = 1 << p.group_log2, kvh = pages.kvh;
  const int floats = (kHeadDim << p.group_log2) + (2 * group + 3) / 4 * 4;
  const float c = score_factor(sscale);
  AttnAcc acc;
  attn_init(acc);
  bf16x8 q[8];
  attn_load_q(row, q);
  attn_stream(acc, q, row, begin, end, c, pages, len, lds);
  stream_join(acc, c, lds, stats, [&](int i, int part, const float4 (&o)[4], float m, float l) {
    const int r = row0 + i, h = r & (group - 1);
    if (r >= rows) return;
    float* rec = p.records + (((int64_t)(first + (r >> p.group_log2)) * p.kv_heads + kvh) * p.record_count + index) * floats;
#pragma unroll
    for (int n = 0; n < 4; ++n) *reinterpret_cast<float4*>(rec + h * kHeadDim + 16 * part + 4 * n) = o[n];
    if (part == 0) {
      rec[group * kHeadDim + h] = fmaxf(m * sscale, kNoScore);
      rec[group * kHeadDim + group + h] = l;
    }
  });
}

__global__ __launch_bounds__(64 * kAttnWaves, 2) void attn_shared_kernel(const SharedArgs p) {
  __shared__ __attribute__((aligned(16))) uint8_t lds_keys[kRingBytes];
  __shared__ __attribute__((aligned(16))) uint8_t lds_values[kRingBytes];
  __shared__ StreamStats stats;
  __shared__ int smallest[kAttnWaves];
  const TileLds lds{lds_keys, lds_values};
  const int kvh = blockIdx.x % p.kv_heads, item = blockIdx.x / p.kv_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = 1 << p.group_log2;
  const float sscale = p.k_scale[0] * p.sm_scale;
  if (item >= p.prefix_tiles * p.prefix_records) {
    // a sequence's own tokens: record `part` of them, for its own heads
    const int own = item - p.prefix_tiles * p.prefix_records, parts = p.record_count - p.prefix_records;
    const int b = own % p.batch, part = own / p.batch;
    const int g = group_of(p, b);
    const int len = clamped_len(p, b);
    const int from = g < 0 ? 0 : shared_prefix(p, g, min(max(p.group_offsets[g], 0), p.batch - 1));
    const int pages = (len + kPageTokens - 1) / kPageTokens - from / kPageTokens;
    const int per = own_split_pages(pages, parts) * kPageTokens;
    const int begin = from + part * per, end = min(len, begin + per);
    if (begin >= end) return;
    AttnRow row;
    const int head = kvh * group + min(lane & 31, group - 1);
    row.q = p.q + ((int64_t)b * p.kv_heads * group + head) * kHeadDim;
    row.limit = end - 1;                                // (the next record's keys are its own)
    const PagedKv kv{p.k, p.v, p.block_table + (int64_t)b * p.max_blocks, p.num_blocks, p.max_blocks, p.kv_heads, kvh};
    stream_record(p, row, begin, end, len, kv, b, 0, group, p.prefix_records + part, sscale, lds, stats);
    return;
  }
  // a prefix: rows are member r / G of the group, query head r % G of the kv head's
  const int split = item % p.prefix_records;
  if (blockIdx.x == 0) {                                // sequences of no group share nothing
    const int lo = p.group_offsets[0], hi = p.group_offsets[p.groups];
    for (int b = threadIdx.x; b < p.batch; b += 64 * kAttnWaves)
      if (b < lo || b >= hi) p.prefix[b] = 0;
  }
  TileOf at;
  if (!find_tile(p.group_offsets, p.groups, p.batch, p.group_log2, kSharedSmall, kAttnShift, item / p.prefix_records, at)) return;
  at.to_scalars();
  const int rows = at.n << p.group_log2;
  const bool small = rows <= kSharedSmall;
  const int row0 = at.index * (small ? kStreamRows : kAttnRows);
  const int prefix = shared_prefix(p, at.b, at.first);
  const int r = row0 + (small ? 0 : kRowsPerWave * wave) + (lane & 31);
  const int seq = at.first + (min(r, rows - 1) >> p.group_log2);
  const int head = kvh * group + (min(r, rows - 1) & (group - 1));
  if (split == 0 && kvh == 0 && (r & (group - 1)) == 0 && r < rows && lane < 32) p.prefix[seq] = prefix;
  const int begin = split * p.split_keys, end = min(prefix, begin + p.split_keys);
  if (begin >= end) return;
  AttnRow row;
  row.q = p.q + ((int64_t)seq * p.kv_heads * group + head) * kHeadDim;
  row.limit = min(clamped_len(p, seq), prefix) - 1;     // (a member may be shorter than the prefix)
  const PagedKv pages{p.k, p.v, p.block_table + (int64_t)at.first * p.max_blocks, p.num_blocks, p.max_blocks, p.kv_heads, kvh};
  if (small) {
    stream_record(p, row, begin, end, prefix, pages, at.first, row0, rows, split, sscale, lds, stats);
    return;
  }
  const int least = wave_min(row.limit);
  if (lane == 0) smallest[wave] = least;
  __syncthreads();
  row.all_limit = min(min(min(smallest[0], smallest[1]), min(smallest[2], smallest[3])), end - 1);
  const float c = score_factor(sscale);
  AttnAcc acc;
  attn_init(acc);
  bf16x8 q[8];
  attn_load_q(row, q);
  attn_run_fp8(acc, q, row, begin, end, c, pages, prefix, lds);
  if (row.all_limit < end - 1) attn_redo(acc, q, row, begin, end, end, end, c, Fp8Tokens{pages});
  const float l = half_sum(acc.l);
  const bool valid = r < rows;
  const int floats = (kHeadDim << p.group_log2) + (2 * group + 3) / 4 * 4;
  float* rec = p.records + (((int64_t)seq * p.kv_heads + kvh) * p.record_count + split) * floats;
  const int h = head & (group - 1);
  attn_store_f32(acc, rec + h * kHeadDim, valid);
  if (valid && lane < 32) {
    rec[group * kHeadDim + h] = fmaxf(acc.m * sscale, kNoScore);
    rec[group * kHeadDim + group + h] = l;
  }
}

// A sequence's records joined: kFew: eight (sequence, query head) pairs a workgroup, 32 lanes each; otherwise one.
template <int kG, bool kFew>
__global__ __launch_bounds__(kFew ? 256 : 32 * kMergeSets) void attn_shared_merge_kernel(const SharedArgs p) {
  const int pair = kFew ? blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  const int heads = p.kv_heads * kG;
  const int b = pair / heads, head = pair % heads;
  if (b >= p.batch) return;
  const int kvh = head / kG, h = head % kG;
  const int n = clamped_len(p, b), from = p.prefix[b];
  const int np = min((min(n, from) + p.split_keys - 1) / p.split_keys, p.prefix_records);
  const int own = max((n + kPageTokens - 1) / kPageTokens - from / kPageTokens, 0);
  const int per = own_split_pages(own, p.record_count - p.prefix_records);
  const int ns = np + (own + per - 1) / per;
  const float* base = p.records + ((int64_t)b * p.kv_heads + kvh) * p.record_count * partial_floats<kG>();
  uint16_t* out = p.out + (int64_t)pair * kHeadDim;
  if constexpr (kFew)
    merge_few_records<kG>(base, ns, np, p.prefix_records - np, h, p.v_scale, out);
  else
    merge_records<kG>(base, ns, np, p.prefix_records - np, h, p.v_scale, out);
}

}  // namespace

// Records of a sequence and kv head.  The prefixes' keys go into as many shares as end first (attn_shares), where two
// workgroups on a CU take twice as long as one, no longer than it takes to read the cache at 4.7 TB/s, and records,
// which the joining launch reads again, count three times; what the prefixes leave free goes to the sequences' own tokens
// meanwhile.  (Against 256 workgroups, rounded up, us: 6 x 11 sequences of 11040 + 8 tokens, 64 heads over 8, 79 -> 60; 3 x
// 21 of 11936 + 74, 32 over 4, 56 -> 49; 9 x 16 of 9424 + 4, 16 over 8, 50 -> 44; 6 x 23 of 11936 + 1416, 32 over 8,
// 128 -> 132; 4 x 32 of 18000 + 1500 and 16 x 16 of 1808 + 2500 as before, 78 and 160.  512 workgroups: 91 and 170.)
// Own tokens are split where the sequences are fewer than 1024, 256 tokens each at least (8 x 16 of 4000 + up to 800
// tokens, for 512 / 1024 / 2048: 51 / 50 / 55; 4 x 32 as above 80 / 80 / 87).
SharedSplit attn_shared_split(int64_t batch, int64_t groups, int64_t group, int64_t kv_heads, int64_t max_prefix_len,
                              int64_t max_seq_len) {
  const int64_t runs = groups < batch ? groups : batch;
  const int64_t wgs = attn_tile_guess(batch * group, runs, kSharedSmall) * kv_heads;
  const bool small = batch * group <= runs * kSharedSmall;
  const double record = 3 * batch * group * kv_heads * (4.0 * (kHeadDim + 2)) / 5e6;
  const double read = runs * max_prefix_len * kv_heads * (2.0 * kHeadDim) / 4.7e6;
  const ShareCost cost{small ? 0.47 : 1.5, small ? 0.94 : 3.0, 0.0, record, 1.0, read};
  const int64_t keys = attn_share(max_prefix_len, attn_shares(wgs, max_prefix_len, cost));
  const int64_t splits = (max_prefix_len + keys - 1) / keys;
  const int64_t pairs = batch * kv_heads;
  int64_t own = (1024 + pairs - 1) / pairs;
  const int64_t most = (max_seq_len + kOwnMinPages * kPageTokens - 1) / (kOwnMinPages * kPageTokens);
  own = own > most ? most : own;
  SharedSplit s;
  s.prefix_records = splits > 1 ? (int)splits : 1;
  s.split_keys = (int)keys;
  s.records = s.prefix_records + (own > 1 ? (int)own : 1);
  s.partial_floats = (int)(group * kHeadDim + (2 * group + 3) / 4 * 4);
  return s;
}

static int64_t prefix_tiles(int64_t batch, int64_t groups, int64_t group) {
  return attn_tile_bound(batch * group, groups, batch, kSharedSmall, kAttnShift);
}

int64_t attn_shared_workgroups(int64_t batch, int64_t groups, int64_t group, int64_t kv_heads, int64_t max_prefix_len,
                               int64_t max_seq_len) {
  const SharedSplit sp = attn_shared_split(batch, groups, group, kv_heads, max_prefix_len, max_seq_len);
  return kv_heads * (prefix_tiles(batch, groups, group) * sp.prefix_records + batch * (sp.records - sp.prefix_records));
}

hipError_t launch_attention_decode_shared(const uint16_t* q, const uint8_t* k_cache, const uint8_t* v_cache,
                                          int64_t num_blocks, const int32_t* block_table, int64_t max_blocks,
                                          const int32_t* seq_lens, int64_t batch, const int32_t* group_offsets,
                                          const int32_t* prefix_lens, int64_t groups, int64_t max_prefix_len,
                                          int64_t q_heads, int64_t kv_heads, int64_t max_seq_len, const float* k_scale,
                                          const float* v_scale, float sm_scale, uint16_t* out, float* workspace,
                                          hipStream_t stream) {
  const int64_t group = q_heads / kv_heads;
  const SharedSplit sp = attn_shared_split(batch, groups, group, kv_heads, max_prefix_len, max_seq_len);
  SharedArgs p{};
  p.q = q, p.k = k_cache, p.v = v_cache, p.num_blocks = num_blocks, p.block_table = block_table;
  p.max_blocks = (int)max_blocks, p.seq_lens = seq_lens, p.max_seq_len = (int)max_seq_len, p.batch = (int)batch;
  p.group_offsets = group_offsets, p.prefix_lens = prefix_lens, p.groups = (int)groups;
  p.max_prefix_len = (int)max_prefix_len, p.kv_heads = (int)kv_heads, p.group_log2 = group_log2_of(group);
  p.k_scale = k_scale, p.v_scale = v_scale, p.sm_scale = sm_scale, p.out = out;
  p.prefix_tiles = (int)prefix_tiles(batch, groups, group);
  p.prefix_records = sp.prefix_records, p.split_keys = sp.split_keys, p.record_count = sp.records;
  p.records = workspace;
  p.prefix = reinterpret_cast<int32_t*>(workspace + batch * kv_heads * sp.records * sp.partial_floats);
  hipLaunchKernelGGL(attn_shared_kernel,
                     dim3((unsigned)attn_shared_workgroups(batch, groups, group, kv_heads, max_prefix_len, max_seq_len)),
                     dim3(64 * kAttnWaves), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool few = sp.records <= kFewRecords;
  const dim3 grid((unsigned)(few ? (batch * q_heads + 7) / 8 : batch * q_heads)), block(few ? 256 : 32 * kMergeSets);
#define FP8RL_MERGE(G)                                                                                            \
  if (group == G) {                                                                                               \
    if (few) hipLaunchKernelGGL((attn_shared_merge_kernel<G, true>), grid, block, 0, stream, p);                  \
    else hipLaunchKernelGGL((attn_shared_merge_kernel<G, false>), grid, block, 0, stream, p);                     \
  }
  FP8RL_MERGE(1)
  FP8RL_MERGE(2)
  FP8RL_MERGE(4)
  FP8RL_MERGE(8)
#undef FP8RL_MERGE
  return hipGetLastError();
}

}  // namespace fp8rl
