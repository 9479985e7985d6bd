// Decode attention for a batch whose sequences share long prefixes (the samples drawn from one
// prompt): the queries of a group's members, every head that reads a kv head, are the rows of one
// product against the prefix, whose pages are read once for all of them (attn_core.hpp); each
// member's tokens behind the prefix are read by the decode kernel (kv.hip); the records of both
// are joined (attn_merge.hpp).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_core.hpp"
#include "attn_merge.hpp"
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
  int prefix_records, split_keys, record_count;
  float* records;          // (sequence, kv head, record): the prefix's first
  int32_t* first_page;     // of each sequence's own part
};

__device__ __forceinline__ int clamped_len(const SharedArgs& p, int b) {
  return min(max(p.seq_lens[b], 0), p.max_seq_len);
}

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// Rows: member r / G of the group, query head r % G of the kv head's.
__global__ __launch_bounds__(64 * kAttnWaves, 2) void attn_shared_prefix_kernel(const SharedArgs p) {
  __shared__ __attribute__((aligned(16))) uint8_t lds_keys[kTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t lds_values[kTileBytes];
  __shared__ int smallest[kAttnWaves];
  const TileLds lds{lds_keys, lds_values};
  const int kvh = blockIdx.x % p.kv_heads, split = blockIdx.y;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && split == 0) {                  // sequences of no group share nothing
    const int lo = p.group_offsets[0], hi = p.group_offsets[p.groups];
    for (int b = threadIdx.x; b < p.batch; b += 64 * kAttnWaves)
      if (b < lo || b >= hi) p.first_page[b] = 0;
  }
  TileOf at;
  if (!find_tile(p.group_offsets, p.groups, p.batch, p.group_log2, blockIdx.x / p.kv_heads, at)) return;
  at.to_scalars();
  const int group = 1 << p.group_log2;
  const int rows = at.n << p.group_log2, row0 = at.index * kAttnRows;
  // the part that is shared: whole pages of the first member's
  const int prefix = min(min(max(p.prefix_lens[at.b], 0), p.max_prefix_len), clamped_len(p, at.first)) / kPageTokens * kPageTokens;
  const int r = row0 + kRowsPerWave * wave + (lane & 31);
  const int seq = at.first + (min(r, rows - 1) >> p.group_log2);
  const int head = kvh * group + (min(r, rows - 1) & (group - 1));
  if (split == 0 && kvh == 0 && (r & (group - 1)) == 0 && r < rows && lane < 32) p.first_page[seq] = prefix / kPageTokens;
  const int begin = split * p.split_keys, end = min(prefix, begin + p.split_keys);
  if (begin >= end) return;
  AttnRow row;
  row.q = p.q + ((int64_t)seq * p.kv_heads * group + head) * kHeadDim;
  row.limit = min(clamped_len(p, seq), prefix) - 1;     // (a member may be shorter than the prefix)
  row.wave_last = -wave_min(-row.limit);
  const int least = wave_min(row.limit);
  if (lane == 0) smallest[wave] = least;
  __syncthreads();
  row.all_limit = min(min(min(smallest[0], smallest[1]), min(smallest[2], smallest[3])), end - 1);

  AttnAcc acc;
  attn_init(acc);
  bf16x8 q[8];
  attn_load_q(row, q);
  const float sscale = p.k_scale[0] * p.sm_scale;
  const float c = fmaxf(sscale * 1.4426950408889634f, 1.17549435e-38f);   // (0 x -inf would be NaN)
  const PagedKv pages{p.k, p.v, p.block_table + (int64_t)at.first * p.max_blocks, p.num_blocks, p.max_blocks, p.kv_heads, kvh};
  attn_run_fp8(acc, q, row, begin, end, c, pages, prefix, lds);
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

// One workgroup per (query head, sequence).
template <int kG>
__global__ __launch_bounds__(32 * kMergeSets) void attn_shared_merge_kernel(const SharedArgs p) {
  const int head = blockIdx.x, b = blockIdx.y;
  const int kvh = head / kG, h = head % kG;
  const int n = clamped_len(p, b), from = max(p.first_page[b], 0);
  const int shared = min(n, from * kPageTokens);
  const int np = min((shared + p.split_keys - 1) / p.split_keys, p.prefix_records);
  const int own = max((n + kPageTokens - 1) / kPageTokens - from, 0);
  const int per = rest_split_pages(n, from, p.record_count - p.prefix_records);
  const int ns = np + (own + per - 1) / per;
  const float* base = p.records + ((int64_t)b * p.kv_heads + kvh) * p.record_count * partial_floats<kG>();
  merge_records<kG>(base, ns, np, p.prefix_records - np, h, p.v_scale, p.out + ((int64_t)b * p.kv_heads * kG + head) * kHeadDim);
}

}  // namespace

// Records of a sequence and kv head: the prefix's keys are split where its row tiles alone are too
// few for the 512 workgroups that the chip holds, 256 keys each at least; the rest as a decode
// step's keys are.
SharedSplit attn_shared_split(int64_t batch, int64_t groups, int64_t group, int64_t kv_heads, int64_t max_prefix_len,
                              int64_t max_seq_len) {
  const int64_t wgs = attn_tile_bound(batch * group, groups < batch ? groups : batch) * kv_heads;
  int64_t splits = wgs > 0 ? (512 + wgs - 1) / wgs : 1;
  int64_t keys = (max_prefix_len + splits - 1) / splits;
  keys = (keys + kTileKeys - 1) / kTileKeys * kTileKeys;
  if (keys < 256) keys = 256;
  splits = (max_prefix_len + keys - 1) / keys;
  SharedSplit s;
  s.prefix_records = splits > 1 ? (int)splits : 1;
  s.split_keys = (int)keys;
  s.records = s.prefix_records + attn_rest_records(batch, kv_heads, group, max_seq_len);
  s.partial_floats = (int)(group * kHeadDim + (2 * group + 3) / 4 * 4);
  return s;
}

int64_t attn_shared_workgroups(int64_t batch, int64_t groups, int64_t group, int64_t kv_heads) {
  return attn_tile_bound(batch * group, groups < batch ? groups : batch) * kv_heads;
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
  p.prefix_records = sp.prefix_records, p.split_keys = sp.split_keys, p.record_count = sp.records;
  p.records = workspace;
  p.first_page = reinterpret_cast<int32_t*>(workspace + batch * kv_heads * sp.records * sp.partial_floats);
  hipLaunchKernelGGL(attn_shared_prefix_kernel,
                     dim3((unsigned)attn_shared_workgroups(batch, groups, group, kv_heads), (unsigned)sp.prefix_records),
                     dim3(64 * kAttnWaves), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = launch_attention_decode_rest(q, k_cache, v_cache, num_blocks, block_table, max_blocks, seq_lens, batch, group,
                                   kv_heads, max_seq_len, k_scale, v_scale, sm_scale, p.first_page, sp.prefix_records,
                                   sp.records, workspace, stream);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)q_heads, (unsigned)batch), block(32 * kMergeSets);
  if (group == 1) hipLaunchKernelGGL((attn_shared_merge_kernel<1>), grid, block, 0, stream, p);
  if (group == 2) hipLaunchKernelGGL((attn_shared_merge_kernel<2>), grid, block, 0, stream, p);
  if (group == 4) hipLaunchKernelGGL((attn_shared_merge_kernel<4>), grid, block, 0, stream, p);
  if (group == 8) hipLaunchKernelGGL((attn_shared_merge_kernel<8>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace fp8rl
