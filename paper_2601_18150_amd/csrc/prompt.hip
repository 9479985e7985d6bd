// Causal attention over whole prompts (packed sequences of different lengths) and over chunks of
// prompts against the paged FP8 cache; the tiles' arithmetic is in attn_core.hpp.
//
// A workgroup takes 128 rows (64 or 32 where they are few) of one (sequence, kv head): row r is token r / G of the sequence and
// query head r % G of those that read the kv head, so that a prompt's short tiles at the diagonal
// waste few keys, a chunk of a few tokens fills a tile G times better, and the group's heads read
// each key once.  Every wave finds its tile in the sequences' offsets by itself.  Grid
// (kv head + kv_heads * tile, split): the tiles of a kv head share an XCD's L2 where kv_heads is a
// multiple of eight; tiles with the most keys come first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_core.hpp"
#include "attn_merge.hpp"
#include "attn_stream.hpp"
#include "launch.hpp"

namespace fp8rl {
namespace {

struct PromptArgs {
  const uint16_t* q;
  int64_t ld_q;
  const void* k;               // bf16 rows, or the FP8 key pages
  int64_t ld_k;
  const void* v;
  int64_t ld_v;
  int64_t num_blocks;          // (pages from here on)
  const int32_t* block_table;
  int max_blocks;
  const int32_t* seq_lens;
  int max_seq_len;
  const float* k_scale;
  const float* v_scale;
  const int32_t* cu_seqlens;
  int batch, total, kv_heads, group_log2;
  float sm_scale;
  uint16_t* out;
  int64_t ld_out;
  int splits, split_keys;      // splits > 1: records instead of outputs
  float* records;              // (token, kv head, split)
  int32_t* counts;             // records of each token
};
constexpr int kWritten = -1;   // (count) the token's output is there already

// Rows of a run up to which it takes tiles of 32 (FP8 cache; 16 sequences of 32 heads over 4, 8 / 12 / 16 new tokens, us
// with 32: 43.5 / 45.0 / 46.6, 64: 37.5 / 45.4 / 47.5, 96: 37.3 / 42.2 / 47.7, 128: 37.5 / 42.9 / 50.2).
constexpr int kPromptSmall = 96;

// kHalf (bf16): tiles of 64 rows, of which two waves each take half of the keys.
template <bool kFp8, bool kHalf>
__global__ __launch_bounds__(64 * kAttnWaves, kFp8 ? 2 : 3) void attn_prompt_kernel(const PromptArgs p) {
  // (FP8: the rings of the small tiles)
  __shared__ __attribute__((aligned(16))) uint8_t lds_keys[kFp8 ? kRingBytes : kTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t lds_values[kFp8 ? kRingBytes : kTileBytes];
  const TileLds lds{lds_keys, lds_values};
  const int kvh = blockIdx.x % p.kv_heads, tiles = gridDim.x / p.kv_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TileOf at;
  if (!find_tile(p.cu_seqlens, p.batch, p.total, p.group_log2, kFp8 ? kPromptSmall : 0, kHalf ? kHalfShift : kAttnShift,
                 tiles - 1 - (int)(blockIdx.x / p.kv_heads), at))
    return;
  at.to_scalars();
  const int group = 1 << p.group_log2;
  const int len = kFp8 ? min(max(p.seq_lens[at.b], 0), p.max_seq_len) : at.n;
  const int first = len - at.n;                         // position of the call's first token of the sequence
  const int rows = at.n << p.group_log2;
  const bool small = kFp8 && rows <= kPromptSmall;
  const int tile = small ? kStreamRows : kHalf ? kAttnRows / 2 : kAttnRows, row0 = at.index * tile;
  auto position = [&](int r) { return first + (min(r, rows - 1) >> p.group_log2); };
  const int r = row0 + (small ? 0 : kRowsPerWave * (kHalf ? wave & 1 : wave)) + (lane & 31);
  const int token = at.first + (min(r, rows - 1) >> p.group_log2);
  const int head = kvh * group + (min(r, rows - 1) & (group - 1));
  AttnRow row;
  row.q = p.q + token * p.ld_q + head * kHeadDim;
  row.limit = position(r);
  const int split = blockIdx.y;
  const int begin = kFp8 ? split * p.split_keys : 0;
  const int end = min(position(row0 + tile - 1) + 1, kFp8 && p.splits > 1 ? begin + p.split_keys : 0x7FFFFFFF);
  // (a tile whose last row sees keys of the first split alone writes its outputs)
  const bool direct = !kFp8 || p.splits == 1 || position(row0 + tile - 1) < p.split_keys;
  if (kFp8 && p.splits > 1 && split == 0 && kvh == 0 && (r & (group - 1)) == 0 && r < rows && lane < 32)
    p.counts[token] = direct ? kWritten : row.limit < 0 ? 0 : row.limit / p.split_keys + 1;
  if (begin >= end) {                                   // no key to see: 0
    if (direct && split == 0)
      for (int i = threadIdx.x; i < min(rows - row0, tile) * (kHeadDim / 8); i += 64 * kAttnWaves) {
        const int ri = row0 + i / (kHeadDim / 8);
        *reinterpret_cast<uint4*>(p.out + (at.first + (ri >> p.group_log2)) * p.ld_out +
                                  (kvh * group + (ri & (group - 1))) * kHeadDim + i % (kHeadDim / 8) * 8) = make_uint4(0, 0, 0, 0);
      }
    return;
  }
  row.all_limit = min(position(row0), end - 1);

  const float sscale = (kFp8 ? p.k_scale[0] : 1.0f) * p.sm_scale;
  const float c = score_factor(sscale);
  const int floats = (kHeadDim << p.group_log2) + (2 * group + 3) / 4 * 4;
  auto record = [&](int tok) { return p.records + (((int64_t)tok * p.kv_heads + kvh) * p.splits + split) * floats; };
  const PagedKv pages{static_cast<const uint8_t*>(p.k), static_cast<const uint8_t*>(p.v),
                      p.block_table + (int64_t)at.b * p.max_blocks, p.num_blocks, p.max_blocks, p.kv_heads, kvh};
  if (kFp8 && small) {
    __shared__ StreamStats stats;
    AttnAcc part_acc;                                   // (nothing that the large tiles' loop has in registers)
    attn_init(part_acc);
    row.limit = min(row.limit, end - 1);                // (the next split's keys are its own)
    bf16x8 part_q[8];
    attn_load_q(row, part_q);
    attn_stream(part_acc, part_q, row, begin, end, c, pages, len, lds);
    stream_join(part_acc, c, lds, stats, [&](int i, int part, const float4 (&o)[4], float m, float l) {
      const int ri = row0 + i, tok = at.first + (ri >> p.group_log2), hd = ri & (group - 1);
      if (ri >= rows) return;
      if (!direct) {
        float* rec = record(tok);
#pragma unroll
        for (int n = 0; n < 4; ++n) *reinterpret_cast<float4*>(rec + hd * kHeadDim + 16 * part + 4 * n) = o[n];
        if (part == 0) {
          rec[group * kHeadDim + hd] = fmaxf(m * sscale, kNoScore);
          rec[group * kHeadDim + group + hd] = l;
        }
      } else {
        uint16_t* at_out = p.out + tok * p.ld_out + (kvh * group + hd) * kHeadDim + 16 * part;
        const float4 none[4] = {};                        // (no visible key: 0, also times a scale of NaN)
        if (position(ri) < 0) store16_bf16(none, 0.0f, at_out);
        else store16_bf16(o, p.v_scale[0] / l, at_out);
      }
    });
    return;
  }
  AttnAcc acc;
  attn_init(acc);
  bf16x8 q[8];
  attn_load_q(row, q);
  if constexpr (kFp8) {
    attn_run_fp8(acc, q, row, begin, end, c, pages, len, lds);
    if (row.all_limit < end - 1) attn_redo(acc, q, row, begin, end, end, end, c, Fp8Tokens{pages});
  } else {
    const Bf16Rows<false> k(static_cast<const uint16_t*>(p.k) + at.first * p.ld_k + kvh * kHeadDim, p.ld_k, len);
    const Bf16Rows<true> v(static_cast<const uint16_t*>(p.v) + at.first * p.ld_v + kvh * kHeadDim, p.ld_v, len);
    const int from = kHalf ? (wave >> 1) * (kTileKeys / 2) : 0;
    attn_run_bf16<kHalf ? 1 : 2>(acc, q, row, begin, end, c, k, v, lds, from);
    if (row.all_limit < end - 1)
      attn_redo(acc, q, row, begin + from, end, kHalf ? kTileKeys / 2 : end, kHalf ? kTileKeys : end, c,
                Bf16Tokens{k.base, k.ld, v.base, v.ld});
  }
  if constexpr (kHalf) {
    __shared__ HalfStats stats;
    attn_join_halves(acc, c, lds, stats);
    if (wave >= 2) return;
  }
  const float l = kHalf ? acc.l : half_sum(acc.l);
  const bool valid = r < rows;
  if (direct) {
    const float f = position(r) < 0 ? 0.0f : (kFp8 ? p.v_scale[0] : 1.0f) / l;   // no visible key: 0
    attn_store_bf16(acc, f, p.out + token * p.ld_out + head * kHeadDim, valid);
    return;
  }
  float* rec = record(token);
  const int h = head & (group - 1);
  attn_store_f32(acc, rec + h * kHeadDim, valid);
  if (valid && lane < 32) {
    rec[group * kHeadDim + h] = fmaxf(acc.m * sscale, kNoScore);
    rec[group * kHeadDim + group + h] = l;
  }
}

// A token's records joined: kFew: eight (token, query head) pairs a workgroup, 32 lanes each; otherwise one.
template <int kG, bool kFew>
__global__ __launch_bounds__(kFew ? 256 : 32 * kMergeSets) void attn_prompt_merge_kernel(const PromptArgs p) {
  const int64_t pair = kFew ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  const int heads = p.kv_heads * kG;
  const int token = (int)(pair / heads), head = (int)(pair % heads);
  const int lo = min(max(p.cu_seqlens[0], 0), p.total), hi = min(max(p.cu_seqlens[p.batch], 0), p.total);
  if (token < lo || token >= hi) return;                 // rows of no sequence stay as they are
  const int kvh = head / kG, h = head % kG;
  const int ns = min(p.counts[token], p.splits);
  if (ns == kWritten) return;
  const float* base = p.records + ((int64_t)token * p.kv_heads + kvh) * p.splits * partial_floats<kG>();
  uint16_t* out = p.out + token * p.ld_out + head * kHeadDim;
  if constexpr (kFew)
    merge_few_records<kG>(base, ns, ns, 0, h, p.v_scale, out);
  else
    merge_records<kG>(base, ns, ns, 0, h, p.v_scale, out);
}

}  // namespace

int64_t attn_prompt_workgroups(int64_t batch, int64_t total, int64_t group, int64_t kv_heads, bool fp8) {
  return attn_tile_bound(total * group, batch, total, fp8 ? kPromptSmall : 0, kAttnShift) * kv_heads;
}

// bf16 calls of at most so many workgroups take tiles of half the rows, twice as many of them, each in about two thirds
// of the time (one prompt, us in a graph, 128 / 64 rows: 1398 tokens, 16 heads over 8, 35 / 30; 4000 96 / 87; 1000, 32 over
// 8, 30 / 26; above the limit 4000, 32 over 8, 143 / 165; 16 prompts of 128 18 / 22).
constexpr int64_t kHalfTiles = 512;

// Splits of the keys, as if the sequences were all as long as their mean and had max_seq_len keys.  Small tiles, bound
// by reading: as many as fill the 512 places that the chip holds.  Large ones: as many as end first (attn_shares), records
// at 5 TB/s.  (Against 512 places for all, us: 4 chunks of up to 375 behind 707 tokens, 32 heads over 4, 45 -> 38; one of 429
// behind 334, 64 over 8, 39 -> 29; two of 239 behind 3926 66 -> 68; 13 of up to 777 behind 3001 84 -> 83.  A CU's
// workgroups weighed in full instead of 0.8: 83 -> 88 there, 0.5: 38 -> 45 for one of 601 behind 157.)
PromptSplit attn_prompt_split(int64_t batch, int64_t total, int64_t group, int64_t kv_heads, int64_t max_seq_len) {
  const int64_t runs = batch < total ? batch : total;
  const int64_t wgs = attn_tile_guess(total * group, runs, kPromptSmall) * kv_heads;
  int64_t splits = wgs > 0 ? (512 + wgs - 1) / wgs : 1;
  if (total * group > runs * kPromptSmall)
    splits = attn_shares(wgs, max_seq_len, {1.5, 2.6, 4.0, total * group * kv_heads * (4.0 * (kHeadDim + 2)) / 5e6, 0.8, 0.0});
  const int64_t keys = attn_share(max_seq_len, splits);
  splits = (max_seq_len + keys - 1) / keys;
  PromptSplit s;
  s.splits = splits > 1 ? (int)splits : 1;
  s.split_keys = (int)keys;
  s.partial_floats = (int)(group * kHeadDim + (2 * group + 3) / 4 * 4);
  return s;
}

hipError_t launch_attention_prompt_bf16(const uint16_t* q, int64_t ld_q, const uint16_t* k, int64_t ld_k,
                                        const uint16_t* v, int64_t ld_v, const int32_t* cu_seqlens, int64_t batch,
                                        int64_t total, int64_t q_heads, int64_t kv_heads, float sm_scale, uint16_t* out,
                                        int64_t ld_out, hipStream_t stream) {
  const int64_t group = q_heads / kv_heads;
  PromptArgs p{};
  p.q = q, p.ld_q = ld_q, p.k = k, p.ld_k = ld_k, p.v = v, p.ld_v = ld_v;
  p.cu_seqlens = cu_seqlens, p.batch = (int)batch, p.total = (int)total, p.kv_heads = (int)kv_heads;
  p.group_log2 = group_log2_of(group), p.sm_scale = sm_scale, p.out = out, p.ld_out = ld_out, p.splits = 1;
  const int64_t wgs = attn_prompt_workgroups(batch, total, group, kv_heads, false);
  if (wgs <= kHalfTiles) {
    const int64_t halves = attn_tile_bound(total * group, batch, total, 0, kHalfShift) * kv_heads;
    hipLaunchKernelGGL((attn_prompt_kernel<false, true>), dim3((unsigned)halves), dim3(64 * kAttnWaves), 0, stream, p);
  } else {
    hipLaunchKernelGGL((attn_prompt_kernel<false, false>), dim3((unsigned)wgs), dim3(64 * kAttnWaves), 0, stream, p);
  }
  return hipGetLastError();
}

hipError_t launch_attention_prompt_fp8kv(const uint16_t* q, int64_t ld_q, const uint8_t* k_cache, const uint8_t* v_cache,
                                         int64_t num_blocks, const int32_t* block_table, int64_t max_blocks,
                                         const int32_t* seq_lens, const int32_t* cu_seqlens, int64_t batch, int64_t total,
                                         int64_t q_heads, int64_t kv_heads, int64_t max_seq_len, const float* k_scale,
                                         const float* v_scale, float sm_scale, uint16_t* out, int64_t ld_out,
                                         float* workspace, hipStream_t stream) {
  const int64_t group = q_heads / kv_heads;
  const PromptSplit sp = attn_prompt_split(batch, total, group, kv_heads, max_seq_len);
  PromptArgs p{};
  p.q = q, p.ld_q = ld_q, p.k = k_cache, p.v = v_cache, p.num_blocks = num_blocks, p.block_table = block_table;
  p.max_blocks = (int)max_blocks, p.seq_lens = seq_lens, p.max_seq_len = (int)max_seq_len;
  p.k_scale = k_scale, p.v_scale = v_scale;
  p.cu_seqlens = cu_seqlens, p.batch = (int)batch, p.total = (int)total, p.kv_heads = (int)kv_heads;
  p.group_log2 = group_log2_of(group), p.sm_scale = sm_scale, p.out = out, p.ld_out = ld_out;
  p.splits = sp.splits, p.split_keys = sp.split_keys;
  p.records = workspace;
  p.counts = reinterpret_cast<int32_t*>(workspace + total * kv_heads * sp.splits * sp.partial_floats);
  hipLaunchKernelGGL((attn_prompt_kernel<true, false>),
                     dim3((unsigned)attn_prompt_workgroups(batch, total, group, kv_heads, true), (unsigned)sp.splits),
                     dim3(64 * kAttnWaves), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.splits == 1) return e;
  const bool few = sp.splits <= kFewRecords;
  const dim3 grid((unsigned)(few ? (total * q_heads + 7) / 8 : total * q_heads)), block(few ? 256 : 32 * kMergeSets);
#define FP8RL_MERGE(G)                                                                                            \
  if (group == G) {                                                                                               \
    if (few) hipLaunchKernelGGL((attn_prompt_merge_kernel<G, true>), grid, block, 0, stream, p);                  \
    else hipLaunchKernelGGL((attn_prompt_merge_kernel<G, false>), grid, block, 0, stream, p);                     \
  }
  FP8RL_MERGE(1)
  FP8RL_MERGE(2)
  FP8RL_MERGE(4)
  FP8RL_MERGE(8)
#undef FP8RL_MERGE
  return hipGetLastError();
}

}  // namespace fp8rl
