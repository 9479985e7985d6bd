// C ABI of libfp8rl (include/fp8rl.h): prompt attention, decode attention over shared prefixes and
// the pages of the cache.  Argument validation, then launches on the caller's stream, as in api.cpp.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "api_util.hpp"
#include "fp8rl.h"
#include "launch.hpp"

namespace {

constexpr int64_t kMaxGrid = int64_t(1) << 23;   // workgroups (of 256 threads: HIP takes 2^32 threads less one)

// Heads and factor that every attention entry point takes: an FP8RL_* error, or kLaunch.
int check_heads(int64_t q_heads, int64_t kv_heads, int64_t head_dim, float sm_scale) {
  if (kv_heads < 1 || q_heads < 1) return FP8RL_ERR_INVALID_ARG;
  if (!(sm_scale > 0.0f) || !(sm_scale <= 3.4028234663852886e38f)) return FP8RL_ERR_INVALID_ARG;
  if (head_dim != 128 || q_heads % kv_heads || kv_heads > 65535) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  const int64_t group = q_heads / kv_heads;
  if (group != 1 && group != 2 && group != 4 && group != 8) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  return kLaunch;
}

// Packed rows: sizes, then the rows of q and out.
int check_prompt(const uint16_t* q, int64_t ld_q, const int32_t* cu_seqlens, int64_t batch, int64_t total,
                 int64_t q_heads, int64_t kv_heads, int64_t head_dim, float sm_scale, const uint16_t* out,
                 int64_t ld_out, bool fp8) {
  if (batch < 0 || total < 0) return FP8RL_ERR_INVALID_ARG;
  const int st = check_heads(q_heads, kv_heads, head_dim, sm_scale);
  if (st != kLaunch) return st;
  if (batch > 65535 || total >= kMaxDim) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (batch == 0 || total == 0) return FP8RL_OK;
  if (fp8rl::attn_prompt_workgroups(batch, total, q_heads / kv_heads, kv_heads, fp8) >= kMaxGrid)
    return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (!q || !cu_seqlens || !out) return FP8RL_ERR_INVALID_ARG;
  if (ld_q < q_heads * 128 || ld_out < q_heads * 128) return FP8RL_ERR_INVALID_ARG;
  if (ld_q >= kMaxDim || ld_out >= kMaxDim) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(cu_seqlens, 4) || ld_q % 8 || ld_out % 8)
    return FP8RL_ERR_MISALIGNED;
  return kLaunch;
}

// The paged FP8 cache and its block table.
int check_paged(const uint8_t* k_cache, const uint8_t* v_cache, int64_t num_blocks, const int32_t* block_table,
                int64_t max_blocks, const int32_t* seq_lens, int64_t max_seq_len, const float* k_scale,
                const float* v_scale) {
  if (!k_cache || !v_cache || !block_table || !seq_lens || !k_scale || !v_scale) return FP8RL_ERR_INVALID_ARG;
  if (num_blocks < 1 || max_blocks < 1 || max_blocks * 16 < max_seq_len) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(block_table, 4) || !aligned(seq_lens, 4) ||
      !aligned(k_scale, 4) || !aligned(v_scale, 4))
    return FP8RL_ERR_MISALIGNED;
  return kLaunch;
}

bool group_ok(int64_t q_heads, int64_t kv_heads) {
  return check_heads(q_heads, kv_heads, 128, 1.0f) == kLaunch;
}

int check_caches(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks) {
  if (num_caches < 1 || block_bytes < 0 || num_blocks < 0 || !caches) return FP8RL_ERR_INVALID_ARG;
  if (num_caches > 65536 || num_blocks >= kMaxDim || block_bytes >= kMaxDim) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  for (int64_t i = 0; i < num_caches; ++i)
    if (!caches[i]) return FP8RL_ERR_INVALID_ARG;
  if (block_bytes % 16) return FP8RL_ERR_MISALIGNED;
  for (int64_t i = 0; i < num_caches; ++i)
    if (!aligned(caches[i], 16)) return FP8RL_ERR_MISALIGNED;
  return kLaunch;
}

int check_table(const int32_t* block_table, int64_t rows, int64_t max_blocks, const int32_t* seq_lens,
                const int32_t* block_refs) {
  if (rows < 0 || max_blocks < 0) return FP8RL_ERR_INVALID_ARG;
  if (rows >= kMaxDim || max_blocks >= kMaxDim) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if ((rows > 0 && (!seq_lens || (max_blocks > 0 && !block_table))) || !block_refs) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(block_refs, 4)) return FP8RL_ERR_MISALIGNED;
  return kLaunch;
}

constexpr int64_t kMaxCount = int64_t(1) << 24;

}  // namespace

extern "C" {

int fp8rl_attention_prompt_bf16(const uint16_t* q, int64_t ld_q, const uint16_t* k, int64_t ld_k, const uint16_t* v,
                                int64_t ld_v, const int32_t* cu_seqlens, int64_t batch, int64_t total, int64_t q_heads,
                                int64_t kv_heads, int64_t head_dim, float sm_scale, uint16_t* out, int64_t ld_out,
                                void* stream) {
  const int st =
      check_prompt(q, ld_q, cu_seqlens, batch, total, q_heads, kv_heads, head_dim, sm_scale, out, ld_out, false);
  if (st != kLaunch) return st;
  if (!k || !v) return FP8RL_ERR_INVALID_ARG;
  if (ld_k < kv_heads * 128 || ld_v < kv_heads * 128) return FP8RL_ERR_INVALID_ARG;
  if (ld_k >= kMaxLd || ld_v >= kMaxLd) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(k, 16) || !aligned(v, 16) || ld_k % 8 || ld_v % 8) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_attention_prompt_bf16(q, ld_q, k, ld_k, v, ld_v, cu_seqlens, batch, total, q_heads,
                                                        kv_heads, sm_scale, out, ld_out, as_stream(stream)));
}

int64_t fp8rl_attention_prompt_workspace_size(int64_t batch, int64_t total, int64_t q_heads, int64_t kv_heads,
                                              int64_t max_seq_len) {
  if (batch < 1 || total < 1 || batch > 65535 || total >= kMaxDim || max_seq_len < 0 ||
      max_seq_len >= (int64_t(1) << 30) || !group_ok(q_heads, kv_heads))
    return 0;
  const fp8rl::PromptSplit sp = fp8rl::attn_prompt_split(batch, total, q_heads / kv_heads, kv_heads, max_seq_len);
  return sp.splits == 1 ? 0 : (total * kv_heads * sp.splits * sp.partial_floats + total) * 4;
}

int fp8rl_attention_prompt_fp8kv(const uint16_t* q, int64_t ld_q, const uint8_t* k_cache, const uint8_t* v_cache,
                                 int64_t num_blocks, const int32_t* block_table, int64_t max_blocks,
                                 const int32_t* seq_lens, const int32_t* cu_seqlens, int64_t batch, int64_t total,
                                 int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_seq_len,
                                 const float* k_scale, const float* v_scale, float sm_scale, uint16_t* out,
                                 int64_t ld_out, void* workspace, int64_t workspace_bytes, void* stream) {
  if (max_seq_len < 0 || num_blocks < 0 || max_blocks < 0 || workspace_bytes < 0) return FP8RL_ERR_INVALID_ARG;
  if (max_seq_len >= (int64_t(1) << 30) || max_blocks >= kMaxDim || num_blocks >= kMaxDim)
    return FP8RL_ERR_UNSUPPORTED_SHAPE;
  int st = check_prompt(q, ld_q, cu_seqlens, batch, total, q_heads, kv_heads, head_dim, sm_scale, out, ld_out, true);
  if (st != kLaunch) return st;
  st = check_paged(k_cache, v_cache, num_blocks, block_table, max_blocks, seq_lens, max_seq_len, k_scale, v_scale);
  if (st != kLaunch) return st;
  const int64_t need = fp8rl_attention_prompt_workspace_size(batch, total, q_heads, kv_heads, max_seq_len);
  if (workspace_bytes < need || (need > 0 && !workspace)) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_attention_prompt_fp8kv(q, ld_q, k_cache, v_cache, num_blocks, block_table, max_blocks,
                                                         seq_lens, cu_seqlens, batch, total, q_heads, kv_heads,
                                                         max_seq_len, k_scale, v_scale, sm_scale, out, ld_out,
                                                         static_cast<float*>(workspace), as_stream(stream)));
}

int64_t fp8rl_attention_decode_shared_workspace_size(int64_t batch, int64_t num_groups, int64_t q_heads,
                                                     int64_t kv_heads, int64_t max_prefix_len, int64_t max_seq_len) {
  if (batch < 1 || batch > 65535 || num_groups < 1 || num_groups > 65535 || max_prefix_len < 0 ||
      max_prefix_len > max_seq_len || max_seq_len >= (int64_t(1) << 30) || !group_ok(q_heads, kv_heads))
    return 0;
  const fp8rl::SharedSplit sp =
      fp8rl::attn_shared_split(batch, num_groups, q_heads / kv_heads, kv_heads, max_prefix_len, max_seq_len);
  return (batch * kv_heads * sp.records * sp.partial_floats + batch) * 4;
}

int fp8rl_attention_decode_shared_fp8kv(const uint16_t* q, const uint8_t* k_cache, const uint8_t* v_cache,
                                        int64_t num_blocks, const int32_t* block_table, int64_t max_blocks,
                                        const int32_t* seq_lens, int64_t batch, const int32_t* group_offsets,
                                        const int32_t* prefix_lens, int64_t num_groups, int64_t max_prefix_len,
                                        int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_seq_len,
                                        const float* k_scale, const float* v_scale, float sm_scale, uint16_t* out,
                                        void* workspace, int64_t workspace_bytes, void* stream) {
  if (batch < 0 || num_groups < 1 || max_seq_len < 0 || max_prefix_len < 0 || max_prefix_len > max_seq_len ||
      max_blocks < 0 || num_blocks < 0)
    return FP8RL_ERR_INVALID_ARG;
  int st = check_heads(q_heads, kv_heads, head_dim, sm_scale);
  if (st != kLaunch) return st;
  if (batch > 65535 || num_groups > 65535 || max_seq_len >= (int64_t(1) << 30) || max_blocks >= kMaxDim ||
      num_blocks >= kMaxDim)
    return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (batch == 0) return FP8RL_OK;
  if (batch * q_heads >= kMaxGrid / 2 ||
      fp8rl::attn_shared_workgroups(batch, num_groups, q_heads / kv_heads, kv_heads, max_prefix_len, max_seq_len) >=
          2 * kMaxGrid)                             // (a workgroup for each sequence and kv head, and for each prefix)
    return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (!q || !out || !group_offsets || !prefix_lens || !workspace) return FP8RL_ERR_INVALID_ARG;
  st = check_paged(k_cache, v_cache, num_blocks, block_table, max_blocks, seq_lens, max_seq_len, k_scale, v_scale);
  if (st != kLaunch) return st;
  if (workspace_bytes < fp8rl_attention_decode_shared_workspace_size(batch, num_groups, q_heads, kv_heads,
                                                                     max_prefix_len, max_seq_len))
    return FP8RL_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 4) || !aligned(group_offsets, 4) || !aligned(prefix_lens, 4) ||
      !aligned(workspace, 16))
    return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_attention_decode_shared(
      q, k_cache, v_cache, num_blocks, block_table, max_blocks, seq_lens, batch, group_offsets, prefix_lens, num_groups,
      max_prefix_len, q_heads, kv_heads, max_seq_len, k_scale, v_scale, sm_scale, out, static_cast<float*>(workspace),
      as_stream(stream)));
}

int fp8rl_kv_copy_blocks(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks,
                         const int32_t* src, const int32_t* dst, int64_t count, void* stream) {
  if (count < 0) return FP8RL_ERR_INVALID_ARG;
  const int st = check_caches(caches, num_caches, block_bytes, num_blocks);
  if (st != kLaunch) return st;
  if (count >= kMaxCount) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (count == 0 || num_blocks == 0 || block_bytes == 0) return FP8RL_OK;
  if (!src || !dst) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(src, 4) || !aligned(dst, 4)) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_kv_copy_blocks(caches, num_caches, block_bytes, num_blocks, src, dst, count,
                                                 as_stream(stream)));
}

int fp8rl_kv_fork_sequences(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks,
                            int32_t* block_table, int64_t rows, int64_t max_blocks, int32_t* seq_lens,
                            int32_t* block_refs, const int32_t* parents, const int32_t* children,
                            const int32_t* new_blocks, int64_t count, void* stream) {
  if (count < 0) return FP8RL_ERR_INVALID_ARG;
  int st = check_caches(caches, num_caches, block_bytes, num_blocks);
  if (st != kLaunch) return st;
  st = check_table(block_table, rows, max_blocks, seq_lens, block_refs);
  if (st != kLaunch) return st;
  if (count >= kMaxCount) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (count == 0 || rows == 0) return FP8RL_OK;
  if (!parents || !children || !new_blocks) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(parents, 4) || !aligned(children, 4) || !aligned(new_blocks, 4)) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_kv_fork(caches, num_caches, block_bytes, num_blocks, block_table, rows, max_blocks,
                                          seq_lens, block_refs, parents, children, new_blocks, count,
                                          as_stream(stream)));
}

int fp8rl_kv_free_sequences(const int32_t* block_table, int64_t rows, int64_t max_blocks, int32_t* seq_lens,
                            int32_t* block_refs, int64_t num_blocks, const int32_t* sequences, int64_t count,
                            void* stream) {
  if (count < 0 || num_blocks < 0) return FP8RL_ERR_INVALID_ARG;
  const int st = check_table(block_table, rows, max_blocks, seq_lens, block_refs);
  if (st != kLaunch) return st;
  if (count >= kMaxCount || num_blocks >= kMaxDim) return FP8RL_ERR_UNSUPPORTED_SHAPE;
  if (count == 0 || rows == 0) return FP8RL_OK;
  if (!sequences) return FP8RL_ERR_INVALID_ARG;
  if (!aligned(sequences, 4)) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_kv_free(block_table, rows, max_blocks, seq_lens, block_refs, num_blocks, sequences,
                                          count, as_stream(stream)));
}

int64_t fp8rl_kv_compact_workspace_size(int64_t num_blocks) {
  return num_blocks < 1 || num_blocks >= kMaxDim ? 0 : fp8rl::kv_compact_workspace_words(num_blocks) * 4;
}

int fp8rl_kv_compact(void* const* caches, int64_t num_caches, int64_t block_bytes, int64_t num_blocks,
                     int32_t* block_table, int64_t rows, int64_t max_blocks, const int32_t* seq_lens,
                     int32_t* block_refs, int32_t* live, void* workspace, int64_t workspace_bytes, void* stream) {
  int st = check_caches(caches, num_caches, block_bytes, num_blocks);
  if (st != kLaunch) return st;
  st = check_table(block_table, rows, max_blocks, seq_lens, block_refs);
  if (st != kLaunch) return st;
  if (num_blocks < 1 || !live || !workspace || workspace_bytes < fp8rl_kv_compact_workspace_size(num_blocks))
    return FP8RL_ERR_INVALID_ARG;
  if (!aligned(live, 4) || !aligned(workspace, 4)) return FP8RL_ERR_MISALIGNED;
  return hip_status(fp8rl::launch_kv_compact(caches, num_caches, block_bytes, num_blocks, block_table, rows, max_blocks,
                                             seq_lens, block_refs, live, static_cast<int32_t*>(workspace),
                                             as_stream(stream)));
}

}  // extern "C"
