// Host-only build of the argument validation of csrc/api_attention.cpp with AddressSanitizer and
// UndefinedBehaviorSanitizer, the launchers replaced by stubs that count calls.  The fake device
// pointers are never dereferenced; the host array of caches is, and is exactly as long as said.  Each
// entry point is called once as it should be (one launch), and with one argument changed at a time.
// Built and run by tests/test_abi_attention.py.
#include <cstdio>
#include <functional>
#include <vector>

#include "../../paper_2601_18150_amd/csrc/api_attention.cpp"

namespace {
int g_launches = 0, g_fail = 0;
hipError_t stub() { ++g_launches; return hipSuccess; }
}  // namespace

namespace fp8rl {
PromptSplit attn_prompt_split(int64_t batch, int64_t, int64_t, int64_t, int64_t max_seq_len) {
  return PromptSplit{batch < 8 && max_seq_len > 512 ? 3 : 1, 256, 132};
}
int64_t attn_prompt_workgroups(int64_t batch, int64_t total, int64_t group, int64_t kv_heads, bool) {
  return (total * group / 128 + batch) * kv_heads;
}
hipError_t launch_attention_prompt_bf16(const uint16_t*, int64_t, const uint16_t*, int64_t, const uint16_t*, int64_t,
                                        const int32_t*, int64_t, int64_t, int64_t, int64_t, float, uint16_t*, int64_t,
                                        hipStream_t) { return stub(); }
hipError_t launch_attention_prompt_fp8kv(const uint16_t*, int64_t, const uint8_t*, const uint8_t*, int64_t,
                                         const int32_t*, int64_t, const int32_t*, const int32_t*, int64_t, int64_t,
                                         int64_t, int64_t, int64_t, const float*, const float*, float, uint16_t*, int64_t,
                                         float*, hipStream_t) { return stub(); }
SharedSplit attn_shared_split(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return SharedSplit{2, 256, 3, 132}; }
int64_t attn_shared_workgroups(int64_t batch, int64_t, int64_t, int64_t kv_heads, int64_t, int64_t) {
  return batch * kv_heads * 3;
}
hipError_t launch_attention_decode_shared(const uint16_t*, const uint8_t*, const uint8_t*, int64_t, const int32_t*,
                                          int64_t, const int32_t*, int64_t, const int32_t*, const int32_t*, int64_t,
                                          int64_t, int64_t, int64_t, int64_t, const float*, const float*, float, uint16_t*,
                                          float*, hipStream_t) { return stub(); }
hipError_t launch_kv_copy_blocks(void* const*, int64_t, int64_t, int64_t, const int32_t*, const int32_t*, int64_t,
                                 hipStream_t) { return stub(); }
hipError_t launch_kv_fork(void* const*, int64_t, int64_t, int64_t, int32_t*, int64_t, int64_t, int32_t*, int32_t*,
                          const int32_t*, const int32_t*, const int32_t*, int64_t, hipStream_t) { return stub(); }
hipError_t launch_kv_free(const int32_t*, int64_t, int64_t, int32_t*, int32_t*, int64_t, const int32_t*, int64_t,
                          hipStream_t) { return stub(); }
int64_t kv_compact_workspace_words(int64_t num_blocks) { return 3 * num_blocks + 10; }
hipError_t launch_kv_compact(void* const*, int64_t, int64_t, int64_t, int32_t*, int64_t, int64_t, const int32_t*, int32_t*,
                             int32_t*, int32_t*, hipStream_t) { return stub(); }
}  // namespace fp8rl

namespace {

typedef std::vector<int64_t> Args;                       // pointers as numbers, the factor as an index into kFactors
const float kFactors[] = {0.1f, 0.0f, -1.0f, INFINITY, NAN};
void* p(int64_t v) { return reinterpret_cast<void*>(uintptr_t(v)); }
template <class T> T* as(int64_t v) { return reinterpret_cast<T*>(uintptr_t(v)); }

constexpr int64_t A = 1 << 20;                           // aligned to anything
constexpr int OK = FP8RL_OK, ARG = FP8RL_ERR_INVALID_ARG, SHAPE = FP8RL_ERR_UNSUPPORTED_SHAPE, ALIGN = FP8RL_ERR_MISALIGNED;
constexpr int64_t BIG = int64_t(1) << 31, HUGE62 = int64_t(1) << 62;

struct Change { int arg; int64_t value; int status; };   // (status OK: a call with nothing to do)

void check(const char* name, const std::function<int(const Args&)>& call, const Args& good, const std::vector<Change>& bad) {
  g_launches = 0;
  if (call(good) != OK || g_launches != 1) {
    std::printf("FAIL %s: the good call gives %d, %d launches\n", name, call(good), g_launches);
    ++g_fail;
  }
  for (const Change& c : bad) {
    Args a = good;
    a[c.arg] = c.value;
    g_launches = 0;
    const int got = call(a);
    if (got != c.status || g_launches != 0) {
      std::printf("FAIL %s, argument %d = %lld: status %d, want %d, %d launches\n", name, c.arg, (long long)c.value, got,
                  c.status, g_launches);
      ++g_fail;
    }
  }
}

}  // namespace

int main() {
  // q, ld_q, k, ld_k, v, ld_v, cu, batch, total, q_heads, kv_heads, head_dim, factor, out, ld_out
  check("prompt_bf16",
        [](const Args& a) {
          return fp8rl_attention_prompt_bf16(as<uint16_t>(a[0]), a[1], as<uint16_t>(a[2]), a[3], as<uint16_t>(a[4]), a[5],
                                             as<int32_t>(a[6]), a[7], a[8], a[9], a[10], a[11], kFactors[a[12]],
                                             as<uint16_t>(a[13]), a[14], nullptr);
        },
        {A, 1024, A, 256, A, 256, A, 3, 100, 8, 2, 128, 0, A, 1024},
        {{0, 0, ARG}, {0, A + 2, ALIGN}, {1, 1016, ARG}, {1, 1025, ALIGN}, {2, 0, ARG}, {2, A + 8, ALIGN}, {3, 248, ARG},
         {3, 257, ALIGN}, {3, 1 << 24, SHAPE}, {4, 0, ARG}, {4, A + 8, ALIGN}, {5, 0, ARG}, {5, 260, ALIGN},
         {5, HUGE62, SHAPE}, {6, 0, ARG}, {6, A + 2, ALIGN}, {7, -1, ARG}, {7, 0, OK}, {7, BIG, SHAPE}, {7, 1 << 23, SHAPE}, {7, 65536, SHAPE},
         {8, -1, ARG}, {8, 0, OK}, {8, BIG - 1, SHAPE}, {8, HUGE62, SHAPE}, {9, 0, ARG}, {9, 3, SHAPE}, {9, 6, SHAPE},
         {9, 32, SHAPE}, {10, 0, ARG}, {10, -2, ARG}, {10, 3, SHAPE}, {11, 64, SHAPE}, {11, 0, SHAPE}, {12, 1, ARG},
         {12, 2, ARG}, {12, 3, ARG}, {12, 4, ARG}, {13, 0, ARG}, {13, A + 4, ALIGN}, {14, 1000, ARG}, {14, 1028, ALIGN},
         {14, BIG, SHAPE}});
  // q, ld_q, k, v, blocks, table, max_blocks, lens, cu, batch, total, q_heads, kv_heads, dim, max_len, ks, vs, factor,
  // out, ld_out, ws, ws bytes
  const int64_t need = (100 * 2 * 3 * 132 + 100) * 4;
  const auto fp8kv = [](const Args& a) {
    return fp8rl_attention_prompt_fp8kv(as<uint16_t>(a[0]), a[1], as<uint8_t>(a[2]), as<uint8_t>(a[3]), a[4],
                                        as<int32_t>(a[5]), a[6], as<int32_t>(a[7]), as<int32_t>(a[8]), a[9], a[10], a[11],
                                        a[12], a[13], a[14], as<float>(a[15]), as<float>(a[16]), kFactors[a[17]],
                                        as<uint16_t>(a[18]), a[19], p(a[20]), a[21], nullptr);
  };
  check("prompt_fp8kv", fp8kv,
        {A, 1024, A, A, 50, A, 63, A, A, 3, 100, 8, 2, 128, 1000, A, A, 0, A, 1024, A, need},
        {{0, 0, ARG}, {1, 1000, ARG}, {2, 0, ARG}, {2, A + 8, ALIGN}, {3, 0, ARG}, {3, A + 1, ALIGN}, {4, 0, ARG},
         {4, -1, ARG}, {4, BIG, SHAPE}, {5, 0, ARG}, {5, A + 1, ALIGN}, {6, 62, ARG}, {6, 0, ARG}, {6, HUGE62, SHAPE},
         {7, 0, ARG}, {7, A + 2, ALIGN}, {8, 0, ARG}, {8, A + 2, ALIGN}, {9, -1, ARG}, {9, 0, OK}, {10, 0, OK},
         {10, HUGE62, SHAPE}, {11, 5, SHAPE}, {12, 0, ARG}, {13, 64, SHAPE}, {14, -1, ARG}, {14, 1009, ARG},
         {14, int64_t(1) << 30, SHAPE}, {15, 0, ARG}, {15, A + 2, ALIGN}, {16, 0, ARG}, {17, 1, ARG}, {18, 0, ARG},
         {19, 1023, ARG}, {20, 0, ARG}, {20, A + 8, ALIGN}, {21, need - 1, ARG}, {21, -1, ARG}});
  g_launches = 0;                                        // nothing split: no workspace needed
  if (fp8kv({A, 1024, A, A, 50, A, 63, A, A, 3, 100, 8, 2, 128, 500, A, A, 0, A, 1024, 0, 0}) != OK || g_launches != 1 ||
      fp8rl_attention_prompt_workspace_size(3, 100, 8, 2, 500) != 0 ||
      fp8rl_attention_prompt_workspace_size(3, 100, 8, 2, 1000) != need ||
      fp8rl_attention_prompt_workspace_size(-3, 100, 8, 2, 1000) != 0 ||
      fp8rl_attention_prompt_workspace_size(3, 100, 6, 2, 1000) != 0 ||
      fp8rl_attention_prompt_workspace_size(3, HUGE62, 8, 2, 1000) != 0)
    std::printf("FAIL prompt_fp8kv: workspace sizes\n"), ++g_fail;
  // q, k, v, blocks, table, max_blocks, lens, batch, offsets, prefixes, groups, max_prefix, q_heads, kv_heads, dim,
  // max_len, ks, vs, factor, out, ws, ws bytes
  const int64_t shared_need = (5 * 2 * 3 * 132 + 5) * 4;
  check("decode_shared",
        [](const Args& a) {
          return fp8rl_attention_decode_shared_fp8kv(
              as<uint16_t>(a[0]), as<uint8_t>(a[1]), as<uint8_t>(a[2]), a[3], as<int32_t>(a[4]), a[5], as<int32_t>(a[6]),
              a[7], as<int32_t>(a[8]), as<int32_t>(a[9]), a[10], a[11], a[12], a[13], a[14], a[15], as<float>(a[16]),
              as<float>(a[17]), kFactors[a[18]], as<uint16_t>(a[19]), p(a[20]), a[21], nullptr);
        },
        {A, A, A, 50, A, 63, A, 5, A, A, 2, 400, 8, 2, 128, 1000, A, A, 0, A, A, shared_need},
        {{0, 0, ARG}, {0, A + 8, ALIGN}, {1, 0, ARG}, {2, A + 4, ALIGN}, {3, 0, ARG}, {3, -1, ARG}, {4, 0, ARG}, {5, 10, ARG},
         {6, 0, ARG}, {7, -1, ARG}, {7, 0, OK}, {7, 65536, SHAPE}, {8, 0, ARG}, {8, A + 1, ALIGN}, {9, 0, ARG},
         {9, A + 2, ALIGN}, {10, 0, ARG}, {10, 65536, SHAPE}, {11, -1, ARG}, {11, 1001, ARG}, {12, 7, SHAPE}, {12, 0, ARG},
         {13, 0, ARG}, {13, 70000, SHAPE}, {14, 127, SHAPE}, {15, -1, ARG}, {15, 399, ARG}, {15, HUGE62, SHAPE},
         {16, 0, ARG}, {17, 0, ARG}, {18, 4, ARG}, {19, 0, ARG}, {19, A + 2, ALIGN}, {20, 0, ARG}, {20, A + 4, ALIGN},
         {21, shared_need - 1, ARG}});
  // caches as an index, count, bytes, blocks, ...
  void* three[] = {p(A), p(2 * A), p(3 * A)};
  void* hole[] = {p(A), nullptr, p(A)};
  void* odd[] = {p(A), p(A + 8), p(A)};
  void* const* lists[] = {three, nullptr, hole, odd};
  const std::vector<Change> caches = {{0, 1, ARG}, {0, 2, ARG}, {0, 3, ALIGN}, {1, 0, ARG}, {1, -1, ARG}, {1, 65537, SHAPE},
                                      {2, -16, ARG}, {2, 24, ALIGN}, {2, BIG, SHAPE}, {3, -1, ARG}, {3, BIG, SHAPE}};
  const auto plus = [&](std::vector<Change> more) { more.insert(more.end(), caches.begin(), caches.end()); return more; };
  check("copy_blocks",
        [&](const Args& a) {
          return fp8rl_kv_copy_blocks(lists[a[0]], a[1], a[2], a[3], as<int32_t>(a[4]), as<int32_t>(a[5]), a[6], nullptr);
        },
        {0, 3, 4096, 50, A, A, 7},
        plus({{2, 0, OK}, {3, 0, OK}, {4, 0, ARG}, {4, A + 2, ALIGN}, {5, 0, ARG}, {5, A + 1, ALIGN}, {6, -1, ARG}, {6, 0, OK},
              {6, 1 << 24, SHAPE}}));
  check("fork",
        [&](const Args& a) {
          return fp8rl_kv_fork_sequences(lists[a[0]], a[1], a[2], a[3], as<int32_t>(a[4]), a[5], a[6], as<int32_t>(a[7]),
                                         as<int32_t>(a[8]), as<int32_t>(a[9]), as<int32_t>(a[10]), as<int32_t>(a[11]),
                                         a[12], nullptr);
        },
        {0, 3, 4096, 50, A, 20, 8, A, A, A, A, A, 4},
        plus({{4, 0, ARG}, {4, A + 2, ALIGN}, {5, -1, ARG}, {5, 0, OK}, {5, BIG, SHAPE}, {6, -1, ARG}, {6, BIG, SHAPE},
              {7, 0, ARG}, {7, A + 2, ALIGN}, {8, 0, ARG}, {8, A + 2, ALIGN}, {9, 0, ARG}, {10, 0, ARG}, {10, A + 2, ALIGN},
              {11, 0, ARG}, {12, -1, ARG}, {12, 0, OK}, {12, 1 << 24, SHAPE}}));
  check("free",
        [&](const Args& a) {
          return fp8rl_kv_free_sequences(as<int32_t>(a[0]), a[1], a[2], as<int32_t>(a[3]), as<int32_t>(a[4]), a[5],
                                         as<int32_t>(a[6]), a[7], nullptr);
        },
        {A, 20, 8, A, A, 50, A, 4},
        {{0, 0, ARG}, {0, A + 2, ALIGN}, {1, -1, ARG}, {1, 0, OK}, {1, HUGE62, SHAPE}, {2, -1, ARG}, {3, 0, ARG}, {4, 0, ARG},
         {5, -1, ARG}, {5, BIG, SHAPE}, {6, 0, ARG}, {6, A + 2, ALIGN}, {7, -1, ARG}, {7, 0, OK}, {7, 1 << 24, SHAPE}});
  check("compact",
        [&](const Args& a) {
          return fp8rl_kv_compact(lists[a[0]], a[1], a[2], a[3], as<int32_t>(a[4]), a[5], a[6], as<int32_t>(a[7]),
                                  as<int32_t>(a[8]), as<int32_t>(a[9]), p(a[10]), a[11], nullptr);
        },
        {0, 3, 4096, 50, A, 20, 8, A, A, A, A, 640},
        plus({{3, 0, ARG}, {4, 0, ARG}, {5, -1, ARG}, {6, -1, ARG}, {7, 0, ARG}, {8, 0, ARG}, {8, A + 1, ALIGN}, {9, 0, ARG},
              {9, A + 2, ALIGN}, {10, 0, ARG}, {10, A + 2, ALIGN}, {11, 639, ARG}, {11, -1, ARG}}));
  if (fp8rl_kv_compact_workspace_size(50) != 640 || fp8rl_kv_compact_workspace_size(0) != 0 ||
      fp8rl_kv_compact_workspace_size(-4) != 0 || fp8rl_kv_compact_workspace_size(HUGE62) != 0)
    std::printf("FAIL compact: workspace sizes\n"), ++g_fail;
  if (g_fail) return 1;
  std::printf("ok\n");
  return 0;
}
