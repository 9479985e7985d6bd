// Joining the records that the splits of one (sequence, kv head) leave: each holds, for the heads
// that read the kv head, the values weighted by e^(score - m) and their sum l, with its own m.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace fp8rl {
namespace {

// A running maximum before its first score: finite, so that scores of -inf (a query-key
// product past the range of fp32) weigh exp(-inf) = 0 also where they are the first ones
// seen, instead of exp(-inf + inf) = NaN; below or equal to every finite score.
constexpr float kNoScore = -3.4028234663852886e38f;

// Partial record per (sequence, kv head, split): o[G][128], then m[G], l[G],
// padded to a multiple of 4 floats (16-byte aligned records).
template <int kG>
constexpr int partial_floats() { return kG * 128 + (2 * kG + 3) / 4 * 4; }
template <int kG>
constexpr int rec_m() { return kG * 128; }
template <int kG>
constexpr int rec_l() { return kG * 128 + kG; }

// out[d] = bf16( v_scale * sum_s e^(m_s - M) o_s[d] / sum_s e^(m_s - M) l_s ) of head h of the
// group, over ns records of `base`: record s for s < np, s + gap behind it.  One workgroup: 32
// lanes hold the head's dims, kMergeSets such sets take the records in turn (their loads are then
// independent of each other) and are combined in LDS.  No record gives 0.
constexpr int kMergeSets = 4;

template <int kG>
__device__ __forceinline__ void merge_records(const float* __restrict__ base, int ns, int np, int gap, int h,
                                              const float* __restrict__ v_scale, uint16_t* __restrict__ out) {
  __shared__ float red[kMergeSets][128 + 2];
  const int set = threadIdx.x >> 5, d = 4 * (threadIdx.x & 31);
  float m = kNoScore, l = 0.0f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = set; s < ns; s += kMergeSets) {
    const float* r = base + (int64_t)(s < np ? s : s + gap) * partial_floats<kG>();
    const float ms = r[rec_m<kG>() + h], ls = r[rec_l<kG>() + h];
    const float4 o = *reinterpret_cast<const float4*>(r + h * 128 + d);
    const float mn = fmaxf(m, ms), f = expf(m - mn), w = expf(ms - mn);
    l = l * f + ls * w;
    a.x = a.x * f + o.x * w;
    a.y = a.y * f + o.y * w;
    a.z = a.z * f + o.z * w;
    a.w = a.w * f + o.w * w;
    m = mn;
  }
  *reinterpret_cast<float2*>(&red[set][d]) = make_float2(a.x, a.y);
  *reinterpret_cast<float2*>(&red[set][d + 2]) = make_float2(a.z, a.w);
  if (d == 0) {
    red[set][128] = m;
    red[set][128 + 1] = l;
  }
  __syncthreads();
  if (set != 0) return;
  float mm = kNoScore, lsum = 0.0f;
#pragma unroll
  for (int s = 0; s < kMergeSets; ++s) mm = fmaxf(mm, red[s][128]);
  a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int s = 0; s < kMergeSets; ++s) {
    const float w = ns > 0 ? expf(red[s][128] - mm) : 0.0f;               // (a set without splits adds 0)
    lsum += red[s][128 + 1] * w;
    a.x += red[s][d] * w;
    a.y += red[s][d + 1] * w;
    a.z += red[s][d + 2] * w;
    a.w += red[s][d + 3] * w;
  }
  const float f = ns > 0 ? (v_scale ? v_scale[0] : 1.0f) / lsum : 0.0f;
  uint2 o2;
  o2.x = f32_to_bf16_rne(a.x * f) | (f32_to_bf16_rne(a.y * f) << 16);
  o2.y = f32_to_bf16_rne(a.z * f) | (f32_to_bf16_rne(a.w * f) << 16);
  uint32_t* orow = reinterpret_cast<uint32_t*>(out + d);
  orow[0] = o2.x;                                  // (out is 4-byte aligned)
  orow[1] = o2.y;
}

// The same with 32 lanes (lane: threadIdx.x % 32) alone, for a few records.
template <int kG>
__device__ __forceinline__ void merge_few_records(const float* __restrict__ base, int ns, int np, int gap, int h,
                                                  const float* __restrict__ v_scale, uint16_t* __restrict__ out) {
  const int d = 4 * (threadIdx.x & 31);
  float m = kNoScore, l = 0.0f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < ns; ++s) {
    const float* r = base + (int64_t)(s < np ? s : s + gap) * partial_floats<kG>();
    const float ms = r[rec_m<kG>() + h], ls = r[rec_l<kG>() + h];
    const float4 o = *reinterpret_cast<const float4*>(r + h * 128 + d);
    const float mn = fmaxf(m, ms), f = expf(m - mn), w = expf(ms - mn);
    l = l * f + ls * w;
    a.x = a.x * f + o.x * w;
    a.y = a.y * f + o.y * w;
    a.z = a.z * f + o.z * w;
    a.w = a.w * f + o.w * w;
    m = mn;
  }
  const float f = ns > 0 ? v_scale[0] / l : 0.0f;
  uint32_t* orow = reinterpret_cast<uint32_t*>(out + d);
  orow[0] = f32_to_bf16_rne(a.x * f) | (f32_to_bf16_rne(a.y * f) << 16);
  orow[1] = f32_to_bf16_rne(a.z * f) | (f32_to_bf16_rne(a.w * f) << 16);
}

// Records up to which 32 lanes join them alone.
constexpr int kFewRecords = 16;

}  // namespace
}  // namespace fp8rl
