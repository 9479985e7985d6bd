// Attention of at most 32 query rows to a run of cached keys: what a few drafted tokens, or a few
// members of a group, have to do.  Such rows are bound by reading the cache, and a tile that four waves
// share (attn_core.hpp) would leave three of them without rows; here the waves share the keys instead:
// wave w attends all rows to chunks w, w + 4, .. of 32 keys (two pages), and the four results are
// joined at the end.  A wave's codes come by DMA, whole 1 KiB runs, into a ring that only it touches, so
// the loop has no barrier, and are widened when they are read.  (24 sequences of up to 4000 tokens, 1 to 8 new
// each, 32 heads over 8: 101 MB in 27 us, 3.7 TB/s; with the tiles of attn_core.hpp 53.)  Arithmetic and operand layouts are
// those of attn_core.hpp: S^T = K Q^T, O^T += V^T P^T with v_mfma_f32_32x32x16.
#pragma once

#include "attn_core.hpp"

namespace fp8rl {
namespace {

constexpr int kStreamRows = kRowsPerWave;
constexpr int kChunkKeys = 32;
constexpr int kChunkBytes = kChunkKeys * kHeadDim;         // of keys, and of values
constexpr int kStreamDepth = 2;                            // chunks on their way per wave
constexpr int kRingBytes = kAttnWaves * kStreamDepth * kChunkBytes;   // of keys, and of values
static_assert(kRingBytes >= kTileBytes, "a large tile's keys, and its values, fit into the rings' space");
static_assert(2 * kRingBytes >= kAttnWaves * kStreamRows * kHeadDim * 4, "the waves' results are joined in the rings");

// m and l of every wave and row, beside their results.
struct StreamStats { float m[kAttnWaves][kStreamRows], l[kAttnWaves][kStreamRows]; };

__device__ __forceinline__ void stream_fetch(const PagedKv& c, const int (&blk)[2], uint8_t* keys, uint8_t* values) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t base = page_offset(c, blk[i]);
    const __amdgpu_buffer_rsrc_t rk = buffer_rsrc(c.k + base), rv = buffer_rsrc(c.v + base);
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      // keys: 16-byte chunks permuted inside their rows (swz, gemm_core.hpp) by the source address
      lds_dma16(rk, (uint32_t)swz(8 * o + (lane >> 3), lane & 7), 0, keys + i * 2048 + o * 1024);
      lds_dma16(rv, lane * 16, o * 1024, values + i * 2048 + o * 1024);
    }
  }
}

__device__ __forceinline__ uint32_t lds_offset(const uint8_t* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p;
}

// A lane's keys and values of a chunk, and the wait for them.  As assembly, because the compiler takes the slot that
// is read for the one that a chunk is on its way into, and would wait for that one too (with the queries' wait in the
// loop as well, attn_stream: 16 x 16 sequences of up to 2500 own tokens 176 us, 164 so).
__device__ __forceinline__ void stream_read(const uint8_t* ks, const int (&key_off)[8], const uint8_t* vs, uint2 (&kf)[8],
                                            uint2 (&vf)[2][2][2]) {
  const uint32_t k = lds_offset(ks), v = lds_offset(vs);
  uint64_t a[8], w[8];
  asm volatile(
      "ds_read_b64 %0, %16\n\tds_read_b64 %1, %17\n\tds_read_b64 %2, %18\n\tds_read_b64 %3, %19\n\t"
      "ds_read_b64 %4, %20\n\tds_read_b64 %5, %21\n\tds_read_b64 %6, %22\n\tds_read_b64 %7, %23\n\t"
      "ds_read2_b32 %8, %24 offset0:0 offset1:32\n\tds_read2_b32 %9, %25 offset0:0 offset1:32\n\t"
      "ds_read2_b32 %10, %24 offset0:64 offset1:96\n\tds_read2_b32 %11, %25 offset0:64 offset1:96\n\t"
      "ds_read2_b32 %12, %26 offset0:0 offset1:32\n\tds_read2_b32 %13, %27 offset0:0 offset1:32\n\t"
      "ds_read2_b32 %14, %26 offset0:64 offset1:96\n\tds_read2_b32 %15, %27 offset0:64 offset1:96\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(a[4]), "=&v"(a[5]), "=&v"(a[6]), "=&v"(a[7]), "=&v"(w[0]),
        "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7])
      : "v"(k + key_off[0]), "v"(k + key_off[1]), "v"(k + key_off[2]), "v"(k + key_off[3]), "v"(k + key_off[4]),
        "v"(k + key_off[5]), "v"(k + key_off[6]), "v"(k + key_off[7]), "v"(v), "v"(v + 1024), "v"(v + 2 * 1024), "v"(v + 3 * 1024)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    kf[i] = __builtin_bit_cast(uint2, a[i]);
    vf[i >> 2][(i >> 1) & 1][i & 1] = __builtin_bit_cast(uint2, w[i]);
  }
}

// Keys begin .. end - 1 (begin a multiple of 16; no row's limit is above end - 1) of the len that the
// sequence has; afterwards every wave has its part in acc.
__device__ __forceinline__ void attn_stream(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int begin, int end,
                                            float c, const PagedKv& pages, int len, const TileLds& lds) {
  c = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c)));
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  const int wave = wave_of();
  uint8_t* keys = lds.k + wave * (kStreamDepth * kChunkBytes);
  uint8_t* values = lds.v + wave * (kStreamDepth * kChunkBytes);
  const int last_page = (len - 1) / kPageTokens;
  auto entries = [&](int i, int (&blk)[2]) {               // of this wave's chunk i
    const int page = (begin + (wave + kAttnWaves * i) * kChunkKeys) / kPageTokens;
#pragma unroll
    for (int u = 0; u < 2; ++u) blk[u] = page_entry(pages, min(page + u, last_page));
  };
  const int chunks = max(0, (end - begin - wave * kChunkKeys + kAttnWaves * kChunkKeys - 1) / (kAttnWaves * kChunkKeys));
  int next[2];
#pragma unroll
  for (int d = 0; d < kStreamDepth; ++d) {                 // (a wave with fewer chunks reads the last page, as others do)
    entries(d, next);
    stream_fetch(pages, next, keys + d * kChunkBytes, values + d * kChunkBytes);
  }
  // The queries were asked for before.  The wait is here, behind a known number of loads that it leaves on their way:
  // the compiler would put it into the loop, in front of every chunk's products, and there for every load.
  wait_vmcnt<8 * kStreamDepth>();
  entries(kStreamDepth, next);
  // this lane's operands: keys of row j, 8 dims of half h of 16-byte chunk kk; values of dim j
  int key_off[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) key_off[kk] = swz(j, kk) + 8 * h;
  const int value_off = (h * kHeadDim + j) * 4;
  int slot = 0;
  for (int i = 0; i < chunks; ++i) {
    wait_own_ring<8, kStreamDepth>(chunks - 1 - i);
    asm volatile("" ::: "memory");
    uint8_t* ks = keys + slot * kChunkBytes;
    uint8_t* vs = values + slot * kChunkBytes;
    uint2 kf[8];
    uint2 vf[2][2][2];                                     // (16-key step, pair of 32 dims, four of the half)
    stream_read(ks, key_off, vs + value_off, kf, vf);
    if (i + kStreamDepth < chunks) stream_fetch(pages, next, ks, vs);
    entries(i + kStreamDepth + 1, next);
    slot = slot + 1 == kStreamDepth ? 0 : slot + 1;

    const int k0 = begin + (wave + kAttnWaves * i) * kChunkKeys;
    f32x16 s = (f32x16)(0.0f);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint2 a = bf16_of_fp8(kf[kk].x), b = bf16_of_fp8(kf[kk].y);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y)), q[kk], s, 0, 0, 0);
    }
    const int from = row.limit - k0 - 4 * h;               // (key - k0 - 4 h above it: not visible)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r >> 2) + (r & 3) > from) s[r] = -INFINITY;
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 15; r += 2) mx = fmaxf(fmaxf(s[r], s[r + 1]), mx);
    mx = half_max(fmaxf(mx, s[15]));
    const bool grown = (mx - acc.m) * c > kMaxGrowth;
    const float m = grown ? mx : acc.m;
    const Exponent at_m(m, c, kF16Lift);
    const float alpha = __builtin_amdgcn_exp2f((acc.m - m) * c);   // (exactly 1 where the maximum stays)
    acc.m = m;
    acc.l *= alpha;
    scale_if(__ballot(grown), acc.o, alpha);
    at_m.rebase<16>(s);
    if (k0 + kChunkKeys > len) {                           // (uniform) tokens of the fours that exist
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int n = len - (k0 + 16 * t + 8 * u + 4 * h);
            vf[t][d][u] = make_uint2(keep_bytes(vf[t][d][u].x, n), keep_bytes(vf[t][d][u].y, n));
          }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float e[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) e[r] = at_m.weight(s[8 * t + r], c);
      acc.l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      const uint4 p = make_uint4(pack_f16(e[0], e[1]), pack_f16(e[2], e[3]), pack_f16(e[4], e[5]), pack_f16(e[6], e[7]));
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint2 x = vf[t][d >> 1][0], y = vf[t][d >> 1][1];
        const uint2 a = f16_of_fp8(d & 1 ? x.y : x.x), b = f16_of_fp8(d & 1 ? y.y : y.x);
        acc.o[d] = value_mfma<true>(make_uint4(a.x, a.y, b.x, b.y), p, acc.o[d]);
      }
    }
  }
  wait_vmcnt<0>();
  if (__ballot(row.limit < end - 1))
    attn_redo(acc, q, row, begin + wave * kChunkKeys, end, kChunkKeys, kAttnWaves * kChunkKeys, c, Fp8Tokens{pages});
  acc.l = half_sum(acc.l);
}

// Joins the four waves' results: store(row, chunk, o, m, l) for the 16 dims 16 chunk .. of every row, with o
// relative to m.
template <class Store>
__device__ __forceinline__ void stream_join(const AttnAcc& acc, float c, const TileLds& lds, StreamStats& stats, Store store) {
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  const int wave = wave_of();
  __syncthreads();                                         // the rings are idle
  // (two waves' results in each ring's space)
  auto result = [&](int w) {
    return reinterpret_cast<float*>(w < 2 ? lds.k : lds.v) + (w & 1) * kStreamRows * kHeadDim;
  };
  float* mine = result(wave);
  // 16-byte chunk n of row j at n ^ j, so that the rows' chunks lie in different banks
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(mine + j * kHeadDim + 4 * ((8 * d + 2 * g + h) ^ j)) =
          make_float4(acc.o[d][4 * g], acc.o[d][4 * g + 1], acc.o[d][4 * g + 2], acc.o[d][4 * g + 3]);
  if (h == 0) {
    stats.m[wave][j] = acc.m;
    stats.l[wave][j] = acc.l;
  }
  __syncthreads();
  const int r = threadIdx.x >> 3, part = threadIdx.x & 7;  // 256 threads: 8 for each row
  float m = kNoScore, l = 0.0f, w[kAttnWaves];
#pragma unroll
  for (int i = 0; i < kAttnWaves; ++i) m = fmaxf(m, stats.m[i][r]);
  float4 o[4];
#pragma unroll
  for (int i = 0; i < kAttnWaves; ++i) {
    w[i] = __builtin_amdgcn_exp2f((stats.m[i][r] - m) * c);
    l += stats.l[i][r] * w[i];
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    o[n] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kAttnWaves; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(result(i) + r * kHeadDim + 4 * ((4 * part + n) ^ r));
      o[n].x += v.x * w[i];
      o[n].y += v.y * w[i];
      o[n].z += v.z * w[i];
      o[n].w += v.w * w[i];
    }
  }
  store(r, part, o, m, l);
}

// 16 values as bf16, times f.
__device__ __forceinline__ void store16_bf16(const float4 (&o)[4], float f, uint16_t* out) {
#pragma unroll
  for (int n = 0; n < 4; n += 2)
    *reinterpret_cast<uint4*>(out + 4 * n) =
        make_uint4(pack_bf16(o[n].x * f, o[n].y * f), pack_bf16(o[n].z * f, o[n].w * f),
                   pack_bf16(o[n + 1].x * f, o[n + 1].y * f), pack_bf16(o[n + 1].z * f, o[n + 1].w * f));
}

}  // namespace
}  // namespace fp8rl
