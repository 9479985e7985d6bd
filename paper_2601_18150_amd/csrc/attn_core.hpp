// Attention of many query rows to one run of keys: the part that a whole prompt, a chunk of
// one against the cache, and the shared prefix of a group of decoding sequences have in common.
//
// A row is a (token, query head) pair; the heads that read one kv head are rows beside each
// other, so a workgroup's 128 rows (four waves of 32) share every key and value they read.  For
// 64 keys at a time (a tile, in LDS):
//   S^T = K Q^T   v_mfma_f32_32x32x16_bf16, A = 32 keys x 16 dims, B = 16 dims x 32 rows: lane L
//                 then holds, of row L % 32 and half h = L / 32, keys 8 (i / 4) + 4 h + i % 4;
//   softmax       running maximum m and sum l of each row, in fp32: a lane has its own row's
//                 keys, its partner lane L ^ 32 the others, so the maximum takes one exchange a
//                 tile and the sum one at the end;
//   O^T += V^T P^T  A = 32 dims x 16 keys, B = 16 keys x 32 rows.  The order of the keys inside
//                 the product is free as long as both operands keep it, so P goes in as it came
//                 out of the first product: element e of half h is key 8 (e / 4) + 4 h + e % 4.
// Scores are exact products of bf16 values summed in fp32 (every E4M3 code is a bf16 value).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_merge.hpp"
#include "common.hpp"
#include "gemm_core.hpp"

namespace fp8rl {
namespace {

constexpr int kHeadDim = 128;
constexpr int kPageTokens = 16;
constexpr int kRowsPerWave = 32;
constexpr int kAttnWaves = 4;
constexpr int kAttnRows = kRowsPerWave * kAttnWaves;   // rows of a workgroup
constexpr int kTileKeys = 64;
constexpr int kTileBytes = kTileKeys * kHeadDim * 2;   // of keys, and of values, in LDS
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Keys in LDS: rows of 256 bytes, 16-byte chunk c of row r at chunk c ^ (r % 16), so that the
// 16 rows which read one logical chunk together lie in different banks.
__device__ __forceinline__ int key_at(int r, int c) { return r * 256 + ((c ^ (r & 15)) << 4); }
// bf16 values in LDS: rows as the keys', chunk c of row r at c ^ 4 (r % 4): the transposing read
// takes 64 bytes of each of four rows, which then lie in different banks.
__device__ __forceinline__ int value_at(int r, int c) { return r * 256 + ((c ^ ((r & 3) << 2)) << 4); }
// f16 values in LDS (from FP8 pages, which hold four tokens of a dim together): 16 bytes for
// (16-key step, half, dim), the eight keys of that half in the order of the value product.
__device__ __forceinline__ int value16_at(int step, int h, int dim) { return ((step * 2 + h) * kHeadDim + dim) * 16; }

// Sequence of tile `t`, each with ceil(length * G / 128) of them, and the tile's index inside it.
// Offsets are clamped into [0, total], lengths below 0 count as 0.  false: behind the last tile.
struct TileOf {
  int b, index, first, n;      // sequence, tile inside it, its first token, its tokens
};

__device__ __forceinline__ bool find_tile(const int32_t* offsets, int count, int total, int group_log2, int t, TileOf& out) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < count; base += 64) {
    const int i = base + lane;
    const int lo = min(max(offsets[min(i, count)], 0), total), hi = min(max(offsets[min(i + 1, count)], 0), total);
    const int n = i < count ? max(hi - lo, 0) : 0;
    const int tiles = (int)((((int64_t)n << group_log2) + kAttnRows - 1) / kAttnRows);
    const int sum = wave_inclusive_sum(tiles);
    const uint64_t hit = __ballot(before + sum > t);
    if (hit) {
      const int w = __builtin_ctzll(hit);
      out.b = base + w;
      out.index = t - before - (__builtin_amdgcn_readlane(sum, w) - __builtin_amdgcn_readlane(tiles, w));
      out.first = __builtin_amdgcn_readlane(lo, w);
      out.n = __builtin_amdgcn_readlane(n, w);
      return true;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// Tiles of all runs: an upper bound, each run's last one may be partly filled.
inline int64_t attn_tile_bound(int64_t rows, int64_t runs) { return rows / kAttnRows + runs; }

inline int group_log2_of(int64_t g) { return g == 1 ? 0 : g == 2 ? 1 : g == 4 ? 2 : 3; }

// Rows of the workgroup as this lane sees its own (lane % 32 of its wave).
struct AttnRow {
  const uint16_t* q;       // its 128 query values
  int limit;               // last key it attends to (below the first key: none)
  int wave_limit;          // the smallest limit of the wave's rows (no mask is needed up to it)
  int wave_last;           // the largest (tiles behind it are skipped)
};

// Running state of a wave: lane L holds dims 8 (i / 4) + 4 (L / 32) + i % 4 of each 32 of row L % 32.
struct AttnAcc {
  f32x16 o[4];
  float m, l;              // l: this lane's keys alone until attn_finish
};

__device__ __forceinline__ float half_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
}

__device__ __forceinline__ void attn_init(AttnAcc& acc) {
#pragma unroll
  for (int d = 0; d < 4; ++d) acc.o[d] = (f32x16)(0.0f);
  acc.m = kNoScore;
  acc.l = 0.0f;
}

// The wave's queries as the B operand of the first product.
__device__ __forceinline__ void attn_load_q(const AttnRow& row, bf16x8 (&q)[8]) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
    q[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row.q + 16 * kk + 8 * h));
}

// One tile of keys k0 .. k0 + 63 in LDS.  c: the scores' factor times log2(e).
template <bool kF16Values>
__device__ __forceinline__ void attn_tile(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int k0, float c,
                                          const uint8_t* keys, const uint8_t* values) {
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  f32x16 s[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    s[b] = (f32x16)(0.0f);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const bf16x8 k = *reinterpret_cast<const bf16x8*>(keys + key_at(32 * b + j, 2 * kk + h));
      s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[kk], s[b], 0, 0, 0);
    }
  }
  if (k0 + kTileKeys - 1 > row.wave_limit) {              // (uniform over the wave)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3) > row.limit) s[b][i] = -INFINITY;
  }
  float mx = acc.m;
#pragma unroll
  for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fmaxf(s[0][i], s[1][i]));
  mx = half_max(mx);
  const float mc = fmaxf(mx * c, kNoScore);                // (finite where m is)
  const float alpha = __builtin_amdgcn_exp2f(fmaf(acc.m, c, -mc));
  acc.m = mx;
  acc.l *= alpha;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc.o[d][i] *= alpha;
  // P rounded to the type of the values: against f16 values (E4M3 codes, exact there) 2^-12
  // relative, against bf16 ones 2^-9, of the size of the output's own rounding.
  uint32_t p[16];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -mc));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], c, -mc));
      acc.l += e0 + e1;
      p[8 * b + i / 2] = kF16Values ? pack_f16(e0, e1) : pack_bf16(e0, e1);
    }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint4 pw = make_uint4(p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if constexpr (kF16Values) {
        const f16x8 v = *reinterpret_cast<const f16x8*>(values + value16_at(t, h, 32 * d + j));
        acc.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, __builtin_bit_cast(f16x8, pw), acc.o[d], 0, 0, 0);
      } else {
        // ds_read_b64_tr_b16: of 16 lanes that point at four rows x 16 columns, lane i gets column i
        const int r = 16 * t + 4 * h + ((lane & 15) >> 2);
        const int ch = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const uint8_t* at = values + value_at(r, ch) + (lane & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * 256));
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        acc.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, pw), acc.o[d], 0, 0, 0);
      }
    }
  }
}

// Keys and values of one tile from rows of bf16: token k0 + r at base + (k0 + r) * ld; rows from
// `len` on are read as row len - 1 (no row attends to them: they only have to be finite).  1 KiB
// (four rows) an instruction, straight into LDS, the chunks permuted by their source addresses.
__device__ __forceinline__ void load_tile_bf16(const uint16_t* k, int64_t ld_k, const uint16_t* v, int64_t ld_v, int k0,
                                               int len, uint8_t* keys, uint8_t* values) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int o = wave * 4 + i;
    const int r = 4 * o + (lane >> 4), ch = lane & 15;
    const int64_t t = min(k0 + r, len - 1);
    lds_dma16(reinterpret_cast<const uint8_t*>(k + t * ld_k + 8 * (ch ^ (r & 15))), keys + o * 1024);
    lds_dma16(reinterpret_cast<const uint8_t*>(v + t * ld_v + 8 * (ch ^ ((r & 3) << 2))), values + o * 1024);
  }
}

// The same from pages of the FP8 cache: block ids table[k0 / 16 ..], pages past the last one
// that holds a token below `len` repeat that one, ids outside the cache are clamped into it.
// Codes are widened on the way, keys to bf16, values to f16 (both exact); values of tokens from
// `len` on become 0 (unwritten bytes may be NaN codes, and 0 x NaN is NaN).
__device__ __forceinline__ uint2 f16_of_fp8(uint32_t w) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true);
  return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
__device__ __forceinline__ uint2 bf16_of_fp8(uint32_t w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true);
  return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}

struct PagedKv {
  const uint8_t* k;
  const uint8_t* v;
  const int32_t* table;    // this sequence's row
  int64_t num_blocks;
  int max_blocks, kv_heads, kvh;
};

__device__ __forceinline__ int64_t page_offset(const PagedKv& c, int page) {
  const int blk = c.table[min(page, c.max_blocks - 1)];
  const int64_t b = blk < 0 ? 0 : ((int64_t)blk >= c.num_blocks ? c.num_blocks - 1 : blk);
  return (b * c.kv_heads + c.kvh) * (kPageTokens * kHeadDim);
}

// Thread t of 256: page (t >> 7) + 2 i of the tile for i = 0, 1; 16 bytes of keys, and of values
// two dims x eight tokens (the two dwords of a half).
struct Fp8TileRegs {
  uint4 k[2];
  uint2 va[2], vb[2];
};

__device__ __forceinline__ void fetch_tile_fp8(const PagedKv& c, int k0, int len, Fp8TileRegs& f) {
  const int u = threadIdx.x & 127;
  const int last = (len - 1) / kPageTokens;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t base = page_offset(c, min(k0 / kPageTokens + (int)(threadIdx.x >> 7) + 2 * i, last));
    f.k[i] = *reinterpret_cast<const uint4*>(c.k + base + u * 16);
    const uint8_t* v = c.v + base + (u >> 6) * 512 + (u & 63) * 8;   // [a][dim][4], a = half, then half + 2
    f.va[i] = *reinterpret_cast<const uint2*>(v);
    f.vb[i] = *reinterpret_cast<const uint2*>(v + 1024);
  }
}

__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int n) {   // the first n bytes, the others 0
  return n >= 4 ? w : (n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u));
}

__device__ __forceinline__ void store_tile_fp8(const Fp8TileRegs& f, int k0, int len, uint8_t* keys, uint8_t* values) {
  const int u = threadIdx.x & 127;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int page = (int)(threadIdx.x >> 7) + 2 * i;
    const int r = page * kPageTokens + (u >> 3), ch = 2 * (u & 7);
    const uint2 k0w = bf16_of_fp8(f.k[i].x), k1w = bf16_of_fp8(f.k[i].y), k2w = bf16_of_fp8(f.k[i].z),
                k3w = bf16_of_fp8(f.k[i].w);
    *reinterpret_cast<uint4*>(keys + key_at(r, ch)) = make_uint4(k0w.x, k0w.y, k1w.x, k1w.y);
    *reinterpret_cast<uint4*>(keys + key_at(r, ch + 1)) = make_uint4(k2w.x, k2w.y, k3w.x, k3w.y);
    const int h = u >> 6, dim = 2 * (u & 63);
    const int na = len - (k0 + page * kPageTokens + 4 * h), nb = na - 8;   // tokens of the two dwords that exist
    const uint2 a0 = f16_of_fp8(keep_bytes(f.va[i].x, na)), b0 = f16_of_fp8(keep_bytes(f.vb[i].x, nb));
    const uint2 a1 = f16_of_fp8(keep_bytes(f.va[i].y, na)), b1 = f16_of_fp8(keep_bytes(f.vb[i].y, nb));
    *reinterpret_cast<uint4*>(values + value16_at(page, h, dim)) = make_uint4(a0.x, a0.y, b0.x, b0.y);
    *reinterpret_cast<uint4*>(values + value16_at(page, h, dim + 1)) = make_uint4(a1.x, a1.y, b1.x, b1.y);
  }
}

// Dims 32 d + 8 g + 4 h .. + 3 of this lane's row, of the eight that the half's pair of lanes share:
// after the exchange half 0 holds the first pair of fours (8 dims) of each 16, half 1 the second.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// out[0 .. 127] = bf16(acc.o * f) of this lane's row (both halves of the wave take part).
__device__ __forceinline__ void attn_store_bf16(const AttnAcc& acc, float f, uint16_t* out, bool valid) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 2; ++g) {                         // 16 dims: fours 2g and 2g + 1
      const int i = 8 * g;
      uint32_t a0 = pack_bf16(acc.o[d][i] * f, acc.o[d][i + 1] * f), a1 = pack_bf16(acc.o[d][i + 2] * f, acc.o[d][i + 3] * f);
      uint32_t b0 = pack_bf16(acc.o[d][i + 4] * f, acc.o[d][i + 5] * f), b1 = pack_bf16(acc.o[d][i + 6] * f, acc.o[d][i + 7] * f);
      swap_halves(a0, b0);                                // half 0: own a, partner's a; half 1: partner's b, own b
      swap_halves(a1, b1);
      if (valid) *reinterpret_cast<uint4*>(out + 32 * d + 16 * g + 8 * h) = make_uint4(a0, a1, b0, b1);
    }
}

// The record of one row in a split: o[128] in fp32 at rec, m (times the scores' factor, natural
// units) and l at their own places.
__device__ __forceinline__ void attn_store_f32(const AttnAcc& acc, float* rec, bool valid) {
  const int h = (threadIdx.x & 63) >> 5;
  if (!valid) return;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(rec + 32 * d + 8 * g + 4 * h) =
          make_float4(acc.o[d][4 * g], acc.o[d][4 * g + 1], acc.o[d][4 * g + 2], acc.o[d][4 * g + 3]);
}

}  // namespace
}  // namespace fp8rl
