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

// Tiles of a run of `rows`: of 2^shift rows, or of 32 where `small` says that so few rows take those.
constexpr int kAttnShift = 7, kHalfShift = 6;
static_assert(kRowsPerWave == 32 && kAttnRows == 1 << kAttnShift, "shifts");
__device__ __forceinline__ int run_tiles(int rows, int small, int shift) {
  return rows <= small ? (rows + 31) >> 5 : (rows + (1 << shift) - 1) >> shift;
}

// Tiles of up to kScanned sequences are numbered one behind the other, and every wave counts them.  With more
// that would be most of the work (65535 prompts of one token: 77 ms, 3.8 so; 1024 of 32 tokens 225 us, 149 so), and the sequences get places by their offsets
// alone: sequence b's start at place(b) and are no more than place(b + 1) - place(b), of which some stay empty.
// (A place more every third sequence: places that are empty at regular distances would leave the same shader engines idle.)
constexpr int kScanned = 256;

struct Places {
  int shift, step;             // rows a place; further places a sequence

  __host__ __device__ Places(int64_t rows, int64_t count, int small, int tile_shift) {
    // large tiles, and up to three of 32 for a run that takes those; or places of 32 rows for all
    const int few = (small + kRowsPerWave - 1) / kRowsPerWave;
    const bool wide = small == 0 || (rows >> tile_shift) + few * count <= rows / kRowsPerWave + count;
    shift = wide ? tile_shift : 5;
    step = wide && small > 0 ? few : 1;
  }
  template <class T>
  __host__ __device__ T operator()(T row, T b) const { return (row >> shift) + step * b + b / 3; }
};

// Sequence of tile `t`, each with ceil(length * G / rows of a tile) of them, and the tile's index inside it.
// Offsets are clamped into [0, total], lengths below 0 count as 0.  false: no such tile.
struct TileOf {
  int b, index, first, n;      // sequence, tile inside it, its first token, its tokens

  __device__ __forceinline__ void to_scalars() {
    b = __builtin_amdgcn_readfirstlane(b);
    index = __builtin_amdgcn_readfirstlane(index);
    first = __builtin_amdgcn_readfirstlane(first);
    n = __builtin_amdgcn_readfirstlane(n);
  }
};

// (total rows < 2^30; four sequences a lane.)
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int count, int total, int group_log2, int small, int shift, int t,
                                          TileOf& out) {
  constexpr int kPerLane = 4;
  static_assert(kScanned == 64 * kPerLane, "one step");
  const int lane = threadIdx.x & 63;
  auto offset = [&](int i) { return min(max(offsets[i], 0), total); };
  if (count > kScanned) {                                  // the last sequence whose place is not above t, by 64 probes at a time
    const Places place((int64_t)total << group_log2, count, small, shift);
    int lo = 0, n = count;
    for (;;) {
      const int stride = (n + 63) / 64;
      const int i = lo + lane * stride;
      const int at = min(i, count - 1);
      const int below = __popcll(__ballot(i < lo + n && place(offset(at) << group_log2, at) <= t));
      if (below == 0) return false;
      lo += (below - 1) * stride;
      n = min(stride, count - lo);
      if (stride == 1) break;
    }
    out.b = lo;
    out.first = offset(lo);
    out.n = max(offset(lo + 1) - out.first, 0);
    out.index = t - place(out.first << group_log2, lo);
    return out.index >= 0 && out.index < run_tiles(out.n << group_log2, small, shift);
  }
  const int first = kPerLane * lane;
  int at[kPerLane + 1], n[kPerLane], tiles[kPerLane], mine = 0;
#pragma unroll
  for (int u = 0; u <= kPerLane; ++u) at[u] = offsets[min(first + u, count)];
#pragma unroll
  for (int u = 0; u <= kPerLane; ++u) at[u] = min(max(at[u], 0), total);
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {                     // (behind the last sequence: at[count] - at[count])
    n[u] = max(at[u + 1] - at[u], 0);
    tiles[u] = run_tiles(n[u] << group_log2, small, shift);
    mine += tiles[u];
  }
  // (runs that overlap may have more tiles than the grid: kept from an overflow)
  const int sum = wave_inclusive_sum(min(mine, 1 << 24));
  const uint64_t hit = __ballot(sum > t);
  if (hit == 0) return false;
  const int w = __builtin_ctzll(hit);
  int r = t - (w > 0 ? __builtin_amdgcn_readlane(sum, w - 1) : 0);
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    const int here = __builtin_amdgcn_readlane(tiles[u], w);
    if (r < here) {
      out.b = kPerLane * w + u;
      out.index = r;
      out.first = __builtin_amdgcn_readlane(at[u], w);
      out.n = __builtin_amdgcn_readlane(n[u], w);
      return true;
    }
    r -= here;
  }
  return false;
}

// Tiles that the grid has to hold for `rows` rows of `count` sequences, of which `tokens` at most are not empty.
inline int64_t attn_tile_bound(int64_t rows, int64_t count, int64_t tokens, int small, int shift) {
  if (count > kScanned) return Places(rows, count, small, shift)(rows, count);
  const int64_t runs = count < tokens ? count : tokens;    // (the last tile of each may be partly filled)
  if (small == 0) return (rows >> shift) + runs;
  const int64_t mixed = (rows >> shift) + runs * ((small + kRowsPerWave - 1) / kRowsPerWave);
  const int64_t all_small = rows / kRowsPerWave + runs;
  return mixed < all_small ? mixed : all_small;
}

// The tiles if the runs were all as long as their mean (what a rule that fills the chip goes by).
inline int64_t attn_tile_guess(int64_t rows, int64_t runs, int small) {
  const int64_t mean = (rows + runs - 1) / (runs > 0 ? runs : 1);
  const int64_t tile = mean <= small ? kRowsPerWave : kAttnRows;
  return runs * ((mean + tile - 1) / tile);
}

// Keys of each of n shares of `keys`: whole tiles, 256 at least.
inline int64_t attn_share(int64_t keys, int64_t n) {
  const int64_t share = ((keys + n - 1) / n + kTileKeys - 1) / kTileKeys * kTileKeys;
  return share < 256 ? 256 : share;
}

// In how many shares of the keys `wgs` workgroups end first, in us: 64 keys of a workgroup alone on a
// CU and beside another, 5 for its start and end, the launch that joins shares where there would be none, a share's records.
// weight: of the sum of a CU's workgroups (below 1 where they differ); the longest is a bound, and reading the cache.
// The callers' numbers start from measured ones (alone 1.5; beside 2.2 in long chunks to 2.9 in mixed ones) and were then
// fitted over some hundred random cases each, where they gain 1.5 to 2.3% on average and single cases lose 3%: that the
// callers differ in them (2.6 and 3.0, records once and three times) is that fit, not the hardware.
struct ShareCost { double alone, beside, join, record, weight, read; };

inline int64_t attn_shares(int64_t wgs, int64_t keys, const ShareCost& c) {
  const int64_t most = (keys + 255) / 256;
  int64_t best = 1;
  double least = 0.0;
  auto consider = [&](int64_t n) {
    const int64_t tiles = attn_share(keys, n) / kTileKeys, on_cu = (wgs * n + 255) / 256;
    const double one = (on_cu > 1 ? c.beside : c.alone) * tiles + 5.0;
    const double all = on_cu / 2 * (c.beside * tiles + 5.0) + on_cu % 2 * (c.alone * tiles + 5.0);
    const double busy = one > c.weight * all ? one : c.weight * all;
    const double us = (busy > c.read ? busy : c.read) + n * c.record + (n > 1 ? c.join : 0.0);
    if (n == 1 || us < least) best = n, least = us;
  };
  consider(1);
  if (most < 2 || wgs < 1 || wgs >= 768) return best;
  // the largest number for each count of workgroups on a CU, and parts of the first
  for (int64_t k = 1; (256 * k / wgs - 1) * wgs < 768; ++k) {
    const int64_t n = 256 * k / wgs;
    if (n > 1) consider(n < most ? n : most);
    if (n >= most) break;
  }
  for (int64_t part = 3; 256 / wgs >= 4 && part > 0; --part) {
    const int64_t n = 256 / wgs * part / 4;
    if (n > 1 && n < most) consider(n);
  }
  return best;
}

inline int group_log2_of(int64_t g) { return g == 1 ? 0 : g == 2 ? 1 : g == 4 ? 2 : 3; }

// Rows of the workgroup as this lane sees its own (lane % 32 of its wave).
struct AttnRow {
  const uint16_t* q;       // its 128 query values
  int limit;               // last key it attends to (below the first key: none)
  int all_limit;           // the smallest limit of the workgroup's rows (no mask is needed up to it)
};

// Running state of a wave: lane L holds dims 8 (i / 4) + 4 (L / 32) + i % 4 of each 32 of row L % 32.
struct AttnAcc {
  f32x16 o[4];
  float m, l;              // l: this lane's keys alone (half_sum: both lanes')
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

// Where a lane's operands lie in a tile: keys of 16-dim step kk and 32-key half b, values of dims 32 d and
// 16-key step t.
template <bool kF16Values>
struct LaneOffsets {
  int k, v;                // of kk = 0, and of d = 0: the permutations are exclusive ors, so that the others' offsets
                           // differ in one bit field each, and no register has to hold them

  __device__ __forceinline__ LaneOffsets() {
    const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
    k = key_at(j, h);
    // ds_read_b64_tr_b16: of 16 lanes that point at four rows x 16 columns, lane i gets column i
    v = kF16Values ? value16_at(0, h, j)
                   : value_at(4 * h + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8;
  }
  // The offsets as they are needed (and not held across the loop).
  __device__ __forceinline__ LaneOffsets fresh() const {
    LaneOffsets f = *this;
    asm volatile("" : "+v"(f.k), "+v"(f.v));
    return f;
  }
  __device__ __forceinline__ bf16x8 key(const uint8_t* keys, int i) const {     // i: 8 * half + step
    return *reinterpret_cast<const bf16x8*>(keys + (k ^ ((i & 7) << 5)) + (i >> 3) * 32 * 256);
  }
  __device__ __forceinline__ uint4 value(const uint8_t* values, int i) const {  // i: 4 * step + d
    if constexpr (kF16Values) {
      return *reinterpret_cast<const uint4*>(values + v + value16_at(i >> 2, 0, 32 * (i & 3)));
    } else {
      const uint8_t* at = values + (v ^ ((i & 3) << 6)) + (i >> 2) * 16 * 256;
      const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at)));
      const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * 256)));
      return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  }
};

template <bool kF16Values>
__device__ __forceinline__ f32x16 value_mfma(const uint4& v, const uint4& p, const f32x16& o) {
  if constexpr (kF16Values)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, p), o, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), o, 0, 0, 0);
}

// Instruction order inside a block: sched<kind, n> asks for n of that kind next.
constexpr int kSchedMfma = 0x8, kSchedLdsRead = 0x100;
template <int kKind, int kCount>
__device__ __forceinline__ void sched() { __builtin_amdgcn_sched_group_barrier(kKind, kCount, 0); }

template <bool kF16Values>
__device__ __forceinline__ uint32_t pack_p(float a, float b) {
  return kF16Values ? pack_f16(a, b) : pack_bf16(a, b);
}

// A row's maximum is only followed once it has grown by this much (a factor of 2^8 in P), so that its
// accumulator is rarely scaled.  P stays at most 2^8, and every sum at least 1.
constexpr float kMaxGrowth = 8.0f;
// What goes into fp16 is 2^7 P, 2^15 at most, and l is the sum of the same.  fp16 has all its bits down to 2^-14 and ends at
// 2^-25: of P itself a long tail of small weights would be cut off in the values while l counts it (weights of 2^-26 behind
// one of 1 had no values at all in its share of the keys); so it ends at 2^-32.  bf16 has the exponents of fp32.
constexpr float kF16Lift = 7.0f;
static_assert(kMaxGrowth + kF16Lift < 15.9f, "fp16 ends at 65504");

// A row's weights are e = 2^((s - base) c + off), 2^lift times those relative to its maximum m: one fma with base = 0,
// off = lift - m c where the rounding of that, which is then a factor of all of them, is below 2^-13.  Far from zero it would
// be a power of two or many (and overflow fp16 from m c = 2^28 on): there the difference is taken first, a subtraction a score
// more.  (For all rows: long prompts + 2.5%, long chunks + 2.2%; behind this branch + 0.5% and + 1.5%.)
struct Exponent {
  float base, off;
  uint64_t any_far;        // rows of the wave that are far: a bit per lane

  __device__ __forceinline__ Exponent(float m, float c, float lift) {
    const float mc = m * c;
    const bool far = !(fabsf(mc) < 1024.0f);
    base = far ? m : 0.0f;
    off = far ? lift : lift - mc;
    any_far = __ballot(far);
  }
  template <int kCount, class Scores>
  __device__ __forceinline__ void rebase(Scores& s) const {      // s: vectors of kCount scores (rows that are near stay as they are)
    if (__builtin_expect(any_far != 0, 0))
#pragma unroll
      for (int i = 0; i < kCount; ++i) s[i] -= base;
  }
  __device__ __forceinline__ float weight(float rebased, float c) const {
    return __builtin_amdgcn_exp2f(fmaf(rebased, c, off));
  }
};

// o *= alpha, where any row needs it (any: a bit per lane).  The branches are inside the assembly: as a
// branch of the program the compiler keeps the accumulators in two places and copies all of them past
// it in every tile (8191 and 16384 tokens, before other steps: 2.80 ms; always scaled 2.63; so 2.54).  The products
// that made o have ended: alpha comes out of products issued after them.
__device__ __forceinline__ void scale_if(uint64_t any, f32x16 (&o)[4], float alpha) {
  asm volatile("s_cmp_eq_u64 %14, 0\n\ts_cbranch_scc1 L%=_as_it_is\n\tv_mul_f32 %0, %0, %13\n\tv_mul_f32 %1, %1, %13\n\t"
      "v_mul_f32 %2, %2, %13\n\tv_mul_f32 %3, %3, %13\n\tv_mul_f32 %4, %4, %13\n\tv_mul_f32 %5, %5, %13\n\t"
      "v_mul_f32 %6, %6, %13\n\tv_mul_f32 %7, %7, %13\n\tv_mul_f32 %8, %8, %13\n\tv_mul_f32 %9, %9, %13\n\t"
      "v_mul_f32 %10, %10, %13\n\tv_mul_f32 %11, %11, %13\n\tv_mul_f32 %12, %12, %13\n\tL%=_as_it_is:"
      : "+v"(o[0][0]), "+v"(o[0][1]), "+v"(o[0][2]), "+v"(o[0][3]), "+v"(o[0][4]), "+v"(o[0][5]), "+v"(o[0][6]),
      "+v"(o[0][7]), "+v"(o[0][8]), "+v"(o[0][9]), "+v"(o[0][10]), "+v"(o[0][11]), "+v"(o[0][12])
      : "v"(alpha), "s"(any) : "scc");
  asm volatile("s_cmp_eq_u64 %14, 0\n\ts_cbranch_scc1 L%=_as_it_is\n\tv_mul_f32 %0, %0, %13\n\tv_mul_f32 %1, %1, %13\n\t"
      "v_mul_f32 %2, %2, %13\n\tv_mul_f32 %3, %3, %13\n\tv_mul_f32 %4, %4, %13\n\tv_mul_f32 %5, %5, %13\n\t"
      "v_mul_f32 %6, %6, %13\n\tv_mul_f32 %7, %7, %13\n\tv_mul_f32 %8, %8, %13\n\tv_mul_f32 %9, %9, %13\n\t"
      "v_mul_f32 %10, %10, %13\n\tv_mul_f32 %11, %11, %13\n\tv_mul_f32 %12, %12, %13\n\tL%=_as_it_is:"
      : "+v"(o[0][13]), "+v"(o[0][14]), "+v"(o[0][15]), "+v"(o[1][0]), "+v"(o[1][1]), "+v"(o[1][2]), "+v"(o[1][3]),
      "+v"(o[1][4]), "+v"(o[1][5]), "+v"(o[1][6]), "+v"(o[1][7]), "+v"(o[1][8]), "+v"(o[1][9])
      : "v"(alpha), "s"(any) : "scc");
  asm volatile("s_cmp_eq_u64 %14, 0\n\ts_cbranch_scc1 L%=_as_it_is\n\tv_mul_f32 %0, %0, %13\n\tv_mul_f32 %1, %1, %13\n\t"
      "v_mul_f32 %2, %2, %13\n\tv_mul_f32 %3, %3, %13\n\tv_mul_f32 %4, %4, %13\n\tv_mul_f32 %5, %5, %13\n\t"
      "v_mul_f32 %6, %6, %13\n\tv_mul_f32 %7, %7, %13\n\tv_mul_f32 %8, %8, %13\n\tv_mul_f32 %9, %9, %13\n\t"
      "v_mul_f32 %10, %10, %13\n\tv_mul_f32 %11, %11, %13\n\tv_mul_f32 %12, %12, %13\n\tL%=_as_it_is:"
      : "+v"(o[1][10]), "+v"(o[1][11]), "+v"(o[1][12]), "+v"(o[1][13]), "+v"(o[1][14]), "+v"(o[1][15]),
      "+v"(o[2][0]), "+v"(o[2][1]), "+v"(o[2][2]), "+v"(o[2][3]), "+v"(o[2][4]), "+v"(o[2][5]), "+v"(o[2][6])
      : "v"(alpha), "s"(any) : "scc");
  asm volatile("s_cmp_eq_u64 %14, 0\n\ts_cbranch_scc1 L%=_as_it_is\n\tv_mul_f32 %0, %0, %13\n\tv_mul_f32 %1, %1, %13\n\t"
      "v_mul_f32 %2, %2, %13\n\tv_mul_f32 %3, %3, %13\n\tv_mul_f32 %4, %4, %13\n\tv_mul_f32 %5, %5, %13\n\t"
      "v_mul_f32 %6, %6, %13\n\tv_mul_f32 %7, %7, %13\n\tv_mul_f32 %8, %8, %13\n\tv_mul_f32 %9, %9, %13\n\t"
      "v_mul_f32 %10, %10, %13\n\tv_mul_f32 %11, %11, %13\n\tv_mul_f32 %12, %12, %13\n\tL%=_as_it_is:"
      : "+v"(o[2][7]), "+v"(o[2][8]), "+v"(o[2][9]), "+v"(o[2][10]), "+v"(o[2][11]), "+v"(o[2][12]), "+v"(o[2][13]),
      "+v"(o[2][14]), "+v"(o[2][15]), "+v"(o[3][0]), "+v"(o[3][1]), "+v"(o[3][2]), "+v"(o[3][3])
      : "v"(alpha), "s"(any) : "scc");
  asm volatile("s_cmp_eq_u64 %13, 0\n\ts_cbranch_scc1 L%=_as_it_is\n\tv_mul_f32 %0, %0, %12\n\tv_mul_f32 %1, %1, %12\n\t"
      "v_mul_f32 %2, %2, %12\n\tv_mul_f32 %3, %3, %12\n\tv_mul_f32 %4, %4, %12\n\tv_mul_f32 %5, %5, %12\n\t"
      "v_mul_f32 %6, %6, %12\n\tv_mul_f32 %7, %7, %12\n\tv_mul_f32 %8, %8, %12\n\tv_mul_f32 %9, %9, %12\n\t"
      "v_mul_f32 %10, %10, %12\n\tv_mul_f32 %11, %11, %12\n\tL%=_as_it_is:"
      : "+v"(o[3][4]), "+v"(o[3][5]), "+v"(o[3][6]), "+v"(o[3][7]), "+v"(o[3][8]), "+v"(o[3][9]), "+v"(o[3][10]),
      "+v"(o[3][11]), "+v"(o[3][12]), "+v"(o[3][13]), "+v"(o[3][14]), "+v"(o[3][15])
      : "v"(alpha), "s"(any) : "scc");
}

// c, the scores' factor times log2(e); not 0, which times -inf would be NaN, but NaN where the scale is.
__device__ __forceinline__ float score_factor(float sscale) {
  const float c = sscale * 1.4426950408889634f;
  return c < 1.17549435e-38f ? 1.17549435e-38f : c;
}

// Scores of the tile of keys k0 .. k0 + 63 in LDS, and P from them (in the type of the values), in
// the order of the value product.  c: the scores' factor times log2(e).  kMask: keys behind a row's
// limit, which only the last tiles have.
// P is rounded to the type of the values: against f16 values (E4M3 codes, exact there) by 2^-11 of it at
// most, against bf16 ones by 2^-8, which is the output's own rounding.
template <bool kF16Values, bool kMask, int kBlocks = 2>
__device__ __forceinline__ void attn_scores(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int k0, float c,
                                            const LaneOffsets<kF16Values>& lane_at, const uint8_t* keys,
                                            uint32_t (&p)[8 * kBlocks]) {
  const LaneOffsets<kF16Values> at = lane_at.fresh();
  const int h = (threadIdx.x & 63) >> 5;
  f32x16 s[kBlocks];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) s[b] = (f32x16)(0.0f);
#pragma unroll
  for (int i = 0; i < 8 * kBlocks; ++i)
    s[i % kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.key(keys, 8 * (i % kBlocks) + i / kBlocks), q[i / kBlocks],
                                                             s[i % kBlocks], 0, 0, 0);
  sched<kSchedLdsRead, 4>();
#pragma unroll
  for (int i = 0; i < 8 * kBlocks - 4; ++i) {
    sched<kSchedMfma, 1>();
    sched<kSchedLdsRead, 1>();
  }
  sched<kSchedMfma, 4>();
  if constexpr (kMask) {
    const int from = row.limit - k0 - 4 * h;               // (key - k0 - 4 h above it: not visible)
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * b + 8 * (i >> 2) + (i & 3) > from) s[b][i] = -INFINITY;
  }
  float mx = fmaxf(s[0][0], s[kBlocks - 1][kBlocks == 1]);
#pragma unroll
  for (int i = 1; i < 16; ++i) mx = fmaxf(kBlocks == 1 ? s[0][i] : fmaxf(s[0][i], s[kBlocks - 1][i]), mx);
  mx = half_max(mx);
  const bool grown = (mx - acc.m) * c > kMaxGrowth;       // (of this row alone: rows do not affect each other)
  const float m = grown ? mx : acc.m;
  const Exponent at_m(m, c, kF16Values ? kF16Lift : 0.0f);
  // (a difference first: 1 where the maximum stays.  2^(acc.m c - m c) would be the rounding of m c, in l alone and tile after tile)
  const float alpha = __builtin_amdgcn_exp2f((acc.m - m) * c);
  acc.m = m;
  acc.l *= alpha;
  scale_if(__ballot(grown), acc.o, alpha);
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) at_m.rebase<16>(s[b]);
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float e0 = at_m.weight(s[b][i], c), e1 = at_m.weight(s[b][i + 1], c);
      acc.l += e0 + e1;
      p[8 * b + i / 2] = pack_p<kF16Values>(e0, e1);
    }
}

// O^T += V^T P^T over the tile's values in LDS.
template <bool kF16Values, int kBlocks = 2>
__device__ __forceinline__ void attn_values(AttnAcc& acc, const uint32_t (&p)[8 * kBlocks], const LaneOffsets<kF16Values>& lane_at,
                                            const uint8_t* values) {
  const LaneOffsets<kF16Values> at = lane_at.fresh();
#pragma unroll
  for (int i = 0; i < 8 * kBlocks; ++i) {
    const int t = i >> 2;
    acc.o[i & 3] = value_mfma<kF16Values>(at.value(values, i), make_uint4(p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]), acc.o[i & 3]);
  }
  constexpr int kReads = kF16Values ? 1 : 2;
  sched<kSchedLdsRead, 3 * kReads>();
#pragma unroll
  for (int i = 0; i < 8 * kBlocks - 3; ++i) {
    sched<kSchedMfma, 1>();
    sched<kSchedLdsRead, kReads>();
  }
  sched<kSchedMfma, 3>();
}

// Rows of bf16 keys or values of one sequence (len rows of pitch ld), moved to LDS a tile at a time by
// DMA, 1 KiB (four rows) an instruction, the chunks permuted by their source addresses.  The buffer
// resource of a tile ends with the sequence's last row: rows behind it are not read and become 0.
constexpr int kTileLoads = kTileBytes / 1024 / kAttnWaves;   // instructions a wave

template <bool kValues>
struct Bf16Rows {
  const uint16_t* base;
  int64_t ld;
  int len;

  __device__ __forceinline__ Bf16Rows(const uint16_t* b, int64_t pitch, int n) : base(b), ld(pitch), len(n) {}
  __device__ __forceinline__ void load(int k0, uint8_t* tile) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
    const int first = k0 + 4 * kTileLoads * wave;            // this wave's rows
    const int rows = min(len - first, 4 * kTileLoads);
    const uint32_t bytes = rows > 0 ? (uint32_t)((rows - 1) * ld * 2) + 2 * kHeadDim : 0u;   // (ld < 2^24: below 2^29)
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base + first * ld), (short)0, bytes, 0x00020000);
    uint32_t lane;                                           // (made here, so that nothing is held across the loop)
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    const uint32_t four = lane >> 4, ch = 16 * ((lane & 15) ^ (kValues ? four << 2 : four));
#pragma unroll
    for (int i = 0; i < kTileLoads; ++i)
      lds_dma16(r, (four + 4 * i) * (uint32_t)(2 * ld) + (kValues ? ch : ch ^ (64 * i)), 0,
                tile + (wave * kTileLoads + i) * 1024);
  }
};
static_assert(kTileLoads == 4, "a wave's rows start at a multiple of 16, so that chunk ^ 4 i permutes those of instruction i");

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

// (the table does not change under the kernel: a scalar load)
__device__ __forceinline__ int page_entry(const PagedKv& c, int page) {
  typedef const __attribute__((address_space(4))) int32_t const_i32;
  return *(const_i32*)(c.table + min(page, c.max_blocks - 1));
}

__device__ __forceinline__ int64_t page_offset(const PagedKv& c, int blk) {
  const int64_t b = blk < 0 ? 0 : ((int64_t)blk >= c.num_blocks ? c.num_blocks - 1 : blk);
  return (b * c.kv_heads + c.kvh) * (kPageTokens * kHeadDim);
}

// Thread t of 256: pages t / 128 and t / 128 + 2 of the tile; 16 bytes of keys each, and of values the
// dwords of dims L and L + 64 of tokens 4 h .. and 4 h + 8 .., with L = t % 64 and h = t / 64 % 2.
struct Fp8Keys { uint4 w[2]; };
struct Fp8Values { uint32_t w[2][4]; };                   // dim L of both fours, dim L + 64 of both
struct Fp8Pages { int blk[2]; };                          // this wave's pages' entries in the block table

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6; }
__device__ __forceinline__ int tile_page(int i) { return (wave_of() >> 1) + 2 * i; }

__device__ __forceinline__ Fp8Pages tile_pages(const PagedKv& c, int k0, int len) {
  Fp8Pages g;
#pragma unroll
  for (int i = 0; i < 2; ++i) g.blk[i] = page_entry(c, min(k0 / kPageTokens + tile_page(i), (len - 1) / kPageTokens));
  return g;
}

__device__ __forceinline__ void fetch_keys(const PagedKv& c, const Fp8Pages& g, Fp8Keys& f) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    f.w[i] = *reinterpret_cast<const uint4*>(c.k + page_offset(c, g.blk[i]) + (threadIdx.x & 127) * 16);
}

__device__ __forceinline__ void fetch_values(const PagedKv& c, const Fp8Pages& g, Fp8Values& f) {
  const int lane = threadIdx.x & 63, h = wave_of() & 1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t* v = reinterpret_cast<const uint32_t*>(c.v + page_offset(c, g.blk[i])) + h * kHeadDim + lane;   // [a][dim]
#pragma unroll
    for (int u = 0; u < 4; ++u) f.w[i][u] = v[(u & 1) * 2 * kHeadDim + (u >> 1) * 64];
  }
}

__device__ __forceinline__ void store_keys(const Fp8Keys& f, uint8_t* keys) {
  const int u = threadIdx.x & 127;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = tile_page(i) * kPageTokens + (u >> 3), ch = 2 * (u & 7);
    const uint2 k0 = bf16_of_fp8(f.w[i].x), k1 = bf16_of_fp8(f.w[i].y), k2 = bf16_of_fp8(f.w[i].z), k3 = bf16_of_fp8(f.w[i].w);
    *reinterpret_cast<uint4*>(keys + key_at(r, ch)) = make_uint4(k0.x, k0.y, k1.x, k1.y);
    *reinterpret_cast<uint4*>(keys + key_at(r, ch + 1)) = make_uint4(k2.x, k2.y, k3.x, k3.y);
  }
}

__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int n) {   // the first n bytes, the others 0
  return n >= 4 ? w : (n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u));
}

__device__ __forceinline__ void store_values(Fp8Values f, int k0, int len, uint8_t* values) {
  const int lane = threadIdx.x & 63, h = wave_of() & 1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (k0 + kTileKeys > len) {                            // (uniform) tokens of the fours that exist
      const int n = len - (k0 + tile_page(i) * kPageTokens + 4 * h);
#pragma unroll
      for (int u = 0; u < 4; ++u) f.w[i][u] = keep_bytes(f.w[i][u], n - 8 * (u & 1));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint2 a = f16_of_fp8(f.w[i][2 * u]), b = f16_of_fp8(f.w[i][2 * u + 1]);
      *reinterpret_cast<uint4*>(values + value16_at(tile_page(i), h, lane + 64 * u)) = make_uint4(a.x, a.y, b.x, b.y);
    }
  }
}

// All tiles of keys begin .. end - 1 (one at least).  LDS holds one tile of keys and one of values, each refilled while
// the other is in use: the values land under the score product, the next keys under the softmax and the
// value product.  Two barriers a tile: behind the first (next_values) every wave has read the values
// before and the keys are there, behind the second (next_keys) every wave has read the keys and the
// values are there.  Keys and values are LDS objects of their own, so that the compiler sees that a
// read of one need not wait for the other's loads.  32 KiB and at most 168 registers leave room for
// three workgroups on a CU, whose matrix and vector work overlaps: a wave's tile is 1024 cycles of the one and some
// 1150 of the other (32 heads over 4, 8191 and 16384 tokens: 2.48 ms, 1.11 PFLOP/s; two tiles of each in LDS, the score
// product of the next tile between the instructions of this one's softmax, two workgroups: a tenth longer, and
// short prompts took 1.7 times as long).  The library's largest bf16 product reaches 1.19 PFLOP/s here, at
// a clock that falls under load: that is what bounds long prompts.  Short ones pay the start and the end of
// every workgroup (33 of up to 1500 tokens: 0.27 ms, 0.78 PFLOP/s).
// Tiles that every row sees in full come first and need no mask.
struct TileLds {
  uint8_t* k;
  uint8_t* v;
};

// kBlocks 1: of each tile the wave takes 32 keys, from key `from` on; lds begins with those.
template <bool kF16Values, int kBlocks, class Keys, class Values>
__device__ __forceinline__ void attn_run(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int begin, int end,
                                         float c, const TileLds& lds, int from, Keys next_keys, Values next_values) {
  c = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c)));
  const LaneOffsets<kF16Values> at;
  uint32_t p[8 * kBlocks];
  int k0 = begin;
  for (; k0 + kTileKeys - 1 <= row.all_limit; k0 += kTileKeys) {
    next_values(k0);
    attn_scores<kF16Values, false, kBlocks>(acc, q, row, k0 + from, c, at, lds.k, p);
    next_keys(k0 + kTileKeys);
    attn_values<kF16Values, kBlocks>(acc, p, at, lds.v);
  }
  for (; k0 < end; k0 += kTileKeys) {
    next_values(k0);
    attn_scores<kF16Values, true, kBlocks>(acc, q, row, k0 + from, c, at, lds.k, p);
    next_keys(k0 + kTileKeys);
    attn_values<kF16Values, kBlocks>(acc, p, at, lds.v);
  }
}

template <int kBlocks>
__device__ __forceinline__ void attn_run_bf16(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int begin, int end,
                                              float c, const Bf16Rows<false>& k, const Bf16Rows<true>& v,
                                              const TileLds& lds, int from = 0) {
  k.load(begin, lds.k);
  v.load(begin, lds.v);                                    // (the first tile's come with its keys)
  const TileLds mine{lds.k + from * 256, lds.v + from * 256};
  attn_run<false, kBlocks>(acc, q, row, begin, end, c, mine, from, [&](int k0) {
    wait_vmcnt<0>();
    lds_barrier();
    if (k0 < end) k.load(k0, lds.k);
  }, [&](int k0) {
    if (k0 == begin) {
      wait_vmcnt<kTileLoads>();
      lds_barrier();
    } else {
      wait_vmcnt<0>();
      lds_barrier();
      v.load(k0, lds.v);
    }
  });
}

// The same from the FP8 cache, through registers, where the codes are widened: a tile's codes are asked
// for when those of the one before it have been stored, its page ids a step earlier.  What is asked for
// behind the last tile repeats the last pages.  (The codes held in registers leave room for two
// workgroups on a CU; three took longer, with the codes brought through LDS by DMA by 5 to 10%, with the
// codes asked for and stored around the value product alone by 4 to 13%: a tile moves 160 KB through LDS, 1280 cycles
// of it.  Codes asked for two tiles ahead: the same time.)  Three
// chunks of 2048 against up to 18432 tokens: 1.20 ms, 0.94 PFLOP/s; the widening adds a fifth to the vector work,
// which a CU with two workgroups overlaps less.
__device__ __forceinline__ void attn_run_fp8(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int begin, int end,
                                             float c, const PagedKv& pages, int len, const TileLds& lds) {
  Fp8Keys fk;
  Fp8Values fv;
  Fp8Pages at = tile_pages(pages, begin, len), after = tile_pages(pages, begin + kTileKeys, len);
  fetch_keys(pages, at, fk);
  fetch_values(pages, at, fv);
  at = after;                                              // of the tile whose values are asked for next
  store_keys(fk, lds.k);
  fetch_keys(pages, at, fk);
  attn_run<true, 2>(acc, q, row, begin, end, c, lds, 0, [&](int k0) {
    lds_barrier();
    store_keys(fk, lds.k);
    fetch_keys(pages, after, fk);
    at = after;
  }, [&](int k0) {
    lds_barrier();
    after = tile_pages(pages, k0 + 2 * kTileKeys, len);
    store_values(fv, k0, len, lds.v);
    fetch_values(pages, at, fv);
  });
}

// Single keys and values as the lanes of attn_redo take them: the half's part of q . k (dims 16 kk + 8 h ..), and
// the values of four dims.
struct Bf16Tokens {
  static constexpr float kLift = 0.0f;
  const uint16_t* k;
  int64_t ld_k;
  const uint16_t* v;
  int64_t ld_v;

  __device__ __forceinline__ float score(const bf16x8 (&q)[8], int t, int h) const {
    float s = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const bf16x8 x = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(k + t * ld_k + 16 * kk + 8 * h));
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf((float)x[i], (float)q[kk][i], s);
    }
    return s;
  }
  __device__ __forceinline__ float4 values(int t, int dim) const {
    const uint2 x = *reinterpret_cast<const uint2*>(v + t * ld_v + dim);
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xFFFF0000u));
  }
};

struct Fp8Tokens {
  static constexpr float kLift = kF16Lift;
  const PagedKv& c;

  __device__ __forceinline__ float score(const bf16x8 (&q)[8], int t, int h) const {
    const uint8_t* at = c.k + page_offset(c, page_entry(c, t / kPageTokens)) + t % kPageTokens * kHeadDim + 8 * h;
    float s = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint2 w = *reinterpret_cast<const uint2*>(at + 16 * kk), a = bf16_of_fp8(w.x), b = bf16_of_fp8(w.y);
      const bf16x8 x = __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y));
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf((float)x[i], (float)q[kk][i], s);
    }
    return s;
  }
  __device__ __forceinline__ float4 values(int t, int dim) const {   // (a dword holds four tokens of a dim)
    const uint4 w = *reinterpret_cast<const uint4*>(c.v + page_offset(c, page_entry(c, t / kPageTokens)) +
                                                    (t % kPageTokens / 4 * kHeadDim + dim) * 4);
    const int b = 8 * (t % 4);
    return make_float4(__builtin_amdgcn_cvt_f32_fp8((int)(w.x >> b), 0), __builtin_amdgcn_cvt_f32_fp8((int)(w.y >> b), 0),
                       __builtin_amdgcn_cvt_f32_fp8((int)(w.z >> b), 0), __builtin_amdgcn_cvt_f32_fp8((int)(w.w >> b), 0));
  }
};

// In a tile of which some rows see less, a value that is not finite would make their sums NaN too (0 x NaN in the
// product).  Rows whose sums are not finite are summed anew here, over the keys that they see alone and in the
// order of the keys: runs of `run` keys, `step` apart.  Slow, and only for such values; a row that sees one gets the same
// again.  Everything else pays a sum of 64 products with zero for each lane at the end.
template <class Tokens>
__device__ __forceinline__ void attn_redo(AttnAcc& acc, const bf16x8 (&q)[8], const AttnRow& row, int begin, int end, int run,
                                          int step, float c, const Tokens& tokens) {
  float z = 0.0f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = fmaf(acc.o[d][i], 0.0f, z);
  const uint64_t bad = __ballot(z != 0.0f);
  if (bad == 0) return;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const bool mine = ((bad | bad >> 32) >> (lane & 31)) & 1;
  const Exponent at_m(acc.m, c, Tokens::kLift);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc.o[d][i] = mine ? 0.0f : acc.o[d][i];
  for (int k0 = begin; k0 < end; k0 += step)
    for (int t = k0; t < min(k0 + run, end); ++t) {
      const float s = half_sum(tokens.score(q, t, h));
      const bool sees = mine && t <= row.limit;
      const float e = at_m.weight(s - at_m.base, c);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 v = tokens.values(t, 32 * d + 8 * g + 4 * h);
          acc.o[d][4 * g] = sees ? fmaf(e, v.x, acc.o[d][4 * g]) : acc.o[d][4 * g];
          acc.o[d][4 * g + 1] = sees ? fmaf(e, v.y, acc.o[d][4 * g + 1]) : acc.o[d][4 * g + 1];
          acc.o[d][4 * g + 2] = sees ? fmaf(e, v.z, acc.o[d][4 * g + 2]) : acc.o[d][4 * g + 2];
          acc.o[d][4 * g + 3] = sees ? fmaf(e, v.w, acc.o[d][4 * g + 3]) : acc.o[d][4 * g + 3];
        }
    }
}

// Waves 2 and 3 have taken the other keys of the rows of waves 0 and 1, which get their sums (l: of both lanes' halves).
struct HalfStats { float m[2][kRowsPerWave], l[2][kRowsPerWave]; };

__device__ __forceinline__ void attn_join_halves(AttnAcc& acc, float c, const TileLds& lds, HalfStats& stats) {
  const int lane = threadIdx.x & 63, j = lane & 31, h = lane >> 5;
  const int wave = wave_of();
  int rows = wave & 1;
  asm volatile("" : "+s"(rows));                           // (a table of LDS addresses, which there cannot be, otherwise)
  acc.l = half_sum(acc.l);
  float* area = reinterpret_cast<float*>(rows ? lds.v : lds.k);
  __syncthreads();                                         // (the tiles are read)
  // 16-byte chunk n of row j at n ^ j, so that the rows' chunks lie in different banks
  auto at = [&](int d, int g) { return reinterpret_cast<float4*>(area + j * kHeadDim + 4 * ((8 * d + 2 * g + h) ^ j)); };
  if (wave >= 2) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *at(d, g) = make_float4(acc.o[d][4 * g], acc.o[d][4 * g + 1], acc.o[d][4 * g + 2], acc.o[d][4 * g + 3]);
    if (h == 0) {
      stats.m[rows][j] = acc.m;
      stats.l[rows][j] = acc.l;
    }
  }
  __syncthreads();
  if (wave >= 2) return;
  const float other = stats.m[rows][j], m = fmaxf(acc.m, other);
  const float a = __builtin_amdgcn_exp2f((acc.m - m) * c), b = __builtin_amdgcn_exp2f((other - m) * c);
  acc.l = acc.l * a + stats.l[rows][j] * b;
  acc.m = m;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 o = *at(d, g);
      acc.o[d][4 * g] = acc.o[d][4 * g] * a + o.x * b;
      acc.o[d][4 * g + 1] = acc.o[d][4 * g + 1] * a + o.y * b;
      acc.o[d][4 * g + 2] = acc.o[d][4 * g + 2] * a + o.z * b;
      acc.o[d][4 * g + 3] = acc.o[d][4 * g + 3] * a + o.w * b;
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
