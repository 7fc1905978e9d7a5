// Tiles of the attention kernels: rows of one head in shared memory (64 or 128 of them) as blocks of their rows x 64 values with the
// 128-byte swizzle, which TMA writes and reads and the products take as operands (rows by rows or transposed).
#pragma once
#include "swarm_attention.h"
#include "swarm_tc.cuh"

namespace swarm {

constexpr int kTile = 128;                              // rows of a tile
constexpr int kBlockBytes = kTile * 128;                // 128 rows x 64 values

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Weights exp(s - max) <= 1 are rounded to T before their products, which take 16-bit operands at twice the rate of any wider
// ones: o and dv are 1.35 to 1.45 times as far from their value as their own rounding leaves them. In fp16 those below 2^-14 would lose bits, so they
// are held as multiples of 2^-shift, with room below the largest fp16 number; bf16 has fp32's range. The exponent's
// argument takes the shift for nothing, and a power of two is taken out of the sums exactly.
template <typename T> constexpr float kWeightShift = 0.0f;
template <> constexpr float kWeightShift<__half> = 15.0f;              // weights against the row's final lse: at most 1
template <typename T> constexpr float kRunningShift = 0.0f;
template <> constexpr float kRunningShift<__half> = 7.0f;              // weights against a running maximum: at most 2^8
__device__ __forceinline__ constexpr float pow2_of(float shift) { return shift == 15.0f ? 0x1p-15f : 1.0f; }

// Whether numbers of T have so small a range that ds, which follows the size of dout, needs a power of two of its own.
template <typename T> constexpr bool kNarrow = false;
template <> constexpr bool kNarrow<__half> = true;
// The power of two that brings a number (not negative) to at least 2^TO and below twice that, 2^80 at most: zeros, and with
// dout of 2^-24 beside values of 2^16, stay far inside fp32's range.
template <int TO>
__device__ __forceinline__ float power_to(float v) {
  const int n = 127 + TO - (int)(__float_as_uint(v) >> 23);
  return __uint_as_float((uint32_t)(127 + min(n, 80)) << 23);
}

// Offset of 16 bytes (8 values) of a row in a block.
__device__ __forceinline__ uint32_t swizzled(int row, int chunk) { return (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

// Zeroes rows [first, last) of a tile of DB blocks; called by one warp. The rows are in an operand of a product whose
// other factor is 0 there, and hold whatever lies past a sentence's end.
template <int DB, int ROWS = kTile>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int first, int last, int lane) {
  for (int i = lane; i < (last - first) * 8 * DB; i += 32) {
    const int row = first + i / (8 * DB), c = i % (8 * DB);
    *reinterpret_cast<uint4*>(tile + (c >> 3) * (ROWS * 128) + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async();
  __syncwarp();
}

// One thread: the copies of a tile (the barrier is told of its bytes beforehand).
template <int DB, int ROWS = kTile>
__device__ __forceinline__ void load_tile(uint32_t dst, const TileMap& m, int row0, int head, int b, uint32_t bar) {
#pragma unroll
  for (int d = 0; d < DB; ++d)
    tma_load_4d(dst + d * (ROWS * 128), &m.map, d * 64, row0 * m.token_step, head * m.head_step, b * m.batch_step, bar);
}
template <int DB>
__device__ __forceinline__ void store_tile(const TileMap& m, uint32_t src, int row0, int head, int b) {
#pragma unroll
  for (int d = 0; d < DB; ++d)
    tma_store_4d(&m.map, src + d * kBlockBytes, d * 64, row0 * m.token_step, head * m.head_step, b * m.batch_step);
}

// One thread: D[128 x cols] = A[128 x dim] B[cols x dim]^T, dim = 16 ksteps <= 64 DB; tile A in shared memory with 128
// rows, tile B with ROWS. The whole width is unrolled: issue, not the tensor pipe, would otherwise set the pace.
template <typename T, int DB, int ROWS>
__device__ __forceinline__ void mma_rows(uint32_t tmem_d, uint32_t tile_a, uint32_t tile_b, int cols, int ksteps) {
  const uint32_t idesc = instr_desc_16<T>(kTile, 0, 0, 0) + ((uint32_t)(cols >> 3) << 17);
  const uint64_t da = smem_desc_sw128(tile_a, 16, 1024), db = smem_desc_sw128(tile_b, 16, 1024);
#pragma unroll
  for (int ks = 0; ks < DB * 4; ++ks)
    if (ks < ksteps)
      tc_mma(tmem_d, da + (uint64_t)(((ks >> 2) * kBlockBytes + (ks & 3) * 32) >> 4),
             db + (uint64_t)(((ks >> 2) * (ROWS * 128) + (ks & 3) * 32) >> 4), idesc, ks != 0);
}

// One thread: D[128 x 64 DB] (+)= W[128 x 16 ksteps] B, the left factor in tensor memory (16-bit pairs, columns 64 apart for
// each 64 of it if SPLIT, else consecutive), tile B in shared memory with ROWS rows.
template <typename T, int DB, int ROWS, bool SPLIT>
__device__ __forceinline__ void mma_weights(uint32_t tmem_d, uint32_t tmem_w, uint32_t tile_b, int ksteps, bool accumulate) {
  constexpr uint32_t idesc = instr_desc_16<T>(kTile, DB * 64, 0, 1);
  const uint64_t db = smem_desc_sw128(tile_b, ROWS * 128, 1024);
#pragma unroll
  for (int ks = 0; ks < ROWS / 16; ++ks)
    if (ks < ksteps)
      tc_mma_ts(tmem_d, tmem_w + (SPLIT ? (ks >> 2) * 64 + (ks & 3) * 8 : ks * 8), db + (uint64_t)((ks * 2048) >> 4), idesc,
                accumulate || ks != 0);
}

// 32 values of a row times `factor` (zeros unless live) into columns col .. col + 31 of a tile.
template <typename T>
__device__ __forceinline__ void store_row32(uint8_t* tile, int row, int col, const float* v, float factor, bool live) {
#pragma unroll
  for (int ch = 0; ch < 4; ++ch) {
    uint32_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = live ? pack2<T>(v[ch * 8 + 2 * u] * factor, v[ch * 8 + 2 * u + 1] * factor) : 0u;
    *reinterpret_cast<uint4*>(tile + (col >> 6) * kBlockBytes + swizzled(row, ((col & 63) >> 3) + ch)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A number per row as an operand of a product: 16 values of bf16 of which the first three add up to it (24 bits), against a row
// of ones in the same places. bf16 whatever the call's type, so that fp32's range is held (a product of its own: an fp16
// call's others are fp16). Rows are stored as the unswizzled operand wants them, eight of them in 256 bytes: their first
// eight values (16 bytes a row), then the others.
using StatType = __nv_bfloat16;
__device__ __forceinline__ int64_t stat_offset(int64_t row) { return (row >> 3) * 256 + (row & 7) * 16; }
__device__ __forceinline__ void store_stat(uint8_t* p, float v) {
  const float hi = to_float(from_float<StatType>(v)), r1 = isinf(hi) ? 0.0f : v - hi;
  const float mid = to_float(from_float<StatType>(r1)), lo = r1 - mid;
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2<StatType>(hi, mid), pack2<StatType>(lo, 0.0f), 0u, 0u);
  *reinterpret_cast<uint4*>(p + 128) = make_uint4(0u, 0u, 0u, 0u);
}

}  // namespace swarm
