// Cross attention, backward pass on the tensor cores.
//
// Two kernels, so that every gradient is summed by one CTA in a fixed order and nothing is added with atomics:
//   attention_dq_kernel   CTA = 128 query rows: s and dp = dout v^T once per tile of states, dq = sum ds k; it also
//                         writes delta = rowsum(dout * o)
//   attention_dkv_kernel  CTA = 128 states of a key head: the transposed products, over all rows of all its query
//                         heads: dv = sum p^T dout, dk = sum ds^T q
// The price is s and dp computed twice: 7 products instead of 5.
#include <mutex>

#include "swarm_attention.h"
#include "swarm_attention_tile.cuh"

namespace swarm {
namespace {

constexpr int kBwdThreads = 320;                        // two warpgroups on the tile's values, copying warp, issuing warp

template <int DB> constexpr int kBwdStages = DB == 2 ? 2 : 4;          // pairs of tiles in flight
template <int DB> constexpr int kBwdSmem = (2 + 2 * kBwdStages<DB>) * DB * kBlockBytes + 1024;

struct BwdBars {
  uint64_t fixed_full, full[4], empty[4], s_full, s_empty, dp_full, dp_empty, ds_full, ds_empty, done, drain;
};

// =================================================================================================
// dq. Tensor memory: s at 0, dp at 128, ds (16 bits, 64 columns) at 256, dq at 384. While the warps turn tile j into
// ds, the scores and dp of tile j + 1 are computed: each is overwritten as soon as it has been read into registers.
// The warpgroups share the rows (warp % 4) and split the columns in halves.
// =================================================================================================
template <typename T, int DB>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_dq_kernel(const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv,
                    const __grid_constant__ TileMap mdo, const __grid_constant__ TileMap mdq, AttentionArgs a, int row_tiles) {
  constexpr int kStages = kBwdStages<DB>;
  constexpr uint32_t kTileBytes = DB * kBlockBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;                                   // q, dout; dq on the way out
  uint8_t* sKV = smem + 2 * kTileBytes;                 // ring of (k, v)
  __shared__ BwdBars bars;
  __shared__ uint32_t tmem_slot;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int qt = blockIdx.x % row_tiles, bh = blockIdx.x / row_tiles, h = bh % a.heads, b = bh / a.heads, hk = h / a.group;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const int row0 = qt * kTile, n = row0 < nq ? (nk + kTile - 1) / kTile : 0;

  if (tid == 0) {
    mbar_init(smem_u32(&bars.fixed_full), 1);
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars.full[i]), 1); mbar_init(smem_u32(&bars.empty[i]), 1); }
    mbar_init(smem_u32(&bars.s_full), 1);
    mbar_init(smem_u32(&bars.s_empty), 8);
    mbar_init(smem_u32(&bars.dp_full), 1);
    mbar_init(smem_u32(&bars.dp_empty), 8);
    mbar_init(smem_u32(&bars.ds_full), 8);
    mbar_init(smem_u32(&bars.ds_empty), 1);
    mbar_init(smem_u32(&bars.done), 1);
    mbar_init(smem_u32(&bars.drain), 1);
    fence_mbar_init();
  }
  if (warp == 9) { tmem_alloc(smem_u32(&tmem_slot), 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, limit = a.wait_limit;
  bool ok = true;

  if (warp == 8) {
    if (n) {
      int issued = 0;
      if (limit && lane == 0) {
        const uint32_t bar = smem_u32(&bars.fixed_full);
        mbar_expect_tx(bar, 2 * kTileBytes);
        load_tile<DB>(smem_u32(sQ), mq, row0, h, b, bar);
        load_tile<DB>(smem_u32(sQ) + kTileBytes, mdo, row0, h, b, bar);
      }
      for (int j = 0; j < n; ++j) {
        const int st = j % kStages;
        ok = mbar_wait(smem_u32(&bars.empty[st]), ((j / kStages) & 1) ^ 1, limit);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t bar = smem_u32(&bars.full[st]);
          mbar_expect_tx(bar, 2 * kTileBytes);
          load_tile<DB>(smem_u32(sKV) + 2 * st * kTileBytes, mk, j * kTile, hk, b, bar);
          load_tile<DB>(smem_u32(sKV) + (2 * st + 1) * kTileBytes, mv, j * kTile, hk, b, bar);
        }
        issued = j + 1;
      }
      if (!ok) {
        // gave up: the copies in flight land before the CTA's shared memory is released
        for (int j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
          mbar_wait(smem_u32(&bars.full[j % kStages]), (j / kStages) & 1, kAttentionWaitLimit);
        if (limit) mbar_wait(smem_u32(&bars.fixed_full), 0, kAttentionWaitLimit);
      }
    }
  } else if (warp == 9) {
    if (n) {
      const int ksteps = (a.head_dim + 15) / 16;
      const uint32_t aq = smem_u32(sQ), akv = smem_u32(sKV);
      constexpr uint32_t kIdescDq = instr_desc_16<T>(kTile, DB * 64, 0, 1);
      auto columns = [&](int j) { return (min(kTile, nk - j * kTile) + 15) & ~15; };
      ok = mbar_wait(smem_u32(&bars.fixed_full), 0, limit);
      for (int j = -1; j < n && ok; ++j) {
        if (j + 1 < n) {
          const int st = (j + 1) % kStages;
          ok = mbar_wait(smem_u32(&bars.full[st]), ((j + 1) / kStages) & 1, limit);
          if (!ok) break;
          const int valid = min(kTile, nk - (j + 1) * kTile), cols = columns(j + 1);
          if (valid < cols) zero_rows<DB>(sKV + 2 * st * kTileBytes, valid, cols, lane);   // k is a factor of dq
          ok = mbar_wait(smem_u32(&bars.s_empty), (j & 1), limit);
          tc_fence_after();
          if (ok && elect_one()) {
            mma_rows<T>(tmem, aq, akv + 2 * st * kTileBytes, cols, ksteps);
            tc_commit(smem_u32(&bars.s_full));
          }
          __syncwarp();
          if (ok) ok = mbar_wait(smem_u32(&bars.dp_empty), (j & 1), limit);
          tc_fence_after();
          if (ok && elect_one()) {
            mma_rows<T>(tmem + 128, aq + kTileBytes, akv + (2 * st + 1) * kTileBytes, cols, ksteps);
            tc_commit(smem_u32(&bars.dp_full));
          }
          __syncwarp();
        }
        if (j >= 0 && ok) {
          const int st = j % kStages;
          ok = mbar_wait(smem_u32(&bars.ds_full), j & 1, limit);
          tc_fence_after();
          if (ok && elect_one()) {
            const uint64_t dk = smem_desc_sw128(akv + 2 * st * kTileBytes, kBlockBytes, 1024);
            for (int ks = 0; ks < columns(j) / 16; ++ks)
              tc_mma_ts(tmem + 384, tmem + 256 + ks * 8, dk + (uint64_t)((ks * 2048) >> 4), kIdescDq, (j | ks) != 0);
            tc_commit(smem_u32(&bars.ds_empty));
            tc_commit(smem_u32(&bars.empty[st]));
            if (j == n - 1) tc_commit(smem_u32(&bars.done));
          }
          __syncwarp();
        }
      }
      if (!ok) {                                        // gave up: no product may be in flight when tensor memory is freed
        if (elect_one()) tc_commit(smem_u32(&bars.drain));
        mbar_wait(smem_u32(&bars.drain), 0, kAttentionWaitLimit);
      }
    }
  } else {
    const int half = warp >> 2, quad = warp & 3, tile_row = quad * 32 + lane, row = row0 + tile_row;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = tmem + lane_base + half * 64, tdp = ts + 128, tds = tmem + lane_base + 256 + half * 32;
    const float c = a.scale * kLog2e;
    const int64_t at = ((int64_t)b * a.heads + h) * a.queries + row;
    const bool live = row < nq && n > 0;
    float delta = 0.0f, lse2 = INFINITY;
    if (live) {
      const T* g = reinterpret_cast<const T*>(a.dout) + offset_of(a.dos, b, row, h);
      const T* o = reinterpret_cast<const T*>(a.o) + offset_of(a.os, b, row, h);
      for (int d = 0; d < a.head_dim; d += 8) {
        float x[8], y[8];
        unpack8<T>(load_raw8<T>(g + d), x);
        unpack8<T>(load_raw8<T>(o + d), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) delta = fmaf(x[i], y[i], delta);
      }
      lse2 = a.lse_in[at] * kLog2e;
    }
    if (half == 0 && row < a.queries) a.delta[at] = delta;
    for (int j = 0; j < n; ++j) {
      const int valid = nk - j * kTile - half * 64;     // columns of this half that exist
      float p[64];
      ok = mbar_wait(smem_u32(&bars.s_full), j & 1, limit);
      if (!ok) break;
      tc_fence_after();
      tmem_ld32(ts, p);
      tmem_ld32(ts + 32, p + 32);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.s_empty));
#pragma unroll
      for (int i = 0; i < 64; ++i) p[i] = ex2(fmaf(p[i], c, -lse2));
      ok = mbar_wait(smem_u32(&bars.dp_full), j & 1, limit);
      if (!ok) break;
      tc_fence_after();
      float dp[64];
      tmem_ld32(tdp, dp);
      tmem_ld32(tdp + 32, dp + 32);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.dp_empty));
#pragma unroll
      for (int i = 0; i < 64; ++i) p[i] = p[i] * (dp[i] - delta);
      if (valid < 64) {
#pragma unroll
        for (int i = 0; i < 64; ++i) p[i] = i < valid ? p[i] : 0.0f;
      }
      ok = mbar_wait(smem_u32(&bars.ds_empty), (j & 1) ^ 1, limit);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = pack2<T>(p[g * 32 + 2 * i], p[g * 32 + 2 * i + 1]);
        tmem_st16(tds + g * 16, w);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.ds_full));
    }
    if (ok && n) {
      ok = mbar_wait(smem_u32(&bars.done), 0, limit);
      tc_fence_after();
    }
    if (named_barrier_and(1, 256, ok)) {
      // warpgroup `half` takes the output's columns [32 DB half, +32 DB)
#pragma unroll
      for (int g = 0; g < DB; ++g) {
        const int col = half * 32 * DB + g * 32;
        float o[32];
        if (n) { tmem_ld32(tmem + lane_base + 384 + col, o); tmem_wait_ld(); }
        store_row32<T>(sQ, tile_row, col, o, live ? a.scale : 0.0f, live);
      }
      fence_proxy_async();
      named_barrier(1, 256);
      if (tid == 0) {
        store_tile<DB>(mdq, smem_u32(sQ), row0, h, b);
        bulk_commit();
        bulk_wait_read();
      }
    }
  }
  if (!ok && lane == 0) atomicExch(a.status, 1);
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// =================================================================================================
// dk and dv. Rows of the transposed tile are states (lanes), columns are query rows. Tensor memory: s^T at 0 with p^T
// (16 bits) written over the half that each warpgroup read, dp^T at 128 with ds^T over it, dv at 256, dk at 384. The
// warps turn s^T(i) into p^T while dp^T(i) is computed, and dp^T(i) into ds^T while dv takes p^T(i) and s^T(i + 1) is
// computed.
// =================================================================================================
template <typename T, int DB>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_dkv_kernel(const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv,
                     const __grid_constant__ TileMap mdo, const __grid_constant__ TileMap mdk, const __grid_constant__ TileMap mdv,
                     AttentionArgs a, int key_tiles) {
  constexpr int kStages = kBwdStages<DB>;
  constexpr uint32_t kTileBytes = DB * kBlockBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sKV = smem;                                  // k, v; dk, dv on the way out
  uint8_t* sQ = smem + 2 * kTileBytes;                  // ring of (q, dout)
  __shared__ BwdBars bars;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_lse[2][kTile], s_delta[2][kTile];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kt = blockIdx.x % key_tiles, bh = blockIdx.x / key_tiles, hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const int key0 = kt * kTile, row_tiles = (nq + kTile - 1) / kTile;
  const int n = key0 < nk ? row_tiles * a.group : 0;

  if (tid == 0) {
    mbar_init(smem_u32(&bars.fixed_full), 1);
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars.full[i]), 1); mbar_init(smem_u32(&bars.empty[i]), 1); }
    mbar_init(smem_u32(&bars.s_full), 1);
    mbar_init(smem_u32(&bars.s_empty), 8);              // p^T has been written
    mbar_init(smem_u32(&bars.dp_full), 1);
    mbar_init(smem_u32(&bars.ds_full), 8);
    mbar_init(smem_u32(&bars.done), 1);
    mbar_init(smem_u32(&bars.drain), 1);
    fence_mbar_init();
  }
  if (warp == 9) { tmem_alloc(smem_u32(&tmem_slot), 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, limit = a.wait_limit;
  bool ok = true;

  if (warp == 8) {
    if (n) {
      int issued = 0;
      if (limit && lane == 0) {
        const uint32_t bar = smem_u32(&bars.fixed_full);
        mbar_expect_tx(bar, 2 * kTileBytes);
        load_tile<DB>(smem_u32(sKV), mk, key0, hk, b, bar);
        load_tile<DB>(smem_u32(sKV) + kTileBytes, mv, key0, hk, b, bar);
      }
      for (int i = 0; i < n; ++i) {
        const int st = i % kStages, h = hk * a.group + i / row_tiles, row0 = i % row_tiles * kTile;
        ok = mbar_wait(smem_u32(&bars.empty[st]), ((i / kStages) & 1) ^ 1, limit);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t bar = smem_u32(&bars.full[st]);
          mbar_expect_tx(bar, 2 * kTileBytes);
          load_tile<DB>(smem_u32(sQ) + 2 * st * kTileBytes, mq, row0, h, b, bar);
          load_tile<DB>(smem_u32(sQ) + (2 * st + 1) * kTileBytes, mdo, row0, h, b, bar);
        }
        issued = i + 1;
      }
      if (!ok) {
        // gave up: the copies in flight land before the CTA's shared memory is released
        for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
          mbar_wait(smem_u32(&bars.full[i % kStages]), (i / kStages) & 1, kAttentionWaitLimit);
        if (limit) mbar_wait(smem_u32(&bars.fixed_full), 0, kAttentionWaitLimit);
      }
    }
  } else if (warp == 9) {
    if (n) {
      const int ksteps = (a.head_dim + 15) / 16;
      const uint32_t akv = smem_u32(sKV), aq = smem_u32(sQ);
      constexpr uint32_t kIdescOut = instr_desc_16<T>(kTile, DB * 64, 0, 1);
      auto columns = [&](int i) { return (min(kTile, nq - i % row_tiles * kTile) + 15) & ~15; };
      // products with p^T or ds^T: column 16 ks of the tile lies at 8 ks of its warpgroup's half
      auto outer = [&](uint32_t d, uint32_t left, uint32_t right, int i) {
        const uint64_t db = smem_desc_sw128(right, kBlockBytes, 1024);
        for (int ks = 0; ks < columns(i) / 16; ++ks)
          tc_mma_ts(d, left + (ks >> 2) * 64 + (ks & 3) * 8, db + (uint64_t)((ks * 2048) >> 4), kIdescOut, (i | ks) != 0);
      };
      ok = mbar_wait(smem_u32(&bars.fixed_full), 0, limit);
      for (int i = -1; i < n && ok; ++i) {
        const int st = i % kStages, next = (i + 1) % kStages;
        if (i >= 0) {
          ok = mbar_wait(smem_u32(&bars.s_empty), i & 1, limit);
          tc_fence_after();
          if (ok && elect_one()) outer(tmem + 256, tmem, aq + (2 * st + 1) * kTileBytes, i);
          __syncwarp();
        }
        if (i + 1 < n && ok) {
          ok = mbar_wait(smem_u32(&bars.full[next]), ((i + 1) / kStages) & 1, limit);
          if (!ok) break;
          const int valid = min(kTile, nq - (i + 1) % row_tiles * kTile), cols = columns(i + 1);
          if (valid < cols) {                           // q and dout are factors of dk and dv
            zero_rows<DB>(sQ + 2 * next * kTileBytes, valid, cols, lane);
            zero_rows<DB>(sQ + (2 * next + 1) * kTileBytes, valid, cols, lane);
          }
          if (elect_one()) {
            mma_rows<T>(tmem, akv, aq + 2 * next * kTileBytes, cols, ksteps);
            tc_commit(smem_u32(&bars.s_full));
          }
          __syncwarp();
        }
        if (i >= 0 && ok) {
          ok = mbar_wait(smem_u32(&bars.ds_full), i & 1, limit);
          tc_fence_after();
          if (ok && elect_one()) {
            outer(tmem + 384, tmem + 128, aq + 2 * st * kTileBytes, i);
            tc_commit(smem_u32(&bars.empty[st]));
            if (i == n - 1) tc_commit(smem_u32(&bars.done));
          }
          __syncwarp();
        }
        if (i + 1 < n && ok && elect_one()) {
          mma_rows<T>(tmem + 128, akv + kTileBytes, aq + (2 * next + 1) * kTileBytes, columns(i + 1), ksteps);
          tc_commit(smem_u32(&bars.dp_full));
        }
        __syncwarp();
      }
      if (!ok) {                                        // gave up: no product may be in flight when tensor memory is freed
        if (elect_one()) tc_commit(smem_u32(&bars.drain));
        mbar_wait(smem_u32(&bars.drain), 0, kAttentionWaitLimit);
      }
    }
  } else {
    const int half = warp >> 2, quad = warp & 3, tile_row = quad * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = tmem + lane_base + half * 64, tdp = ts + 128;
    const float c = a.scale * kLog2e;
    constexpr float kUnshift = pow2_of(kWeightShift<T>);
    // lse and delta of tile i, shifted so that p comes out as a multiple of 2^-shift and ds does not: thread r of a warpgroup fetches row r (warpgroup 0 lse, warpgroup 1 delta)
    auto fetch = [&](int i) {
      const int h = hk * a.group + i / row_tiles, row = i % row_tiles * kTile + tile_row;
      const int64_t at = ((int64_t)b * a.heads + h) * a.queries + row;
      if (row >= nq) return half == 0 ? INFINITY : 0.0f;
      return half == 0 ? a.lse_in[at] * kLog2e - kWeightShift<T> : a.delta[at] * kUnshift;
    };
    float ahead = n ? fetch(0) : 0.0f;
    for (int i = 0; i < n; ++i) {
      const int cols = min(kTile, nq - i % row_tiles * kTile) - half * 64;            // columns of this half that exist
      (half == 0 ? s_lse : s_delta)[i & 1][tile_row] = ahead;
      named_barrier(1, 256);                            // both sets are there; their last readers passed two barriers ago
      if (i + 1 < n) ahead = fetch(i + 1);
      const float* lse2 = s_lse[i & 1] + half * 64;
      const float* delta = s_delta[i & 1] + half * 64;
      float p[64];
      ok = mbar_wait_if(smem_u32(&bars.s_full), i & 1, limit, ok);
      tc_fence_after();
      if (ok) {
        tmem_ld32(ts, p);
        tmem_ld32(ts + 32, p + 32);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 64; q += 4) {
          const float4 l4 = *reinterpret_cast<const float4*>(lse2 + q);
          p[q] = ex2(fmaf(p[q], c, -l4.x));
          p[q + 1] = ex2(fmaf(p[q + 1], c, -l4.y));
          p[q + 2] = ex2(fmaf(p[q + 2], c, -l4.z));
          p[q + 3] = ex2(fmaf(p[q + 3], c, -l4.w));
        }
        if (cols < 64) {
#pragma unroll
          for (int q = 0; q < 64; ++q) p[q] = q < cols ? p[q] : 0.0f;                 // what lies there is not a score
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t w[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) w[q] = pack2<T>(p[g * 32 + 2 * q], p[g * 32 + 2 * q + 1]);
          tmem_st16(ts + g * 16, w);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.s_empty));
      }
      ok = mbar_wait_if(smem_u32(&bars.dp_full), i & 1, limit, ok);
      tc_fence_after();
      if (ok) {
        float dp[64];
        tmem_ld32(tdp, dp);
        tmem_ld32(tdp + 32, dp + 32);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 64; q += 4) {
          const float4 d4 = *reinterpret_cast<const float4*>(delta + q);
          dp[q] = p[q] * fmaf(dp[q], kUnshift, -d4.x);
          dp[q + 1] = p[q + 1] * fmaf(dp[q + 1], kUnshift, -d4.y);
          dp[q + 2] = p[q + 2] * fmaf(dp[q + 2], kUnshift, -d4.z);
          dp[q + 3] = p[q + 3] * fmaf(dp[q + 3], kUnshift, -d4.w);
        }
        if (cols < 64) {
#pragma unroll
          for (int q = 0; q < 64; ++q) dp[q] = q < cols ? dp[q] : 0.0f;
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t w[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) w[q] = pack2<T>(dp[g * 32 + 2 * q], dp[g * 32 + 2 * q + 1]);
          tmem_st16(tdp + g * 16, w);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.ds_full));
      }
    }
    if (ok && n) {
      ok = mbar_wait(smem_u32(&bars.done), 0, limit);
      tc_fence_after();
    }
    if (named_barrier_and(1, 256, ok)) {
      // warpgroup 0 writes dv, warpgroup 1 dk
      const bool live = n > 0 && key0 + tile_row < nk;
      uint8_t* out = sKV + (half == 0 ? kTileBytes : 0u);
#pragma unroll
      for (int g = 0; g < DB * 2; ++g) {
        float o[32];
        if (n) { tmem_ld32(tmem + lane_base + 256 + half * 128 + g * 32, o); tmem_wait_ld(); }
        store_row32<T>(out, tile_row, g * 32, o, half == 0 ? kUnshift : a.scale, live);
      }
      fence_proxy_async();
      named_barrier(2 + half, 128);
      if ((warp & 3) == 0 && lane == 0) {
        store_tile<DB>(half == 0 ? mdv : mdk, smem_u32(out), key0, hk, b);
        bulk_commit();
        bulk_wait_read();
      }
    }
  }
  if (!ok && lane == 0) atomicExch(a.status, 1);
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

template <typename T, int DB>
cudaError_t launch_backward(const AttentionArgs& a, int dtype, cudaStream_t st) {
  static bool attr_set[64] = {};
  static std::mutex attr_mutex;
  {
    std::lock_guard<std::mutex> lock(attr_mutex);
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
      cudaError_t e = cudaFuncSetAttribute(attention_dq_kernel<T, DB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBwdSmem<DB>);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(attention_dkv_kernel<T, DB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBwdSmem<DB>);
      if (e != cudaSuccess) return e;
      attr_set[dev] = true;
    }
  }
  TileMap mq, mk, mv, mdo, mdq, mdk, mdv;
  cudaError_t e = make_tile_map(&mq, a.q, a.qs, dtype, a.batch, a.queries, a.heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mdo, a.dout, a.dos, dtype, a.batch, a.queries, a.heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mdq, a.dq, a.dqs, dtype, a.batch, a.queries, a.heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mk, a.k, a.ks, dtype, a.batch, a.keys, a.kv_heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mv, a.v, a.vs, dtype, a.batch, a.keys, a.kv_heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mdk, a.dk, a.dks, dtype, a.batch, a.keys, a.kv_heads, a.head_dim);
  if (e == cudaSuccess) e = make_tile_map(&mdv, a.dv, a.dvs, dtype, a.batch, a.keys, a.kv_heads, a.head_dim);
  if (e != cudaSuccess) return e;
  const int row_tiles = (a.queries + kTile - 1) / kTile, key_tiles = (a.keys + kTile - 1) / kTile;
  attention_dq_kernel<T, DB><<<(unsigned)((int64_t)row_tiles * a.heads * a.batch), kBwdThreads, kBwdSmem<DB>, st>>>(mq, mk, mv, mdo, mdq, a, row_tiles);
  attention_dkv_kernel<T, DB><<<(unsigned)((int64_t)key_tiles * a.kv_heads * a.batch), kBwdThreads, kBwdSmem<DB>, st>>>(mq, mk, mv, mdo, mdk, mdv, a, key_tiles);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_backward_tc(const AttentionArgs& a, int dtype, cudaStream_t st) {
  if (dtype == SWARM_BF16)
    return a.head_dim <= 64 ? launch_backward<__nv_bfloat16, 1>(a, dtype, st) : launch_backward<__nv_bfloat16, 2>(a, dtype, st);
  return a.head_dim <= 64 ? launch_backward<__half, 1>(a, dtype, st) : launch_backward<__half, 2>(a, dtype, st);
}

}  // namespace swarm
