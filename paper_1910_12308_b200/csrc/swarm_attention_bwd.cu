// Cross attention, backward pass on the tensor cores.
//
// Two kernels, so that every gradient is summed by one CTA in a fixed order and nothing is added with atomics:
//   attention_dq_kernel   CTA = tiles of 128 query rows: s and dp = dout v^T once per 64 states, dq = sum ds k; it also
//                         leaves lse and delta = rowsum(dout * o) as the other kernel wants them
//   attention_dkv_kernel  CTA = 128 states of a key head: the transposed products, over all rows of all its query
//                         heads: dv = sum p^T dout, dk = sum ds^T q
// The price is s and dp computed twice: 8 products instead of 5 (one for ds's second part, see dq).
// Measured: 32 x 16 heads of 64, 512 rows and states, bf16 227 us (dq 126, dkv 100), fp16 267 us; 4 x 16 heads of 128 on 4 key
// heads, 2048 rows, 4096 states, fp16, 1046 us (dq 573, dkv 465), 657 TFLOP/s of the five products. There the tensor pipe is
// busy 43 % (dq) and 59 % (dkv) of the time, in the first case 21 % and 29 %; a tile's chain of products, their latency (about
// 350 cycles from the issue to the barrier) and the warps' arithmetic is what the other tile covers in part.
#include <mutex>

#include "swarm_attention_tile.cuh"

namespace swarm {
namespace {

// =================================================================================================
// dq. NT row tiles per CTA, a warpgroup each (thread = row). Tensor memory of a tile: s (64 columns, two sets of them for
// NT = 1), dp (64) with ds (16 bits) over it, dq. The scores are computed one step ahead (NT = 1) or as soon as those of the
// step have been read into registers; dp follows once dq has taken ds. While one tile's warps are at their exponentials,
// the other tile's products (NT = 2) or the other CTA's of the multiprocessor (NT = 1, heads of up to 64 values) run. With
// two tiles the issuing thread takes up whichever barrier has completed: in a fixed order either tile's scores waited for
// the other's ds.
// delta = rowsum(dout * o) is off by what the rounding of o left; the sum of ds over a row, 0 in exact arithmetic, is that
// error, and the other kernel gets delta without it. Here it stays in ds (but for sentences of one step, where it can be
// taken out: with 6 states it doubled the error of dq), beside the rounding of ds to T; the two together would leave dq 1.55
// times as far from its value as its own rounding does. So ds is the sum of two numbers of T, both of which dq takes (the
// second lies beside the first, over the rest of dp): 1.02 to 1.2 times. That is for values around zero. The rounding of o, and
// with it delta's error, grows with a part that the values of a sentence share: of one deviation dq is 2.3 (512 states) to 3.4 times
// (4096) as far from its value as its own rounding leaves it, of four 8 and 13 times. To take it out for longer sentences needs
// sum p k, a further product and tensor memory that is not there.
// In fp16 a row's ds is held times a power of two, since its size is that of dout / states and fp16 ends at 2^-24 and 2^16:
// the first step's largest is brought to 2^7, and where a later one passes 2^15 the row's power and its sums so far come down
// (their product has completed when the step's dp has). It is taken out with the result's factor. Price: fp16 heads of 64, 512 rows
// and states, 32 x 16, backward 254 -> 267 us; heads of 128 1 %.
// =================================================================================================
constexpr int kStep = 64;                               // states of a step
constexpr int kStepBlock = kStep * 128;                 // bytes of 64 rows x 64 values

template <int DB, int NT> struct DqShape {
  static constexpr int kThreads = 128 * (NT + 1);
  static constexpr int kCtasPerSm = NT == 1 ? 2 : 1;
  static constexpr int kRegs = NT == 1 ? 192 : 208, kRegsRest = NT == 1 ? 64 : 88;
  static constexpr int kStages = NT == 1 ? 4 : 3;       // of (k, v)
  static constexpr int kSmem = NT * 2 * DB * kBlockBytes + kStages * 2 * DB * kStepBlock + 1024;
  static constexpr uint32_t kColumns = NT == 1 ? 256 : 512, kDp = NT == 1 ? 128 : 64, kDq = kDp + 64;
};

struct DqBars {
  uint64_t q_full[2], kv_full[4], kv_empty[4], s_full[2],   // s_full: of the tiles, or of the two sets of one tile's scores
      s_empty[2], dp_full[2], ds_full[2], done[2], edge_here, edge_done, drain;
};

template <typename T, int DB, int NT, bool SPLIT>
__global__ void __launch_bounds__(DqShape<DB, NT>::kThreads, DqShape<DB, NT>::kCtasPerSm)
attention_dq_kernel(const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv,
                    const __grid_constant__ TileMap mdo, const __grid_constant__ TileMap mdq, AttentionArgs a, int row_tiles,
                    int tile_groups, SplitPlan plan) {
  using Shape = DqShape<DB, NT>;
  constexpr int kStages = Shape::kStages;
  constexpr uint32_t kTileBytes = DB * kBlockBytes, kHalfBytes = DB * kStepBlock;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;                                   // per tile q, dout; dq on the way out
  uint8_t* sKV = smem + NT * 2 * kTileBytes;            // ring of (k, v)
  __shared__ DqBars bars;
  __shared__ uint32_t tmem_slot;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // the row tiles of this CTA: tiles are numbered head after head within the group of a key head
  const int split = SPLIT ? blockIdx.x % plan.splits : 0, cta = SPLIT ? blockIdx.x / plan.splits : blockIdx.x;
  const int first = cta % tile_groups * NT, bh = cta / tile_groups, hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const int all = (nk + kStep - 1) / kStep;             // steps; this CTA has n of them, the first of them `start`
  const int start = SPLIT ? (int)((int64_t)all * split / plan.splits) : 0;
  const int n = SPLIT ? (int)((int64_t)all * (split + 1) / plan.splits) - start : all;
  auto head_of = [&](int t) { return hk * a.group + (first + t) / row_tiles; };
  auto row_of = [&](int t) { return (first + t) % row_tiles * kTile; };
  auto exists = [&](int t) { return first + t < row_tiles * a.group; };
  uint32_t act = 0;                                     // bit t: tile t has work
#pragma unroll
  for (int t = 0; t < NT; ++t) act |= exists(t) && row_of(t) < nq && n > 0 ? 1u << t : 0u;
  auto active = [&](int t) { return (act >> t & 1u) != 0; };
  const int edge = nk % 16 && start + n == all ? nk % kStep : 0;       // states of the last step, where they end inside a product's sixteen

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars.q_full[i]), 1);
      mbar_init(smem_u32(&bars.s_full[i]), 1);
      mbar_init(smem_u32(&bars.s_empty[i]), 4);
      mbar_init(smem_u32(&bars.dp_full[i]), 1);
      mbar_init(smem_u32(&bars.ds_full[i]), 4);
      mbar_init(smem_u32(&bars.done[i]), 1);
    }
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars.kv_full[i]), 1); mbar_init(smem_u32(&bars.kv_empty[i]), 1); }
    mbar_init(smem_u32(&bars.edge_here), 1);
    mbar_init(smem_u32(&bars.edge_done), 1);
    mbar_init(smem_u32(&bars.drain), 1);
    fence_mbar_init();
  }
  if (warp == 4 * NT + 1) { tmem_alloc(smem_u32(&tmem_slot), Shape::kColumns); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, limit = a.wait_limit;
  bool ok = true;

  if (warp >= 4 * NT) {
    regs_lower<Shape::kRegsRest>();
    if (warp == 4 * NT && act && elect_one()) {
      // ---- copies (one thread) ----------------------------------------------------------------
      int issued = 0;
      if (limit) {
        for (int t = 0; t < NT; ++t)
          if (active(t)) {
            const uint32_t bar = smem_u32(&bars.q_full[t]), dst = smem_u32(sQ) + 2 * t * kTileBytes;
            mbar_expect_tx(bar, 2 * kTileBytes);
            load_tile<DB>(dst, mq, row_of(t), head_of(t), b, bar);
            load_tile<DB>(dst + kTileBytes, mdo, row_of(t), head_of(t), b, bar);
          }
      }
      for (int j = 0; j < n; ++j) {
        const int st = j % kStages;
        ok = mbar_wait_one(smem_u32(&bars.kv_empty[st]), ((j / kStages) & 1) ^ 1, limit);
        if (!ok) break;
        const uint32_t bar = smem_u32(&bars.kv_full[st]), dst = smem_u32(sKV) + 2 * st * kHalfBytes;
        mbar_expect_tx(bar, 2 * kHalfBytes);
        load_tile<DB, kStep>(dst, mk, (start + j) * kStep, hk, b, bar);
        load_tile<DB, kStep>(dst + kHalfBytes, mv, (start + j) * kStep, hk, b, bar);
        issued = j + 1;
      }
      // every copy lands before the CTA's shared memory is released, whichever of its threads gives up
      for (int j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
        mbar_wait_one(smem_u32(&bars.kv_full[j % kStages]), (j / kStages) & 1, kAttentionWaitLimit);
      for (int t = 0; t < NT; ++t)
        if (active(t) && limit) mbar_wait_one(smem_u32(&bars.q_full[t]), 0, kAttentionWaitLimit);
    } else if (warp == 4 * NT + 2 && act && edge) {
      // ---- the last step's end: k is a factor of dq -------------------------------------------
      const int st = (n - 1) % kStages;
      ok = mbar_wait(smem_u32(&bars.edge_here), 0, limit);
      if (ok) {
        zero_rows<DB, kStep>(sKV + 2 * st * kHalfBytes, edge, (edge + 15) & ~15, lane);
        if (lane == 0) mbar_arrive(smem_u32(&bars.edge_done));
      }
    } else if (warp == 4 * NT + 1 && act && elect_one()) {
      // ---- products (one thread) --------------------------------------------------------------
      const int ksteps = (a.head_dim + 15) / 16;
      const uint32_t aq = smem_u32(sQ), akv = smem_u32(sKV);
      auto columns = [&](int j) { return (min(kStep, nk - (start + j) * kStep) + 15) & ~15; };
      auto scores = [&](int t, int j) {
        mma_rows<T, DB, kStep>(tmem + 256 * t + (NT == 1 ? 64 * (j & 1) : 0), aq + 2 * t * kTileBytes,
                               akv + 2 * (j % kStages) * kHalfBytes, columns(j), ksteps);
        tc_commit(smem_u32(&bars.s_full[NT == 1 ? j & 1 : t]));
      };
      auto dps = [&](int t, int j) {
        mma_rows<T, DB, kStep>(tmem + 256 * t + Shape::kDp, aq + (2 * t + 1) * kTileBytes, akv + (2 * (j % kStages) + 1) * kHalfBytes,
                               columns(j), ksteps);
        tc_commit(smem_u32(&bars.dp_full[t]));
      };
      auto dqs = [&](int t, int j) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
          mma_weights<T, DB, kStep, false>(tmem + 256 * t + Shape::kDq, tmem + 256 * t + Shape::kDp + 32 * part,
                                           akv + 2 * (j % kStages) * kHalfBytes, columns(j) / 16, part != 0 || j != 0);
        if (j == n - 1) tc_commit(smem_u32(&bars.done[t]));
      };
      // the states of step j have landed, and what lies past their end is zeros where they end inside a product's sixteen
      auto wait_kv = [&](int j) {
        if (!mbar_wait_one(smem_u32(&bars.kv_full[j % kStages]), (j / kStages) & 1, limit)) return false;
        if (j < n - 1 || !edge) return true;
        mbar_arrive(smem_u32(&bars.edge_here));
        return mbar_wait_one(smem_u32(&bars.edge_done), 0, limit);
      };
      ok = wait_kv(0);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (active(t) && ok) {
          ok = mbar_wait_one(smem_u32(&bars.q_full[t]), 0, limit);
          tc_fence_after();
          if (ok) { scores(t, 0); dps(t, 0); }
        }
      if constexpr (NT == 1) {
        if (n > 1 && ok) {
          ok = wait_kv(1);
          tc_fence_after();
          if (ok) scores(0, 1);
        }
        for (int j = 0; j < n && ok; ++j) {
          ok = mbar_wait_one(smem_u32(&bars.ds_full[0]), j & 1, limit);
          if (!ok) break;
          tc_fence_after();
          dqs(0, j);
          if (j + 1 < n) dps(0, j + 1);
          tc_commit(smem_u32(&bars.kv_empty[j % kStages]));
          if (j + 2 < n) {                              // ds(j) has been written, so s(j) has been read
            ok = wait_kv(j + 2);
            tc_fence_after();
            if (ok) scores(0, j + 2);
          }
        }
      } else {
        int next_s[2] = {active(0) ? 1 : n, active(1) ? 1 : n}, next_ds[2] = {active(0) ? 0 : n, active(1) ? 0 : n};
        int here = 1, freed = 0;                        // steps whose states have landed; whose states are done with
        bool waits_edge = false;
        uint32_t idle = 0;
        while (ok && (next_ds[0] < n || next_ds[1] < n)) {
          bool moved = false;
          if (here < n && (next_s[0] == here || next_s[1] == here)) {
            if (!waits_edge && mbar_test(smem_u32(&bars.kv_full[here % kStages]), (here / kStages) & 1)) {
              waits_edge = here == n - 1 && edge;
              if (waits_edge) mbar_arrive(smem_u32(&bars.edge_here));
              else ++here;
              moved = true;
            } else if (waits_edge && mbar_test(smem_u32(&bars.edge_done), 0)) {
              ++here;
              moved = true;
            }
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (next_s[t] < here && mbar_test(smem_u32(&bars.s_empty[t]), (next_s[t] - 1) & 1)) {
              tc_fence_after();
              scores(t, next_s[t]);
              ++next_s[t];
              moved = true;
            }
            if (next_ds[t] < n && next_s[t] > min(next_ds[t] + 1, n - 1) && mbar_test(smem_u32(&bars.ds_full[t]), next_ds[t] & 1)) {
              tc_fence_after();
              dqs(t, next_ds[t]);
              ++next_ds[t];
              if (next_ds[t] < n) dps(t, next_ds[t]);
              if (min(next_ds[0], next_ds[1]) > freed) { tc_commit(smem_u32(&bars.kv_empty[freed % kStages])); ++freed; }
              moved = true;
            }
          }
          if (moved) idle = 0;
          else if (++idle >= limit) ok = false;             // reached for every limit, 2^32 - 1 included
        }
      }
      // no product is in flight when tensor memory is freed, whichever thread gives up
      tc_commit(smem_u32(&bars.drain));
      mbar_wait_one(smem_u32(&bars.drain), 0, kAttentionWaitLimit);
    }
    __syncwarp();
  } else {
    // ---- ds -----------------------------------------------------------------------------------
    regs_raise<Shape::kRegs>();
    const int t = NT == 1 ? 0 : warp >> 2, quad = warp & 3, head = head_of(t), row0 = row_of(t), tile_row = quad * 32 + lane;
    const bool work = active(t);
    const int row = row0 + tile_row;
    const uint32_t tile = tmem + 256 * t + ((uint32_t)(quad * 32) << 16), tdp = tile + Shape::kDp;
    const float c = a.scale * kLog2e;
    const bool live = work && row < nq;
    float up = 1.0f, peak = 0.0f;                       // fp16: what ds is held times, and the largest so far
    float delta = 0.0f, size = 0.0f, taken = 0.0f, lse2 = INFINITY, off[2] = {0.0f, 0.0f};
    if (live) {
      const T* g = reinterpret_cast<const T*>(a.dout) + offset_of(a.dos, b, row, head);
      const T* o = reinterpret_cast<const T*>(a.o) + offset_of(a.os, b, row, head);
      lse2 = a.lse_in[((int64_t)b * a.heads + head) * a.queries + row] * kLog2e;
#pragma unroll 4
      for (int d = 0; d < a.head_dim; d += 8) {
        float x[8], y[8];
        unpack8<T>(load_raw8<T>(g + d), x);
        unpack8<T>(load_raw8<T>(o + d), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          delta = fmaf(x[i], y[i], delta);
          if constexpr (kNarrow<T>) size += fabsf(x[i]);
        }
      }
    }
    if (work) {
      bool ahead = false;                               // the scores of the step have been seen to be there
      for (int j = 0; j < n; ++j) {
        const int valid = nk - (start + j) * kStep;
        float p[kStep], dp[kStep];
        ok = NT == 1 ? mbar_wait_after(ahead, smem_u32(&bars.s_full[j & 1]), (j >> 1) & 1, limit)
                     : mbar_wait_after(ahead, smem_u32(&bars.s_full[t]), j & 1, limit);
        if (!ok) break;
        tc_fence_after();
        const uint32_t ts = tile + (NT == 1 ? 64 * (j & 1) : 0);
        tmem_ld32(ts, p);
        tmem_ld32(ts + 32, p + 32);
        tmem_wait_ld();
        if (NT == 2) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars.s_empty[t]));
        }
#pragma unroll
        for (int i = 0; i < kStep; i += 2) {
          fma2(p[i], p[i + 1], p[i], p[i + 1], c, c, -lse2, -lse2);
          p[i] = ex2(p[i]);
          p[i + 1] = ex2(p[i + 1]);
        }
        ok = mbar_wait(smem_u32(&bars.dp_full[t]), j & 1, limit);
        if (!ok) break;
        tc_fence_after();
        tmem_ld32(tdp, dp);
        tmem_ld32(tdp + 32, dp + 32);
        tmem_wait_ld();
        if (all == 1) {                                 // all states are here: take delta's error out
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < kStep; ++i) sum += i < valid ? p[i] * (dp[i] - delta) : 0.0f;
          delta += sum;
          taken = sum;
        }
#pragma unroll
        for (int i = 0; i < kStep; i += 2) {
          if constexpr (kNarrow<T>) fma2(dp[i], dp[i + 1], dp[i], dp[i + 1], up, up, -delta * up, -delta * up);
          else add2(dp[i], dp[i + 1], dp[i], dp[i + 1], -delta, -delta);
          mul2(p[i], p[i + 1], p[i], p[i + 1], dp[i], dp[i + 1]);
        }
        if (valid < kStep) {
#pragma unroll
          for (int i = 0; i < kStep; ++i) p[i] = i < valid ? p[i] : 0.0f;
        }
        if constexpr (kNarrow<T>) {
          float top = 0.0f;
#pragma unroll
          for (int i = 0; i < kStep; i += 2) top = max3(top, fabsf(p[i]), fabsf(p[i + 1]));
          if (j == 0 || __any_sync(0xFFFFFFFFu, top > 0x1p15f)) {
            const float f = j == 0 || top > 0x1p15f ? power_to<7>(top) : 1.0f;
            up *= f;
            peak *= f;
            top *= f;
            off[0] *= f;
            off[1] *= f;
#pragma unroll
            for (int i = 0; i < kStep; ++i) p[i] *= f;
            if (j > 0) {
#pragma unroll
              for (int g = 0; g < DB * 2; ++g) {
                float o[32];
                tmem_ld32(tile + Shape::kDq + g * 32, o);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= f;
                tmem_st32(tile + Shape::kDq + g * 32, o);
              }
            }
          }
          peak = fmaxf(peak, top);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            add2(off[0], off[1], off[0], off[1], p[g * 32 + 2 * i], p[g * 32 + 2 * i + 1]);
            w[i] = pack2<T>(p[g * 32 + 2 * i], p[g * 32 + 2 * i + 1]);
          }
          tmem_st16(tdp + g * 16, w);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float a0, a1;
            unpack2<T>(w[i], a0, a1);
            fma2(a0, a1, a0, a1, -1.0f, -1.0f, p[g * 32 + 2 * i], p[g * 32 + 2 * i + 1]);
            w[i] = pack2<T>(a0, a1);
          }
          tmem_st16(tdp + 32 + g * 16, w);
        }
        ahead = j + 1 < n && (NT == 1 ? mbar_test(smem_u32(&bars.s_full[(j + 1) & 1]), ((j + 1) >> 1) & 1)
                                      : mbar_test(smem_u32(&bars.s_full[t]), (j + 1) & 1));
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.ds_full[t]));
      }
      if (ok) {
        ok = mbar_wait(smem_u32(&bars.done[t]), 0, limit);
        tc_fence_after();
      }
    }
    const int64_t stat = stat_offset(((int64_t)b * a.heads + head) * row_tiles * kTile + row);
    const float down = 1.0f / up;                       // a power of two
    const bool write = exists(t) && named_barrier_and(1 + t, 128, ok);
    if (kNarrow<T> && write) {
      peak = live ? fmaxf(peak * down, size * 0x1p-7f) : 0.0f;         // size: sum of |dout|
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, o));
      if (lane == 0)
        a.stat_peak[((((int64_t)b * a.heads + head) * row_tiles + row0 / kTile) * 4 + quad) * plan.splits + split] = peak;
    }
    if (!write) {
      // nothing to write
    } else if (SPLIT) {
      // this CTA's part of the row: dq without its factor, and delta's error: the sum of ds and what was taken out before
      const int64_t at = (((int64_t)bh * a.queries + row) * a.group + (head - hk * a.group)) * plan.splits + split;
#pragma unroll
      for (int g = 0; g < DB * 2; ++g) {
        float o[32];
        if (work) { tmem_ld32(tile + Shape::kDq + g * 32, o); tmem_wait_ld(); }
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          if (row < a.queries && g * 32 + i < a.head_dim)
            *reinterpret_cast<float4*>(plan.part_o + at * a.head_dim + g * 32 + i) =
                live ? make_float4(o[i] * down, o[i + 1] * down, o[i + 2] * down, o[i + 3] * down) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if (row < a.queries) *reinterpret_cast<float2*>(plan.part_ml + at * 2) = make_float2(live ? taken + (off[0] + off[1]) * down : 0.0f, 0.0f);
      else if (split == 0) {                            // rows of the tile past the tensor's
        store_stat(a.stat_lse + stat, -INFINITY);
        store_stat(a.stat_delta + stat, 0.0f);
      }
    } else {
      store_stat(a.stat_lse + stat, (kWeightShift<T> - lse2) / c);    // in units of a score; -infinity in rows that take no part
      store_stat(a.stat_delta + stat, live ? -(delta + (off[0] + off[1]) * down) : 0.0f);
      uint8_t* out = sQ + 2 * t * kTileBytes;
#pragma unroll
      for (int g = 0; g < DB * 2; ++g) {
        float o[32];
        if (work) { tmem_ld32(tile + Shape::kDq + g * 32, o); tmem_wait_ld(); }
        store_row32<T>(out, tile_row, g * 32, o, a.scale * down, live);
      }
      fence_proxy_async();
      named_barrier(1 + t, 128);
      if (quad == 0 && lane == 0) {
        store_tile<DB>(mdq, smem_u32(out), row0, head, b);
        bulk_commit();
        bulk_wait_read();
      }
    }
  }
  if (!ok) atomicExch(a.status, 1);
  tc_fence_before();
  __syncthreads();
  if (warp == 4 * NT + 1) tmem_dealloc(tmem, Shape::kColumns);
}

// Joins the parts of a row's dq and leaves its statistics: warp = one row, lane = four of its values, the parts in order.
template <typename T>
__global__ void __launch_bounds__(128) attention_dq_join_kernel(AttentionArgs a, SplitPlan plan, int row_tiles) {
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (i >= (int64_t)a.batch * a.kv_heads * plan.rows) return;
  const int r = (int)(i % plan.rows), bh = (int)(i / plan.rows), hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int t = r / a.group, h = hk * a.group + r % a.group;
  const bool live = t < length_of(a.query_lengths, b, a.queries) && length_of(a.key_lengths, b, a.keys) > 0;
  const bool mine = lane * 4 < a.head_dim;
  float delta = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (live && mine) {
    const uint2 g = *reinterpret_cast<const uint2*>(reinterpret_cast<const T*>(a.dout) + offset_of(a.dos, b, t, h) + lane * 4);
    const uint2 o = *reinterpret_cast<const uint2*>(reinterpret_cast<const T*>(a.o) + offset_of(a.os, b, t, h) + lane * 4);
    float g0, g1, o0, o1;
    unpack2<T>(g.x, g0, g1); unpack2<T>(o.x, o0, o1);
    delta = fmaf(g0, o0, g1 * o1);
    unpack2<T>(g.y, g0, g1); unpack2<T>(o.y, o0, o1);
    delta = fmaf(g0, o0, fmaf(g1, o1, delta));
  }
  delta = warp_sum(delta) + warp_sum(lane < plan.splits ? plan.part_ml[(i * plan.splits + lane) * 2] : 0.0f);
  const float* part = plan.part_o + i * plan.splits * a.head_dim + lane * 4;
#pragma unroll 8
  for (int s = 0; s < plan.splits; ++s)
    if (mine) {
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)s * a.head_dim);
      v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
  if (mine) {
    const uint2 w = live ? make_uint2(pack2<T>(v[0] * a.scale, v[1] * a.scale), pack2<T>(v[2] * a.scale, v[3] * a.scale)) : make_uint2(0, 0);
    *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.dq) + offset_of(a.dqs, b, t, h) + lane * 4) = w;
  }
  if (lane == 0) {
    const int64_t head = (int64_t)b * a.heads + h, stat = stat_offset(head * row_tiles * kTile + t);
    store_stat(a.stat_lse + stat, live ? (kWeightShift<T> - a.lse_in[head * a.queries + t] * kLog2e) / (a.scale * kLog2e) : -INFINITY);
    store_stat(a.stat_delta + stat, live ? -delta : 0.0f);
  }
}

// As for the forward pass (make_forward_plan): few row tiles over many states are split, eight steps of 64 or more to each
// part, where that saves 24 steps of about 1 us.
SplitPlan make_dq_plan(const AttentionArgs& a) {
  SplitPlan p{};
  const int nt = a.head_dim <= 64 ? 1 : 2;
  const int64_t row_tiles = (a.queries + kTile - 1) / kTile, steps = (a.keys + kStep - 1) / kStep;
  const int64_t ctas = (row_tiles * a.group + nt - 1) / nt * a.kv_heads * a.batch, room = 148 * (nt == 1 ? 2 : 1);
  int64_t s = room / ctas;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s > steps / 8) s = steps / 8;
  if (s < 2 || steps - (steps + s - 1) / s < 24) s = 1;
  p.splits = (int32_t)s;
  p.rows = s > 1 ? a.queries * a.group : 0;
  return p;
}

// =================================================================================================
// dk and dv. Rows of the transposed tile are states (lanes), columns are 64 NW query rows, 64 for each of NW warpgroups.
// Tensor memory: s^T with p^T (16 bits) over the columns that the same warpgroup read, dp^T with ds^T over it, dv, dk. The
// warps turn s^T(i) into p^T while dp^T(i) is computed, and dp^T(i) into ds^T while dv takes p^T(i) and s^T(i + 1) is
// computed. lse and delta belong to columns here, so no thread can keep its own: they join the products as a further
// sixteen of the contraction, q's row with -lse against a row of ones beside k, and dout's with -delta beside v. (Read
// from shared memory by every thread they took 32 loads a step, which waited behind the special functions: 1.17 ms
// against 1.05 ms for the backward pass of 4 x 16 heads of 64, 4096 rows and states.)
// In fp16 ds^T is held times one power of two for all rows that a state's dk sums, which brings the largest |ds| that the dq
// kernel saw among them to 2^13: room for four times as much above (p is formed again here, from scores of another product), 27
// powers of two below it before bits are lost. It takes the place of the power that p is held times. Where ds cancels to nothing
// what is left of it here may be any multiple of what is left there: at most a few roundings of dout v^T, 2^-21 of
// sum |dout| * 2^16. So the largest |ds| counts as at least 2^-7 of sum |dout|, which keeps that below fp16's end as well.
// =================================================================================================
template <int DB, int NW> struct DkvShape {
  static constexpr int kThreads = 128 * (NW + 1);
  static constexpr int kCtasPerSm = NW == 1 ? 2 : 1;
  static constexpr int kRegs = NW == 1 ? 192 : 208, kRegsRest = NW == 1 ? 64 : 88;
  static constexpr int kRows = 64 * NW;                 // query rows of a step
  static constexpr int kHalfBytes = DB * kRows * 128;   // of q or dout
  static constexpr int kStages = NW == 1 ? 3 : 2;
  static constexpr int kStatBytes = kRows * 32;         // of lse or delta
  static constexpr int kOnesBytes = kTile * 32;
  static constexpr int kSmem = 2 * DB * kBlockBytes + kStages * 2 * (kHalfBytes + kStatBytes) + kOnesBytes + 1024;
  static constexpr uint32_t kColumns = NW == 1 ? 256 : 512;
  static constexpr uint32_t kDp = kRows, kDv = 2 * kRows, kDk = 2 * kRows + DB * 64;
};

struct DkvBars {
  uint64_t kv_full, full[4], empty[4], s_full, p_full, dp_full, ds_full, done, edge_here, edge_done, drain;
};

template <typename T, int DB, int NW, bool SPLIT>
__global__ void __launch_bounds__(DkvShape<DB, NW>::kThreads, DkvShape<DB, NW>::kCtasPerSm)
attention_dkv_kernel(const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv,
                     const __grid_constant__ TileMap mdo, const __grid_constant__ TileMap mdk, const __grid_constant__ TileMap mdv,
                     AttentionArgs a, int key_tiles, int row_tiles, int dq_splits, SplitPlan plan) {
  using Shape = DkvShape<DB, NW>;
  constexpr int kStages = Shape::kStages, kRows = Shape::kRows;
  constexpr uint32_t kTileBytes = DB * kBlockBytes, kHalfBytes = Shape::kHalfBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sKV = smem;                                  // k, v; dk, dv on the way out
  uint8_t* sQ = smem + 2 * kTileBytes;                  // ring of (q, dout)
  uint8_t* sStat = sQ + kStages * 2 * kHalfBytes;       // ring of (lse, delta)
  uint8_t* sOnes = sStat + kStages * 2 * Shape::kStatBytes;
  __shared__ DkvBars bars;
  __shared__ uint32_t tmem_slot;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = SPLIT ? blockIdx.x % plan.splits : 0, cta = SPLIT ? blockIdx.x / plan.splits : blockIdx.x;
  const int kt = cta % key_tiles, bh = cta / key_tiles, hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const int key0 = kt * kTile, steps = (nq + kRows - 1) / kRows;       // steps of one head
  const int64_t all = key0 < nk ? (int64_t)steps * a.group : 0;        // steps of all heads; this CTA has n, from `start`
  const int start = SPLIT ? (int)(all * split / plan.splits) : 0;
  const int n = SPLIT ? (int)(all * (split + 1) / plan.splits) - start : (int)all;
  const int step0 = SPLIT && n ? start % steps : 0;                    // the first one's place within its head
  const int edge = nq % 16 ? nq % kRows : 0;            // rows of a head's last step, where they end inside a product's sixteen

  if (tid == 0) {
    mbar_init(smem_u32(&bars.kv_full), 1);
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars.full[i]), 1); mbar_init(smem_u32(&bars.empty[i]), 1); }
    mbar_init(smem_u32(&bars.s_full), 1);
    mbar_init(smem_u32(&bars.p_full), 4 * NW);
    mbar_init(smem_u32(&bars.dp_full), 1);
    mbar_init(smem_u32(&bars.ds_full), 4 * NW);
    mbar_init(smem_u32(&bars.done), 1);
    mbar_init(smem_u32(&bars.edge_here), 1);
    mbar_init(smem_u32(&bars.edge_done), 1);
    mbar_init(smem_u32(&bars.drain), 1);
    fence_mbar_init();
  }
  if (warp == 4 * NW + 1) { tmem_alloc(smem_u32(&tmem_slot), Shape::kColumns); tmem_relinquish(); }
  if (tid < kTile) {                                    // the row of ones, for 128 states
    const uint32_t one = pack2<StatType>(1.0f, 1.0f);
    uint8_t* p = sOnes + stat_offset(tid);
    *reinterpret_cast<uint4*>(p) = make_uint4(one, one & 0xFFFFu, 0u, 0u);
    *reinterpret_cast<uint4*>(p + 128) = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, limit = a.wait_limit;
  bool ok = true;

  if (warp >= 4 * NW) {
    regs_lower<Shape::kRegsRest>();
    if (warp == 4 * NW && n && elect_one()) {
      // ---- copies (one thread) ----------------------------------------------------------------
      int issued = 0;
      if (limit) {
        const uint32_t bar = smem_u32(&bars.kv_full);
        mbar_expect_tx(bar, 2 * kTileBytes);
        load_tile<DB>(smem_u32(sKV), mk, key0, hk, b, bar);
        load_tile<DB>(smem_u32(sKV) + kTileBytes, mv, key0, hk, b, bar);
      }
      int h = hk * a.group + (SPLIT ? start / steps : 0), row0 = step0 * kRows;
      for (int i = 0; i < n; ++i) {
        const int st = i % kStages;
        ok = mbar_wait_one(smem_u32(&bars.empty[st]), ((i / kStages) & 1) ^ 1, limit);
        if (!ok) break;
        const uint32_t bar = smem_u32(&bars.full[st]), dst = smem_u32(sQ) + 2 * st * kHalfBytes;
        const uint32_t stat = smem_u32(sStat) + 2 * st * Shape::kStatBytes;
        const int64_t at = stat_offset(((int64_t)b * a.heads + h) * row_tiles * kTile + row0);
        mbar_expect_tx(bar, 2 * (kHalfBytes + Shape::kStatBytes));
        load_tile<DB, kRows>(dst, mq, row0, h, b, bar);
        load_tile<DB, kRows>(dst + kHalfBytes, mdo, row0, h, b, bar);
        bulk_load(stat, a.stat_lse + at, Shape::kStatBytes, bar);
        bulk_load(stat + Shape::kStatBytes, a.stat_delta + at, Shape::kStatBytes, bar);
        issued = i + 1;
        row0 += kRows;
        if (row0 >= nq) { row0 = 0; ++h; }
      }
      // every copy lands before the CTA's shared memory is released, whichever of its threads gives up
      for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
        mbar_wait_one(smem_u32(&bars.full[i % kStages]), (i / kStages) & 1, kAttentionWaitLimit);
      if (limit) mbar_wait_one(smem_u32(&bars.kv_full), 0, kAttentionWaitLimit);
    } else if (warp == 4 * NW + 2 && edge) {
      // ---- the end of each head's last step: q and dout are factors of dk and dv ----------------
      for (int i = steps - 1 - step0, g = 0; i < n && ok; i += steps, ++g) {
        const int st = i % kStages;
        ok = mbar_wait(smem_u32(&bars.edge_here), g & 1, limit);
        if (!ok) break;
        zero_rows<DB, kRows>(sQ + 2 * st * kHalfBytes, edge, (edge + 15) & ~15, lane);
        zero_rows<DB, kRows>(sQ + (2 * st + 1) * kHalfBytes, edge, (edge + 15) & ~15, lane);
        if (lane == 0) mbar_arrive(smem_u32(&bars.edge_done));
      }
    } else if (warp == 4 * NW + 1 && n && elect_one()) {
      // ---- products (one thread) --------------------------------------------------------------
      const int ksteps = (a.head_dim + 15) / 16;
      const uint32_t akv = smem_u32(sKV), aq = smem_u32(sQ);
      const int last_cols = (nq - (steps - 1) * kRows + 15) & ~15;     // columns of a head's last step
      const uint64_t d_ones = smem_desc_plain(smem_u32(sOnes), 128, 256);
      // d += ones x stat^T: the number `which` (0 lse, 1 delta) of the stage's rows
      auto add_stat = [&](uint32_t d, int stage, int which, int columns) {
        tc_mma(d, d_ones, smem_desc_plain(smem_u32(sStat) + (2 * stage + which) * Shape::kStatBytes, 128, 256),
               instr_desc_16<StatType>(kTile, 0, 0, 0) + ((uint32_t)(columns >> 3) << 17), 1);
      };
      ok = mbar_wait_one(smem_u32(&bars.kv_full), 0, limit);
      int cols = 0, cols_next = 0, step = step0, head = 0;  // columns of steps i and i + 1; the latter's place
      for (int i = -1; i < n && ok; ++i) {
        const int st = i % kStages, next = (i + 1) % kStages;
        const bool last = step == steps - 1, at_edge = i + 1 < n && last && edge;
        cols = cols_next;
        if (at_edge) {
          ok = mbar_wait_one(smem_u32(&bars.full[next]), ((i + 1) / kStages) & 1, limit);
          if (!ok) break;
          mbar_arrive(smem_u32(&bars.edge_here));
        }
        if (i >= 0) {
          ok = mbar_wait_one(smem_u32(&bars.p_full), i & 1, limit);
          if (!ok) break;
          tc_fence_after();
          mma_weights<T, DB, kRows, true>(tmem + Shape::kDv, tmem, aq + (2 * st + 1) * kHalfBytes, cols / 16, i != 0);
        }
        if (i + 1 < n) {
          ok = mbar_wait_one(smem_u32(&bars.full[next]), ((i + 1) / kStages) & 1, limit) &&
               (!at_edge || mbar_wait_one(smem_u32(&bars.edge_done), head & 1, limit));
          if (!ok) break;
          cols_next = last ? last_cols : kRows;
          if (last) { step = 0; ++head; } else ++step;
          tc_fence_after();
          mma_rows<T, DB, kRows>(tmem, akv, aq + 2 * next * kHalfBytes, cols_next, ksteps);
          add_stat(tmem, next, 0, cols_next);
          tc_commit(smem_u32(&bars.s_full));
        }
        if (i >= 0) {
          ok = mbar_wait_one(smem_u32(&bars.ds_full), i & 1, limit);
          if (!ok) break;
          tc_fence_after();
          mma_weights<T, DB, kRows, true>(tmem + Shape::kDk, tmem + Shape::kDp, aq + 2 * st * kHalfBytes, cols / 16, i != 0);
          tc_commit(smem_u32(&bars.empty[st]));
          if (i == n - 1) tc_commit(smem_u32(&bars.done));
        }
        if (i + 1 < n) {
          mma_rows<T, DB, kRows>(tmem + Shape::kDp, akv + kTileBytes, aq + (2 * next + 1) * kHalfBytes, cols_next, ksteps);
          add_stat(tmem + Shape::kDp, next, 1, cols_next);
          tc_commit(smem_u32(&bars.dp_full));
        }
      }
      // no product is in flight when tensor memory is freed, whichever thread gives up
      tc_commit(smem_u32(&bars.drain));
      mbar_wait_one(smem_u32(&bars.drain), 0, kAttentionWaitLimit);
    }
    __syncwarp();
  } else {
    // ---- p and ds -----------------------------------------------------------------------------
    regs_raise<Shape::kRegs>();
    const int half = NW == 1 ? 0 : warp >> 2, quad = warp & 3, tile_row = quad * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = tmem + lane_base + half * 64, tdp = ts + Shape::kDp;
    const float c = a.scale * kLog2e;
    constexpr float kUnshift = pow2_of(kWeightShift<T>);
    float up = 1.0f;                                    // fp16: what ds is held times
    if (kNarrow<T> && n) {
      const int64_t peaks = (int64_t)a.group * row_tiles * 4 * dq_splits;
      const float* of_head = a.stat_peak + ((int64_t)b * a.kv_heads + hk) * peaks;
      float peak = 0.0f;
#pragma unroll 4
      for (int64_t i = lane; i < peaks; i += 32) peak = fmaxf(peak, of_head[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, o));
      up = isinf(peak) ? 1.0f : power_to<13>(peak);
    }
    const float p_to_ds = kUnshift * up, dk_factor = a.scale / up;
    int step = step0;
    for (int i = 0; i < n; ++i) {
      const int cols = (step == steps - 1 ? nq - step * kRows : kRows) - half * 64;   // columns of this warpgroup that exist
      if (++step == steps) step = 0;
      float p[64];
      ok = mbar_wait(smem_u32(&bars.s_full), i & 1, limit);
      if (!ok) break;
      tc_fence_after();
      tmem_ld32(ts, p);
      tmem_ld32(ts + 32, p + 32);
      tmem_wait_ld();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t w[16];
#pragma unroll
        for (int q = g * 32; q < g * 32 + 32; q += 2) {
          mul2(p[q], p[q + 1], p[q], p[q + 1], c, c);
          p[q] = ex2(p[q]);
          p[q + 1] = ex2(p[q + 1]);
        }
        if (cols < 64) {
#pragma unroll
          for (int q = g * 32; q < g * 32 + 32; ++q) p[q] = q < cols ? p[q] : 0.0f;   // what lies there is not a score
        }
#pragma unroll
        for (int q = 0; q < 16; ++q) w[q] = pack2<T>(p[g * 32 + 2 * q], p[g * 32 + 2 * q + 1]);
        tmem_st16(ts + g * 16, w);
      }
      const bool ahead = mbar_test(smem_u32(&bars.dp_full), i & 1);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.p_full));
      ok = mbar_wait_after(ahead, smem_u32(&bars.dp_full), i & 1, limit);
      if (!ok) break;
      tc_fence_after();
      float dp[64];
      tmem_ld32(tdp, dp);
      tmem_ld32(tdp + 32, dp + 32);
      tmem_wait_ld();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t w[16];
#pragma unroll
        for (int q = g * 32; q < g * 32 + 32; q += 2) {
          if constexpr (kNarrow<T>) mul2(dp[q], dp[q + 1], dp[q], dp[q + 1], p_to_ds, p_to_ds);
          mul2(dp[q], dp[q + 1], dp[q], dp[q + 1], p[q], p[q + 1]);
        }
        if (cols < 64) {
#pragma unroll
          for (int q = g * 32; q < g * 32 + 32; ++q) dp[q] = q < cols ? dp[q] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 16; ++q) w[q] = pack2<T>(dp[g * 32 + 2 * q], dp[g * 32 + 2 * q + 1]);
        tmem_st16(tdp + g * 16, w);
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
    const bool live = n > 0 && key0 + tile_row < nk;
    // two warpgroups write dv and dk, one writes both
    if (!named_barrier_and(1, 128 * NW, ok)) {
      // nothing to write
    } else if (SPLIT) {
      // this CTA's part of the state's dk and dv, with their factors
      const int64_t at = ((int64_t)bh * a.keys + key0 + tile_row) * plan.splits + split;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (NW == 2 && which != half) continue;
        const float factor = which == 0 ? kUnshift : dk_factor;
#pragma unroll
        for (int g = 0; g < DB * 2; ++g) {
          float o[32];
          if (n) { tmem_ld32(tmem + lane_base + (which == 0 ? Shape::kDv : Shape::kDk) + g * 32, o); tmem_wait_ld(); }
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            if (key0 + tile_row < a.keys && g * 32 + i < a.head_dim)
              *reinterpret_cast<float4*>(plan.part_o + (at * 2 + which) * a.head_dim + g * 32 + i) =
                  live ? make_float4(o[i] * factor, o[i + 1] * factor, o[i + 2] * factor, o[i + 3] * factor) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
    } else {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (NW == 2 && which != half) continue;
        uint8_t* out = sKV + (which == 0 ? kTileBytes : 0u);
#pragma unroll
        for (int g = 0; g < DB * 2; ++g) {
          float o[32];
          if (n) { tmem_ld32(tmem + lane_base + (which == 0 ? Shape::kDv : Shape::kDk) + g * 32, o); tmem_wait_ld(); }
          store_row32<T>(out, tile_row, g * 32, o, which == 0 ? kUnshift : dk_factor, live);
        }
      }
      fence_proxy_async();
      named_barrier(1, 128 * NW);
      if (tid == 0) {
        store_tile<DB>(mdv, smem_u32(sKV) + kTileBytes, key0, hk, b);
        store_tile<DB>(mdk, smem_u32(sKV), key0, hk, b);
        bulk_commit();
        bulk_wait_read();
      }
    }
  }
  if (!ok) atomicExch(a.status, 1);
  tc_fence_before();
  __syncthreads();
  if (warp == 4 * NW + 1) tmem_dealloc(tmem, Shape::kColumns);
}

// Joins the parts of a state's dk and dv: warp = one state of one key head, lane = four values of each, the parts in order.
template <typename T>
__global__ void __launch_bounds__(128) attention_dkv_join_kernel(AttentionArgs a, SplitPlan plan) {
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (i >= (int64_t)a.batch * a.kv_heads * a.keys || lane * 4 >= a.head_dim) return;
  const int j = (int)(i % a.keys), bh = (int)(i / a.keys), hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const float* part = plan.part_o + i * plan.splits * 2 * a.head_dim + lane * 4;
  float v[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
  for (int s = 0; s < plan.splits; ++s)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)(2 * s + which) * a.head_dim);
      v[which][0] += x.x; v[which][1] += x.y; v[which][2] += x.z; v[which][3] += x.w;
    }
  *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.dv) + offset_of(a.dvs, b, j, hk) + lane * 4) = make_uint2(pack2<T>(v[0][0], v[0][1]), pack2<T>(v[0][2], v[0][3]));
  *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.dk) + offset_of(a.dks, b, j, hk) + lane * 4) = make_uint2(pack2<T>(v[1][0], v[1][1]), pack2<T>(v[1][2], v[1][3]));
}

// The same for few states under many rows: eight steps of 64 rows (or four of 128) or more to each part, where that saves 24
// (or 12) of them.
SplitPlan make_dkv_plan(const AttentionArgs& a) {
  SplitPlan p{};
  const int rows = a.head_dim <= 64 ? DkvShape<1, 1>::kRows : DkvShape<2, 2>::kRows;
  const int64_t steps = (int64_t)((a.queries + rows - 1) / rows) * a.group;
  const int64_t ctas = (int64_t)((a.keys + kTile - 1) / kTile) * a.kv_heads * a.batch, room = 148 * (a.head_dim <= 64 ? 2 : 1);
  int64_t s = room / ctas;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s > steps * rows / 512) s = steps * rows / 512;
  if (s < 2 || (steps - (steps + s - 1) / s) * rows < 24 * 64) s = 1;
  p.splits = (int32_t)s;
  return p;
}
size_t dkv_part_bytes(const AttentionArgs& a, const SplitPlan& p) {
  return p.splits == 1 ? 0 : (size_t)a.batch * a.kv_heads * a.keys * p.splits * 2 * a.head_dim * sizeof(float);
}

template <typename T, int DB>
cudaError_t launch_backward(const AttentionArgs& a, const SplitPlan& plan, const SplitPlan& dkv, int dtype, cudaStream_t st) {
  using Dq = DqShape<DB, DB>;                           // heads of up to 64 values: one tile and two CTAs per multiprocessor
  using Dkv = DkvShape<DB, DB>;
  static bool attr_set[64] = {};
  static std::mutex attr_mutex;
  {
    std::lock_guard<std::mutex> lock(attr_mutex);
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
      cudaError_t e = cudaFuncSetAttribute(attention_dq_kernel<T, DB, DB, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Dq::kSmem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(attention_dq_kernel<T, DB, DB, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Dq::kSmem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(attention_dkv_kernel<T, DB, DB, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Dkv::kSmem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(attention_dkv_kernel<T, DB, DB, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Dkv::kSmem);
      if (e != cudaSuccess) return e;
      attr_set[dev] = true;
    }
  }
  TileMap mq, mk, mv, mdo, mdq, mdk, mdv;
  auto rows = [&](TileMap* m, const void* p, const swarm_strides& s, int box) { return make_tile_map(m, p, s, dtype, a.batch, a.queries, a.heads, a.head_dim, box); };
  auto states = [&](TileMap* m, const void* p, const swarm_strides& s, int box) { return make_tile_map(m, p, s, dtype, a.batch, a.keys, a.kv_heads, a.head_dim, box); };
  cudaError_t e = rows(&mq, a.q, a.qs, kTile);
  if (e == cudaSuccess) e = rows(&mdo, a.dout, a.dos, kTile);
  if (e == cudaSuccess) e = rows(&mdq, a.dq, a.dqs, kTile);
  if (e == cudaSuccess) e = states(&mk, a.k, a.ks, kStep);
  if (e == cudaSuccess) e = states(&mv, a.v, a.vs, kStep);
  if (e != cudaSuccess) return e;
  const int row_tiles = (a.queries + kTile - 1) / kTile, key_tiles = (a.keys + kTile - 1) / kTile;
  const int tile_groups = (int)(((int64_t)row_tiles * a.group + DB - 1) / DB);
  const unsigned dq_ctas = (unsigned)((int64_t)tile_groups * a.kv_heads * a.batch * plan.splits);
  if (plan.splits > 1) {
    attention_dq_kernel<T, DB, DB, true><<<dq_ctas, Dq::kThreads, Dq::kSmem, st>>>(mq, mk, mv, mdo, mdq, a, row_tiles, tile_groups, plan);
    attention_dq_join_kernel<T><<<(unsigned)(((int64_t)a.batch * a.kv_heads * plan.rows + 3) / 4), 128, 0, st>>>(a, plan, row_tiles);
  } else {
    attention_dq_kernel<T, DB, DB, false><<<dq_ctas, Dq::kThreads, Dq::kSmem, st>>>(mq, mk, mv, mdo, mdq, a, row_tiles, tile_groups, plan);
  }
  e = cudaGetLastError();
  if (e == cudaSuccess) e = rows(&mq, a.q, a.qs, Dkv::kRows);
  if (e == cudaSuccess) e = rows(&mdo, a.dout, a.dos, Dkv::kRows);
  if (e == cudaSuccess) e = states(&mk, a.k, a.ks, kTile);
  if (e == cudaSuccess) e = states(&mv, a.v, a.vs, kTile);
  if (e == cudaSuccess) e = states(&mdk, a.dk, a.dks, kTile);
  if (e == cudaSuccess) e = states(&mdv, a.dv, a.dvs, kTile);
  if (e != cudaSuccess) return e;
  const unsigned dkv_ctas = (unsigned)((int64_t)key_tiles * a.kv_heads * a.batch * dkv.splits);
  if (dkv.splits > 1) {
    attention_dkv_kernel<T, DB, DB, true><<<dkv_ctas, Dkv::kThreads, Dkv::kSmem, st>>>(mq, mk, mv, mdo, mdk, mdv, a, key_tiles, row_tiles, plan.splits, dkv);
    attention_dkv_join_kernel<T><<<(unsigned)(((int64_t)a.batch * a.kv_heads * a.keys + 3) / 4), 128, 0, st>>>(a, dkv);
  } else {
    attention_dkv_kernel<T, DB, DB, false><<<dkv_ctas, Dkv::kThreads, Dkv::kSmem, st>>>(mq, mk, mv, mdo, mdk, mdv, a, key_tiles, row_tiles, plan.splits, dkv);
  }
  return cudaGetLastError();
}

int64_t stat_count(const AttentionArgs& a) { return (int64_t)a.batch * a.heads * ((a.queries + kTile - 1) / kTile) * kTile; }
size_t peak_bytes(const AttentionArgs& a, const SplitPlan& dq) { return (size_t)(stat_count(a) / 32) * dq.splits * sizeof(float); }

}  // namespace

size_t attention_backward_workspace(const AttentionArgs& a) {
  const SplitPlan dq = make_dq_plan(a);
  return (size_t)stat_count(a) * 2 * 32 + dkv_part_bytes(a, make_dkv_plan(a)) + split_bytes(a, dq) + peak_bytes(a, dq);
}

cudaError_t launch_attention_backward_tc(AttentionArgs a, int dtype, void* workspace, cudaStream_t st) {
  a.stat_lse = reinterpret_cast<uint8_t*>(workspace);
  a.stat_delta = a.stat_lse + stat_count(a) * 32;
  SplitPlan dq = make_dq_plan(a), dkv = make_dkv_plan(a);
  uint8_t* rest = a.stat_delta + stat_count(a) * 32;
  dkv.part_o = reinterpret_cast<float*>(rest);          // head_dim is a multiple of 8: 16-byte boundaries throughout
  if (dq.splits > 1) place_parts(a, &dq, rest + dkv_part_bytes(a, dkv));
  a.stat_peak = reinterpret_cast<float*>(rest + dkv_part_bytes(a, dkv) + split_bytes(a, dq));
  if (dtype == SWARM_BF16)
    return a.head_dim <= 64 ? launch_backward<__nv_bfloat16, 1>(a, dq, dkv, dtype, st) : launch_backward<__nv_bfloat16, 2>(a, dq, dkv, dtype, st);
  return a.head_dim <= 64 ? launch_backward<__half, 1>(a, dq, dkv, dtype, st) : launch_backward<__half, 2>(a, dq, dkv, dtype, st);
}

}  // namespace swarm
