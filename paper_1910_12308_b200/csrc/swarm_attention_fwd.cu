// Cross attention, forward pass on the tensor cores (many query rows): S = Q K^T and O += P V with tcgen05.mma, all four in
// tensor memory, tiles brought by TMA into a ring.
//
// What bounds it. A tile of 128 rows x 128 states costs 1024 cycles of exponentials on the special-function unit, and 512
// (heads of 64) or 1024 (heads of 128) cycles of products. Heads of 64: two CTAs share those units, a warpgroup's step takes
// about 2700 cycles of which 2048 are both CTAs' exponentials; 4 x 16 heads, 4096 rows and states, 380 us, 720 TFLOP/s.
// A part of the exponentials as polynomials on the fp32 pipe gave nothing: a warp's other 600 instructions a step
// then take as long. Heads of 128: a tile's chain of softmax (1900 cycles), products (1024) and their latency is what
// two tiles in turn cover to 56 %; 460 us there, 1190 TFLOP/s. Sentences of 128: 25 us for 64 x 16 heads, mostly the
// CTAs' start and end.
#include <mutex>

#include "swarm_attention_tile.cuh"

namespace swarm {
namespace {

// Shape of a CTA. NT tiles of 128 query rows, each with a softmax warpgroup; a further warpgroup holds the copying warp
// and the issuing warp. Registers are moved from it to the others: the sum stays what the block was launched with.
template <int DB, int NT> struct FwdShape {
  static constexpr int kThreads = 128 * (NT + 1);
  static constexpr int kCtasPerSm = NT == 1 ? 2 : 1;
  static constexpr int kRegs = NT == 1 ? 200 : 208, kRegsRest = NT == 1 ? 56 : 88;
  static constexpr int kStages = NT == 1 ? 4 : DB == 2 ? 4 : 6;
  static constexpr int kSmem = (NT + kStages) * DB * kBlockBytes + 1024;
  // tensor memory: scores, weights, sums of tile 0, then of tile 1
  static constexpr uint32_t kColumns = NT == 1 ? 256 : 512;
  static constexpr uint32_t kWeights = NT == 1 ? 128 : 0;              // two tiles: the weights overwrite the scores
  static constexpr uint32_t kSums = NT == 1 ? 192 : 256;
};

struct FwdBars {
  uint64_t q_full[2], kv_full[6], kv_empty[6], s_full[2], s_empty[2], p_full[2], pv_done[2], edge_here, edge_done, drain;
};

// NT = 1 (heads of up to 64 values): scores and weights have tensor memory of their own, so the scores of the next tile
// are computed while the warps take the exponentials of this one, and two such CTAs share a multiprocessor.
// NT = 2: two row tiles share every tile of states; while one's products run, the other's softmax does.
template <typename T, int DB, int NT, bool SPLIT>
__global__ void __launch_bounds__(FwdShape<DB, NT>::kThreads, FwdShape<DB, NT>::kCtasPerSm)
attention_forward_kernel(const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv,
                         const __grid_constant__ TileMap mo, AttentionArgs a, int row_tiles, int tile_groups, SplitPlan plan) {
  using Shape = FwdShape<DB, NT>;
  constexpr int kStages = Shape::kStages;
  constexpr uint32_t kTileBytes = DB * kBlockBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;                                   // NT tiles
  uint8_t* sKV = smem + NT * kTileBytes;                // ring of K, V tiles
  __shared__ FwdBars bars;
  __shared__ uint32_t tmem_slot;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // the row tiles of this CTA: tiles are numbered head after head within the group of a key head
  const int split = SPLIT ? blockIdx.x % plan.splits : 0, cta = SPLIT ? blockIdx.x / plan.splits : blockIdx.x;
  const int first = cta % tile_groups * NT, bh = cta / tile_groups, hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const int tiles = (nk + kTile - 1) / kTile;           // of states; this CTA has n of them, the first of them `start`
  const int start = SPLIT ? (int)((int64_t)tiles * split / plan.splits) : 0;
  const int n = SPLIT ? (int)((int64_t)tiles * (split + 1) / plan.splits) - start : tiles;
  auto head_of = [&](int t) { return hk * a.group + (first + t) / row_tiles; };
  auto row_of = [&](int t) { return (first + t) % row_tiles * kTile; };
  auto exists = [&](int t) { return first + t < row_tiles * a.group; };
  uint32_t act = 0;                                     // bit t: tile t has work
#pragma unroll
  for (int t = 0; t < NT; ++t) act |= exists(t) && row_of(t) < nq && n > 0 ? 1u << t : 0u;
  auto active = [&](int t) { return (act >> t & 1u) != 0; };
  const bool any = act != 0;
  const int edge = nk % 16 && start + n == tiles ? nk % kTile : 0;     // rows of the last tile, where they end inside a product's sixteen

  if (tid == 0) {
    for (int i = 0; i < NT; ++i) {
      mbar_init(smem_u32(&bars.q_full[i]), 1);
      mbar_init(smem_u32(&bars.s_full[i]), 1);
      mbar_init(smem_u32(&bars.s_empty[i]), 4);
      mbar_init(smem_u32(&bars.p_full[i]), 4);
      mbar_init(smem_u32(&bars.pv_done[i]), 1);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&bars.kv_full[i]), 1);
      mbar_init(smem_u32(&bars.kv_empty[i]), 1);
    }
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
    if (warp == 4 * NT && any && elect_one()) {
      // ---- copies (one thread) ----------------------------------------------------------------
      int issued = 0;
      if (limit) {
        for (int t = 0; t < NT; ++t)
          if (active(t)) {
            const uint32_t bar = smem_u32(&bars.q_full[t]);
            mbar_expect_tx(bar, kTileBytes);
            load_tile<DB>(smem_u32(sQ) + t * kTileBytes, mq, row_of(t), head_of(t), b, bar);
          }
      }
      for (int f = 0; f < 2 * n; ++f) {                 // K of tile 0, V of tile 0, K of tile 1, ...
        const int st = f % kStages;
        ok = mbar_wait_one(smem_u32(&bars.kv_empty[st]), ((f / kStages) & 1) ^ 1, limit);
        if (!ok) break;
        const uint32_t bar = smem_u32(&bars.kv_full[st]);
        mbar_expect_tx(bar, kTileBytes);
        load_tile<DB>(smem_u32(sKV) + st * kTileBytes, f & 1 ? mv : mk, (start + (f >> 1)) * kTile, hk, b, bar);
        issued = f + 1;
      }
      // every copy lands before the CTA's shared memory is released, whichever of its threads gives up
      for (int f = issued > kStages ? issued - kStages : 0; f < issued; ++f)
        mbar_wait_one(smem_u32(&bars.kv_full[f % kStages]), (f / kStages) & 1, kAttentionWaitLimit);
      for (int t = 0; t < NT; ++t)
        if (active(t) && limit) mbar_wait_one(smem_u32(&bars.q_full[t]), 0, kAttentionWaitLimit);
    } else if (warp == 4 * NT + 2 && any && edge) {
      // ---- the last tile's end: v is a factor of the sums ---------------------------------------
      const int f = 2 * n - 1;
      ok = mbar_wait(smem_u32(&bars.edge_here), 0, limit);
      if (ok) {
        zero_rows<DB, kTile>(sKV + f % kStages * kTileBytes, edge, (edge + 15) & ~15, lane);
        if (lane == 0) mbar_arrive(smem_u32(&bars.edge_done));
      }
    } else if (warp == 4 * NT + 1 && any && elect_one()) {
      // ---- products (one thread) --------------------------------------------------------------
      const int ksteps = (a.head_dim + 15) / 16;
      const uint32_t aq = smem_u32(sQ), akv = smem_u32(sKV);
      auto columns = [&](int j) { return (min(kTile, nk - (start + j) * kTile) + 15) & ~15; };
      auto scores = [&](int t, int j) {                 // S_t = Q_t K_j^T
        mma_rows<T, DB, kTile>(tmem + 128 * t, aq + t * kTileBytes, akv + (2 * j) % kStages * kTileBytes, columns(j), ksteps);
        tc_commit(smem_u32(&bars.s_full[t]));
      };
      auto sums = [&](int t, int j) {                   // O_t += P_t V_j
        mma_weights<T, DB, kTile, false>(tmem + 128 * t + Shape::kSums, tmem + 128 * t + Shape::kWeights,
                                         akv + (2 * j + 1) % kStages * kTileBytes, columns(j) / 16, j != 0);
        if (NT == 1 || j == n - 1) tc_commit(smem_u32(&bars.pv_done[t]));
      };
      auto wait_kv = [&](int f) { return mbar_wait_one(smem_u32(&bars.kv_full[f % kStages]), (f / kStages) & 1, limit); };
      ok = wait_kv(0);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (active(t) && ok) {
          ok = mbar_wait_one(smem_u32(&bars.q_full[t]), 0, limit);
          tc_fence_after();
          if (ok) scores(t, 0);
        }
      if (ok) tc_commit(smem_u32(&bars.kv_empty[0]));
      for (int j = 0; j < n && ok; ++j) {
        const int sv = (2 * j + 1) % kStages, sk = (2 * j + 2) % kStages;
        if (NT == 1 && j + 1 < n) {                     // the next scores as soon as these have been read
          ok = wait_kv(2 * j + 2) && mbar_wait_one(smem_u32(&bars.s_empty[0]), j & 1, limit);
          if (!ok) break;
          tc_fence_after();
          scores(0, j + 1);
          tc_commit(smem_u32(&bars.kv_empty[sk]));
        }
        ok = wait_kv(2 * j + 1);
        if (j == n - 1 && edge && ok) mbar_arrive(smem_u32(&bars.edge_here));
#pragma unroll
        for (int t = 0; t < NT; ++t)
          if (active(t) && ok) {
            ok = mbar_wait_one(smem_u32(&bars.p_full[t]), j & 1, limit) &&
                 (j < n - 1 || !edge || mbar_wait_one(smem_u32(&bars.edge_done), 0, limit));
            tc_fence_after();
            if (ok) sums(t, j);
            if (NT == 2 && j + 1 < n && ok) {
              ok = wait_kv(2 * j + 2);
              tc_fence_after();
              if (ok) scores(t, j + 1);
            }
          }
        if (ok) {
          tc_commit(smem_u32(&bars.kv_empty[sv]));
          if (NT == 2 && j + 1 < n) tc_commit(smem_u32(&bars.kv_empty[sk]));
        }
      }
      // no product is in flight when tensor memory is freed, whichever thread gives up
      tc_commit(smem_u32(&bars.drain));
      mbar_wait_one(smem_u32(&bars.drain), 0, kAttentionWaitLimit);
    }
    __syncwarp();
  } else {
    // ---- softmax ------------------------------------------------------------------------------
    regs_raise<Shape::kRegs>();
    const int t = NT == 1 ? 0 : warp >> 2, quad = warp & 3, head = head_of(t), row0 = row_of(t);
    const bool work = active(t);
    const int row = row0 + quad * 32 + lane;            // this thread's query row
    const uint32_t ts = tmem + 128 * t + ((uint32_t)(quad * 32) << 16), tp = ts + Shape::kWeights, to = ts + Shape::kSums;
    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.0f;                      // m: the maximum that the weights are taken against
    if (work) {
      bool ahead = false;                               // the scores of the step have been seen to be there
      for (int j = 0; j < n; ++j) {
        ok = mbar_wait_after(ahead, smem_u32(&bars.s_full[t]), j & 1, limit);
        if (!ok) break;
        tc_fence_after();
        const int valid = nk - (start + j) * kTile;
        float s[kTile];
#pragma unroll
        for (int g = 0; g < 4; ++g) tmem_ld32(ts + g * 32, s + g * 32);
        tmem_wait_ld();
        if (NT == 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars.s_empty[t]));
        }
        if (valid < kTile) {
#pragma unroll
          for (int i = 0; i < kTile; ++i) s[i] = i < valid ? s[i] : -INFINITY;
        }
        float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i + 8 <= kTile; i += 8) {
#pragma unroll
          for (int u = 0; u < 4; ++u) top[u] = max3(top[u], s[i + u], s[i + 4 + u]);
        }
        const float m_tile = fmaxf(max3(top[0], s[124], s[125]), max3(max3(top[1], s[126], s[127]), top[2], top[3]));
        // NT = 1: the weights and sums of the last tile are free again once its product has completed
        bool pv_waits = NT == 1 && j > 0;
        auto wait_pv = [&]() {
          if (pv_waits) {
            ok = mbar_wait(smem_u32(&bars.pv_done[t]), (j - 1) & 1, limit);
            tc_fence_after();
          }
          pv_waits = false;
        };
        if (j == 0) m = m_tile;
        else if (__any_sync(0xFFFFFFFFu, (m_tile - m) * c > 8.0f)) {
          wait_pv();
          if (!ok) break;
          // the maximum moved by more than a factor of 2^8 in some row of the warp: rescale the sums so far. Smaller
          // moves keep the old reference; the weights then reach 2^8, which fp32 sums and 16-bit weights hold as well.
          const float m_new = fmaxf(m, m_tile), f = m_new == m ? 1.0f : ex2((m - m_new) * c);
          l *= f;
          m = m_new;
#pragma unroll
          for (int g = 0; g < DB * 2; ++g) {
            float o[32];
            tmem_ld32(to + g * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= f;
            tmem_st32(to + g * 32, o);
          }
        }
        const float mc = m == -INFINITY ? 0.0f : m * c - kRunningShift<T>;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p0, p1;
            fma2(p0, p1, s[g * 32 + 2 * i], s[g * 32 + 2 * i + 1], c, c, -mc, -mc);
            p0 = ex2(p0);
            p1 = ex2(p1);
            add2(sum[2 * (i & 1)], sum[2 * (i & 1) + 1], sum[2 * (i & 1)], sum[2 * (i & 1) + 1], p0, p1);
            p[i] = pack2<T>(p0, p1);
          }
          if (NT == 1 && g == 0) {
            wait_pv();
            if (!ok) break;
          }
          tmem_st16(tp + g * 16, p);
        }
        if (!ok) break;
        if (NT == 1) ahead = j + 1 < n && mbar_test(smem_u32(&bars.s_full[t]), (j + 1) & 1);
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.p_full[t]));
      }
      if (ok) {
        ok = mbar_wait(smem_u32(&bars.pv_done[t]), NT == 1 ? (n - 1) & 1 : 0, limit);
        tc_fence_after();
      }
    }
    // ---- output -------------------------------------------------------------------------------
    const bool live = work && row < nq;
    if (!exists(t) || !named_barrier_and(1 + t, 128, ok)) {
      // nothing to write
    } else if (SPLIT) {
      // this CTA's part of the row: its sums as they are, their maximum and the sum of the weights
      const int64_t at = (((int64_t)bh * a.queries + row) * a.group + (head - hk * a.group)) * plan.splits + split;
#pragma unroll
      for (int g = 0; g < DB * 2; ++g) {
        float o[32];
        if (work) { tmem_ld32(to + g * 32, o); tmem_wait_ld(); }
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          if (row < a.queries && g * 32 + i < a.head_dim)
            *reinterpret_cast<float4*>(plan.part_o + at * a.head_dim + g * 32 + i) =
                live ? make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if (row < a.queries) *reinterpret_cast<float2*>(plan.part_ml + at * 2) = live ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
    } else {
      const float inv = live && l != 0.0f ? 1.0f / l : 0.0f;
      uint8_t* out = sQ + t * kTileBytes;               // the query tile has been read by now
#pragma unroll
      for (int g = 0; g < DB * 2; ++g) {
        float o[32];
        if (work) { tmem_ld32(to + g * 32, o); tmem_wait_ld(); }
        store_row32<T>(out, quad * 32 + lane, g * 32, o, inv, live);
      }
      if (a.lse && row < a.queries)
        a.lse[((int64_t)b * a.heads + head) * a.queries + row] = live ? m * a.scale + (logf(l) - kRunningShift<T> * 0.69314718f) : -INFINITY;
      fence_proxy_async();
      named_barrier(1 + t, 128);
      if (quad == 0 && lane == 0) {
        store_tile<DB>(mo, smem_u32(out), row0, head, b);
        bulk_commit();
        bulk_wait_read();
      }
    }
  }
  if (!ok) atomicOr(a.status, kStatusWait);
  tc_fence_before();
  __syncthreads();
  if (warp == 4 * NT + 1) tmem_dealloc(tmem, Shape::kColumns);
}

template <typename T, int DB, int NT, bool SPLIT>
cudaError_t launch_forward_as(const AttentionArgs& a, const SplitPlan& plan, const TileMap& mq, const TileMap& mk, const TileMap& mv,
                           const TileMap& mo, cudaStream_t st) {
  using Shape = FwdShape<DB, NT>;
  static bool attr_set[64] = {};
  static std::mutex attr_mutex;
  {
    std::lock_guard<std::mutex> lock(attr_mutex);
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
      const cudaError_t e = cudaFuncSetAttribute(attention_forward_kernel<T, DB, NT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem);
      if (e != cudaSuccess) return e;
      attr_set[dev] = true;
    }
  }
  const int row_tiles = (a.queries + kTile - 1) / kTile, tile_groups = (int)(((int64_t)row_tiles * a.group + NT - 1) / NT);
  const int64_t ctas = (int64_t)tile_groups * a.kv_heads * a.batch * plan.splits;
  attention_forward_kernel<T, DB, NT, SPLIT><<<(unsigned)ctas, Shape::kThreads, Shape::kSmem, st>>>(mq, mk, mv, mo, a, row_tiles, tile_groups, plan);
  return cudaGetLastError();
}

template <typename T, int DB, int NT>
cudaError_t launch_forward(const AttentionArgs& a, const SplitPlan& plan, const TileMap& mq, const TileMap& mk, const TileMap& mv,
                           const TileMap& mo, cudaStream_t st) {
  return plan.splits > 1 ? launch_forward_as<T, DB, NT, true>(a, plan, mq, mk, mv, mo, st)
                         : launch_forward_as<T, DB, NT, false>(a, plan, mq, mk, mv, mo, st);
}

// Few row tiles leave multiprocessors idle while each CTA walks all states: these are then split, as far as the CTAs still
// run at once and four steps or more are left to each, where that saves twelve steps (a step is about 1.4 us, the parts'
// way through memory and the joining kernel 10 to 15). Measured: 8 heads of 64, 128 rows, 4096 states 42 us whole and 24 in
// parts, 8 heads of 128, 512 rows 66 and 26; 2 x 8 heads of 64, 300 rows, 1000 states (eight steps) 16 and 25.
SplitPlan make_forward_plan(const AttentionArgs& a) {
  SplitPlan p{};
  const int nt = a.head_dim <= 64 ? 1 : 2;
  const int64_t row_tiles = (a.queries + kTile - 1) / kTile, steps = (a.keys + kTile - 1) / kTile;
  const int64_t ctas = (row_tiles * a.group + nt - 1) / nt * a.kv_heads * a.batch, room = 148 * (nt == 1 ? 2 : 1);
  int64_t s = room / ctas;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s > steps / 4) s = steps / 4;
  if (s < 2 || steps - (steps + s - 1) / s < 12) s = 1;
  p.splits = (int32_t)s;
  p.rows = s > 1 ? a.queries * a.group : 0;             // at most 128 rows for each of the 296 CTAs
  return p;
}

}  // namespace

cudaError_t make_tile_map(TileMap* out, const void* p, const swarm_strides& s, int dtype, int batch, int tokens, int heads,
                          int head_dim, int rows) {
  typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static encode_fn encode = nullptr;
  static std::mutex mutex;
  {
    std::lock_guard<std::mutex> lock(mutex);
    if (!encode) {
      void* f = nullptr;
      cudaDriverEntryPointQueryResult found;
      const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
      if (e != cudaSuccess) return e;
      if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
      encode = (encode_fn)f;
    }
  }
  const int64_t stride[3] = {s.token, s.head, s.batch};
  const int extent[3] = {tokens, heads, batch};
  int32_t* step[3] = {&out->token_step, &out->head_step, &out->batch_step};
  cuuint64_t dims[4] = {(cuuint64_t)head_dim, 1, 1, 1}, bytes[3] = {16, 16, 16};
  for (int i = 0; i < 3; ++i) {
    *step[i] = 0;
    if (extent[i] > 1 && stride[i] != 0) {
      dims[i + 1] = (cuuint64_t)extent[i];
      bytes[i] = (cuuint64_t)stride[i] * 2;
      *step[i] = 1;
    }
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, ones[4] = {1, 1, 1, 1};
  const CUresult r = encode(&out->map, dtype == SWARM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                            const_cast<void*>(p), dims, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

size_t attention_forward_workspace(const AttentionArgs& a) { return split_bytes(a, make_forward_plan(a)); }

cudaError_t launch_attention_forward_tc(const AttentionArgs& a, int dtype, void* workspace, cudaStream_t st) {
  SplitPlan plan = make_forward_plan(a);
  if (plan.splits > 1) place_parts(a, &plan, workspace);
  TileMap mq, mk, mv, mo;
  cudaError_t e = make_tile_map(&mq, a.q, a.qs, dtype, a.batch, a.queries, a.heads, a.head_dim, kTile);
  if (e == cudaSuccess) e = make_tile_map(&mo, a.out, a.os, dtype, a.batch, a.queries, a.heads, a.head_dim, kTile);
  if (e == cudaSuccess) e = make_tile_map(&mk, a.k, a.ks, dtype, a.batch, a.keys, a.kv_heads, a.head_dim, kTile);
  if (e == cudaSuccess) e = make_tile_map(&mv, a.v, a.vs, dtype, a.batch, a.keys, a.kv_heads, a.head_dim, kTile);
  if (e != cudaSuccess) return e;
  if (dtype == SWARM_BF16)
    e = a.head_dim <= 64 ? launch_forward<__nv_bfloat16, 1, 1>(a, plan, mq, mk, mv, mo, st) : launch_forward<__nv_bfloat16, 2, 2>(a, plan, mq, mk, mv, mo, st);
  else
    e = a.head_dim <= 64 ? launch_forward<__half, 1, 1>(a, plan, mq, mk, mv, mo, st) : launch_forward<__half, 2, 2>(a, plan, mq, mk, mv, mo, st);
  if (e == cudaSuccess && plan.splits > 1) e = launch_attention_join(a, plan, dtype, st);
  return e;
}

}  // namespace swarm
