// Attention of a sentence's newest tokens over its paged cache: every visible key and value is read once, HBM is the bound.
//
// An item is 16 rows (tokens x query heads of a key head) of a sentence and all the positions that one of them sees, in blocks of 16.
// The blocks of all items in a row are dealt to the device's warps in equal runs, whatever the sentences' lengths: a warp may end
// one item, take several whole ones and begin another. Each warp works alone: a ring of blocks that cp.async fills
// past the ends of items, so that loads never pause (about 170 KB in flight on a multiprocessor), ldmatrix, m16n8k16 products with
// the running maximum and sum of the softmax in registers. An item that was cut leaves parts (maximum, sum, o): those of
// a CTA's warps, whose runs follow one another, are joined at the CTA's end, those of several CTAs by a second kernel, whose
// launch overlaps the first one's end; always in the items' order.
//
// Weights enter their product as the sum of two numbers of the type: rounded once, o would be 1.4 times as far from its value as
// its own rounding leaves it. The products are a small part of a block's time, so the second costs nothing.
#include <mutex>

#include "swarm_attention_tile.cuh"
#include "swarm_paged.h"

namespace swarm {
namespace {

constexpr int kBlock = 16;                              // positions of a block
constexpr int kRows = 16;
constexpr int kWarps = 8;
constexpr int kMinShare = 4;                            // blocks that a warp's run has at least
constexpr int kWholeBlocks = 8;                         // items of no more blocks are not cut
constexpr int kSms = 148;

// DB: heads of up to 64 DB values.
template <int DB> struct Shape {
  static constexpr int kCtasPerSm = DB == 1 ? 2 : 1;
  static constexpr int kStages = 3;
  static constexpr int kTileBytes = kBlock * DB * 128;  // of keys, and of values
  static constexpr int kSmem = kWarps * kStages * 2 * kTileBytes;
};

struct PagedPlan {
  int32_t row_groups;                 // of `tokens` rows
  int32_t rows;                       // that a part holds
  int32_t whole;                      // items are not cut
  int32_t ctas;
  int32_t join_warps;                 // for each row
  uint32_t page_multiplier, page_shift;                 // division by the size of a page
  int64_t* prefix;                    // [batch + 1] blocks of the items before a sentence's
  // parts of the warps, two each, then of the CTAs
  float* part_ml;                     // [parts][rows][2] maximum and sum
  float* part_o;                      // [parts][rows][head_dim]
};

// What a sentence's rows see, in blocks: the first `sink_blocks`, then those from position lo / 16 * 16.
struct Sentence {
  int length, n, lo, sink_blocks, blocks, row_groups;
};
__device__ __forceinline__ Sentence sentence_of(const PagedArgs& a, int b) {
  Sentence s;
  s.length = length_in(a, b);
  s.n = rows_in(a, b, s.length);
  s.lo = a.window > 0 ? max(0, s.length - s.n - a.window + 1) : 0;
  const int sinks = min(a.sinks, s.lo);
  s.sink_blocks = min(sinks / kBlock + (sinks % kBlock != 0), s.lo / kBlock);
  s.blocks = s.n > 0 ? s.sink_blocks + (s.length - 1) / kBlock + 1 - s.lo / kBlock : 0;
  s.row_groups = (s.n * a.group + kRows - 1) / kRows;
  return s;
}
__device__ __forceinline__ int64_t blocks_of_items(const PagedArgs& a, const Sentence& s) {
  return (int64_t)s.blocks * a.kv_heads * s.row_groups;
}

// The runs that `total` blocks are dealt in: `warps` runs, `per_cta` of them in each CTA, the first `more` one block longer.
struct Runs {
  int64_t each, more;
  int warps, per_cta;
  __device__ __forceinline__ Runs(int64_t total, int ctas) {
    warps = (int)max((int64_t)1, min((int64_t)ctas * kWarps, total / kMinShare));
    per_cta = (warps + ctas - 1) / ctas;                // few runs go to many multiprocessors
    each = total / warps;
    more = total % warps;
  }
  __device__ __forceinline__ int64_t begin(int w) const { return w * each + min((int64_t)w, more); }
  __device__ __forceinline__ int owner(int64_t x) const {
    const int64_t wide = more * (each + 1);
    return (int)(x < wide ? x / (each + 1) : more + (x - wide) / each);
  }
};

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t r[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t r[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Offset of chunk c (16 bytes) of row r of a tile: eight rows' same chunk, and a row's eight, lie in different banks.
template <int DB> __device__ __forceinline__ uint32_t tile_offset(int r, int c) {
  return (uint32_t)(r * (DB * 128) + (c >> 3) * 128 + (((c & 7) ^ (r & 7)) << 4));
}
// Whether a word holds an infinity or a NaN.
template <typename T> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t e = sizeof(T) == 2 && kNarrow<T> ? 0x7C00u : 0x7F80u;
  return (w & e) == e || ((w >> 16) & e) == e;
}

// A block in the ring: what it is of, and which of its positions were read.
struct __align__(16) BlockInfo {
  int32_t b, head, row0, n;           // sentence, key head, first row of the item; the sentence's rows are n tokens'
  int32_t position;
  int32_t first_new;                  // position of the first row: what lies past it, not every row sees
  int32_t last_gone;                  // what lies before it, the last row does not see
  uint32_t flags;                     // bits 0..15: the position is there
};
constexpr uint32_t kFirst = 1u << 16, kLast = 2u << 16, kFromStart = 4u << 16, kToEnd = 8u << 16, kNone = 16u << 16;

// Parts of a cut item that a warp holds: the run's first item may have begun elsewhere (0), its last one may go on (1).
struct __align__(16) PartInfo {
  int32_t there, b, head, row0, n, to_end;
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= kBlock ? 0xFFFFu : (1u << n) - 1u; }

// Two parts of a row joined: maximum and sum, and the factors of their o.
__device__ __forceinline__ void join_ml(float& m, float& l, float m1, float l1, float c, float& f0, float& f1) {
  const float top = fmaxf(m, m1), base = top == -INFINITY ? 0.0f : top;
  f0 = ex2((m - base) * c);
  f1 = ex2((m1 - base) * c);
  l = l * f0 + l1 * f1;
  m = top;
}

// Four values of a row from its sum, and its lse.
template <typename T>
__device__ __forceinline__ void write_row(const PagedArgs& a, int b, int t, int h, int lane, float m, float l, const float v[4]) {
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  if (lane * 4 < a.head_dim)
    *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h) + lane * 4) =
        l != 0.0f ? make_uint2(pack2<T>(v[0] * inv, v[1] * inv), pack2<T>(v[2] * inv, v[3] * inv)) : make_uint2(0, 0);
  if (a.lse && lane == 0)
    a.lse[((int64_t)b * a.heads + h) * a.tokens + t] = l != 0.0f ? m * a.scale + (logf(l) - kRunningShift<T> * 0.69314718f) : -INFINITY;
}

// ONE_PAGE: pages hold a multiple of 16 positions, so a block lies in one. Then its page is the same number in every lane and
// a row's address is one addition away from the last one's; else each position has its own, and a lane gets them by shuffles.
template <typename T, int DB, bool ONE_PAGE>
__global__ void __launch_bounds__(kWarps * 32, Shape<DB>::kCtasPerSm)
paged_attention_kernel(PagedArgs a, PagedPlan plan) {
  using S = Shape<DB>;
  constexpr int kStages = S::kStages, kChunks = DB * 8, kRowsPerCopy = 32 / kChunks;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ BlockInfo s_info[kWarps][kStages];
  __shared__ PartInfo s_part[kWarps][2];
  __shared__ int64_t s_prefix[kWarps * 32 + 1];
  __shared__ int64_t s_warp[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r8 = lane >> 2, c4 = lane & 3, chunks = a.head_dim / 8;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (lane < 2) s_part[warp][lane].there = 0;

  // rows past a sentence's count
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    const int n = rows_in(a, b, length_in(a, b));
    for (int i = tid; i < (a.tokens - n) * a.heads * chunks; i += kWarps * 32) {
      const int ch = i % chunks, h = i / chunks % a.heads, t = n + i / chunks / a.heads;
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h) + ch * 8) = make_uint4(0, 0, 0, 0);
      if (a.lse && ch == 0) a.lse[((int64_t)b * a.heads + h) * a.tokens + t] = -INFINITY;
    }
  }

  // this warp's run
  int b = 0, hk = 0, rg = 0, block = 0, w = 0;
  int64_t left = 0, item_end = 0;                       // blocks to take; past the last item, where items are not cut
  Sentence s;
  if (plan.whole) {
    const int64_t each = a.kv_heads * (int64_t)plan.row_groups, items = a.batch * each;
    const int all = gridDim.x * kWarps, turn = warp * gridDim.x + blockIdx.x;          // few items go to many multiprocessors
    const int64_t per = items / all, more = items % all, item = turn * per + min((int64_t)turn, more);
    item_end = item + per + (turn < more);
    b = (int)(item / each); hk = (int)(item % each) / plan.row_groups; rg = (int)(item % plan.row_groups);
    left = item < item_end;
    if (left) s = sentence_of(a, b);
  } else {
    const int per = (a.batch + kWarps * 32 - 1) / (kWarps * 32);
    const int b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
    int64_t sum = 0;
    for (int i = b0; i < b1; ++i) sum += blocks_of_items(a, sentence_of(a, i));
    int64_t before = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, before, o);
      if (lane >= o) before += x;
    }
    if (lane == 31) s_warp[warp] = before;
    __syncthreads();
    for (int i = 0; i < warp; ++i) before += s_warp[i];
    s_prefix[tid + 1] = before;
    if (tid == 0) s_prefix[0] = 0;
    if (blockIdx.x == 0) {                              // for the joining kernel
      int64_t at = before - sum;
      for (int i = b0; i < b1; ++i) { plan.prefix[i] = at; at += blocks_of_items(a, sentence_of(a, i)); }
      if (b1 == a.batch && b0 < b1) plan.prefix[a.batch] = at;
    }
    __syncthreads();
    const Runs runs(s_prefix[kWarps * 32], gridDim.x);
    w = blockIdx.x * runs.per_cta + warp;
    const bool takes = warp < runs.per_cta && w < runs.warps;
    const int64_t begin = takes ? runs.begin(w) : 0;
    left = takes ? runs.begin(w + 1) - begin : 0;
    if (left > 0) {
      int lo = 0, hi = kWarps * 32;                     // the slice of sentences that holds the run's first block
      while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (s_prefix[mid] <= begin) lo = mid; else hi = mid; }
      int64_t at = begin - s_prefix[lo];
      b = lo * per;
      s = sentence_of(a, b);
      while (at >= blocks_of_items(a, s)) { at -= blocks_of_items(a, s); ++b; s = sentence_of(a, b); }
      const int64_t item = at / s.blocks;
      block = (int)(at % s.blocks);
      hk = (int)(item / s.row_groups);
      rg = (int)(item % s.row_groups);
    }
  }
  bool fresh = true;                                    // the next block is the first of its item here
  // moves on to an item that exists
  auto skip = [&]() {
    while (rg >= s.row_groups) {                        // none in a sentence without rows
      rg = 0;
      ++hk;
      if (hk >= a.kv_heads || s.row_groups == 0) {
        hk = 0;
        if (++b >= a.batch) { left = 0; return; }
        s = sentence_of(a, b);
      }
    }
    if (plan.whole && ((int64_t)b * a.kv_heads + hk) * plan.row_groups + rg >= item_end) left = 0;
  };
  if (left > 0) skip();

  // the next block: its position, and its page (ONE_PAGE) or lane i < 16 that of its position i, looked up a block ahead
  int p0 = 0, page = -1, slot = 0;
  auto look_up = [&]() {
    page = -1;
    if (left <= 0) return;
    p0 = (block < s.sink_blocks ? block : block - s.sink_blocks + s.lo / kBlock) * kBlock;
    const int p = ONE_PAGE ? p0 : p0 + (lane & (kBlock - 1));
    const int column = (int)((__umulhi((uint32_t)p, plan.page_multiplier) + (uint32_t)p) >> plan.page_shift);
    slot = p - column * a.page_size;
    if (column < a.table_columns && (ONE_PAGE || (p < s.length && (p >= s.lo || p < a.sinks)))) page = a.table[b * a.table_pitch + column];
  };
  look_up();

  uint8_t* ring = smem + warp * kStages * 2 * S::kTileBytes;
  const int row_of_lane = lane / kChunks, c_of_lane = lane % kChunks;
  uint32_t spot[kBlock / kRowsPerCopy];                 // where a lane's pieces of a tile go
#pragma unroll
  for (int i = 0; i < kBlock / kRowsPerCopy; ++i) spot[i] = smem_u32(ring) + tile_offset<DB>(i * kRowsPerCopy + row_of_lane, c_of_lane);
  // starts the copies of the next block, and moves on
  auto fetch = [&](int stage) {
    if (left > 0) {
      const uint32_t dst = stage * 2 * S::kTileBytes;
      const bool there = (uint32_t)page < (uint32_t)a.pages;
      uint32_t present = 0xFFFFu;                       // wanted by some row
      if (p0 < s.lo || p0 > s.length - kBlock) present = low_bits(s.length - p0) & (~low_bits(s.lo - p0) | low_bits(a.sinks - p0));
      if constexpr (ONE_PAGE) {
        if (!there) {
          if (lane == 0 && present) atomicOr(a.status, kStatusPage);
          present = 0;
        }
        const T* kp = reinterpret_cast<const T*>(a.k_pages) + hk * a.kps.head + page * a.kps.batch + (slot + row_of_lane) * a.kps.token + c_of_lane * 8;
        const T* vp = reinterpret_cast<const T*>(a.v_pages) + hk * a.vps.head + page * a.vps.batch + (slot + row_of_lane) * a.vps.token + c_of_lane * 8;
        const int64_t kstep = kRowsPerCopy * a.kps.token, vstep = kRowsPerCopy * a.vps.token;
        if (present == 0xFFFFu && chunks == kChunks) {
#pragma unroll
          for (int i = 0; i < kBlock / kRowsPerCopy; ++i) {
            cp_async16(spot[i] + dst, kp);
            cp_async16(spot[i] + dst + S::kTileBytes, vp);
            kp += kstep;
            vp += vstep;
          }
        } else {
#pragma unroll
          for (int i = 0; i < kBlock / kRowsPerCopy; ++i) {
            const bool copy = (present >> (i * kRowsPerCopy + row_of_lane) & 1u) && c_of_lane < chunks;
            const void* none = a.q;                     // nothing is read there
            cp_async16_or_zero(spot[i] + dst, copy ? kp : none, copy);
            cp_async16_or_zero(spot[i] + dst + S::kTileBytes, copy ? vp : none, copy);
            kp += kstep;
            vp += vstep;
          }
        }
      } else {
        const bool wanted = lane < kBlock && (present >> lane & 1u);
        if (wanted && !there) atomicOr(a.status, kStatusPage);
        present = __ballot_sync(0xFFFFFFFFu, wanted && there);
        const int64_t ko = page * a.kps.batch + slot * a.kps.token, vo = page * a.vps.batch + slot * a.vps.token;
        const T* kb = reinterpret_cast<const T*>(a.k_pages) + hk * a.kps.head + c_of_lane * 8;
        const T* vb = reinterpret_cast<const T*>(a.v_pages) + hk * a.vps.head + c_of_lane * 8;
#pragma unroll
        for (int i = 0; i < kBlock / kRowsPerCopy; ++i) {
          const int r = i * kRowsPerCopy + row_of_lane;
          const int64_t kr = __shfl_sync(0xFFFFFFFFu, ko, r), vr = __shfl_sync(0xFFFFFFFFu, vo, r);
          const bool copy = (present >> r & 1u) && c_of_lane < chunks;
          const void* none = a.q;
          cp_async16_or_zero(spot[i] + dst, copy ? kb + kr : none, copy);
          cp_async16_or_zero(spot[i] + dst + S::kTileBytes, copy ? vb + vr : none, copy);
        }
      }
      const bool ends = block + 1 == s.blocks, last = ends || (!plan.whole && left == 1);
      if (lane == 0) {
        BlockInfo info;
        info.b = b; info.head = hk; info.row0 = rg * kRows; info.n = s.n; info.position = p0;
        info.first_new = s.length - s.n;
        info.last_gone = a.window > 0 ? s.length - a.window : 0;
        info.flags = present | (fresh ? kFirst : 0u) | (fresh && block == 0 ? kFromStart : 0u) | (last ? kLast : 0u) | (ends ? kToEnd : 0u);
        s_info[warp][stage] = info;
      }
      fresh = last;
      ++block;
      if (!plan.whole) --left;
      if (ends) {
        block = 0;
        ++rg;
        if (left > 0) skip();
      }
      look_up();
    } else if (lane == 0) {
      s_info[warp][stage].flags = kNone;
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);

  uint32_t q[DB * 4][4];                                // operands of the products with the keys
  float o[DB * 8][4], m[2], l[2];
  const float c = a.scale * kLog2e;
  int t_of[2] = {0, 0};
  bool from_start = false;
  // a lane's addresses for ldmatrix: keys, 8 positions x 8 values four times; values likewise, transposed
  const int key_row = (lane & 7) + (lane >> 4) * 8, key_half = lane >> 3 & 1, value_row = lane & 15, value_half = lane >> 4;
  for (int stage = 0;; stage = stage + 1 == kStages ? 0 : stage + 1) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    const BlockInfo info = s_info[warp][stage];
    if (info.flags & kNone) break;
    if (info.flags & kFirst) {
      from_start = info.flags & kFromStart;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = info.row0 + r8 + 8 * u, t = r / a.group;
        t_of[u] = t;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(a.q) + offset_of(a.qs, info.b, t, info.head * a.group + r % a.group)) + c4;
#pragma unroll
        for (int ks = 0; ks < DB * 4; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) q[ks][u + 2 * e] = t < info.n && ks * 2 + e < chunks ? src[ks * 8 + e * 4] : 0u;
        m[u] = -INFINITY;
        l[u] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < DB * 8; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) o[i][u] = 0.0f;
    }
    const uint32_t tile_k = smem_u32(ring) + stage * 2 * S::kTileBytes, tile_v = tile_k + S::kTileBytes;
    // scores: s[8 positions][row r8: positions 2 c4, 2 c4 + 1; row r8 + 8: the same]
    float sc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int ks = 0; ks < DB * 4; ++ks) {
      uint32_t k[4];                                    // positions 0..7, values 0..7 and 8..15 of sixteen; positions 8..15
      ldmatrix4(tile_k + tile_offset<DB>(key_row, ks * 2 + key_half), k);
      mma16816<T>(sc[0], q[ks], k[0], k[1]);
      mma16816<T>(sc[1], q[ks], k[2], k[3]);
    }
    // some position of the block is hidden from some row
    const bool edge = (info.flags & 0xFFFFu) != 0xFFFFu || info.position + (kBlock - 1) > info.first_new ||
                      (a.window > 0 && info.position < info.last_gone && info.position + (kBlock - 1) >= a.sinks);
    auto sees = [&](int p, int t) {
      const int own = info.first_new + t;
      return p <= own && (a.window == 0 || p > own - a.window || p < a.sinks);
    };
    if (edge) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = g * 8 + c4 * 2 + (u & 1);
          if (!(info.flags >> i & 1u) || !sees(info.position + i, t_of[u >> 1])) sc[g][u] = -INFINITY;
        }
    }
    float top[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = fmaxf(fmaxf(sc[0][2 * u], sc[0][2 * u + 1]), fmaxf(sc[1][2 * u], sc[1][2 * u + 1]));
      t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 1));
      top[u] = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 2));
    }
    if (__any_sync(0xFFFFFFFFu, (top[0] - m[0]) * c > 8.0f || (top[1] - m[1]) * c > 8.0f)) {
      // the maximum moved by more than 2^8 in some row (or the first block): rescale; smaller moves keep the reference
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float m_new = fmaxf(m[u], top[u]), f = m_new == m[u] ? 1.0f : ex2((m[u] - m_new) * c);
        m[u] = m_new;
        l[u] *= f;
#pragma unroll
        for (int i = 0; i < DB * 8; ++i) { o[i][2 * u] *= f; o[i][2 * u + 1] *= f; }
      }
    }
    const float base[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        sc[g][u] = ex2(fmaf(sc[g][u] - base[u >> 1], c, kRunningShift<T>));
        l[u >> 1] += sc[g][u];
      }
    uint32_t hi[4], lo[4];                              // weights as an operand: the numbers and what rounding left of them
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = sc[i >> 1][2 * (i & 1)], y = sc[i >> 1][2 * (i & 1) + 1];
      float rx, ry;
      hi[i] = pack2<T>(x, y);
      unpack2<T>(hi[i], rx, ry);
      lo[i] = pack2<T>(x - rx, y - ry);
    }
    bool apart = false;                                 // an infinity or a NaN that not every row sees: 0 times it would be NaN
    if (edge && a.tokens > 1) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < kBlock / kRowsPerCopy; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(ring + stage * 2 * S::kTileBytes + S::kTileBytes + tile_offset<DB>(i * kRowsPerCopy + row_of_lane, c_of_lane));
        bad |= not_finite<T>(x.x) || not_finite<T>(x.y) || not_finite<T>(x.z) || not_finite<T>(x.w);
      }
      apart = __any_sync(0xFFFFFFFFu, bad);
    }
    if (!apart) {
#pragma unroll
      for (int d = 0; d < DB * 4; ++d) {
        uint32_t v[4];                                  // sixteen values: the first eight of positions 0..7 and 8..15, the others
        ldmatrix4_trans(tile_v + tile_offset<DB>(value_row, d * 2 + value_half), v);
        mma16816<T>(o[2 * d], hi, v[0], v[1]);
        mma16816<T>(o[2 * d + 1], hi, v[2], v[3]);
        mma16816<T>(o[2 * d], lo, v[0], v[1]);
        mma16816<T>(o[2 * d + 1], lo, v[2], v[3]);
      }
    } else {
      // one token after the other, its rows alone and what it does not see as zeros: the same bits as above for these
      for (int t = 0; t < a.tokens; ++t) {
        uint32_t keep[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int p = info.position + g * 8 + c4 * 2;
          keep[g] = (sees(p, t) ? 0xFFFFu : 0u) | (sees(p + 1, t) ? 0xFFFF0000u : 0u);
        }
#pragma unroll
        for (int d = 0; d < DB * 4; ++d) {
          uint32_t v[4];
          ldmatrix4_trans(tile_v + tile_offset<DB>(value_row, d * 2 + value_half), v);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x[4] = {o[2 * d + e][0], o[2 * d + e][1], o[2 * d + e][2], o[2 * d + e][3]};
            mma16816<T>(x, hi, v[2 * e] & keep[0], v[2 * e + 1] & keep[1]);
            mma16816<T>(x, lo, v[2 * e] & keep[0], v[2 * e + 1] & keep[1]);
#pragma unroll
            for (int u = 0; u < 4; ++u) o[2 * d + e][u] = t_of[u >> 1] == t ? x[u] : o[2 * d + e][u];
          }
        }
      }
    }
    if (info.flags & kLast) {
      const bool done = from_start && (info.flags & kToEnd);
      if (!done && lane == 0) {
        PartInfo part;
        part.there = 1; part.b = info.b; part.head = info.head; part.row0 = info.row0; part.n = info.n;
        part.to_end = (info.flags & kToEnd) != 0;
        s_part[warp][from_start] = part;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 1);
        l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 2);
        const int r = info.row0 + r8 + 8 * u, t = t_of[u];
        if (t >= info.n) continue;
        if (done) {
          const int h = info.head * a.group + r % a.group;
          const float inv = l[u] != 0.0f ? 1.0f / l[u] : 0.0f;
          uint32_t* dst = reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + offset_of(a.os, info.b, t, h)) + c4;
#pragma unroll
          for (int i = 0; i < DB * 8; ++i)
            if (i < chunks) dst[i * 4] = pack2<T>(l[u] != 0.0f ? o[i][2 * u] * inv : 0.0f, l[u] != 0.0f ? o[i][2 * u + 1] * inv : 0.0f);
          if (a.lse && c4 == 0)
            a.lse[((int64_t)info.b * a.heads + h) * a.tokens + t] = l[u] != 0.0f ? m[u] * a.scale + (logf(l[u]) - kRunningShift<T> * 0.69314718f) : -INFINITY;
        } else {
          const int64_t at = (int64_t)(2 * (blockIdx.x * kWarps + warp) + from_start) * plan.rows + r8 + 8 * u;
          if (c4 == 0) *reinterpret_cast<float2*>(plan.part_ml + at * 2) = make_float2(m[u], l[u]);
          float2* dst = reinterpret_cast<float2*>(plan.part_o + at * a.head_dim) + c4;
#pragma unroll
          for (int i = 0; i < DB * 8; ++i)
            if (i < chunks) dst[i * 4] = make_float2(o[i][2 * u], o[i][2 * u + 1]);
        }
      }
    }
  }
  cp_async_wait<0>();
  if (plan.whole) return;

  // the CTA's parts: an item's are warp j's second and the first of those after it, up to one that ends it. warp = one row of an item
  __syncthreads();
  int turn = 0;
  for (int j = 0; j < kWarps; ++j)
#pragma unroll 1
    for (int second = 0; second < 2; ++second) {
      if (!s_part[j][second].there || (second == 0 && j > 0)) continue;      // a later warp's first part follows another
      int last = j;
      bool ended = s_part[j][second].to_end;
      while (!ended && last + 1 < kWarps && s_part[last + 1][0].there) ended = s_part[++last][0].to_end;
      const PartInfo item = s_part[j][second];
      const int rows = min(kRows, item.n * a.group - item.row0);
      for (int r = 0; r < rows; ++r, ++turn) {
        if (turn % kWarps != warp) continue;
        float m0 = -INFINITY, l0 = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = j; k <= last; ++k) {
          const int64_t at = (int64_t)(2 * (blockIdx.x * kWarps + k) + (k == j ? second : 0)) * plan.rows + r;
          const float2 ml = __ldcg(reinterpret_cast<const float2*>(plan.part_ml + at * 2));
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (lane * 4 < a.head_dim) x = __ldcg(reinterpret_cast<const float4*>(plan.part_o + at * a.head_dim + lane * 4));
          float f0, f1;
          join_ml(m0, l0, ml.x, ml.y, c, f0, f1);
          v[0] = v[0] * f0 + x.x * f1; v[1] = v[1] * f0 + x.y * f1; v[2] = v[2] * f0 + x.z * f1; v[3] = v[3] * f0 + x.w * f1;
        }
        if (second && ended) {
          const int row = item.row0 + r;
          write_row<T>(a, item.b, row / a.group, item.head * a.group + row % a.group, lane, m0, l0, v);
        } else {
          const int64_t at = (int64_t)(2 * (gridDim.x * kWarps + blockIdx.x) + second) * plan.rows + r;
          if (lane == 0) *reinterpret_cast<float2*>(plan.part_ml + at * 2) = make_float2(m0, l0);
          if (lane * 4 < a.head_dim) *reinterpret_cast<float4*>(plan.part_o + at * a.head_dim + lane * 4) = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
    }
}

// Joins the CTAs' parts of a row: `join_warps` warps for each, lane = four values, the parts in order; the warps meet in shared memory.
template <typename T>
__global__ void __launch_bounds__(1024) paged_join_kernel(PagedArgs a, PagedPlan plan) {
  extern __shared__ float s_join[];                     // [warps][head_dim + 2]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % plan.join_warps, pitch = a.head_dim + 2;
  const uint32_t rows = a.tokens * a.group, index = blockIdx.x * (blockDim.x / 32 / plan.join_warps) + warp / plan.join_warps;
  const bool exists = index < (uint32_t)a.batch * a.kv_heads * rows;
  const int row = index % rows, hk = index / rows % a.kv_heads, b = exists ? index / rows / a.kv_heads : 0;
  const int t = row / a.group, h = hk * a.group + row % a.group;
  const Sentence s = sentence_of(a, b);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int c0 = 0, c1 = 0;                                   // the CTAs that hold parts
  if (exists && t < s.n) {
    const Runs runs(plan.prefix[a.batch], plan.ctas);
    const int64_t start = plan.prefix[b] + ((int64_t)hk * s.row_groups + row / kRows) * s.blocks;
    c0 = runs.owner(start) / runs.per_cta;
    c1 = runs.owner(start + s.blocks - 1) / runs.per_cta;
  }
  const float c = a.scale * kLog2e;
  float top = -INFINITY, sum = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (c1 > c0) {
    const int count = c1 - c0 + 1, from = count * sub / plan.join_warps, to = count * (sub + 1) / plan.join_warps;
    for (int p0 = from; p0 < to; p0 += 8) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = p0 + i;
        const int64_t at = (int64_t)(2 * (plan.ctas * kWarps + c0 + k) + (k == 0)) * plan.rows + row % kRows;
        ml[i] = k < to ? *reinterpret_cast<const float2*>(plan.part_ml + at * 2) : make_float2(-INFINITY, 0.0f);
        x[i] = k < to && lane * 4 < a.head_dim ? *reinterpret_cast<const float4*>(plan.part_o + at * a.head_dim + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f0, f1;
        join_ml(top, sum, ml[i].x, ml[i].y, c, f0, f1);
        v[0] = v[0] * f0 + x[i].x * f1; v[1] = v[1] * f0 + x[i].y * f1; v[2] = v[2] * f0 + x[i].z * f1; v[3] = v[3] * f0 + x[i].w * f1;
      }
    }
  }
  if (plan.join_warps > 1) {
    float* mine = s_join + warp * pitch;
    if (lane * 4 < a.head_dim)
      for (int e = 0; e < 4; ++e) mine[2 + lane * 4 + e] = v[e];
    if (lane == 0) { mine[0] = top; mine[1] = sum; }
    __syncthreads();
    if (sub == 0) {
      for (int i = 1; i < plan.join_warps; ++i) {
        const float* x = mine + i * pitch;
        float f0, f1;
        join_ml(top, sum, x[0], x[1], c, f0, f1);
        if (lane * 4 < a.head_dim)
          for (int e = 0; e < 4; ++e) v[e] = v[e] * f0 + x[2 + lane * 4 + e] * f1;
      }
    }
  }
  if (c1 > c0 && sub == 0) write_row<T>(a, b, t, h, lane, top, sum, v);
}

PagedPlan make_plan(const PagedArgs& a) {
  PagedPlan p{};
  const int64_t rows = (int64_t)a.tokens * a.group;
  p.row_groups = (int32_t)((rows + kRows - 1) / kRows);
  p.rows = (int32_t)(rows < kRows ? rows : kRows);
  // the most blocks that an item can have: the table's, or the window's with the first tokens'
  int64_t most = ((int64_t)a.table_columns * a.page_size + kBlock - 1) / kBlock;
  if (a.window > 0) {
    const int64_t seen = ((int64_t)a.window + a.tokens - 1) / kBlock + 2 + (a.sinks + (int64_t)kBlock - 1) / kBlock;
    if (seen < most) most = seen;
  }
  const int64_t items = (int64_t)a.batch * a.kv_heads * p.row_groups, room = (int64_t)kSms * (a.head_dim <= 64 ? 2 : 1);
  p.whole = most <= kWholeBlocks;
  const int64_t warps = p.whole ? items : items * (most / kMinShare + 1);
  p.ctas = (int32_t)(warps < room ? (warps < 1 ? 1 : warps) : room);
  const int64_t join = p.ctas / (items > 0 ? items : 1) / 8;           // about 8 parts or more to a warp
  p.join_warps = 1;
  while (p.join_warps < 32 && p.join_warps < join) p.join_warps *= 2;
  // x / size = (high word of x * multiplier + x) >> shift for every x below 2^31 (Granlund and Montgomery's division by invariants)
  while (p.page_shift < 31 && (1u << p.page_shift) < (uint32_t)a.page_size) ++p.page_shift;
  p.page_multiplier = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << p.page_shift) - (uint64_t)a.page_size)) / (uint64_t)a.page_size + 1);
  return p;
}

template <typename T, int DB, bool ONE_PAGE>
cudaError_t launch(const PagedArgs& a, const PagedPlan& p, cudaStream_t st) {
  using S = Shape<DB>;
  static bool attr_set[64] = {};
  static std::mutex attr_mutex;
  {
    std::lock_guard<std::mutex> lock(attr_mutex);
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
      const cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<T, DB, ONE_PAGE>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
      if (e != cudaSuccess) return e;
      attr_set[dev] = true;
    }
  }
  paged_attention_kernel<T, DB, ONE_PAGE><<<p.ctas, kWarps * 32, S::kSmem, st>>>(a, p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || p.whole) return e;
  const int warps = p.join_warps > 8 ? p.join_warps : 8;
  const int64_t rows = (int64_t)a.batch * a.heads * a.tokens, each = warps / p.join_warps;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((rows + each - 1) / each));
  cfg.blockDim = dim3(warps * 32);
  cfg.dynamicSmemBytes = p.join_warps > 1 ? warps * (a.head_dim + 2) * sizeof(float) : 0;
  cfg.stream = st;
  cudaLaunchAttribute early{};                          // its CTAs start while the first kernel ends, and wait for its end
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_join_kernel<T>, a, p);
}

size_t parts_of(const PagedPlan& p) { return (size_t)2 * p.ctas * (kWarps + 1) * p.rows; }

}  // namespace

size_t paged_attention_workspace(const PagedArgs& a) {
  const PagedPlan p = make_plan(a);
  return p.whole ? 0 : parts_of(p) * (a.head_dim + 2) * sizeof(float) + ((size_t)a.batch + 1) * sizeof(int64_t);
}

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, void* workspace, cudaStream_t st) {
  PagedPlan p = make_plan(a);
  if (!p.whole) {
    p.part_o = reinterpret_cast<float*>(workspace);
    p.part_ml = p.part_o + parts_of(p) * a.head_dim;
    p.prefix = reinterpret_cast<int64_t*>(p.part_ml + parts_of(p) * 2);
  }
#define SWARM_PAGED_LAUNCH(T)                                                                                             \
  (a.page_size % kBlock == 0 ? a.head_dim <= 64 ? launch<T, 1, true>(a, p, st) : launch<T, 2, true>(a, p, st)             \
                             : a.head_dim <= 64 ? launch<T, 1, false>(a, p, st) : launch<T, 2, false>(a, p, st))
  return dtype == SWARM_BF16 ? SWARM_PAGED_LAUNCH(__nv_bfloat16) : SWARM_PAGED_LAUNCH(__half);
#undef SWARM_PAGED_LAUNCH
}

}  // namespace swarm
