// Attention of a sentence's newest tokens over its paged cache: every visible key and value is read once, HBM is the bound.
//
// An item is up to 16 rows (tokens x query heads of a key head) of a sentence and all the positions that one of them sees, in
// blocks of 16 or 32. The blocks of all items in a row are dealt to the device's warps in equal runs, whatever the sentences'
// lengths: a warp may end one item, take several whole ones and begin another. Each warp works alone: a ring of blocks that
// cp.async fills past the ends of items, so that loads never pause (64 to 128 KB in flight on a multiprocessor), ldmatrix,
// m16n8k16 products with the running maximum and sum of the softmax in registers. An item that was cut leaves parts (maximum,
// sum, o): those of a CTA's warps, whose runs follow one another, are joined at the CTA's end, those of several CTAs by a
// second kernel, which may be launched before the first has ended (up to 1 us less); always in the items' order.
//
// Positions and values are the sixteen rows of the products, the item's rows their eight columns: s^T = K q^T, o^T = V^T p^T.
// A decoding step has few rows, and the other way round half of every product and of the softmax would go to rows that
// are not there.
//
// Weights enter their product as the sum of two numbers of the type: rounded once, o would be 1.4 times as far from its value as
// its own rounding leaves it. The products are a small part of a block's time, so the second costs nothing.
//
// Measured on the device, whole call: 8 sentences of 16384 positions, 8 key heads of 128 with four query heads each, 537 MB, 90 us, 6.0
// TB/s; 128 sentences of 128 to 1024 positions, 16 heads of 64, 327 MB, 63 us, 5.2 TB/s; 64 sentences' drafts of four
// tokens through a window of 1024, 32 heads of 128 on 8, 264 MB, 61 us. Of these 5 us pass until the first copies are on their way, 4 us in
// the joining kernel, and about 8 us while some multiprocessors have ended: runs are equal, not what HBM gives each
// multiprocessor. Runs given to whoever is free would change the order of sums from call to call. The tensor pipe is 10 to 18 % busy.
#include <mutex>

#include "swarm_attention_tile.cuh"
#include "swarm_paged.h"

namespace swarm {
namespace {

constexpr int kRows = 16;
constexpr int kWarps = 8;
constexpr int kCtasPerSm = 1;                         // two of four warps: long documents 96 -> 101 us
// Positions that a warp's run has at least. Small calls, 32 / 64 / 128: 4 x 8 heads of 64 on 490 positions 12.2 / 14.0 / 15.0 us, 32 x 4
// key heads of 128 on 230 14.1 / 16.0 / 20.0; large ones are the same.
constexpr int kMinShare = 32;
// Items of no more positions are not cut: a warp takes each, and no kernel joins. 4 x 8 heads of 64 on 100 positions 9.1 us, cut 10.7;
// on 230 positions 13.6 and 12.1, 32 x 4 key heads of 128 on 230 20.6 and 14.1. The host knows no lengths: this, and what is kept in L2, go
// by the room that the table and the pages have (77 positions 8.0 us, in a table for more 10.4).
constexpr int kWholePositions = 128;
// The tensor core cuts off what its sum has no bits for, always towards 0, so sums shrink by as many cuts as a warp takes products
// of an item: 2^20 positions in one run, fp16, left o 0.8 % too small. Where a run may be longer than this, a block's products
// are added up from nothing and then to o in fp32; below, it is 256 cuts and by that measure 1.6e-5, a thirtieth of fp16's
// own rounding. Added always, drafts through a window 61 -> 63 us, 8 sentences of 16384 positions, heads of 64, 88 -> 92.
constexpr int kLongRun = 2048;
constexpr int kSms = 148;

// DB: heads of up to 64 DB values. Blocks in flight to a warp, measured with one page to sixteen positions: heads of 128, pages of 64,
// long documents two ahead 95 us, one 89; drafts through a window 61 and 60. Heads of 64, 8 sentences of 16384, 88 and 91;
// with a page to each position, heads of 128, 88 and 90.
template <int DB, bool ONE_PAGE> struct Shape {
  static constexpr int kBlock = 32 / DB;                // positions of a block
  static constexpr int kStages = DB == 2 && ONE_PAGE ? 2 : 3;
  static constexpr int kTileBytes = kBlock * DB * 128;  // of keys, and of values
  static constexpr int kRing = kStages * 2 * kTileBytes;
  static constexpr int kSmem = kWarps * kRing;
};

struct PagedPlan {
  int32_t row_groups;                 // of `tokens` rows
  int32_t rows;                       // that a part holds
  int32_t whole;                      // items are not cut
  int32_t long_runs;                  // a warp may take more than kLongRun positions of an item
  int32_t streams;                    // the cache is larger than L2
  int32_t ctas;
  int32_t beside;                     // key heads that warps of a CTA take side by side: 1 or 2
  int32_t head_groups;                // kv_heads / beside
  int32_t joined;                     // items that the joining kernel has at most, those side by side counted once
  int32_t join_warps;                 // for each row of them
  uint32_t page_multiplier, page_shift;                 // division by the size of a page
  int32_t* joins;                     // [ctas][8], see JoinInfo
  // parts: two for each CTA and key head side by side; then, without ml, the first of each warp
  float* part_ml;                     // [parts][rows][2] maximum and sum
  float* part_o;                      // [parts][rows][pitch], the warps' as their lanes hold them
  int32_t pitch;
};

// What a sentence's rows see, in blocks of B: the first `sink_blocks`, then those from position lo / B * B. A length beyond what the
// table has room for adds no blocks, and a sentence without blocks has no items.
struct Sentence {
  int length, n, lo, sink_blocks, blocks, row_groups;
};
template <int B> __device__ __forceinline__ Sentence sentence_of(const PagedArgs& a, int b) {
  Sentence s;
  s.length = length_in(a, b);
  s.n = rows_in(a, b, s.length);
  s.lo = a.window > 0 ? max(0, s.length - s.n - a.window + 1) : 0;
  const int sinks = min(min(a.sinks, s.lo), a.capacity), end = min(s.length, a.capacity);
  s.sink_blocks = sinks / B + (sinks % B != 0);
  s.blocks = s.sink_blocks;
  if (end > s.lo) {
    s.sink_blocks = min(s.sink_blocks, s.lo / B);
    s.blocks = s.sink_blocks + (end - 1) / B + 1 - s.lo / B;
  }
  if (s.n == 0) s.blocks = 0;
  s.row_groups = s.blocks > 0 ? (s.n * a.group + kRows - 1) / kRows : 0;
  return s;
}
// Blocks of a sentence's items, those of the key heads beside one another counted once.
__device__ __forceinline__ int64_t blocks_of_items(const PagedPlan& p, const Sentence& s) {
  return (int64_t)s.blocks * (p.head_groups * s.row_groups);
}
__device__ __forceinline__ int64_t divide(int64_t x, int64_t d) {      // of numbers that are not negative
  return ((x | d) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)d) : x / d;
}

// The runs that `total` blocks are dealt in, `per_cta` of them in each CTA, the first `more` one block longer.
struct Runs {
  int64_t each, more;
  int count, per_cta;
  __device__ __forceinline__ Runs(int64_t total, int most, int ctas, int min_share) {
    count = (int)max((int64_t)1, min((int64_t)most, total / min_share));
    per_cta = count == most ? most / ctas : (count + ctas - 1) / ctas;        // few runs go to many multiprocessors
    each = divide(total, count);
    more = total - each * count;
  }
  __device__ __forceinline__ int64_t begin(int r) const { return r * each + min((int64_t)r, more); }
  __device__ __forceinline__ int owner(int64_t x) const {
    const int64_t wide = more * (each + 1);
    return (int)(x < wide ? divide(x, each + 1) : more + divide(x - wide, each));
  }
};

// Copies of 16 bytes under a cache policy; zeros where nothing is there.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void copy16_or_zero(uint32_t dst, const void* src, bool there, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" :: "r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t r[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t r[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" :: "l"(p)); }
// An 8 x 8 matrix of 16-bit numbers (lane: two neighbours of row lane / 4) transposed. All lanes of the warp.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// Offset of chunk c (16 bytes) of row r of a tile: eight rows' same chunk, and a row's eight, lie in different banks.
template <int DB> __device__ __forceinline__ uint32_t tile_offset(int r, int c) {
  return (uint32_t)(r * (DB * 128) + (c >> 3) * 128 + (((c & 7) ^ (r & 7)) << 4));
}
// Whether a word holds an infinity or a NaN.
template <typename T> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t e = kNarrow<T> ? 0x7C00u : 0x7F80u;
  return (w & e) == e || ((w >> 16) & e) == e;
}

// The numbers of a word that are NaN or the infinity with this sign bit (in each half), as ones of the type.
template <typename T> __device__ __forceinline__ uint32_t infinities(uint32_t w, uint32_t sign) {
  constexpr uint32_t e = kNarrow<T> ? 0x7C007C00u : 0x7F807F80u, least = e & ~(e << 1), one = kNarrow<T> ? 0x3C00u : 0x3F80u;
  const uint32_t all = (w & e) + least;                 // the top bit: an exponent of ones
  const uint32_t some = ((w & ~e & 0x7FFF7FFFu) + 0x7FFF7FFFu) | ~(w ^ sign);           // the top bit: a NaN, or that sign
  return ((all & some) >> 15 & 0x00010001u) * one;
}

// A block in the ring: what it is of, and which of its positions were read.
struct __align__(16) BlockInfo {
  int32_t b, head, row0, n;           // sentence, key head, first row of the item; the sentence's rows are n tokens'
  int32_t block;                      // of the item
  int32_t position;
  int32_t first_new;                  // position of the first row: what lies past it, not every row sees
  int32_t last_gone;                  // what lies before it, the last row does not see
  uint32_t present;                   // a bit for each position
  uint32_t flags;
};
enum : uint32_t {
  kFirst = 1, kLast = 2,              // of the blocks of the item that this run has
  kFromStart = 4, kToEnd = 8,         // the item's first, its last
  kRunEnds = 16, kNone = 32
};

// Whether the row of token t sees position p.
__device__ __forceinline__ bool sees(const PagedArgs& a, const BlockInfo& info, int p, int t) {
  const int own = info.first_new + t;
  return p <= own && (a.window == 0 || p > own - a.window || p < a.sinks);
}

// Parts of a cut item that a warp holds: the run's first item may have begun elsewhere (0), its last one may go on (1).
struct __align__(16) PartInfo {
  int32_t there, b, head, row0, rows, to_end, in_ring;   // rows: from row0 on; in_ring: in shared memory, else in the workspace
};
// A row of a cut item: where it goes (values of out, or below 0 the CTA's part -1 - row), its parts' first and last warp.
struct __align__(16) CutRow {
  int64_t to;
  float sum;
  int8_t first, last, second, there;
};
// The item (of the first of the key heads beside one another) that a CTA begins and does not end, for the joining kernel; rows 0: none.
struct __align__(16) JoinInfo {
  int32_t b, head, row0, rows, last_cta, unused[3];
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// The factor of a part's sums whose maximum is `m` beside one of `base`; never 0, so that infinities of its o stay.
__device__ __forceinline__ float part_factor(float m, float base, float c) { return fmaxf(ex2((m - base) * c), 1.17549435e-38f); }
// Two parts of a row joined: maximum and sum, and the factors of their o.
__device__ __forceinline__ void join_ml(float& m, float& l, float m1, float l1, float c, float& f0, float& f1) {
  const float top = fmaxf(m, m1), base = top == -INFINITY ? 0.0f : top;
  f0 = part_factor(m, base, c);
  f1 = part_factor(m1, base, c);
  l = l * f0 + l1 * f1;
  m = top;
}

// The lse of a row from its maximum and sum.
template <typename T>
__device__ __forceinline__ void write_lse(const PagedArgs& a, int b, int t, int h, float m, float l) {
  a.lse[((int64_t)b * a.heads + h) * a.tokens + t] = l != 0.0f ? m * a.scale + (logf(l) - kRunningShift<T> * 0.69314718f) : -INFINITY;
}
// Four values of a row, from the row's sum.
template <typename T>
__device__ __forceinline__ void write_values(T* to, float l, const float v[4]) {
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2*>(to) = l != 0.0f ? make_uint2(pack2<T>(v[0] * inv, v[1] * inv), pack2<T>(v[2] * inv, v[3] * inv)) : make_uint2(0, 0);
}

// Puts infinities in the places of NaN that stand for them. A row's infinite value becomes NaN where what rounding left of its weight
// is 0 or of the other sign. The item's values are read once more, the infinities of either sign that a row sees are counted by
// products with ones. sums: a warp's, [NT][DB * 4][4], of the blocks from `first_block` to the one of `block`. Not inlined: where
// all is finite it would cost 2 us of 90 by being there. With infinities in every page those 90 us are 750.
template <typename T, int DB, int NT>
__device__ __noinline__ void put_infinities(const PagedArgs& a, const BlockInfo* block, int first_block, float* sums) {
  constexpr int B = 32 / DB, kSixteens = B / 16;
  constexpr uint32_t kOne = kNarrow<T> ? 0x3C00u : 0x3F80u;
  const BlockInfo info = *block;
  const int lane = threadIdx.x & 31, r8 = lane >> 2, c4 = lane & 3;
  const Sentence of = sentence_of<B>(a, info.b);
  const T* values = reinterpret_cast<const T*>(a.v_pages) + info.head * a.vps.head;
  // -0 stands for a NaN that nothing has taken the place of
  for (int i = 0; i < NT * DB * 16; ++i) sums[i] = isnan(sums[i]) ? -0.0f : sums[i] + 0.0f;
  for (int sixteen = first_block * kSixteens; sixteen < (info.block + 1) * kSixteens; ++sixteen) {
    const int at = sixteen / kSixteens, p0 = (at < of.sink_blocks ? at : at - of.sink_blocks + of.lo / B) * B + sixteen % kSixteens * 16;
    const T* row[4];                                    // of positions 2 c4, + 1, + 8, + 9
    uint32_t see[NT][2];                                // row r8 sees them
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + c4 * 2 + (i & 1) + (i >> 1) * 8, page = p >= 0 ? page_of(a, info.b, p / a.page_size) : -1;
      row[i] = page >= 0 ? values + page * a.vps.batch + p % a.page_size * a.vps.token : nullptr;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint32_t one = page >= 0 && sees(a, info, p, (info.row0 + nt * 8 + r8) / a.group) ? kOne : 0u;
        see[nt][i >> 1] = i & 1 ? see[nt][i >> 1] | one << 16 : one;
      }
    }
    for (int d = 0; d < DB * 4; ++d) {
      uint32_t up[4], down[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {                     // values r8 (and 8 more), positions as in `see`
        const int value = d * 16 + r8 + (e & 1) * 8;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (row[(e >> 1) * 2 + i] && value < a.head_dim) w |= (uint32_t)reinterpret_cast<const uint16_t*>(row[(e >> 1) * 2 + i])[value] << (16 * i);
        up[e] = infinities<T>(w, 0u);
        down[e] = infinities<T>(w, 0x80008000u);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float plus[4] = {}, minus[4] = {}, *to = sums + (nt * DB * 4 + d) * 4;
        mma16816<T>(plus, up, see[nt][0], see[nt][1]);
        mma16816<T>(minus, down, see[nt][0], see[nt][1]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (plus[u] > 0.0f) to[u] += INFINITY;
          if (minus[u] > 0.0f) to[u] -= INFINITY;
        }
      }
    }
  }
  for (int i = 0; i < NT * DB * 16; ++i) sums[i] = __float_as_uint(sums[i]) == 0x80000000u ? NAN : sums[i];
}

// NT: items of up to 8 NT rows. ONE_PAGE: pages hold a multiple of 16 positions, so sixteen of a block lie in one. Then a row's
// address is one addition away from the last one's; else each position has its own, and a lane gets them by shuffles.
template <typename T, int DB, int NT, bool ONE_PAGE, bool LONG>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm)
paged_attention_kernel(const __grid_constant__ PagedArgs a, const PagedPlan plan) {
  using S = Shape<DB, ONE_PAGE>;
  constexpr int kPartBytes = kRows * DB * 64 * 4;
  static_assert(2 * kPartBytes <= S::kRing, "a warp's two parts fit its ring");
  constexpr int B = S::kBlock, kSixteens = B / 16, kStages = S::kStages, kChunks = DB * 8, kRowsPerCopy = 32 / kChunks;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ BlockInfo s_info[kWarps][kStages];
  __shared__ PartInfo s_part[kWarps][2];
  __shared__ int64_t s_prefix[kWarps * 32 + 1];
  __shared__ int64_t s_warp[kWarps];
  __shared__ int s_last_cta;
  __shared__ int s_first_block[kWarps];                 // that a run has of its item
  __shared__ float2 s_ml[kWarps][2][kRows];             // maximum and sum of the rows of a part, then (factor of their o, .)
  __shared__ CutRow s_rows[(kWarps + 2) * kRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r8 = lane >> 2, c4 = lane & 3, chunks = a.head_dim / 8;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (lane < 2) s_part[warp][lane].there = 0;
  if (tid == 0) s_last_cta = blockIdx.x;                // no run of the CTA ends inside an item
  const int beside = plan.beside, sub_runs = beside == 2 ? kWarps / 2 : kWarps, side = warp & (beside - 1), sub = warp >> (beside - 1);

  uint64_t policy;
  if (plan.streams) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));

  // this warp's run
  int b = 0, hk = 0, rg = 0, block = 0;
  int64_t left = 0, item_end = 0;                       // blocks to take; past the last item, where items are not cut
  Sentence s;
  if (plan.whole) {
    const uint32_t each = a.kv_heads * plan.row_groups, items = a.batch * each;         // below 2^31
    const uint32_t all = gridDim.x * kWarps, turn = warp * gridDim.x + blockIdx.x;      // few items go to many multiprocessors
    const uint32_t per = items / all, more = items % all, item = turn * per + min(turn, more);
    item_end = item + per + (turn < more);
    b = item / each; hk = item % each / plan.row_groups; rg = item % plan.row_groups;
    left = item < item_end;
    if (left) s = sentence_of<B>(a, b);
  } else {
    const int per = (a.batch + kWarps * 32 - 1) / (kWarps * 32);
    const int b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
    int64_t before = 0;
    for (int i = b0; i < b1; ++i) before += blocks_of_items(plan, sentence_of<B>(a, i));
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
    __syncthreads();
    const Runs runs(s_prefix[kWarps * 32], gridDim.x * sub_runs, gridDim.x, kMinShare / B);
    const int run = blockIdx.x * runs.per_cta + sub;
    const bool takes = sub < runs.per_cta && run < runs.count;
    const int64_t begin = takes ? runs.begin(run) : 0;
    left = takes ? runs.begin(run + 1) - begin : 0;
    if (left > 0) {
      int lo = 0, hi = kWarps * 32;                     // the slice of sentences that holds the run's first block
      while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (s_prefix[mid] <= begin) lo = mid; else hi = mid; }
      int64_t at = begin - s_prefix[lo];
      b = lo * per;
      s = sentence_of<B>(a, b);
      while (at >= blocks_of_items(plan, s) && b + 1 < a.batch) { at -= blocks_of_items(plan, s); ++b; s = sentence_of<B>(a, b); }
      // Lengths are read more than once: should somebody write them meanwhile, the results are undefined, but nothing out of
      // range is touched. Runs and items then may not fit together: this run is left out, items begun before it are not ended.
      if (at >= blocks_of_items(plan, s)) {
        left = 0;
      } else {
        const int item = (int)divide(at, s.blocks);
        block = (int)(at - (int64_t)item * s.blocks);
        hk = item / s.row_groups * beside + side;
        rg = item % s.row_groups;
      }
    }
  }
  bool fresh = true;                                    // the next block is the first of its item here
  // moves on to an item that exists
  auto skip = [&]() {
    while (rg >= s.row_groups) {                        // none in a sentence without rows
      rg = 0;
      hk += beside;
      if (hk >= a.kv_heads || s.row_groups == 0) {
        hk = side;
        if (++b >= a.batch) { left = 0; return; }
        s = sentence_of<B>(a, b);
      }
    }
    if (plan.whole && ((int64_t)b * a.kv_heads + hk) * plan.row_groups + rg >= item_end) left = 0;
  };
  if (left > 0) skip();

  // The next block: its position, and the pages of its sixteens (ONE_PAGE), or lane i that of position i. The table is read 64
  // columns at a time, the second 32 before they are needed: lane i holds columns seen + i and seen + 32 + i of row seen_b.
  int p0 = 0, page[ONE_PAGE ? kSixteens : 1], slot[ONE_PAGE ? kSixteens : 1], near = 0, far = 0, seen = 0, seen_b = -1;
  auto look_up = [&]() {
    if (left <= 0) return;
    p0 = (block < s.sink_blocks ? block : block - s.sink_blocks + s.lo / B) * B;
    auto column_of = [&](int p) { return (int)((__umulhi((uint32_t)p, plan.page_multiplier) + (uint32_t)p) >> plan.page_shift); };
    auto entries = [&](uint32_t column) { return column + lane < (uint32_t)a.table_columns ? a.table[b * a.table_pitch + column + lane] : -1; };
    const int first = column_of(p0);
    const uint32_t ahead = (uint32_t)(first - seen);
    if (b != seen_b || ahead >= 64u) {
      seen_b = b;
      seen = first;
      near = entries(first);
      far = entries((uint32_t)first + 32u);
    } else if (ahead >= 32u) {
      seen += 32;
      near = far;
      far = entries((uint32_t)seen + 32u);
    }
#pragma unroll
    for (int g = 0; g < (ONE_PAGE ? kSixteens : 1); ++g) {
      const int p = ONE_PAGE ? p0 + g * 16 : p0 + (lane & (B - 1)), column = column_of(p), at = column - seen;
      slot[g] = p - column * a.page_size;
      const int x = __shfl_sync(0xFFFFFFFFu, near, at & 31), y = __shfl_sync(0xFFFFFFFFu, far, at & 31);
      page[g] = at < 32 ? x : y;                        // a block has at most 32 columns from its first one on
    }
  };
  look_up();

  uint8_t* ring = smem + warp * S::kRing;
  const int row_of_lane = lane / kChunks, c_of_lane = lane % kChunks;
  const uint32_t ring_at = smem_u32(ring);
  // where a lane's pieces of a tile go: rows 4 (DB = 1) or 2 apart, so that swizzling repeats after two or four
  uint32_t spot[8 / kRowsPerCopy];
#pragma unroll
  for (int i = 0; i < 8 / kRowsPerCopy; ++i) spot[i] = ring_at + tile_offset<DB>(i * kRowsPerCopy + row_of_lane, c_of_lane);
  // starts the copies of the next block, and moves on
  auto fetch = [&](int stage) {
    if (left > 0) {
      const uint32_t dst = stage * 2 * S::kTileBytes;
      auto spot_of = [&](int i) { return spot[i % (8 / kRowsPerCopy)] + i / (8 / kRowsPerCopy) * (8 * DB * 128) + dst; };
      uint32_t present = low_bits(B);                   // seen by some row
      if (p0 < s.lo || p0 > s.length - B) present = low_bits(s.length - p0) & (~low_bits(s.lo - p0) | low_bits(a.sinks - p0)) & low_bits(B);
      if constexpr (ONE_PAGE) {
        uint32_t gone = 0;
#pragma unroll
        for (int g = 0; g < kSixteens; ++g)
          if ((uint32_t)page[g] >= (uint32_t)a.pages) gone |= 0xFFFFu << (16 * g);
        if (gone & present) {
          if (lane == 0) atomicOr(a.status, kStatusPage);
        }
        present &= ~gone;
        const int64_t kstep = kRowsPerCopy * a.kps.token, vstep = kRowsPerCopy * a.vps.token;
#pragma unroll
        for (int g = 0; g < kSixteens; ++g) {
          const T* kp = reinterpret_cast<const T*>(a.k_pages) + hk * a.kps.head + page[g] * a.kps.batch + (slot[g] + row_of_lane) * a.kps.token + c_of_lane * 8;
          const T* vp = reinterpret_cast<const T*>(a.v_pages) + hk * a.vps.head + page[g] * a.vps.batch + (slot[g] + row_of_lane) * a.vps.token + c_of_lane * 8;
          if (present == low_bits(B) && chunks == kChunks) {
#pragma unroll
            for (int i = 0; i < 16 / kRowsPerCopy; ++i) {
              const uint32_t to = spot_of(g * (16 / kRowsPerCopy) + i);
              copy16(to, kp, policy);
              copy16(to + S::kTileBytes, vp, policy);
              kp += kstep;
              vp += vstep;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 16 / kRowsPerCopy; ++i) {
              const bool copy = (present >> (g * 16 + i * kRowsPerCopy + row_of_lane) & 1u) && c_of_lane < chunks;
              const void* none = a.q;                   // nothing is read there
              const uint32_t to = spot_of(g * (16 / kRowsPerCopy) + i);
              copy16_or_zero(to, copy ? kp : none, copy, policy);
              copy16_or_zero(to + S::kTileBytes, copy ? vp : none, copy, policy);
              kp += kstep;
              vp += vstep;
            }
          }
        }
      } else {
        const bool wanted = lane < B && (present >> lane & 1u), there = (uint32_t)page[0] < (uint32_t)a.pages;
        if (wanted && !there) atomicOr(a.status, kStatusPage);
        present = __ballot_sync(0xFFFFFFFFu, wanted && there);
        const int64_t ko = page[0] * a.kps.batch + slot[0] * a.kps.token, vo = page[0] * a.vps.batch + slot[0] * a.vps.token;
        const T* kb = reinterpret_cast<const T*>(a.k_pages) + hk * a.kps.head + c_of_lane * 8;
        const T* vb = reinterpret_cast<const T*>(a.v_pages) + hk * a.vps.head + c_of_lane * 8;
#pragma unroll
        for (int i = 0; i < B / kRowsPerCopy; ++i) {
          const int r = i * kRowsPerCopy + row_of_lane;
          const int64_t kr = __shfl_sync(0xFFFFFFFFu, ko, r), vr = __shfl_sync(0xFFFFFFFFu, vo, r);
          const bool copy = (present >> r & 1u) && c_of_lane < chunks;
          const void* none = a.q;
          copy16_or_zero(spot_of(i), copy ? kb + kr : none, copy, policy);
          copy16_or_zero(spot_of(i) + S::kTileBytes, copy ? vb + vr : none, copy, policy);
        }
      }
      const bool ends = block + 1 == s.blocks, run_ends = !plan.whole && left == 1, last = ends || run_ends;
      if (lane == 0) {
        BlockInfo info;
        info.b = b; info.head = hk; info.row0 = rg * kRows; info.n = s.n; info.block = block; info.position = p0;
        info.first_new = s.length - s.n;
        info.last_gone = a.window > 0 ? s.length - a.window : 0;
        info.present = present;
        info.flags = (fresh ? kFirst : 0u) | (fresh && block == 0 ? kFromStart : 0u) | (last ? kLast : 0u) | (ends ? kToEnd : 0u) | (run_ends ? kRunEnds : 0u);
        s_info[warp][stage] = info;
      }
      if (fresh) {                                      // its rows, needed a block or two from now, behind what is in flight
        const int r = rg * kRows + lane / DB, t = r / a.group;
        if (lane < NT * 8 * DB && t < s.n && lane % DB * 64 < a.head_dim)
          prefetch_l2(reinterpret_cast<const T*>(a.q) + offset_of(a.qs, b, t, hk * a.group + r % a.group) + lane % DB * 64);
      }
      if (run_ends && !ends && lane == 0 && side == 0) {
        // the CTA that holds the item's last block; of a CTA's runs the last one's counts
        const Runs runs(s_prefix[kWarps * 32], gridDim.x * sub_runs, gridDim.x, kMinShare / B);
        const int run = blockIdx.x * runs.per_cta + sub;
        if (sub + 1 == runs.per_cta || run + 1 == runs.count) s_last_cta = min(runs.owner(runs.begin(run + 1) + (s.blocks - 2 - block)) / runs.per_cta, (int)gridDim.x - 1);
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

  // rows past a sentence's count, or of a sentence of which nothing is there
  for (int z = blockIdx.x; z < a.batch; z += gridDim.x) {
    const Sentence x = sentence_of<B>(a, z);
    const int n = x.blocks > 0 ? x.n : 0;
    if (x.n > 0 && x.length > a.capacity && tid == 0) atomicOr(a.status, kStatusPage);
    for (int i = tid; i < (a.tokens - n) * a.heads * chunks; i += kWarps * 32) {
      const int ch = i % chunks, h = i / chunks % a.heads, t = n + i / chunks / a.heads;
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + offset_of(a.os, z, t, h) + ch * 8) = make_uint4(0, 0, 0, 0);
      if (a.lse && ch == 0) a.lse[((int64_t)z * a.heads + h) * a.tokens + t] = -INFINITY;
    }
  }

  uint32_t q[NT][DB * 4][2];                            // operands of the products with the keys: row r8
  float o[NT][DB * 4][4], m[NT][2], l[NT][2];           // values r8, r8 + 8 of sixteen; rows 2 c4, 2 c4 + 1
  int t_of[NT][2];                                      // the tokens of these rows
  const float c = a.scale * kLog2e;
  bool from_start = false;
  // a part of a cut item, as rows, in the ring when the run has ended; one that ends earlier is kept in the workspace till then
  auto store_part = [&](int second, auto value) {
    float* to = reinterpret_cast<float*>(ring) + second * (kPartBytes / 4);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < DB * 4; ++d) {
        const float4 x = value(nt, d);
        const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) to[(nt * 8 + c4 * 2 + (u & 1)) * (DB * 64) + d * 16 + (u >> 1) * 8 + r8] = xs[u];
      }
  };
  float4* kept = reinterpret_cast<float4*>(plan.part_o + ((int64_t)2 * gridDim.x * beside * plan.rows + (int64_t)(blockIdx.x * kWarps + warp) * kRows) * (DB * 64)) + lane;
  // a lane's rows and halves for ldmatrix: eight rows x 8 values four times
  const int key_row = lane & 15, key_half = lane >> 4, value_row = (lane & 7) + (lane >> 4) * 8, value_half = lane >> 3 & 1;
  for (int stage = 0;; stage = stage + 1 == kStages ? 0 : stage + 1) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    const BlockInfo info = s_info[warp][stage];
    if (info.flags & kNone) break;
    if (info.flags & kFirst) {
      from_start = info.flags & kFromStart;
      if (lane == 0) s_first_block[warp] = info.block;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = info.row0 + nt * 8 + r8, t = r / a.group;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(a.q) + offset_of(a.qs, info.b, t, info.head * a.group + r % a.group)) + c4;
#pragma unroll
        for (int ks = 0; ks < DB * 4; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) q[nt][ks][e] = t < info.n && ks * 2 + e < chunks ? src[ks * 8 + e * 4] : 0u;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          t_of[nt][u] = (info.row0 + nt * 8 + c4 * 2 + u) / a.group;
          m[nt][u] = -INFINITY;
          l[nt][u] = 0.0f;
        }
#pragma unroll
        for (int d = 0; d < DB * 4; ++d)
#pragma unroll
          for (int u = 0; u < 4; ++u) o[nt][d][u] = 0.0f;
      }
    }
    const uint32_t tile_k = ring_at + stage * 2 * S::kTileBytes, tile_v = tile_k + S::kTileBytes;
    // scores: sc[sixteen positions][rows 2 c4, 2 c4 + 1 of position r8; of position r8 + 8]
    float sc[NT][kSixteens][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int g = 0; g < kSixteens; ++g)
#pragma unroll
        for (int u = 0; u < 4; ++u) sc[nt][g][u] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < DB * 4; ++ks)
#pragma unroll
      for (int g = 0; g < kSixteens; ++g) {
        uint32_t k[4];
        ldmatrix4(tile_k + g * (16 * DB * 128) + tile_offset<DB>(key_row, ks * 2 + key_half), k);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816<T>(sc[nt][g], k, q[nt][ks][0], q[nt][ks][1]);
      }
    // some position of the block is hidden from some row
    const bool edge = info.present != low_bits(B) || info.position + (B - 1) > info.first_new ||
                      (a.window > 0 && info.position < info.last_gone && info.position + (B - 1) >= a.sinks);
    if (edge) {
#pragma unroll
      for (int g = 0; g < kSixteens; ++g)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = g * 16 + r8 + (u >> 1) * 8;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            if (!(info.present >> i & 1u) || !sees(a, info, info.position + i, t_of[nt][u & 1])) sc[nt][g][u] = -INFINITY;
        }
    }
    bool moved = false;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float t = fmaxf(sc[nt][0][u], sc[nt][0][u + 2]);
        if constexpr (kSixteens == 2) t = max3(t, sc[nt][1][u], sc[nt][1][u + 2]);
        t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
        t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
        top[nt][u] = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
        moved |= (top[nt][u] - m[nt][u]) * c > 8.0f;
      }
    if (__any_sync(0xFFFFFFFFu, moved)) {
      // the maximum moved by more than 2^8 in some row (or the first block): rescale; smaller moves keep the reference
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float m_new = fmaxf(m[nt][u], top[nt][u]), f = m_new == m[nt][u] ? 1.0f : ex2((m[nt][u] - m_new) * c);
          m[nt][u] = m_new;
          l[nt][u] *= f;
#pragma unroll
          for (int d = 0; d < DB * 4; ++d) { o[nt][d][u] *= f; o[nt][d][u + 2] *= f; }
        }
    }
    uint32_t hi[NT][kSixteens][2], lo[NT][kSixteens][2];           // weights as an operand: the numbers, and what rounding left of them
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float base[2] = {m[nt][0] == -INFINITY ? 0.0f : m[nt][0], m[nt][1] == -INFINITY ? 0.0f : m[nt][1]};
#pragma unroll
      for (int g = 0; g < kSixteens; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = ex2(fmaf(sc[nt][g][2 * e] - base[0], c, kRunningShift<T>)), y = ex2(fmaf(sc[nt][g][2 * e + 1] - base[1], c, kRunningShift<T>));
          l[nt][0] += x;
          l[nt][1] += y;
          const uint32_t w = pack2<T>(x, y);
          float rx, ry;
          unpack2<T>(w, rx, ry);
          hi[nt][g][e] = transposed(w);
          lo[nt][g][e] = transposed(pack2<T>(x - rx, y - ry));
        }
    }
    bool apart = false;                                 // an infinity or a NaN that not every row sees: 0 times it would be NaN
    if (edge && a.tokens > 1) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < B / kRowsPerCopy; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(ring + stage * 2 * S::kTileBytes + S::kTileBytes + tile_offset<DB>(i * kRowsPerCopy + row_of_lane, c_of_lane));
        bad |= not_finite<T>(x.x) || not_finite<T>(x.y) || not_finite<T>(x.z) || not_finite<T>(x.w);
      }
      apart = __any_sync(0xFFFFFFFFu, bad);
    }
    // Adds the block's products to o, for the rows that `of_rows` says; `masked` leaves of the cache's values what is to be seen.
    // Sums of 64 values side by side: they wait for one another less often.
    constexpr int kSide = DB == 1 ? 4 : 1;
    auto add_products = [&](auto masked, auto of_rows) {
#pragma unroll
      for (int d0 = 0; d0 < DB * 4; d0 += kSide) {
        float x[kSide][NT][4];
#pragma unroll
        for (int d = 0; d < kSide; ++d)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < 4; ++u) x[d][nt][u] = LONG ? 0.0f : o[nt][d0 + d][u];
#pragma unroll
        for (int g = 0; g < kSixteens; ++g)
#pragma unroll
          for (int d = 0; d < kSide; ++d) {
            uint32_t v[4];
            ldmatrix4_trans(tile_v + g * (16 * DB * 128) + tile_offset<DB>(value_row, (d0 + d) * 2 + value_half), v);
            masked(g, v);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma16816<T>(x[d][nt], v, hi[nt][g][0], hi[nt][g][1]);
              mma16816<T>(x[d][nt], v, lo[nt][g][0], lo[nt][g][1]);
            }
          }
#pragma unroll
        for (int d = 0; d < kSide; ++d)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (of_rows(t_of[nt][u & 1])) o[nt][d0 + d][u] = LONG ? o[nt][d0 + d][u] + x[d][nt][u] : x[d][nt][u];
      }
    };
    if (!apart) {
      add_products([](int, uint32_t*) {}, [](int) { return true; });
    } else {
      // one token after the other, its rows alone and what it does not see as zeros: the same bits as above for these
      for (int t = 0; t < a.tokens; ++t) {
        uint32_t keep[kSixteens][2];
#pragma unroll
        for (int g = 0; g < kSixteens; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int p = info.position + g * 16 + e * 8 + c4 * 2;
            keep[g][e] = (sees(a, info, p, t) ? 0xFFFFu : 0u) | (sees(a, info, p + 1, t) ? 0xFFFF0000u : 0u);
          }
        add_products([&](int g, uint32_t* v) { v[0] &= keep[g][0]; v[1] &= keep[g][0]; v[2] &= keep[g][1]; v[3] &= keep[g][1]; },
                     [&](int token) { return token == t; });
      }
    }
    if (info.flags & kLast) {
      const bool done = from_start && (info.flags & kToEnd);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l[nt][u] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][u], x);
      // NaN among the sums of a row whose weights are none may stand for an infinite value
      float zero[2] = {0.0f, 0.0f};                     // as long as all sums are finite
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int d = 0; d < DB * 4; ++d) {
          fma2(zero[0], zero[1], o[nt][d][0], o[nt][d][1], 0.0f, 0.0f, zero[0], zero[1]);
          fma2(zero[0], zero[1], o[nt][d][2], o[nt][d][3], 0.0f, 0.0f, zero[0], zero[1]);
        }
      if (__any_sync(0xFFFFFFFFu, zero[0] + zero[1] != 0.0f)) {
        float sums[NT * DB * 16];
        bool some = false;
#pragma unroll
        for (int i = 0; i < NT * DB * 16; ++i) {
          sums[i] = o[i / (DB * 16)][i / 4 % (DB * 4)][i % 4];
          some |= isnan(sums[i]) && !isnan(l[i / (DB * 16)][i & 1]);
        }
        __syncwarp();                                   // the run's first block of the item has been written down
        if (__any_sync(0xFFFFFFFFu, some)) put_infinities<T, DB, NT>(a, &s_info[warp][stage], s_first_block[warp], sums);
#pragma unroll
        for (int i = 0; i < NT * DB * 16; ++i) o[i / (DB * 16)][i / 4 % (DB * 4)][i % 4] = sums[i];
      }
      if (done) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float inv[2] = {l[nt][0] != 0.0f ? 1.0f / l[nt][0] : 0.0f, l[nt][1] != 0.0f ? 1.0f / l[nt][1] : 0.0f};
          const int r = info.row0 + nt * 8 + r8, t = r / a.group;
          uint32_t* dst = reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(a.out) + offset_of(a.os, info.b, t, info.head * a.group + r % a.group)) + c4;
#pragma unroll
          for (int d = 0; d < DB * 4; ++d)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w = transposed(pack2<T>(l[nt][0] != 0.0f ? o[nt][d][2 * e] * inv[0] : 0.0f, l[nt][1] != 0.0f ? o[nt][d][2 * e + 1] * inv[1] : 0.0f));
              if (t < info.n && d * 2 + e < chunks) dst[d * 8 + e * 4] = w;
            }
          if (a.lse && r8 == 0) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (t_of[nt][u] < info.n) write_lse<T>(a, info.b, t_of[nt][u], info.head * a.group + (info.row0 + nt * 8 + c4 * 2 + u) % a.group, m[nt][u], l[nt][u]);
          }
        }
      } else {
        // a part: the last of the run's into its ring, which is done with, the other one into the workspace
        const bool in_ring = info.flags & kRunEnds;
        if (lane == 0) {
          PartInfo part;
          part.there = 1; part.b = info.b; part.head = info.head; part.row0 = info.row0; part.rows = min(kRows, info.n * a.group - info.row0);
          part.to_end = (info.flags & kToEnd) != 0; part.in_ring = in_ring;
          s_part[warp][from_start] = part;
        }
        __syncwarp();
        if (r8 == 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < 2; ++u) s_ml[warp][from_start][nt * 8 + c4 * 2 + u] = make_float2(m[nt][u], l[nt][u]);
        }
        if (in_ring) {
          store_part(from_start, [&](int nt, int d) { return make_float4(o[nt][d][0], o[nt][d][1], o[nt][d][2], o[nt][d][3]); });
        } else {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int d = 0; d < DB * 4; ++d) kept[(nt * DB * 4 + d) * 32] = make_float4(o[nt][d][0], o[nt][d][1], o[nt][d][2], o[nt][d][3]);
        }
      }
    }
  }
  cp_async_wait<0>();
  if (plan.whole) return;
  __syncwarp();
  if (s_part[warp][0].there && !s_part[warp][0].in_ring) {
    float4 x[NT][DB * 4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < DB * 4; ++d) x[nt][d] = kept[(nt * DB * 4 + d) * 32];
    store_part(0, [&](int nt, int d) { return x[nt][d]; });
  }

  // The CTA's parts. Those of an item: the second of the warp that begins it here, or the first warp's first, and the first of
  // the warps after it up to one that ends it. A row of an item: (its key head beside the others, k: its first warp's first
  // part (0) or that of the k-1-th warp's second, row).
  if (tid == 0) reinterpret_cast<JoinInfo*>(plan.joins)[blockIdx.x] = JoinInfo{};
  __syncthreads();
  // thread = a row: maximum and sum over its parts, and the parts' factors
  const int rows = (sub_runs + 1) * beside * plan.rows;
  for (int unit = tid; unit < rows; unit += kWarps * 32) {
    CutRow x{};
    int k = unit / plan.rows;
    const int row = unit - k * plan.rows, i0 = k > sub_runs;
    k -= i0 * (sub_runs + 1);
    const int second = k > 0, first = (k > 0 ? k - 1 : 0) * beside + i0;
    int last = first;
    const PartInfo of = s_part[first][second];
    if (of.there && row < of.rows) {
      bool ended = of.to_end;
      float most = s_ml[first][second][row].x, sum = 0.0f;
      while (!ended && last + beside < kWarps && s_part[last + beside][0].there) {
        last += beside;
        ended = s_part[last][0].to_end;
        most = fmaxf(most, s_ml[last][0][row].x);
      }
      const float base = most == -INFINITY ? 0.0f : most;
      for (int j = first; j <= last; j += beside) {
        float2& ml = s_ml[j][j == first && second][row];
        const float f = part_factor(ml.x, base, c);
        sum = fmaf(ml.y, f, sum);
        ml.x = f;
      }
      x.sum = sum; x.first = first; x.last = last; x.second = second; x.there = 1;
      const int r = of.row0 + row, t = r / a.group, h = of.head * a.group + r - t * a.group;
      if (second && ended) {
        x.to = offset_of(a.os, of.b, t, h);
        if (a.lse) write_lse<T>(a, of.b, t, h, most, sum);
      } else {
        const int64_t part = (int64_t)(2 * (blockIdx.x * beside + i0) + second) * plan.rows + row;
        x.to = -1 - part;
        *reinterpret_cast<float2*>(plan.part_ml + part * 2) = make_float2(most, sum);
        if (second && row == 0 && i0 == 0) {
          JoinInfo join{};
          join.b = of.b; join.head = of.head; join.row0 = of.row0; join.rows = of.rows; join.last_cta = s_last_cta;
          reinterpret_cast<JoinInfo*>(plan.joins)[blockIdx.x] = join;
        }
      }
    }
    s_rows[unit] = x;
  }
  __syncthreads();
  // 16 or 32 lanes take a row, four values each
  constexpr int kLanes = DB * 16;
  const int l4 = tid % kLanes * 4;
  if (l4 >= a.head_dim) return;
#pragma unroll 2
  for (int unit = tid / kLanes; unit < rows; unit += kWarps * 32 / kLanes) {
    const CutRow x = s_rows[unit];
    if (!x.there) continue;
    const int row = unit % plan.rows;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    int second = x.second;
    for (int j = x.first; j <= x.last; j += beside, second = 0) {
      const float f = s_ml[j][second][row].x;
      const float4 y = *reinterpret_cast<const float4*>(smem + j * S::kRing + second * kPartBytes + (row * (DB * 64) + l4) * 4);
      v[0] = fmaf(y.x, f, v[0]); v[1] = fmaf(y.y, f, v[1]); v[2] = fmaf(y.z, f, v[2]); v[3] = fmaf(y.w, f, v[3]);
    }
    if (x.to >= 0) write_values<T>(reinterpret_cast<T*>(a.out) + x.to + l4, x.sum, v);
    else *reinterpret_cast<float4*>(plan.part_o + (-1 - x.to) * (DB * 64) + l4) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// Joins the CTAs' parts of the items that go on past the CTA that began them: `join_warps` warps for each row, lane = four
// values, the parts in order; the warps meet in shared memory.
template <typename T>
__global__ void __launch_bounds__(1024) paged_join_kernel(PagedArgs a, PagedPlan plan) {
  extern __shared__ float s_join[];                     // [warps][head_dim + 2]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % plan.join_warps, pitch = a.head_dim + 2;
  const int index = blockIdx.x * (blockDim.x / 32 / plan.join_warps) + warp / plan.join_warps;
  int c0 = index / plan.rows / plan.beside;             // of the items that have to be joined
  const int side = index / plan.rows % plan.beside, r = index % plan.rows;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (plan.joined < plan.ctas) {                        // fewer than CTAs: which CTA begins the c0-th
    int there[(kSms * kCtasPerSm + 31) / 32], seen = 0, found = plan.ctas;
#pragma unroll
    for (int i = 0; i < (kSms * kCtasPerSm + 31) / 32; ++i)
      there[i] = i * 32 + lane < plan.ctas ? reinterpret_cast<const JoinInfo*>(plan.joins)[i * 32 + lane].rows : 0;
#pragma unroll
    for (int i = 0; i < (kSms * kCtasPerSm + 31) / 32; ++i) {
      const uint32_t has = __ballot_sync(0xFFFFFFFFu, there[i] > 0);
      const int here = __popc(has);
      const uint32_t at = __ballot_sync(0xFFFFFFFFu, there[i] > 0 && __popc(has & ((1u << lane) - 1u)) == c0 - seen);
      if (at) found = i * 32 + __ffs(at) - 1;
      seen += here;
    }
    c0 = found;
  }
  JoinInfo join{};
  if (c0 < plan.ctas) join = reinterpret_cast<const JoinInfo*>(plan.joins)[c0];
  const bool works = r < join.rows;
  const float c = a.scale * kLog2e;
  float top = -INFINITY, sum = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (works) {
    const int count = parts_between(c0, join.last_cta, plan.ctas), from = count * sub / plan.join_warps, to = count * (sub + 1) / plan.join_warps;
    for (int p0 = from; p0 < to; p0 += 8) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = p0 + i;
        const int64_t at = (int64_t)(2 * ((c0 + k) * plan.beside + side) + (k == 0)) * plan.rows + r;
        ml[i] = k < to ? *reinterpret_cast<const float2*>(plan.part_ml + at * 2) : make_float2(-INFINITY, 0.0f);
        x[i] = k < to && lane * 4 < a.head_dim ? *reinterpret_cast<const float4*>(plan.part_o + at * plan.pitch + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
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
    if (works && sub == 0) {                            // lane = a warp's part
      const float m0 = lane < plan.join_warps ? mine[lane * pitch] : -INFINITY;
      top = m0;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
      const float f = part_factor(m0, top == -INFINITY ? 0.0f : top, c);
      sum = warp_sum(lane < plan.join_warps ? mine[lane * pitch + 1] * f : 0.0f);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = 0.0f;
#pragma unroll 8
      for (int i = 0; i < plan.join_warps; ++i) {
        const float fi = __shfl_sync(0xFFFFFFFFu, f, i);
        if (lane * 4 < a.head_dim)
          for (int e = 0; e < 4; ++e) v[e] = fmaf(mine[i * pitch + 2 + lane * 4 + e], fi, v[e]);
      }
    }
  }
  if (!works || sub != 0) return;
  const int t = (join.row0 + r) / a.group, h = (join.head + side) * a.group + (join.row0 + r) % a.group;
  if (lane * 4 < a.head_dim) write_values<T>(reinterpret_cast<T*>(a.out) + offset_of(a.os, join.b, t, h) + lane * 4, sum, v);
  if (a.lse && lane == 0) write_lse<T>(a, join.b, t, h, top, sum);
}

PagedPlan make_plan(const PagedArgs& a) {
  PagedPlan p{};
  const int64_t rows = (int64_t)a.tokens * a.group;
  p.row_groups = (int32_t)((rows + kRows - 1) / kRows);
  p.rows = (int32_t)(rows < kRows ? rows : kRows);
  // the most positions that an item can have: the table's, or the window's with the first tokens'
  int64_t most = a.capacity;
  if (a.window > 0) {
    const int64_t seen = (int64_t)a.window + a.tokens - 1 + a.sinks;
    if (seen < most) most = seen;
  }
  const int64_t items = (int64_t)a.batch * a.kv_heads * p.row_groups;
  p.whole = most <= kWholePositions;
  // A cache that does not fit into L2 passes through it without displacing what other kernels, and the tables, rows and parts
  // of this one, have there: 128 sentences x 16 heads of 64 67 -> 62 us, drafts through a window 65 -> 61, long documents
  // 95 -> 92. One that fits stays for the next step: 100001 positions 24 us, else 25.
  p.streams = (int64_t)a.pages * a.page_size * a.kv_heads * a.head_dim * 4 > (int64_t)96 << 20;
  p.beside = 1;
  p.pitch = a.head_dim <= 64 ? 64 : 128;
  if (!p.whole) {
    // A position's heads of up to 64 values are 128 bytes each; where they lie side by side, two warps that take two of them at
    // a time ask for 256 bytes together: 16 heads of 64, 128 sentences 74 -> 68 us, 8 of 16384 positions 101 -> 96 us; four
    // at a time 68 and 96, eight 68 and 102. Heads of 128 on their own 95 us, two at a time 97.
    if (a.head_dim <= 64 && a.kv_heads % 2 == 0 && a.kps.head < a.kps.token) p.beside = 2;
  }
  p.head_groups = a.kv_heads / p.beside;
  // a run is a warp's equal share of all positions that there can be (or kMinShare of them, and the device is not filled)
  p.long_runs = most > kLongRun && items * most / (kSms * kCtasPerSm * kWarps) > kLongRun;
  const int64_t warps = p.whole ? items : items * (most / kMinShare + 2);
  const int64_t room = (int64_t)kSms * kCtasPerSm;
  p.ctas = (int32_t)(warps < room ? (warps < 1 ? 1 : warps) : room);
  const int64_t join = p.ctas * p.beside / (items > 0 ? items : 1) / 8;           // about 8 parts or more to a warp
  p.join_warps = 1;
  p.joined = (int32_t)(items / p.beside < p.ctas ? items / p.beside : p.ctas);
  while (p.join_warps < 32 && p.join_warps < join) p.join_warps *= 2;
  // x / size = (high word of x * multiplier + x) >> shift for every x below 2^31 (Granlund and Montgomery's division by invariants)
  while (p.page_shift < 31 && (1u << p.page_shift) < (uint32_t)a.page_size) ++p.page_shift;
  p.page_multiplier = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << p.page_shift) - (uint64_t)a.page_size)) / (uint64_t)a.page_size + 1);
  return p;
}

template <typename T, int DB, int NT, bool ONE_PAGE, bool LONG>
cudaError_t launch_as(const PagedArgs& a, const PagedPlan& p, cudaStream_t st) {
  using S = Shape<DB, ONE_PAGE>;
  static bool attr_set[64] = {};
  static std::mutex attr_mutex;
  {
    std::lock_guard<std::mutex> lock(attr_mutex);
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
      const cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<T, DB, NT, ONE_PAGE, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
      if (e != cudaSuccess) return e;
      attr_set[dev] = true;
    }
  }
  paged_attention_kernel<T, DB, NT, ONE_PAGE, LONG><<<p.ctas, kWarps * 32, S::kSmem, st>>>(a, p);
  return cudaGetLastError();
}

template <typename T, int DB, int NT>
cudaError_t launch_of(const PagedArgs& a, const PagedPlan& p, cudaStream_t st) {
  if (a.page_size % 16 == 0) return p.long_runs ? launch_as<T, DB, NT, true, true>(a, p, st) : launch_as<T, DB, NT, true, false>(a, p, st);
  return p.long_runs ? launch_as<T, DB, NT, false, true>(a, p, st) : launch_as<T, DB, NT, false, false>(a, p, st);
}

template <typename T>
cudaError_t launch(const PagedArgs& a, const PagedPlan& p, cudaStream_t st) {
  cudaError_t e;
  if (a.head_dim <= 64) e = p.rows <= 8 ? launch_of<T, 1, 1>(a, p, st) : launch_of<T, 1, 2>(a, p, st);
  else e = p.rows <= 8 ? launch_of<T, 2, 1>(a, p, st) : launch_of<T, 2, 2>(a, p, st);
  if (e != cudaSuccess || p.whole || p.ctas == 1) return e;
  const int warps = p.join_warps > 4 ? p.join_warps : 4, each = warps / p.join_warps;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((p.joined * p.beside * p.rows + each - 1) / each);
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

size_t cta_rows(const PagedPlan& p) { return (size_t)2 * p.ctas * p.beside * p.rows; }
size_t all_rows(const PagedPlan& p) { return cta_rows(p) + (size_t)p.ctas * kWarps * kRows; }

}  // namespace

size_t paged_attention_workspace(const PagedArgs& a) {
  const PagedPlan p = make_plan(a);
  return p.whole ? 0 : (all_rows(p) * p.pitch + cta_rows(p) * 2) * sizeof(float) + (size_t)p.ctas * sizeof(JoinInfo);
}

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, void* workspace, cudaStream_t st) {
  PagedPlan p = make_plan(a);
  if (!p.whole) {
    p.joins = reinterpret_cast<int32_t*>(workspace);
    p.part_o = reinterpret_cast<float*>(p.joins + p.ctas * 8);
    p.part_ml = p.part_o + all_rows(p) * p.pitch;
  }
  return dtype == SWARM_BF16 ? launch<__nv_bfloat16>(a, p, st) : launch<__half>(a, p, st);
}

}  // namespace swarm
