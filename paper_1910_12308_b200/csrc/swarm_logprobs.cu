// Log probabilities of given tokens with entropy and the likeliest tokens, and their gradient with respect to the logits.
//
// Forward: one walk over a row with the running maximum, sum and weighted sum of each thread's logits; HBM is the bound where rows are
// many. Short rows, and many, take a warp each, others a CTA, and where these are too few for the device a
// cluster of up to eight CTAs, which meet in shared memory of the first. The likeliest tokens take a second walk (over L2):
// the first leaves a number that at least `top` logits of the CTA reach, so of the second's logits hardly more than `top` are
// looked at twice. They are kept as (logit, place) in one 64-bit key, a lane each, so that their order is that of numbers.
// Gradient: one walk, a logit read and a gradient written.
//
// Measured on the device: 8192 rows of 32000 in bf16 forward 88 us, 6.0 TB/s (the special-function unit is 72 % busy; in fp32 6.6 TB/s),
// with entropies 102, gradient 165 us, 6.4 TB/s; 128 rows of 131072 9 us, with entropies and the 20 likeliest 19: the bound, the second
// walk and the merging of lists are chains of latencies; 8 rows of 32000 with four likeliest 5.9 us. Where fewer logits are finite than
// wanted, or all are equal, the bound leaves every logit: the 128 rows take 72 us.
#include <cmath>
#include <mutex>

#include "swarm_opsup.cuh"
#include "swarm_tc.cuh"

namespace swarm {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr float kFar = -3.402823466e38f;                // stands for differences of -infinity, whose exponential 0 they are multiplied with

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

struct LogProbsArgs {
  const void* logits;
  const int64_t* tokens;
  float *log_probs, *stats, *entropy, *top_log_probs;
  int64_t* top_tokens;
  const float *dlog_probs, *dentropy;
  void* dlogits;
  int64_t rows, cols, pitch, dlogits_pitch;
  float scale;
  int32_t top;
};

// A logit and its place as one number: larger logits first, of equal ones the lowest place; NaN above all, -0 as 0. 0 is no key.
__device__ __forceinline__ uint32_t rank_of(float v) {
  const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);
  return isnan(v) ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t rank) { return __uint_as_float(rank & 0x80000000u ? rank & 0x7FFFFFFFu : ~rank); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t place) { return (uint64_t)rank_of(v) << 32 | (uint32_t)~place; }

// What a part of a row adds up to: its largest logit, and with d = logit - largest the sums of exp(scale d) and exp(scale d) d.
// A part of nothing but -infinity has sums of 0. c = scale * log2(e).
struct Sums {
  float m, s, w;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// The sums taken against a larger maximum.
template <bool ENTROPY>
__device__ __forceinline__ void rebase(Sums& x, float m, float c) {
  if (x.m == m) return;
  const float d = x.m - m, f = ex2(d * c);
  if (ENTROPY) x.w = f == 0.0f ? 0.0f : (x.w + x.s * d) * f;
  x.s *= f;
  x.m = m;
}
// The sums of LANES neighbouring lanes, in each of them.
template <bool ENTROPY, int LANES>
__device__ __forceinline__ Sums lanes_joined(Sums x, float c) {
  float m = x.m;
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
  rebase<ENTROPY>(x, m, c);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    x.s += __shfl_xor_sync(kAll, x.s, o);
    if (ENTROPY) x.w += __shfl_xor_sync(kAll, x.w, o);
  }
  return x;
}

// Elements [0, n) of a row whose first one may lie anywhere: `head` elements up to a 16-byte boundary, `vectors` of 16 bytes, a tail.
template <typename T> struct Span {
  static constexpr int kPer = 16 / (int)sizeof(T);
  const T* p;
  int head, vectors, n;
  __device__ __forceinline__ Span(const T* row, int64_t cols) {
    p = row;
    n = (int)cols;
    head = min(n, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
    vectors = (n - head) / kPer;
  }
  __device__ __forceinline__ const uint4* at(int v) const { return reinterpret_cast<const uint4*>(p + head) + v; }
  // the elements outside the vectors, at most 2 (kPer - 1): number i of them
  __device__ __forceinline__ int loose() const { return n - vectors * kPer; }
  __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + vectors * kPer; }
};
template <typename T> __device__ __forceinline__ void unpack(const uint4& r, float* v) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  } else {
    unpack2<T>(r.x, v[0], v[1]); unpack2<T>(r.y, v[2], v[3]); unpack2<T>(r.z, v[4], v[5]); unpack2<T>(r.w, v[6], v[7]);
  }
}

// The largest of 16 bytes of logits; a NaN is passed by, or (NAN_TOO) is it. 16-bit ones are compared two at a time.
template <bool NAN_TOO> __device__ __forceinline__ __nv_bfloat162 max_pair(__nv_bfloat162 a, __nv_bfloat162 b) { return NAN_TOO ? __hmax2_nan(a, b) : __hmax2(a, b); }
template <bool NAN_TOO> __device__ __forceinline__ __half2 max_pair(__half2 a, __half2 b) { return NAN_TOO ? __hmax2_nan(a, b) : __hmax2(a, b); }
template <bool NAN_TOO> __device__ __forceinline__ float max_one(float a, float b) {
  if (!NAN_TOO) return fmaxf(a, b);
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T> struct PairOf;
template <> struct PairOf<__nv_bfloat16> { using Type = __nv_bfloat162; };
template <> struct PairOf<__half> { using Type = __half2; };
template <typename T, bool NAN_TOO>
__device__ __forceinline__ float largest(const uint4& r) {
  if constexpr (sizeof(T) == 4) {
    return max_one<NAN_TOO>(max_one<NAN_TOO>(__uint_as_float(r.x), __uint_as_float(r.y)), max_one<NAN_TOO>(__uint_as_float(r.z), __uint_as_float(r.w)));
  } else {
    using P = typename PairOf<T>::Type;
    const P m = max_pair<NAN_TOO>(max_pair<NAN_TOO>(*reinterpret_cast<const P*>(&r.x), *reinterpret_cast<const P*>(&r.y)),
                                  max_pair<NAN_TOO>(*reinterpret_cast<const P*>(&r.z), *reinterpret_cast<const P*>(&r.w)));
    float lo, hi;
    unpack2<T>(*reinterpret_cast<const uint32_t*>(&m), lo, hi);
    return max_one<NAN_TOO>(lo, hi);
  }
}

// N logits, `most` the largest of them, into a thread's sums.
template <bool ENTROPY, int N>
__device__ __forceinline__ void add_logits(Sums& x, const float* v, float most, float c) {
  if (most > x.m) rebase<ENTROPY>(x, most, c);          // rarely after the first few
  const float base = base_of(x.m);
  float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    if (N == 1) {
      const float d = v[0] - base, e = ex2(d * c);
      s[0] = e;
      if (ENTROPY) w[0] = e * fmaxf(d, kFar);
      break;
    }
    float d0, d1, e0, e1;
    add2(d0, d1, v[i], v[i + 1], -base, -base);
    mul2(e0, e1, d0, d1, c, c);
    e0 = ex2(e0);
    e1 = ex2(e1);
    add2(s[0], s[1], s[0], s[1], e0, e1);
    if (ENTROPY) {                                      // a NaN comes in through the exponential
      d0 = fmaxf(d0, kFar);
      d1 = fmaxf(d1, kFar);
      fma2(w[0], w[1], e0, e1, d0, d1, w[0], w[1]);
    }
  }
  x.s += s[0] + s[1];
  if (ENTROPY) x.w += w[0] + w[1];
}

// How many of the lanes' numbers come before this one in descending order (of equal ones the lower lane's).
__device__ __forceinline__ int place_among(uint32_t x, int lane) {
  int before = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t y = __shfl_sync(kAll, x, i);
    before += y > x || (y == x && i < lane);
  }
  return before;
}

// The likeliest of what a warp has seen: lane i holds the i-th key, in descending order.
struct Best {
  uint64_t key;
  // all lanes; keys of the lanes where `has`
  __device__ __forceinline__ void add(uint64_t k, bool has, int top, int lane) {
    if (!__any_sync(kAll, has)) return;
    const uint64_t least = __shfl_sync(kAll, key, top - 1);
    uint32_t todo = __ballot_sync(kAll, has && k > least);
    while (todo) {
      const int from = __ffs(todo) - 1;
      todo &= todo - 1;
      const uint64_t x = __shfl_sync(kAll, k, from), before = __shfl_up_sync(kAll, key, 1);
      const int at = __popc(__ballot_sync(kAll, key > x));
      key = lane < at ? key : lane == at ? x : before;
    }
  }
  // with another list in descending order: the 32 largest of both, in descending order
  __device__ __forceinline__ void merge(uint64_t other, int lane) {
    const uint64_t y = __shfl_sync(kAll, other, 31 - lane);
    uint64_t x = key > y ? key : y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const uint64_t z = __shfl_xor_sync(kAll, x, o);
      x = (lane & o) == 0 ? (x > z ? x : z) : (x < z ? x : z);
    }
    key = x;
  }
};

// The token that is given for a row and its logit, looked up ahead of time; -1: none, or a padded place.
template <typename T> struct Given {
  int64_t token;
  float logit;
  __device__ __forceinline__ Given(const LogProbsArgs& a, int64_t row, const T* x) {
    token = a.tokens ? a.tokens[row] : -1;
    if (token >= a.cols) token = -1;
    logit = token >= 0 ? to_float<T>(x[token]) : 0.0f;
  }
};

// N lists, list w < N held by warp w and in shared memory, into the first warp's; all warps of a CTA.
template <int N>
__device__ __forceinline__ void merge_lists(uint64_t (*lists)[32], Best& mine, int warp, int lane) {
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2) {
    __syncthreads();
    if (warp < n) {
      mine.merge(lists[warp + n][lane], lane);
      lists[warp][lane] = mine.key;
    }
  }
}

// Writes a row's results; one warp, the row's sums and its best keys in every lane.
template <typename T>
__device__ __forceinline__ void write_results(const LogProbsArgs& a, int64_t row, const Given<T>& given, const Sums& sums, const Best& best, int lane) {
  const float base = base_of(sums.m), log_sum = logf(sums.s);
  const bool none = sums.s == 0.0f;                     // not a token is left: else the largest one's exponential is 1
  auto log_prob = [&](float v) { return none ? -INFINITY : (v - base) * a.scale - log_sum; };
  if (lane == 0) {
    a.stats[row * 2] = isnan(sums.s) && sums.m != INFINITY ? sums.s : sums.m;       // maxima pass NaN by
    a.stats[row * 2 + 1] = log_sum;
    if (a.log_probs) a.log_probs[row] = given.token >= 0 ? log_prob(given.logit) : 0.0f;
    if (a.entropy) a.entropy[row] = none ? 0.0f : log_sum - a.scale * (sums.w / sums.s);
  }
  if (lane < a.top) {
    a.top_tokens[row * a.top + lane] = ~(uint32_t)best.key;
    a.top_log_probs[row * a.top + lane] = log_prob(logit_of((uint32_t)(best.key >> 32)));
  }
}

constexpr int kThreads = 256, kWarps = kThreads / 32;

// Warp = a row.
template <typename T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kThreads, TOP ? 4 : 6) log_probs_warp_kernel(LogProbsArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const Span<T> span(reinterpret_cast<const T*>(a.logits) + row * a.pitch, a.cols);
  constexpr int kPer = Span<T>::kPer, kAhead = 4;
  const Given<T> given(a, row, span.p);
  const float c = a.scale * kLog2e;
  Sums sums{-INFINITY, 0.0f, 0.0f};
  for (int i0 = lane; i0 < span.vectors; i0 += kAhead * 32) {
    uint4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * 32 < span.vectors) raw[u] = *span.at(i0 + u * 32);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * 32 < span.vectors) {
        float v[kPer];
        unpack<T>(raw[u], v);
        add_logits<ENTROPY, kPer>(sums, v, largest<T, false>(raw[u]), c);
      }
  }
  if (lane < span.loose()) {
    const float v = to_float<T>(span.p[span.loose_at(lane)]);
    add_logits<ENTROPY, 1>(sums, &v, v, c);
  }
  const uint32_t mine = rank_of(sums.m);
  sums = lanes_joined<ENTROPY, 32>(sums, c);
  Best best{0};
  if constexpr (TOP) {
    // the top-th largest of the lanes' largest logits: `top` logits reach it
    const float floor = logit_of(__shfl_sync(kAll, mine, __ffs(__ballot_sync(kAll, place_among(mine, lane) == a.top - 1)) - 1));
    for (int i0 = 0; i0 < span.n; i0 += 32) {
      const int i = i0 + lane;
      const float v = i < span.n ? to_float<T>(span.p[i]) : 0.0f;
      best.add(key_of(v, (uint32_t)i), i < span.n && !(v < floor), a.top, lane);
    }
  }
  write_results<T>(a, row, given, sums, best, lane);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// The address of the first CTA's copy of a variable in shared memory.
__device__ __forceinline__ uint32_t in_first(const void* p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}
__device__ __forceinline__ void store_remote(uint32_t at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void store_remote(uint32_t at, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(at), "l"(v) : "memory"); }

// CTA, or cluster of CTAS of them, = a row.
template <typename T, bool ENTROPY, bool TOP, int CTAS>
__global__ void __launch_bounds__(kThreads, TOP ? 4 : 6) log_probs_kernel(LogProbsArgs a) {
  constexpr int kPer = Span<T>::kPer;
  __shared__ Sums s_sums[kWarps], s_row[8];
  __shared__ uint64_t s_keys[TOP ? kWarps : 1][32], s_row_keys[TOP ? CTAS : 1][32];
  __shared__ __align__(16) uint32_t s_largest[kWarps][8];
  __shared__ float s_floor;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if constexpr (CTAS > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
  const int64_t row = blockIdx.x / CTAS;
  const int part = CTAS > 1 ? (int)cluster_rank() : 0;
  const Span<T> span(reinterpret_cast<const T*>(a.logits) + row * a.pitch, a.cols);
  const Given<T> given(a, row, span.p);
  // this CTA's vectors; the elements outside them are the first one's
  const int begin = (int)((int64_t)span.vectors * part / CTAS), end = (int)((int64_t)span.vectors * (part + 1) / CTAS);
  const float c = a.scale * kLog2e;
  Sums sums{-INFINITY, 0.0f, 0.0f};
  constexpr int kAhead = 4;
  for (int i0 = begin + tid; i0 < end; i0 += kAhead * kThreads) {
    uint4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * kThreads < end) raw[u] = *span.at(i0 + u * kThreads);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * kThreads < end) {
        float v[kPer];
        unpack<T>(raw[u], v);
        add_logits<ENTROPY, kPer>(sums, v, largest<T, false>(raw[u]), c);
      }
  }
  const bool loose = part == 0 && tid < span.loose();
  const float loose_logit = loose ? to_float<T>(span.p[span.loose_at(tid)]) : 0.0f;
  if (loose) add_logits<ENTROPY, 1>(sums, &loose_logit, loose_logit, c);
  const float mine = sums.m;
  sums = lanes_joined<ENTROPY, 32>(sums, c);
  if (lane == 0) s_sums[warp] = sums;
  if constexpr (TOP) {
    // the top-th largest of the eight largest of each warp's threads' largest logits: `top` logits of this CTA reach it
    const uint32_t r = rank_of(mine);
    const int before = place_among(r, lane);
    if (before < 8) s_largest[warp][before] = r;
  }
  __syncthreads();
  Best best{0};
  if constexpr (TOP) {
    static_assert(kWarps * 8 == 64, "two warps take one of them each");
    if (tid < 64) {
      const uint32_t r = s_largest[0][tid];
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < 64; i += 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(&s_largest[0][i]);
        before += (x.x > r || (x.x == r && i < tid)) + (x.y > r || (x.y == r && i + 1 < tid)) + (x.z > r || (x.z == r && i + 2 < tid)) + (x.w > r || (x.w == r && i + 3 < tid));
      }
      if (before == a.top - 1) s_floor = logit_of(r);
    }
    __syncthreads();
    float floor = s_floor;                              // from here on the larger of that and the warp's top-th best so far
    best.add(key_of(loose_logit, (uint32_t)span.loose_at(tid)), loose && !(loose_logit < floor), a.top, lane);
    for (int i0 = begin + tid; i0 - lane < end; i0 += kAhead * kThreads) {
      uint4 raw[kAhead];
      uint32_t hits = 0;                                // the vectors of which some lane's reaches it, a NaN too
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i0 + u * kThreads < end) raw[u] = *span.at(i0 + u * kThreads);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        hits |= __any_sync(kAll, i0 + u * kThreads < end && !(largest<T, true>(raw[u]) < floor)) ? 1u << u : 0u;
      // one copy of what follows: unrolled, it would not stay in the instruction cache (33 us instead of 22 for a step's 128 rows)
#pragma unroll 1
      for (; hits; hits &= hits - 1) {
        const int u = __ffs(hits) - 1, i = i0 + u * kThreads;
        uint4 r = raw[0];
#pragma unroll
        for (int k = 1; k < kAhead; ++k)
          if (u == k) r = raw[k];
        float v[kPer];
        uint32_t some = 0;                              // which of the lane's logits
        unpack<T>(r, v);
#pragma unroll
        for (int e = 0; e < kPer; ++e) some |= i < end && !(v[e] < floor) ? 1u << e : 0u;
#pragma unroll 1
        for (uint32_t any = __reduce_or_sync(kAll, some); any; any &= any - 1) {
          const int e = __ffs(any) - 1;
          float x = v[0];
#pragma unroll
          for (int k = 1; k < kPer; ++k)
            if (e == k) x = v[k];
          best.add(key_of(x, (uint32_t)(span.head + i * kPer + e)), some >> e & 1u, a.top, lane);
        }
        const uint64_t least = __shfl_sync(kAll, best.key, a.top - 1);
        if (least != 0) floor = fmaxf(floor, logit_of((uint32_t)(least >> 32)));       // of a NaN: stays
      }
    }
    s_keys[warp][lane] = best.key;
    merge_lists<kWarps>(s_keys, best, warp, lane);
  }
  if (warp == 0) {
    sums = lanes_joined<ENTROPY, kWarps>(s_sums[lane % kWarps], c);
  }
  if constexpr (CTAS > 1) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");       // the first CTA has begun: its shared memory is there
    if (warp == 0) {
      if (lane == 0) {
        store_remote(in_first(&s_row[part].m), sums.m);
        store_remote(in_first(&s_row[part].s), sums.s);
        store_remote(in_first(&s_row[part].w), sums.w);
      }
      if constexpr (TOP) store_remote(in_first(&s_row_keys[part][lane]), best.key);
    }
    cluster_sync();
    if (part != 0) return;
    if (warp == 0) sums = lanes_joined<ENTROPY, CTAS>(s_row[lane % CTAS], c);
    if constexpr (TOP) {
      best.key = s_row_keys[warp % CTAS][lane];
      merge_lists<CTAS>(s_row_keys, best, warp, lane);
    }
  }
  if (warp == 0) write_results<T>(a, row, given, sums, best, lane);
}

// Gradient: CTA = a row, or `parts` CTAs for long ones, a warp for short ones. The last rows come first: they are what the forward
// call has left in L2, and the gradients pass through it first to go.
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(kThreads, 4) log_probs_grad_kernel(LogProbsArgs a, int parts, int threads_per_row) {
  constexpr int kPer = Span<T>::kPer;
  const int rows_here = kThreads / threads_per_row, tid = threadIdx.x % threads_per_row;
  const int64_t turn = (int64_t)(blockIdx.x / parts) * rows_here + threadIdx.x / threads_per_row, row = a.rows - 1 - turn;
  const int part = blockIdx.x % parts;
  if (row < 0) return;
  const Span<T> span(reinterpret_cast<const T*>(a.logits) + row * a.pitch, a.cols);
  T* dx = reinterpret_cast<T*>(a.dlogits) + row * a.dlogits_pitch;
  const bool same = (((uintptr_t)dx ^ (uintptr_t)span.p) & 15) == 0;
  const float top = a.stats[row * 2], log_sum = a.stats[row * 2 + 1];
  const int64_t t64 = a.tokens ? a.tokens[row] : -1;
  const int t = t64 >= 0 && t64 < a.cols ? (int)t64 : -1;
  const float g = a.dlog_probs && t >= 0 ? a.dlog_probs[row] * a.scale : 0.0f;
  const float h = ENTROPY ? a.dentropy[row] * a.scale : 0.0f, entropy = ENTROPY ? a.entropy[row] : 0.0f;
  const bool none = top == -INFINITY;
  // with l = log p: p (-g - h (l + entropy)), and g more at the token. The token's is g (1 - p), not g - g p of rounded parts
  auto gradient = [&](float v, int i) {
    const float l = (v - top) * a.scale - log_sum, p = ex2(l * kLog2e);
    float r = i == t ? g * (1.0f - p) : -g * p;
    if (ENTROPY) r -= p == 0.0f ? 0.0f : p * (h * (l + entropy));
    return none ? 0.0f : r;
  };
  const int begin = (int)((int64_t)span.vectors * part / parts), end = (int)((int64_t)span.vectors * (part + 1) / parts);
  constexpr int kAhead = 4;
  for (int i0 = begin + tid; i0 < end; i0 += kAhead * threads_per_row) {
    uint4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * threads_per_row < end) raw[u] = *span.at(i0 + u * threads_per_row);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u * threads_per_row < end) {
        const int first = span.head + (i0 + u * threads_per_row) * kPer;
        float v[kPer];
        unpack<T>(raw[u], v);
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = gradient(v[e], first + e);
        if (same) {
          uint4 w;
          if constexpr (sizeof(T) == 4) w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
          else w = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4 % kPer], v[5 % kPer]), pack2<T>(v[6 % kPer], v[7 % kPer]));
          __stcs(reinterpret_cast<uint4*>(dx + first), w);
        } else {
#pragma unroll
          for (int e = 0; e < kPer; ++e) dx[first + e] = from_float<T>(v[e]);
        }
      }
  }
  if (part == 0 && tid < span.loose()) {
    const int i = span.loose_at(tid);
    dx[i] = from_float<T>(gradient(to_float<T>(span.p[i]), i));
  }
}

template <typename T, bool ENTROPY, bool TOP, int CTAS>
cudaError_t launch_rows(const LogProbsArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.rows * CTAS));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = CTAS;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cfg.attrs = &cluster;
  cfg.numAttrs = CTAS > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, log_probs_kernel<T, ENTROPY, TOP, CTAS>, a);
}

// Whether a warp takes a row: short rows, and longer ones where there are at least as many, so that no warp is left with its row when the
// others have ended. A CTA's rows begin and end with nothing to read. Measured, bf16, us with a CTA / a warp to a row, forward:
//   rows                 100        1000       4000        8000        16000        32000
//   of 1000            2.6 / 2.9                                                 (200000: 507 / 94)
//   of 2000            2.6 / 3.6  4.1 / 3.5  9.4 / 5.6   17 / 8      32 / 13
//   of 4000            2.8 / 5.2  4.7 / 5.3  11 / 9      20 / 13
//   of 8000                                  14 / 15     32 / 29     61 / 47      117 / 85
//   of 16000                                             50 / 54     94 / 87      184 / 161
//   of 32000                                             88 / 116    165 / 182
// The gradient, and fp32, turn at about the same sizes. us with a CTA / a warp to a row:
//                      bf16 gradient   fp32 forward   fp32 gradient
//   1000 of 2000         4.6 / 3.3       4.3 / 4.2      4.9 / 4.4
//   1000 of 4000         5.5 / 5.1       4.8 / 6.5      5.6 / 6.4
//   4000 of 4000          17 / 11         11 / 10        24 / 22
//   4000 of 8000          28 / 25         25 / 24        38 / 46
//   8000 of 8000          53 / 45         45 / 50        82 / 88
//   16000 of 16000       178 / 175       148 / 163      302 / 352
// The rule gives away up to 1.3 us of 4.6 at 1000 rows of 2000, and up to a sixth at the longest rows of fp32.
bool warp_takes_row(const LogProbsArgs& a) { return a.cols <= 1024 || (a.cols <= 16384 && a.rows >= a.cols); }
template <typename T, bool ENTROPY, bool TOP>
cudaError_t launch_forward_as(const LogProbsArgs& a, cudaStream_t st) {
  if (TOP ? a.cols <= 1024 : warp_takes_row(a)) {       // a warp's search for the likeliest is for short rows
    log_probs_warp_kernel<T, ENTROPY, TOP><<<(unsigned)((a.rows + kWarps - 1) / kWarps), kThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  // as many CTAs to a row as leave two thousand logits to each and fill the device's 148 multiprocessors twice over
  int ctas = 1;
  while (ctas < 8 && a.rows * ctas < 296 && a.cols >= ctas * 4096) ctas *= 2;
  return ctas == 1 ? launch_rows<T, ENTROPY, TOP, 1>(a, st) : ctas == 2 ? launch_rows<T, ENTROPY, TOP, 2>(a, st)
       : ctas == 4 ? launch_rows<T, ENTROPY, TOP, 4>(a, st) : launch_rows<T, ENTROPY, TOP, 8>(a, st);
}
template <typename T>
cudaError_t launch_forward(const LogProbsArgs& a, cudaStream_t st) {
  if (a.top > 0) return a.entropy ? launch_forward_as<T, true, true>(a, st) : launch_forward_as<T, false, true>(a, st);
  return a.entropy ? launch_forward_as<T, true, false>(a, st) : launch_forward_as<T, false, false>(a, st);
}
template <typename T>
cudaError_t launch_backward(const LogProbsArgs& a, cudaStream_t st) {
  // several CTAs for a long row where rows are few
  const int threads = warp_takes_row(a) ? 32 : kThreads;
  const int64_t groups = (a.rows * threads + kThreads - 1) / kThreads;
  int parts = 1;
  while (threads == kThreads && groups * parts < 1184 && a.cols >= (int64_t)parts * 8192 && parts < 64) parts *= 2;
  if (a.dentropy) log_probs_grad_kernel<T, true><<<(unsigned)(groups * parts), kThreads, 0, st>>>(a, parts, threads);
  else log_probs_grad_kernel<T, false><<<(unsigned)(groups * parts), kThreads, 0, st>>>(a, parts, threads);
  return cudaGetLastError();
}

// ---- argument checks ------------------------------------------------------------------------
constexpr int64_t kMaxPitch = (int64_t)1 << 38;
bool sizes_ok(int64_t rows, int64_t cols, int64_t pitch, int32_t dtype, float scale) {
  return rows >= 0 && rows < (int64_t)1 << 31 && cols >= 1 && cols < (int64_t)1 << 31 && pitch >= cols && pitch < kMaxPitch &&
         dtype >= SWARM_F32 && dtype <= SWARM_F16 && scale > 0.0f && std::isfinite(scale);
}
bool at_ok(const void* p, size_t size, bool needed) { return (p || !needed) && (uintptr_t)p % size == 0; }

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" {

int swarm_token_log_probs(const void* logits_dev, const int64_t* tokens_dev, float* log_probs_dev, float* stats_dev,
                          float* entropy_dev, float* top_log_probs_dev, int64_t* top_tokens_dev, int64_t rows,
                          int64_t cols, int64_t pitch, int32_t dtype, float scale, int32_t top, void* cuda_stream) {
  if (!sizes_ok(rows, cols, pitch, dtype, scale) || top < 0 || top > SWARM_MAX_TOP || top > cols ||
      (tokens_dev != nullptr) != (log_probs_dev != nullptr))
    return SWARM_EINVAL;
  if (rows == 0) return SWARM_OK;
  if (!at_ok(logits_dev, element_size(dtype), true) || !at_ok(tokens_dev, 8, false) || !at_ok(log_probs_dev, 4, false) ||
      !at_ok(stats_dev, 4, true) || !at_ok(entropy_dev, 4, false) || !at_ok(top_log_probs_dev, 4, top > 0) || !at_ok(top_tokens_dev, 8, top > 0))
    return SWARM_EINVAL;
  LogProbsArgs a{};
  a.logits = logits_dev; a.tokens = tokens_dev; a.log_probs = log_probs_dev; a.stats = stats_dev; a.entropy = entropy_dev;
  a.top_log_probs = top_log_probs_dev; a.top_tokens = top_tokens_dev;
  a.rows = rows; a.cols = cols; a.pitch = pitch; a.scale = scale; a.top = top;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == SWARM_F32) return operator_result(launch_forward<float>(a, st));
  if (dtype == SWARM_BF16) return operator_result(launch_forward<__nv_bfloat16>(a, st));
  return operator_result(launch_forward<__half>(a, st));
}

int swarm_token_log_probs_backward(const float* dlog_probs_dev, const float* dentropy_dev, const void* logits_dev,
                                   const int64_t* tokens_dev, const float* stats_dev, const float* entropy_dev,
                                   void* dlogits_dev, int64_t rows, int64_t cols, int64_t pitch, int64_t dlogits_pitch,
                                   int32_t dtype, float scale, void* cuda_stream) {
  if (!sizes_ok(rows, cols, pitch, dtype, scale) || dlogits_pitch < cols || dlogits_pitch >= kMaxPitch) return SWARM_EINVAL;
  if (rows == 0) return SWARM_OK;
  if (!at_ok(logits_dev, element_size(dtype), true) || !at_ok(dlogits_dev, element_size(dtype), true) || !at_ok(stats_dev, 4, true) ||
      !at_ok(tokens_dev, 8, dlog_probs_dev != nullptr) || !at_ok(dlog_probs_dev, 4, false) || !at_ok(dentropy_dev, 4, false) ||
      !at_ok(entropy_dev, 4, dentropy_dev != nullptr) || (dlogits_dev == logits_dev && dlogits_pitch != pitch))
    return SWARM_EINVAL;
  LogProbsArgs a{};
  a.logits = logits_dev; a.tokens = tokens_dev; a.stats = const_cast<float*>(stats_dev); a.entropy = const_cast<float*>(entropy_dev);
  a.dlog_probs = dlog_probs_dev; a.dentropy = dentropy_dev; a.dlogits = dlogits_dev;
  a.rows = rows; a.cols = cols; a.pitch = pitch; a.dlogits_pitch = dlogits_pitch; a.scale = scale;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == SWARM_F32) return operator_result(launch_backward<float>(a, st));
  if (dtype == SWARM_BF16) return operator_result(launch_backward<__nv_bfloat16>(a, st));
  return operator_result(launch_backward<__half>(a, st));
}

}  // extern "C"
