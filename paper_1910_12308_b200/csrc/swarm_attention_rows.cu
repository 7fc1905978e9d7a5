// Cross attention of few query rows (a decoding step): every state is read once, HBM is the bound.
//
// CTA = up to 16 rows (query tokens x the query heads of a key head) and a part of the states, four warps on 16 states at
// a time each, the next ones fetched before these are used. The products run as m16n8k16 on operands that go from global memory straight into registers:
//   scores  the order of the contraction over the head's values is free, so a lane takes 16 consecutive bytes of a
//           state (values 32 p + 8 c .. + 7, c = lane % 4) as the operands of two products, and the same of a row of q
//   sums    a lane takes 16 bytes (values 8 n .. + 7, n = lane / 4) of the states 2 c, 2 c + 1, 2 c + 8, 2 c + 9 and
//           pairs the states byte-wise; product j then gives values 8 n + j
// so neither needs shared memory or a transposition. Measured: 128 sentences x 16 heads of 64 over 1024 states 103 us, 5.2
// TB/s; 8 sentences x 8 key heads of 128 with four query heads each over 16384 states 99 us, 5.4 TB/s, about 5 of them the
// joining kernel; the tensor pipe is busy a seventh of the time. The four warps meet in shared memory; where there are fewer (key
// head, sentence) pairs than the device has room for, the states are split over CTAs whose parts (maximum, sum, o) a
// second kernel joins in order.
#include "swarm_attention_tile.cuh"

namespace swarm {
namespace {

constexpr int kRows = 16, kRowsWarps = 4;

constexpr int kRowsStep = 16;                           // states that a warp takes at a time

struct RowsPlan : SplitPlan {
  int32_t row_groups;                 // groups of 16 rows
};

template <typename T, int DB>
__global__ void __launch_bounds__(kRowsWarps * 32)
attention_rows_kernel(AttentionArgs a, RowsPlan plan) {
  constexpr int kDim = DB * 64;
  __shared__ float s_ml[kRowsWarps][kRows][2];
  extern __shared__ float s_o[];                        // [warps][rows of this group][head_dim]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r8 = lane >> 2, c4 = lane & 3;
  const int split = blockIdx.x % plan.splits, group = blockIdx.x / plan.splits % plan.row_groups;
  const int bh = blockIdx.x / plan.splits / plan.row_groups, hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int row0 = group * kRows, rows = min(kRows, plan.rows - row0);
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  // this CTA's part of the states: equal runs of whole steps of all warps
  constexpr int kWhole = kRowsStep * kRowsWarps;
  const int steps = (nk + kWhole - 1) / kWhole;
  const int begin = (int)((int64_t)steps * split / plan.splits) * kWhole;
  const int end = min(nk, (int)((int64_t)steps * (split + 1) / plan.splits) * kWhole);
  const int chunks = a.head_dim / 8;                    // 16-byte pieces of a head

  uint32_t q[DB * 2][2][4];                             // [32 values][row r8, row r8 + 8][pair]
#pragma unroll
  for (int p = 0; p < DB * 2; ++p)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = row0 + r8 + 8 * u;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r < plan.rows && p * 4 + c4 < chunks)
        w = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + offset_of(a.qs, b, r / a.group, hk * a.group + r % a.group) + p * 32 + c4 * 8);
      q[p][u][0] = w.x; q[p][u][1] = w.y; q[p][u][2] = w.z; q[p][u][3] = w.w;
    }
  const T* kbase = reinterpret_cast<const T*>(a.k) + b * a.ks.batch + hk * a.ks.head;
  const T* vbase = reinterpret_cast<const T*>(a.v) + b * a.vs.batch + hk * a.vs.head;
  const float c = a.scale * kLog2e;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, o[DB * 8][4];
#pragma unroll
  for (int i = 0; i < DB * 8; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) o[i][u] = 0.0f;

  constexpr int kStep = kRowsStep, kStride = kStep * kRowsWarps;
  struct States { uint4 k[kStep / 8][DB * 2], v[kStep / 16][4][DB]; };
  auto fetch = [&](States& x, int j0) {
#pragma unroll
    for (int g = 0; g < kStep / 8; ++g) {               // eight states at a time: state r8 of the group
      const int j = j0 + g * 8 + r8;
#pragma unroll
      for (int p = 0; p < DB * 2; ++p)
        x.k[g][p] = j < nk && p * 4 + c4 < chunks ? *reinterpret_cast<const uint4*>(kbase + (int64_t)j * a.ks.token + p * 32 + c4 * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int g = 0; g < kStep / 16; ++g)
#pragma unroll
      for (int u = 0; u < 4; ++u) {                     // states 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of sixteen
        const int j = j0 + g * 16 + c4 * 2 + (u & 1) + (u >> 1) * 8;
#pragma unroll
        for (int d = 0; d < DB; ++d)
          x.v[g][u][d] = j < nk && d * 8 + r8 < chunks ? *reinterpret_cast<const uint4*>(vbase + (int64_t)j * a.vs.token + d * 64 + r8 * 8) : make_uint4(0, 0, 0, 0);
      }
  };
  auto compute = [&](const States& x, int j0) {
    float s[kStep / 8][4];
#pragma unroll
    for (int g = 0; g < kStep / 8; ++g) {
#pragma unroll
      for (int u = 0; u < 4; ++u) s[g][u] = 0.0f;
#pragma unroll
      for (int p = 0; p < DB * 2; ++p) {
        const uint32_t a0[4] = {q[p][0][0], q[p][1][0], q[p][0][1], q[p][1][1]};
        const uint32_t a1[4] = {q[p][0][2], q[p][1][2], q[p][0][3], q[p][1][3]};
        mma16816<T>(s[g], a0, x.k[g][p].x, x.k[g][p].y);
        mma16816<T>(s[g], a1, x.k[g][p].z, x.k[g][p].w);
      }
    }
    if (j0 + kStep > nk) {
#pragma unroll
      for (int g = 0; g < kStep / 8; ++g)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (j0 + g * 8 + c4 * 2 + (u & 1) >= nk) s[g][u] = -INFINITY;
    }
    float top[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = fmaxf(s[0][2 * u], s[0][2 * u + 1]);
#pragma unroll
      for (int g = 1; g < kStep / 8; ++g) t = fmaxf(t, fmaxf(s[g][2 * u], s[g][2 * u + 1]));
      t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 1));
      top[u] = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 2));
    }
    if (__any_sync(0xFFFFFFFFu, (top[0] - m[0]) * c > 8.0f || (top[1] - m[1]) * c > 8.0f)) {
      // the maximum moved by more than 2^8 in some row (or the first step): rescale; smaller moves keep the reference
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float m_new = fmaxf(m[u], top[u]), f = m_new == m[u] ? 1.0f : ex2((m[u] - m_new) * c);
        m[u] = m_new;
        l[u] *= f;
#pragma unroll
        for (int i = 0; i < DB * 8; ++i) { o[i][2 * u] *= f; o[i][2 * u + 1] *= f; }
      }
    }
    const float mc[2] = {m[0] == -INFINITY ? 0.0f : m[0] * c - kRunningShift<T>, m[1] == -INFINITY ? 0.0f : m[1] * c - kRunningShift<T>};
#pragma unroll
    for (int g = 0; g < kStep / 8; ++g)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        s[g][u] = ex2(fmaf(s[g][u], c, -mc[u >> 1]));
        l[u >> 1] += s[g][u];
      }
#pragma unroll
    for (int g = 0; g < kStep / 16; ++g) {
      const uint32_t p[4] = {pack2<T>(s[2 * g][0], s[2 * g][1]), pack2<T>(s[2 * g][2], s[2 * g][3]),
                             pack2<T>(s[2 * g + 1][0], s[2 * g + 1][1]), pack2<T>(s[2 * g + 1][2], s[2 * g + 1][3])};
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const uint32_t v[4][4] = {{x.v[g][0][d].x, x.v[g][0][d].y, x.v[g][0][d].z, x.v[g][0][d].w},
                                  {x.v[g][1][d].x, x.v[g][1][d].y, x.v[g][1][d].z, x.v[g][1][d].w},
                                  {x.v[g][2][d].x, x.v[g][2][d].y, x.v[g][2][d].z, x.v[g][2][d].w},
                                  {x.v[g][3][d].x, x.v[g][3][d].y, x.v[g][3][d].z, x.v[g][3][d].w}};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mma16816<T>(o[d * 8 + 2 * i], p, __byte_perm(v[0][i], v[1][i], 0x5410), __byte_perm(v[2][i], v[3][i], 0x5410));
          mma16816<T>(o[d * 8 + 2 * i + 1], p, __byte_perm(v[0][i], v[1][i], 0x7632), __byte_perm(v[2][i], v[3][i], 0x7632));
        }
      }
    }
  };
  int j0 = begin + warp * kStep;
  if (j0 < end) {
    States even, odd;
    fetch(even, j0);
    while (true) {
      if (j0 + kStride < end) fetch(odd, j0 + kStride);
      compute(even, j0);
      j0 += kStride;
      if (j0 >= end) break;
      if (j0 + kStride < end) fetch(even, j0 + kStride);
      compute(odd, j0);
      j0 += kStride;
      if (j0 >= end) break;
    }
  }

  // the warps meet: product j of block d holds values d * 64 + 8 n + j, n = 2 c4, 2 c4 + 1
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 1);
    l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 2);
    const int r = r8 + 8 * u;
    if (r < rows) {
      if (c4 == 0) { s_ml[warp][r][0] = m[u]; s_ml[warp][r][1] = l[u]; }
      float* dst = s_o + (warp * rows + r) * a.head_dim;
#pragma unroll
      for (int i = 0; i < DB * 8; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = (i >> 3) * 64 + 8 * (2 * c4 + e) + (i & 7);
          if (col < a.head_dim) dst[col] = o[i][2 * u + e];
        }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * chunks; i += kRowsWarps * 32) {
    const int r = i / chunks, ch = i % chunks, row = row0 + r, t = row / a.group, h = hk * a.group + row % a.group;
    float top = -INFINITY, sum = 0.0f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) top = fmaxf(top, s_ml[w][r][0]);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < kRowsWarps; ++w) {
      const float f = ex2((s_ml[w][r][0] - base) * c);
      sum = fmaf(s_ml[w][r][1], f, sum);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(s_o[(w * rows + r) * a.head_dim + ch * 8 + e], f, v[e]);
    }
    if (plan.splits == 1) {
      const float inv = t < nq && sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = inv != 0.0f ? v[e] * inv : 0.0f;
      store8<T>(reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h) + ch * 8, v);
      if (a.lse && ch == 0)
        a.lse[((int64_t)b * a.heads + h) * a.queries + t] = t < nq && nk > 0 ? top * a.scale + (logf(sum) - kRunningShift<T> * 0.69314718f) : -INFINITY;
    } else {
      const int64_t at = ((int64_t)bh * plan.rows + row) * plan.splits + split;
      if (ch == 0) { plan.part_ml[at * 2] = top; plan.part_ml[at * 2 + 1] = sum; }
      store8<float>(plan.part_o + at * a.head_dim + ch * 8, v);
    }
  }
}

// Joins the parts of a row: warp = one row, lane = four values of it, the parts in order.
template <typename T>
__global__ void __launch_bounds__(128) attention_join_kernel(AttentionArgs a, SplitPlan plan) {
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (i >= (int64_t)a.batch * a.kv_heads * plan.rows) return;
  const int row = (int)(i % plan.rows), bh = (int)(i / plan.rows), hk = bh % a.kv_heads, b = bh / a.kv_heads;
  const int t = row / a.group, h = hk * a.group + row % a.group;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const float c = a.scale * kLog2e;
  // lane s weighs part s; the parts' values are then added in order
  const float* part = plan.part_o + i * plan.splits * a.head_dim + lane * 4;
  float2 ml = make_float2(-INFINITY, 0.0f);
  if (lane < plan.splits) ml = reinterpret_cast<const float2*>(plan.part_ml)[i * plan.splits + lane];
  float top = ml.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  const float f = ex2((ml.x - (top == -INFINITY ? 0.0f : top)) * c), sum = warp_sum(ml.y * f);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < plan.splits; ++s) {
    const float fs = __shfl_sync(0xFFFFFFFFu, f, s);
    if (lane * 4 < a.head_dim) {
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)s * a.head_dim);
      v[0] = fmaf(x.x, fs, v[0]); v[1] = fmaf(x.y, fs, v[1]); v[2] = fmaf(x.z, fs, v[2]); v[3] = fmaf(x.w, fs, v[3]);
    }
  }
  const bool live = t < nq && nk > 0;
  const float inv = live && sum != 0.0f ? 1.0f / sum : 0.0f;
  if (lane * 4 < a.head_dim) {
    T* out = reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h) + lane * 4;
    uint2 w = make_uint2(0, 0);
    if (inv != 0.0f) w = make_uint2(pack2<T>(v[0] * inv, v[1] * inv), pack2<T>(v[2] * inv, v[3] * inv));
    *reinterpret_cast<uint2*>(out) = w;
  }
  if (a.lse && lane == 0)
    a.lse[((int64_t)b * a.heads + h) * a.queries + t] = live ? top * a.scale + (logf(sum) - kRunningShift<T> * 0.69314718f) : -INFINITY;
}


// The number of parts of the states that this model of a multiprocessor's time likes best, in states of one CTA: its share
// of the CTAs, each with its states and a cost of its own (its start, the meeting of its warps, its share of the join:
// measured, about 64 states and 24 more for each row), divided by the share of the bandwidth that its resident CTAs
// draw (up to three for heads of up to 64 values, two for longer ones); and the join's launch, about 4 us.
// Measured (both sides): 16 x 16 heads of 64 over 2048 states 35 us whole and 40 us in five parts; 8 x 8 grouped heads of
// 128 over 16384 states 101 us in nine parts and 115 us in seven, which leave half a wave empty.
RowsPlan make_plan(const AttentionArgs& a) {
  RowsPlan p{};
  p.rows = a.queries * a.group;
  p.row_groups = (p.rows + kRows - 1) / kRows;
  p.splits = 1;
  const int64_t ctas = (int64_t)a.batch * a.kv_heads * p.row_groups, sms = 148;
  const double own = 64.0 + 24.0 * (p.rows < kRows ? p.rows : kRows), join = a.head_dim <= 64 ? 480.0 : 320.0;
  double best = 0.0;
  for (int s = 1; s <= kMaxSplits && (int64_t)(s - 1) * 128 < a.keys; ++s) {
    const int64_t each = (ctas * s + sms - 1) / sms;
    const double drawn = a.head_dim <= 64 ? (each == 1 ? 0.55 : each == 2 ? 0.85 : 1.0) : each == 1 ? 0.6 : 1.0;
    const double time = (double)each * ((double)a.keys / s + own) / drawn + (s > 1 ? join : 0.0);
    if (s == 1 || time < best * 0.97) { best = time; p.splits = s; }
  }
  return p;
}

template <typename T, int DB>
cudaError_t launch_rows(const AttentionArgs& a, const RowsPlan& p, cudaStream_t st) {
  const int64_t ctas = (int64_t)a.batch * a.kv_heads * p.row_groups * p.splits;
  const int rows = p.rows < kRows ? p.rows : kRows;
  attention_rows_kernel<T, DB><<<(unsigned)ctas, kRowsWarps * 32, kRowsWarps * rows * a.head_dim * sizeof(float), st>>>(a, p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_join(const AttentionArgs& a, const SplitPlan& p, int dtype, cudaStream_t st) {
  const unsigned grid = (unsigned)(((int64_t)a.batch * a.kv_heads * p.rows + 3) / 4);
  if (dtype == SWARM_BF16) attention_join_kernel<__nv_bfloat16><<<grid, 128, 0, st>>>(a, p);
  else attention_join_kernel<__half><<<grid, 128, 0, st>>>(a, p);
  return cudaGetLastError();
}

size_t attention_rows_workspace(const AttentionArgs& a) { return split_bytes(a, make_plan(a)); }

cudaError_t launch_attention_rows(const AttentionArgs& a, int dtype, void* workspace, cudaStream_t st) {
  RowsPlan p = make_plan(a);
  if (p.splits > 1) place_parts(a, &p, workspace);
  cudaError_t e;
  if (dtype == SWARM_BF16) e = a.head_dim <= 64 ? launch_rows<__nv_bfloat16, 1>(a, p, st) : launch_rows<__nv_bfloat16, 2>(a, p, st);
  else e = a.head_dim <= 64 ? launch_rows<__half, 1>(a, p, st) : launch_rows<__half, 2>(a, p, st);
  if (e == cudaSuccess && p.splits > 1) e = launch_attention_join(a, p, dtype, st);
  return e;
}

}  // namespace swarm
