// Attention of a sentence's newest tokens over its paged cache.
#include "swarm_attention_tile.cuh"
#include "swarm_paged.h"

namespace swarm {
namespace {

// Warp = one row of one head, lane = four of its values; one pass over the visible positions with the running maximum and sum.
template <typename T>
__global__ void __launch_bounds__(128) paged_attention_kernel(PagedArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (int64_t)a.batch * a.tokens * a.heads) return;
  const int h = (int)(row % a.heads), t = (int)(row / a.heads % a.tokens), b = (int)(row / a.heads / a.tokens), hk = h / a.group;
  const int length = length_in(a, b), n = rows_in(a, b, length), at = length - n + t, d0 = lane * 4;
  const bool live = t < n, has = d0 < a.head_dim;
  float q[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.0f;
  const float c = a.scale * kLog2e;
  if (live) {
    if (has)
      for (int i = 0; i < 4; ++i) q[i] = to_float<T>((reinterpret_cast<const T*>(a.q) + offset_of(a.qs, b, t, h))[d0 + i]);
    const int low = a.window > 0 && at >= a.window ? at - a.window + 1 : 0;
    for (int j = 0; j <= at; ++j) {
      if (j < low && j >= a.sinks) { j = low - 1; continue; }
      const int page = page_of(a, b, j / a.page_size);
      if (page < 0) { if (lane == 0) atomicOr(a.status, kStatusPage); continue; }
      float s = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
      if (has) {
        const T* k = reinterpret_cast<const T*>(a.k_pages) + offset_of(a.kps, page, j % a.page_size, hk) + d0;
        const T* pv = reinterpret_cast<const T*>(a.v_pages) + offset_of(a.vps, page, j % a.page_size, hk) + d0;
        for (int i = 0; i < 4; ++i) { s = fmaf(q[i], to_float<T>(k[i]), s); v[i] = to_float<T>(pv[i]); }
      }
      s = warp_sum(s);
      const float m_new = fmaxf(m, s), base = m_new == -INFINITY ? 0.0f : m_new, f = ex2((m - base) * c), p = ex2((s - base) * c);
      m = m_new;
      l = fmaf(l, f, p);
      for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], f, p * v[i]);
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : l;             // l = 0: nothing was seen; NaN stays
  if (has)
    for (int i = 0; i < 4; ++i) (reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h))[d0 + i] = from_float<T>(l == 0.0f ? 0.0f : o[i] * inv);
  if (a.lse && lane == 0) a.lse[((int64_t)b * a.heads + h) * a.tokens + t] = l == 0.0f ? -INFINITY : m * a.scale + logf(l);
}

}  // namespace

size_t paged_attention_workspace(const PagedArgs&) { return 0; }

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, void*, cudaStream_t st) {
  const int64_t rows = (int64_t)a.batch * a.tokens * a.heads;
  if (dtype == SWARM_BF16) paged_attention_kernel<__nv_bfloat16><<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(a);
  else paged_attention_kernel<__half><<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace swarm
