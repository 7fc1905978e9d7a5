// The paged cache of keys and values: argument checks, entry points, and the kernel that appends to it.
#include <cmath>

#include "swarm_paged.h"

namespace swarm {
namespace {

// Keys and values of new tokens into their pages, keys and queries rotated on the way: thread = one pair of a head of a token.
template <typename T>
__global__ void __launch_bounds__(256) cache_append_kernel(PagedArgs a, int heads) {
  const int half = a.rotated / 2, pairs = a.head_dim / 2, all = heads + 2 * a.kv_heads;
  const int64_t count = (int64_t)a.batch * a.tokens * all * pairs;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
    const int u = (int)(i % pairs), vh = (int)(i / pairs % all);
    const int64_t token = i / pairs / all;
    const int t = (int)(token % a.tokens), b = (int)(token / a.tokens);
    const int length = length_in(a, b), n = rows_in(a, b, length), at = length - n + t;
    const bool live = t < n, is_q = vh < heads, is_v = vh >= heads + a.kv_heads;
    const int h = is_q ? vh : is_v ? vh - heads - a.kv_heads : vh - heads;
    // pair u: of the rotated values, or two neighbours of the others
    int first = 2 * u, second = 2 * u + 1;
    if (u < half && !a.interleaved) { first = u; second = u + half; }
    const T* src = reinterpret_cast<const T*>(is_q ? a.q : is_v ? a.v : a.k) + offset_of(is_q ? a.qs : is_v ? a.vs : a.ks, b, t, h);
    T* dst;
    if (is_q) {
      dst = reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h);
    } else {
      if (!live) continue;
      const int page = page_of(a, b, at / a.page_size);
      if (page < 0) { atomicOr(a.status, kStatusPage); continue; }
      dst = reinterpret_cast<T*>(is_v ? a.v_pages : a.k_pages) + offset_of(is_v ? a.vps : a.kps, page, at % a.page_size, h);
    }
    float x = live ? to_float<T>(src[first]) : 0.0f, y = live ? to_float<T>(src[second]) : 0.0f;
    if (live && !is_v && u < half) {
      const double angle = (double)at * (double)a.frequencies[u];
      double s, c;
      sincos(angle, &s, &c);
      const float fs = (float)s, fc = (float)c, x0 = x;
      x = fmaf(x0, fc, -(y * fs));
      y = fmaf(y, fc, x0 * fs);
    }
    dst[first] = from_float<T>(x);
    dst[second] = from_float<T>(y);
  }
}

template <typename T>
cudaError_t launch_append(const PagedArgs& a, cudaStream_t st) {
  const int heads = a.out ? a.heads : 0;
  const int64_t count = (int64_t)a.batch * a.tokens * (heads + 2 * a.kv_heads) * (a.head_dim / 2);
  cache_append_kernel<T><<<(unsigned)((count + 255) / 256 < 65535 ? (count + 255) / 256 : 65535), 256, 0, st>>>(a, heads);
  return cudaGetLastError();
}

// ---- argument checks ------------------------------------------------------------------------
constexpr int64_t kMaxStride = (int64_t)1 << 38;
bool one_stride_ok(int64_t s, int64_t extent, bool repeats) {
  return extent <= 1 || (s >= 0 && s < kMaxStride && s % 8 == 0 && (repeats || s != 0));
}
bool strided_ok(const void* p, const swarm_strides& s, int64_t batch, int64_t tokens, int heads, bool output) {
  return p && ((uintptr_t)p & 15) == 0 && one_stride_ok(s.batch, batch, !output) && one_stride_ok(s.token, tokens, false) &&
         one_stride_ok(s.head, heads, !output);
}
bool words_ok(const void* p, bool needed) { return ((uintptr_t)p & 3) == 0 && (p || !needed); }
bool cache_ok(const swarm_paged* d, const void* k_pages, const void* v_pages) {
  return d->pages == 0 || (strided_ok(k_pages, d->k_pages, d->pages, d->page_size, d->kv_heads, true) &&
                           strided_ok(v_pages, d->v_pages, d->pages, d->page_size, d->kv_heads, true));
}
bool desc_ok(const swarm_paged* d) {
  return d && d->batch >= 0 && d->batch <= 65535 && d->kv_heads >= 1 && d->kv_heads <= 65535 && d->tokens >= 0 && d->tokens <= 1 << 30 &&
         d->head_dim >= 8 && d->head_dim <= kMaxDim && d->head_dim % 8 == 0 && (d->dtype == SWARM_BF16 || d->dtype == SWARM_F16) &&
         d->pages >= 0 && d->page_size >= 1 && d->table_columns >= 0 && d->table_pitch >= d->table_columns &&
         d->table_pitch < kMaxStride && words_ok(d->table_dev, d->batch > 0 && d->table_columns > 0) &&
         words_ok(d->lengths_dev, d->batch > 0) && words_ok(d->counts_dev, false);
}
bool heads_ok(const swarm_paged* d) { return d->heads >= 1 && d->heads <= 65535 && d->heads % d->kv_heads == 0; }
bool attention_ok(const swarm_paged* d) {
  return desc_ok(d) && heads_ok(d) && d->tokens <= SWARM_PAGED_MAX_TOKENS &&
         (int64_t)d->batch * d->heads * SWARM_PAGED_MAX_TOKENS < (int64_t)1 << 31 && d->window >= 0 && d->sinks >= 0 && d->scale > 0.0f && std::isfinite(d->scale);
}

void fill(PagedArgs& a, const swarm_paged* d) {
  a.table = d->table_dev; a.lengths = d->lengths_dev; a.counts = d->counts_dev; a.table_pitch = d->table_pitch;
  a.kps = d->k_pages; a.vps = d->v_pages; a.qs = d->q; a.os = d->out; a.ks = d->k; a.vs = d->v;
  a.batch = d->batch; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads;
  a.tokens = d->tokens; a.head_dim = d->head_dim; a.pages = d->pages; a.page_size = d->page_size; a.table_columns = d->table_columns;
  a.rotated = d->rotated; a.interleaved = d->interleaved; a.window = d->window; a.sinks = d->window > 0 ? d->sinks : 0;
  a.scale = d->scale;
}

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" {

int swarm_cache_append(const swarm_paged* desc_host, const void* k_dev, const void* v_dev, void* k_pages_dev,
                       void* v_pages_dev, const void* q_dev, void* out_dev, const float* frequencies_dev, void* cuda_stream) {
  if (!desc_ok(desc_host)) return SWARM_EINVAL;
  const swarm_paged& d = *desc_host;
  if (d.rotated < 0 || d.rotated > d.head_dim || d.rotated % 2 || (d.rotated > 0 && !words_ok(frequencies_dev, true)) ||
      (q_dev != nullptr) != (out_dev != nullptr) || (q_dev && !heads_ok(&d)))
    return SWARM_EINVAL;
  if (d.batch == 0 || d.tokens == 0) return SWARM_OK;
  if (!cache_ok(&d, k_pages_dev, v_pages_dev) || !strided_ok(k_dev, d.k, d.batch, d.tokens, d.kv_heads, false) ||
      !strided_ok(v_dev, d.v, d.batch, d.tokens, d.kv_heads, false) ||
      (q_dev && (!strided_ok(q_dev, d.q, d.batch, d.tokens, d.heads, false) || !strided_ok(out_dev, d.out, d.batch, d.tokens, d.heads, true))))
    return SWARM_EINVAL;
  PagedArgs a{};
  fill(a, desc_host);
  a.q = q_dev; a.k = k_dev; a.v = v_dev; a.k_pages = k_pages_dev; a.v_pages = v_pages_dev; a.out = out_dev; a.frequencies = frequencies_dev;
  cudaError_t e = status_word(&a.status);
  if (e == cudaSuccess) e = d.dtype == SWARM_BF16 ? launch_append<__nv_bfloat16>(a, (cudaStream_t)cuda_stream) : launch_append<__half>(a, (cudaStream_t)cuda_stream);
  return operator_result(e);
}

int swarm_paged_attention_workspace(const swarm_paged* desc_host, size_t* bytes_host) {
  if (!attention_ok(desc_host) || !bytes_host) return SWARM_EINVAL;
  PagedArgs a{};
  fill(a, desc_host);
  *bytes_host = a.batch && a.tokens ? paged_attention_workspace(a) : 0;
  return SWARM_OK;
}

int swarm_paged_attention(const swarm_paged* desc_host, const void* q_dev, const void* k_pages_dev, const void* v_pages_dev,
                          void* out_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  if (!attention_ok(desc_host)) return SWARM_EINVAL;
  const swarm_paged& d = *desc_host;
  if (d.batch == 0 || d.tokens == 0) return SWARM_OK;
  size_t need = 0;
  swarm_paged_attention_workspace(desc_host, &need);
  if (!cache_ok(&d, k_pages_dev, v_pages_dev) || !strided_ok(q_dev, d.q, d.batch, d.tokens, d.heads, false) ||
      !strided_ok(out_dev, d.out, d.batch, d.tokens, d.heads, true) || !words_ok(lse_dev, false) || workspace_bytes < need ||
      (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15))))
    return SWARM_EINVAL;
  PagedArgs a{};
  fill(a, desc_host);
  a.q = q_dev; a.k_pages = const_cast<void*>(k_pages_dev); a.v_pages = const_cast<void*>(v_pages_dev); a.out = out_dev; a.lse = lse_dev;
  cudaError_t e = status_word(&a.status);
  if (e == cudaSuccess) e = launch_paged_attention(a, d.dtype, workspace_dev, (cudaStream_t)cuda_stream);
  return operator_result(e);
}

}  // extern "C"
