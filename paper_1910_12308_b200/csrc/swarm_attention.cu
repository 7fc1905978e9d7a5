// Cross attention of a decoder's rows to an encoder's states, and its gradient.
//
//   s = scale * q k^T,  p = exp(s - lse),  o = p v
//   dv = p^T dout,  ds = scale * p * (dout v^T - rowsum(dout * o)),  dq = ds k,  dk = ds^T q
//
// One pass over the states with the running maximum and sum of the softmax; nothing of size queries x keys is stored.
#include <cmath>
#include <mutex>

#include "swarm_attention.h"

namespace swarm {
namespace {

constexpr int kMaxDevices = 64;
static __device__ int g_operator_status;               // raised by a kernel of this device whose wait gave up
int* g_status_addr[kMaxDevices] = {};
std::mutex g_setup_mutex;

// Device address of the status word of the current device.
cudaError_t status_word(int** out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_setup_mutex);
  if (!g_status_addr[dev]) {
    void* p = nullptr;
    e = cudaGetSymbolAddress(&p, g_operator_status);
    if (e != cudaSuccess) return e;
    g_status_addr[dev] = (int*)p;
  }
  *out = g_status_addr[dev];
  return cudaSuccess;
}

template <typename T>
__device__ __forceinline__ float dot_row(const float* a, const T* p, int dim) {
  float s = 0.0f;
  for (int d = 0; d < dim; d += 8) {
    float v[8];
    unpack8<T>(load_raw8<T>(p + d), v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(a[d + i], v[i], s);
  }
  return s;
}

// Warp = one query row; lane = one state of 32 at a time for the scores, then dims lane, lane + 32, ... of the output.
template <typename T>
__global__ void __launch_bounds__(128) attention_rows_kernel(AttentionArgs a) {
  __shared__ float sq[4][kMaxDim];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * 4 + warp, h = blockIdx.y, b = blockIdx.z, hk = h / a.group;
  if (t >= a.queries) return;
  const int nq = length_of(a.query_lengths, b, a.queries), nk = length_of(a.key_lengths, b, a.keys);
  const T* q = reinterpret_cast<const T*>(a.q) + offset_of(a.qs, b, t, h);
  T* out = reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h);
  const int n = t < nq ? nk : 0;
  for (int d = lane; d < a.head_dim; d += 32) sq[warp][d] = n ? to_float<T>(q[d]) : 0.0f;
  __syncwarp();
  float m = -INFINITY, l = 0.0f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < n; j0 += 32) {
    const int j = j0 + lane;
    const float s = j < n ? a.scale * dot_row<T>(sq[warp], reinterpret_cast<const T*>(a.k) + offset_of(a.ks, b, j, hk), a.head_dim) : -INFINITY;
    float top = s;
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.0f : m_new;
    const float c = exp2f((m - base) * kLog2e), p = exp2f((s - base) * kLog2e);
    l = l * c + warp_sum(p);
    m = m_new;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= c;
    for (int u = 0; u < min(32, n - j0); ++u) {
      const float pu = __shfl_sync(0xFFFFFFFFu, p, u);
      const T* v = reinterpret_cast<const T*>(a.v) + offset_of(a.vs, b, j0 + u, hk);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < a.head_dim) acc[i] = fmaf(pu, to_float<T>(v[lane + 32 * i]), acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < a.head_dim) out[lane + 32 * i] = from_float<T>(n ? acc[i] / l : 0.0f);
  if (a.lse && lane == 0) a.lse[((int64_t)b * a.heads + h) * a.queries + t] = n ? m + logf(l) : -INFINITY;
}

// Zeros into a strided tensor: the outputs of a call that has no rows or no states to sum over.
__global__ void __launch_bounds__(256) attention_zero_kernel(uint4* p, swarm_strides s, int tokens, int heads, int chunks) {
  const int b = blockIdx.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)tokens * heads * chunks; i += (int64_t)gridDim.x * 256) {
    const int ch = (int)(i % chunks), h = (int)(i / chunks % heads), t = (int)(i / chunks / heads);
    p[offset_of(s, b, t, h) / 8 + ch] = make_uint4(0, 0, 0, 0);
  }
}
__global__ void __launch_bounds__(256) attention_no_states_kernel(float* lse, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) lse[i] = -INFINITY;
}
cudaError_t launch_zero(void* p, const swarm_strides& s, int batch, int tokens, int heads, int head_dim, cudaStream_t st) {
  const int64_t count = (int64_t)tokens * heads * (head_dim / 8);
  const unsigned x = (unsigned)(count < 256 * 1024 ? (count + 255) / 256 : 1024);
  attention_zero_kernel<<<dim3(x, (unsigned)batch), 256, 0, st>>>(reinterpret_cast<uint4*>(p), s, tokens, heads, head_dim / 8);
  return cudaGetLastError();
}

// ---- argument checks ------------------------------------------------------------------------
bool desc_ok(const swarm_attention* d) {
  return d && d->batch >= 0 && d->queries >= 0 && d->keys >= 0 && d->heads >= 1 && d->kv_heads >= 1 &&
         d->heads % d->kv_heads == 0 && d->batch <= 65535 && d->heads <= 65535 && d->head_dim >= 8 && d->head_dim <= kMaxDim &&
         d->head_dim % 8 == 0 && (d->dtype == SWARM_BF16 || d->dtype == SWARM_F16) && d->scale > 0.0f && std::isfinite(d->scale);
}
constexpr int64_t kMaxStride = (int64_t)1 << 38;
bool one_stride_ok(int64_t s, int extent, bool repeats) {
  return extent <= 1 || (s >= 0 && s < kMaxStride && s % 8 == 0 && (repeats || s != 0));
}
// A tensor of `tokens` rows and `heads` heads: address and strides; an input may repeat its sentences or heads.
bool strided_ok(const void* p, const swarm_strides& s, int batch, int tokens, int heads, bool output) {
  return p && ((uintptr_t)p & 15) == 0 && one_stride_ok(s.batch, batch, !output) && one_stride_ok(s.token, tokens, false) &&
         one_stride_ok(s.head, heads, !output);
}
bool lengths_ok(const int32_t* p) { return ((uintptr_t)p & 3) == 0; }

void fill(AttentionArgs& a, const swarm_attention* d) {
  a.query_lengths = d->query_lengths_dev; a.key_lengths = d->key_lengths_dev;
  a.qs = d->q; a.ks = d->k; a.vs = d->v; a.os = d->o; a.dos = d->dout; a.dqs = d->dq; a.dks = d->dk; a.dvs = d->dv;
  a.batch = d->batch; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads;
  a.queries = d->queries; a.keys = d->keys; a.head_dim = d->head_dim;
  a.scale = d->scale;
  a.wait_limit = d->wait_limit < 0 ? kAttentionWaitLimit : d->wait_limit < (int64_t)1 << 32 ? (uint32_t)d->wait_limit : 0xFFFFFFFFu;
}

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" {

int swarm_cross_attention_workspace(const swarm_attention* desc_host, int32_t backward, size_t* bytes_host) {
  if (!desc_ok(desc_host) || !bytes_host) return SWARM_EINVAL;
  *bytes_host = backward ? (size_t)desc_host->batch * desc_host->heads * desc_host->queries * sizeof(float) : 0;
  return SWARM_OK;
}

int swarm_cross_attention(const swarm_attention* desc_host, const void* q_dev, const void* k_dev, const void* v_dev,
                          void* o_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  if (!desc_ok(desc_host)) return SWARM_EINVAL;
  const swarm_attention& d = *desc_host;
  if (d.batch == 0 || d.queries == 0) return SWARM_OK;
  size_t need = 0;
  swarm_cross_attention_workspace(desc_host, 0, &need);
  if (!strided_ok(q_dev, d.q, d.batch, d.queries, d.heads, false) || !strided_ok(o_dev, d.o, d.batch, d.queries, d.heads, true) ||
      (d.keys > 0 && (!strided_ok(k_dev, d.k, d.batch, d.keys, d.kv_heads, false) || !strided_ok(v_dev, d.v, d.batch, d.keys, d.kv_heads, false))) ||
      ((uintptr_t)lse_dev & 3) || !lengths_ok(d.query_lengths_dev) || !lengths_ok(d.key_lengths_dev) ||
      workspace_bytes < need || (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15))))
    return SWARM_EINVAL;
  AttentionArgs a{};
  fill(a, desc_host);
  a.q = q_dev; a.k = k_dev; a.v = v_dev; a.out = o_dev; a.lse = lse_dev;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = status_word(&a.status);
  if (e != cudaSuccess) return operator_result(e);
  if (d.keys == 0) {
    if (lse_dev) {
      const int64_t count = (int64_t)d.batch * d.heads * d.queries;
      attention_no_states_kernel<<<(unsigned)(count < 256 * 1024 ? (count + 255) / 256 : 1024), 256, 0, st>>>(lse_dev, count);
    }
    return operator_result(launch_zero(o_dev, d.o, d.batch, d.queries, d.heads, d.head_dim, st));
  }
  if ((int64_t)d.queries * a.group > 16) return operator_result(launch_attention_forward_tc(a, d.dtype, st));
  const dim3 grid((unsigned)((d.queries + 3) / 4), (unsigned)d.heads, (unsigned)d.batch);
  if (d.dtype == SWARM_BF16) attention_rows_kernel<__nv_bfloat16><<<grid, 128, 0, st>>>(a);
  else attention_rows_kernel<__half><<<grid, 128, 0, st>>>(a);
  return operator_result(cudaGetLastError());
}

int swarm_cross_attention_backward(const swarm_attention* desc_host, const void* dout_dev, const void* q_dev,
                                   const void* k_dev, const void* v_dev, const void* o_dev, const float* lse_dev,
                                   void* dq_dev, void* dk_dev, void* dv_dev, void* workspace_dev,
                                   size_t workspace_bytes, void* cuda_stream) {
  if (!desc_ok(desc_host)) return SWARM_EINVAL;
  const swarm_attention& d = *desc_host;
  if (d.batch == 0) return SWARM_OK;
  size_t need = 0;
  swarm_cross_attention_workspace(desc_host, 1, &need);
  if (d.queries > 0 &&
      (!strided_ok(q_dev, d.q, d.batch, d.queries, d.heads, false) || !strided_ok(o_dev, d.o, d.batch, d.queries, d.heads, false) ||
       !strided_ok(dout_dev, d.dout, d.batch, d.queries, d.heads, false) || !strided_ok(dq_dev, d.dq, d.batch, d.queries, d.heads, true) ||
       !lse_dev || ((uintptr_t)lse_dev & 3)))
    return SWARM_EINVAL;
  if (d.keys > 0 &&
      (!strided_ok(dk_dev, d.dk, d.batch, d.keys, d.kv_heads, true) || !strided_ok(dv_dev, d.dv, d.batch, d.keys, d.kv_heads, true) ||
       !strided_ok(k_dev, d.k, d.batch, d.keys, d.kv_heads, false) || !strided_ok(v_dev, d.v, d.batch, d.keys, d.kv_heads, false)))
    return SWARM_EINVAL;
  if (!lengths_ok(d.query_lengths_dev) || !lengths_ok(d.key_lengths_dev) || workspace_bytes < need ||
      (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15))))
    return SWARM_EINVAL;
  AttentionArgs a{};
  fill(a, desc_host);
  a.q = q_dev; a.k = k_dev; a.v = v_dev; a.o = o_dev; a.dout = dout_dev; a.lse_in = lse_dev;
  a.dq = dq_dev; a.dk = dk_dev; a.dv = dv_dev; a.delta = reinterpret_cast<float*>(workspace_dev);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = status_word(&a.status);
  if (d.queries > 0 && d.keys > 0) {
    if (e == cudaSuccess) e = launch_attention_backward_tc(a, d.dtype, st);
  } else if (d.queries > 0) {
    if (e == cudaSuccess) e = launch_zero(dq_dev, d.dq, d.batch, d.queries, d.heads, d.head_dim, st);
  } else if (d.keys > 0) {
    if (e == cudaSuccess) e = launch_zero(dk_dev, d.dk, d.batch, d.keys, d.kv_heads, d.head_dim, st);
    if (e == cudaSuccess) e = launch_zero(dv_dev, d.dv, d.batch, d.keys, d.kv_heads, d.head_dim, st);
  }
  return operator_result(e);
}

int swarm_operator_check(void* cuda_stream) {
  cudaStream_t st = (cudaStream_t)cuda_stream;
  int *word = nullptr, raised = 0;
  cudaError_t e = status_word(&word);
  if (e == cudaSuccess) e = cudaMemcpyAsync(&raised, word, sizeof raised, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && raised) {
    e = cudaMemsetAsync(word, 0, sizeof raised, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess) e = cudaErrorLaunchTimeout;
  }
  return operator_result(e);
}

}  // extern "C"
