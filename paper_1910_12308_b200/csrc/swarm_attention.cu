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
static __device__ int g_operator_status;               // raised by kernels of this device
int* g_status_addr[kMaxDevices] = {};
std::mutex g_setup_mutex;

}  // namespace

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

namespace {

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
constexpr int32_t kMaxTokens = 1 << 30;                 // tile arithmetic stays in 32 bits
// CTAs of the largest grid that any kernel of the call may take.
bool grid_ok(const swarm_attention* d) {
  const int64_t rows = ((int64_t)d->queries + 127) / 128, states = ((int64_t)d->keys + 127) / 128;
  return (rows > 32 ? rows : 32) * d->heads < ((int64_t)1 << 31) / (d->batch > 0 ? d->batch : 1) &&
         states * d->kv_heads < ((int64_t)1 << 31) / (d->batch > 0 ? d->batch : 1);
}
bool desc_ok(const swarm_attention* d) {
  return d && d->queries <= kMaxTokens && d->keys <= kMaxTokens && d->batch >= 0 && d->queries >= 0 && d->keys >= 0 && d->heads >= 1 && d->kv_heads >= 1 &&
         d->heads % d->kv_heads == 0 && d->batch <= 65535 && d->heads <= 65535 && d->head_dim >= 8 && d->head_dim <= kMaxDim &&
         d->head_dim % 8 == 0 && (d->dtype == SWARM_BF16 || d->dtype == SWARM_F16) && d->scale > 0.0f && std::isfinite(d->scale) && grid_ok(d);
}
constexpr int64_t kMaxStride = (int64_t)1 << 38;
bool one_stride_ok(int64_t s, int extent, bool repeats) {
  return extent <= 1 || (s >= 0 && s < kMaxStride && s % 8 == 0 && (repeats || s != 0));
}
// The backward kernels hold lse / scale, which has to stay within fp32's range (lse is below 2^7 where that bounds it).
constexpr float kMinGradScale = 0x1p-120f;
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

// Whether a call goes to the kernel that streams the states past 16 rows (query tokens x heads of a key head) at a time, instead
// of that with tiles of 128 rows of one head. The tiles walk all states once for each head of a group, the other kernel once for
// each 16 rows, so the crossing in tokens hardly moves with the group; at 12 streaming is at most 15 % behind and up to a
// quarter ahead. Measured, 128 sentences of 1024 states, 16 heads of 64, one token: 103 / 122 us; 16 sentences, 16 key heads, bf16,
// cold caches, us streaming / tiles:
//   tokens                            1          8          12         16         24
//   heads of 64,  1 to a key head   29 /  27   29 /  27   31 /  27   33 /  27   49 /  27
//   heads of 64,  4 to a key head   29 /  66   51 /  68   55 /  68   72 /  68   92 /  68
//   heads of 64,  8 to a key head   31 / 119   70 / 121   92 / 121  113 / 121  156 / 121
//   heads of 128, 1 to a key head   39 /  45   43 /  45   45 /  47   47 /  45   70 /  45
//   heads of 128, 4 to a key head   41 /  90   74 /  90   98 /  90  125 /  90  178 /  90
//   heads of 128, 8 to a key head   41 / 150  125 / 152  172 / 152  209 / 152  307 / 154
bool few_rows(const AttentionArgs& a) { return a.queries <= 12; }

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" {

int swarm_cross_attention_workspace(const swarm_attention* desc_host, int32_t backward, size_t* bytes_host) {
  if (!desc_ok(desc_host) || !bytes_host) return SWARM_EINVAL;
  AttentionArgs a{};
  fill(a, desc_host);
  if (backward) *bytes_host = a.batch && a.queries && a.keys ? attention_backward_workspace(a) : 0;
  else if (!a.batch || !a.queries || !a.keys) *bytes_host = 0;
  else *bytes_host = few_rows(a) ? attention_rows_workspace(a) : attention_forward_workspace(a);
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
  return operator_result(few_rows(a) ? launch_attention_rows(a, d.dtype, workspace_dev, st) : launch_attention_forward_tc(a, d.dtype, workspace_dev, st));
}

int swarm_cross_attention_backward(const swarm_attention* desc_host, const void* dout_dev, const void* q_dev,
                                   const void* k_dev, const void* v_dev, const void* o_dev, const float* lse_dev,
                                   void* dq_dev, void* dk_dev, void* dv_dev, void* workspace_dev,
                                   size_t workspace_bytes, void* cuda_stream) {
  if (!desc_ok(desc_host) || desc_host->scale < kMinGradScale) return SWARM_EINVAL;
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
  a.dq = dq_dev; a.dk = dk_dev; a.dv = dv_dev;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = status_word(&a.status);
  if (d.queries > 0 && d.keys > 0) {
    if (e == cudaSuccess) e = launch_attention_backward_tc(a, d.dtype, workspace_dev, st);
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
    if (e == cudaSuccess && !(raised & kStatusWait)) return SWARM_ERANGE;
    if (e == cudaSuccess) e = cudaErrorLaunchTimeout;
  }
  return operator_result(e);
}

}  // extern "C"
