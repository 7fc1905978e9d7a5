// Log probabilities of given tokens with entropy and the likeliest tokens, and their gradient with respect to the logits.
#include <cmath>

#include "swarm_opsup.cuh"

namespace swarm {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

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
__device__ __forceinline__ uint64_t key_of(float v, uint32_t place) {
  uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);
  u = isnan(v) ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (uint32_t)~place;
}

// CTA = one row, three walks over it: its largest logit, its sums, and one for each of the likeliest tokens.
template <typename T>
__global__ void __launch_bounds__(256) log_probs_kernel(LogProbsArgs a) {
  __shared__ float s_f[8], s_g[8];
  __shared__ uint64_t s_k[8];
  const int64_t row = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.pitch;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto largest_below = [&](uint64_t bound) {
    uint64_t best = 0;
    for (int64_t i = threadIdx.x; i < a.cols; i += 256) {
      const uint64_t k = key_of(to_float<T>(x[i]), (uint32_t)i);
      if (k < bound && k > best) best = k;
    }
    for (int o = 16; o > 0; o >>= 1) { const uint64_t k = __shfl_xor_sync(0xFFFFFFFFu, best, o); best = k > best ? k : best; }
    __syncthreads();
    if (lane == 0) s_k[warp] = best;
    __syncthreads();
    for (int w = 0; w < 8; ++w) best = s_k[w] > best ? s_k[w] : best;
    return best;
  };
  const uint64_t first = largest_below(~0ull);
  const float top = to_float<T>(x[~(uint32_t)first]), base = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f, weighted = 0.0f;
  for (int64_t i = threadIdx.x; i < a.cols; i += 256) {
    const float d = (to_float<T>(x[i]) - base) * a.scale, e = ex2(d * kLog2e);
    sum += e;
    weighted += e == 0.0f ? 0.0f : e * d;
  }
  sum = warp_sum(sum);
  weighted = warp_sum(weighted);
  if (lane == 0) { s_f[warp] = sum; s_g[warp] = weighted; }
  __syncthreads();
  sum = weighted = 0.0f;
  for (int w = 0; w < 8; ++w) { sum += s_f[w]; weighted += s_g[w]; }
  const float log_sum = logf(sum);
  auto log_prob = [&](float v) { return top == -INFINITY ? -INFINITY : (v - base) * a.scale - log_sum; };
  if (threadIdx.x == 0) {
    a.stats[row * 2] = top;
    a.stats[row * 2 + 1] = log_sum;
    if (a.log_probs) {
      const int64_t t = a.tokens[row];
      a.log_probs[row] = t >= 0 && t < a.cols ? log_prob(to_float<T>(x[t])) : 0.0f;
    }
    if (a.entropy) a.entropy[row] = top == -INFINITY ? 0.0f : log_sum - weighted / sum;
  }
  uint64_t key = first;
  for (int k = 0; k < a.top; ++k) {
    if (k > 0) key = largest_below(key);
    if (threadIdx.x == 0) {
      const uint32_t place = ~(uint32_t)key;
      a.top_tokens[row * a.top + k] = place;
      a.top_log_probs[row * a.top + k] = log_prob(to_float<T>(x[place]));
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) log_probs_grad_kernel(LogProbsArgs a) {
  const int64_t row = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.pitch;
  T* dx = reinterpret_cast<T*>(a.dlogits) + row * a.dlogits_pitch;
  const float top = a.stats[row * 2], log_sum = a.stats[row * 2 + 1];
  const int64_t t = a.tokens ? a.tokens[row] : -1;
  const float g = a.dlog_probs && t >= 0 && t < a.cols ? a.dlog_probs[row] : 0.0f;
  const float h = a.dentropy ? a.dentropy[row] : 0.0f, entropy = a.dentropy ? a.entropy[row] : 0.0f;
  for (int64_t i = threadIdx.x; i < a.cols; i += 256) {
    const float logp = (to_float<T>(x[i]) - top) * a.scale - log_sum, p = ex2(logp * kLog2e);
    float v = (i == t ? g : 0.0f) - g * p;
    if (a.dentropy && p != 0.0f) v -= h * p * (logp + entropy);
    dx[i] = from_float<T>(top == -INFINITY ? 0.0f : v * a.scale);
  }
}

template <typename T>
cudaError_t launch_forward(const LogProbsArgs& a, cudaStream_t st) {
  log_probs_kernel<T><<<(unsigned)a.rows, 256, 0, st>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch_backward(const LogProbsArgs& a, cudaStream_t st) {
  log_probs_grad_kernel<T><<<(unsigned)a.rows, 256, 0, st>>>(a);
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
