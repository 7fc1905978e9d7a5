// Row operators of the models that the nodes train: dropout with a residual addition, and the root-mean-square norm
// with the residual's addition (dropout included), its 8-bit output and its gradient.
//
// All of them are one pass over their tensors: every element is read once and written once, a row stays in registers
// between its reduction and its output, and HBM bandwidth is the bound; the generator's ~60 integer instructions per
// eight elements run beside the loads.
#include <cuda_fp8.h>

#include <cmath>
#include <mutex>

#include "swarm_opsup.cuh"

namespace swarm {

thread_local int g_operator_error = 0;

cudaError_t operator_sm_count(int* out) {
  static int counts[64] = {};
  static std::mutex mutex;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lock(mutex);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!counts[dev]) {
    e = cudaDeviceGetAttribute(&counts[dev], cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) { counts[dev] = 0; return e; }
  }
  *out = counts[dev];
  return cudaSuccess;
}

namespace {

// =================================================================================================
// Dropout. Warp = one 256-column segment of a row at a time; the warps of the grid walk the (row, segment) list with
// a fixed stride, whose quotient and remainder by the segments of a row come from the host, so that the walk needs
// no division.
// =================================================================================================
constexpr int kDropThreads = 256;

struct DropoutArgs {
  const void* x;
  const void* residual;
  void* out;
  int64_t x_pitch, residual_pitch, out_pitch;
  int64_t rows, cols;
  uint32_t segments;                  // per row
  int64_t row_step;                   // the stride of the walk: this many rows
  uint32_t segment_step;              // and this many segments
};

template <typename T, bool VEC, bool RES>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(DropoutArgs a, DropoutMask m) {
  const int lane = threadIdx.x & 31;
  const int64_t first = (int64_t)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5);
  int64_t row = first / a.segments;
  uint32_t seg = (uint32_t)(first - row * a.segments);
  while (row < a.rows) {
    const int64_t col = (int64_t)seg * kSegment;
    const int valid = (int)min((int64_t)kSegment, a.cols - col);
    float v[8], r[8];
    segment_load<T, VEC>(reinterpret_cast<const T*>(a.x) + row * a.x_pitch + col, valid, lane, v);
    if constexpr (RES) segment_load<T, VEC>(reinterpret_cast<const T*>(a.residual) + row * a.residual_pitch + col, valid, lane, r);
    if (m.threshold != 0) segment_dropout<VEC>(v, seg * (kSegment / 8), (uint32_t)row, lane, m);
    if constexpr (RES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    segment_store<T, VEC>(reinterpret_cast<T*>(a.out) + row * a.out_pitch + col, valid, lane, v);
    row += a.row_step;
    seg += a.segment_step;
    if (seg >= a.segments) { seg -= a.segments; ++row; }
  }
}

template <typename T>
cudaError_t launch_dropout(DropoutArgs a, const DropoutMask& m, bool vec, cudaStream_t st) {
  int sms = 0;
  const cudaError_t e = operator_sm_count(&sms);
  if (e != cudaSuccess) return e;
  const int64_t items = a.rows * (int64_t)a.segments, per_cta = kDropThreads / 32;
  const int64_t most = (int64_t)sms * (2048 / kDropThreads);
  const int64_t ctas = items < most * per_cta ? (items + per_cta - 1) / per_cta : most;
  const int64_t stride = ctas * per_cta;
  a.row_step = stride / a.segments;
  a.segment_step = (uint32_t)(stride % a.segments);
  const unsigned grid = (unsigned)ctas;
  if (vec) {
    if (a.residual) dropout_kernel<T, true, true><<<grid, kDropThreads, 0, st>>>(a, m);
    else dropout_kernel<T, true, false><<<grid, kDropThreads, 0, st>>>(a, m);
  } else {
    if (a.residual) dropout_kernel<T, false, true><<<grid, kDropThreads, 0, st>>>(a, m);
    else dropout_kernel<T, false, false><<<grid, kDropThreads, 0, st>>>(a, m);
  }
  return cudaGetLastError();
}

// =================================================================================================
// Norm. A row belongs to WPR warps (a group), each holding VPL segments of it in registers: segment v of warp w is
// segment w + v * WPR of the row. WPR = 1 reduces with shuffles alone and a CTA holds several rows; a wider row is a
// CTA of its own and meets once in shared memory.
// =================================================================================================
constexpr int kNormBlock = 128;                        // columns that share one scale in the 8-bit output

struct NormArgs {
  const void* x;
  const void* residual;
  const float* weight;
  void* total;
  void* y;
  uint8_t* codes;
  float* scales;
  int64_t x_pitch, residual_pitch, total_pitch, y_pitch;
  int64_t rows, cols, blocks;         // blocks = ceil(cols / 128)
  float eps, inv_cols;
};

template <bool VEC>
__device__ __forceinline__ void weight_load(const float* w, int valid, int lane, bool aligned, float v[8]) {
  if (VEC && aligned) segment_load<float, true>(w, valid, lane, v);
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = segment_column<VEC>(lane, i);
      v[i] = c < valid ? w[c] : 0.0f;
    }
  }
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// Sum over the warps of a row's group: the same value, added in warp order, in every thread.
template <int WPR>
__device__ __forceinline__ float group_sum(float v, float* slots, int warp) {
  v = warp_sum(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 31) == 0) slots[warp] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) v += slots[w];
  }
  return v;
}

template <typename T, bool VEC, int WPR, int VPL, bool CODES>
__global__ void __launch_bounds__(WPR == 1 ? 128 : WPR * 32)
add_rms_norm_kernel(NormArgs a, DropoutMask m) {
  constexpr int kRowsPerCta = WPR == 1 ? 4 : 1;
  __shared__ float slots[2][WPR];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * kRowsPerCta + (WPR == 1 ? warp : 0);
  if (WPR == 1 && row >= a.rows) return;
  const int seg0 = WPR == 1 ? 0 : warp;
  float t[VPL][8], r[VPL][8];
#pragma unroll
  for (int s = 0; s < VPL; ++s) {
    const int64_t col = (int64_t)(seg0 + s * WPR) * kSegment;
    const int valid = (int)min((int64_t)kSegment, a.cols - col);
    segment_load<T, VEC>(reinterpret_cast<const T*>(a.x) + row * a.x_pitch + col, valid, lane, t[s]);
    if (a.residual) segment_load<T, VEC>(reinterpret_cast<const T*>(a.residual) + row * a.residual_pitch + col, valid, lane, r[s]);
  }
  float sq = 0.0f;
#pragma unroll
  for (int s = 0; s < VPL; ++s) {
    const int seg = seg0 + s * WPR;
    if (m.threshold != 0) segment_dropout<VEC>(t[s], (uint32_t)seg * (kSegment / 8), (uint32_t)row, lane, m);
    if (a.residual) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[s][i] += r[s][i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sq = fmaf(t[s][i], t[s][i], sq);
  }
  sq = group_sum<WPR>(sq, slots[0], warp);
  const float rstd = 1.0f / sqrtf(fmaf(sq, a.inv_cols, a.eps));
  const bool w_aligned = (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0;
#pragma unroll
  for (int s = 0; s < VPL; ++s) {
    const int seg = seg0 + s * WPR;
    const int64_t col = (int64_t)seg * kSegment;
    const int valid = (int)min((int64_t)kSegment, a.cols - col);
    if (valid <= 0) continue;                                          // the same for the whole warp
    if (a.total) segment_store<T, VEC>(reinterpret_cast<T*>(a.total) + row * a.total_pitch + col, valid, lane, t[s]);
    float w[8];
    weight_load<VEC>(a.weight + col, valid, lane, w_aligned, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) t[s][i] = t[s][i] * rstd * w[i];
    if constexpr (!CODES) {
      segment_store<T, VEC>(reinterpret_cast<T*>(a.y) + row * a.y_pitch + col, valid, lane, t[s]);
    } else {
      // largest magnitude of each 128-column block, as bit patterns, so that a NaN is the largest: VEC lanes 0..15 hold
      // the first block and 16..31 the second, else elements 0..3 and 4..7 of every lane do
      uint32_t top[2] = {0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t mag = segment_column<VEC>(lane, i) < valid ? __float_as_uint(t[s][i]) & 0x7FFFFFFFu : 0u;
        const int b = VEC ? (lane >> 4) : (i >> 2);
        if (b == 0) top[0] = max(top[0], mag); else top[1] = max(top[1], mag);
      }
      top[0] = __reduce_max_sync(0xFFFFFFFFu, top[0]);
      top[1] = __reduce_max_sync(0xFFFFFFFFu, top[1]);
      float scale[2], inv[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        scale[b] = __uint_as_float(top[b]) * (1.0f / 448.0f);
        if (scale[b] < 0x1p-126f) scale[b] = 0.0f;                     // its reciprocal could overflow
        inv[b] = scale[b] == 0.0f ? 0.0f : 1.0f / scale[b];
        const int64_t block = (int64_t)seg * 2 + b;
        if (lane == 0 && block < a.blocks) a.scales[row * a.blocks + block] = scale[b];
      }
      uint8_t* out = a.codes + row * a.y_pitch + col;
      if constexpr (VEC) {
        const float f = lane >> 4 ? inv[1] : inv[0];
        const uint32_t lo = e4m3x2(t[s][0] * f, t[s][1] * f) | e4m3x2(t[s][2] * f, t[s][3] * f) << 16;
        const uint32_t hi = e4m3x2(t[s][4] * f, t[s][5] * f) | e4m3x2(t[s][6] * f, t[s][7] * f) << 16;
        if (lane * 8 + 8 <= valid) *reinterpret_cast<uint2*>(out + lane * 8) = make_uint2(lo, hi);
        else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (lane * 8 + i < valid) out[lane * 8 + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = i * 32 + lane;
          if (c < valid) out[c] = (uint8_t)e4m3x2(t[s][i] * inv[i >> 2], 0.0f);
        }
      }
    }
  }
}

// =================================================================================================
// Gradient of the norm. The groups of the grid walk the rows with a fixed stride and keep their part of dweight in
// registers; the parts of a CTA meet in shared memory in warp order, those of the CTAs in a second kernel in CTA
// order, so the sum over rows has one fixed association.
// =================================================================================================
struct NormGradArgs {
  const void* dy;
  const void* dtotal;
  const void* total;
  const float* weight;
  void* dresidual;
  void* dx;
  float* partial;                     // [CTAs][cols] or nullptr
  int64_t dy_pitch, dtotal_pitch, total_pitch, dresidual_pitch, dx_pitch;
  int64_t rows, cols;
  float eps, inv_cols;
};

template <typename T, bool VEC, int WPR, int VPL>
__global__ void __launch_bounds__(WPR == 1 ? 128 : WPR * 32)
add_rms_norm_grad_kernel(NormGradArgs a, DropoutMask m) {
  constexpr int kRowsPerCta = WPR == 1 ? 4 : 1;
  __shared__ float slots[2][2][WPR];
  __shared__ float parts[WPR == 1 ? 4 * VPL * kSegment : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int seg0 = WPR == 1 ? 0 : warp;
  const bool w_aligned = (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0;
  float dw[VPL][8];
#pragma unroll
  for (int s = 0; s < VPL; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[s][i] = 0.0f;
  int flip = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRowsPerCta + (WPR == 1 ? warp : 0); row < a.rows; row += (int64_t)gridDim.x * kRowsPerCta) {
    float g[VPL][8], t[VPL][8];                                        // weight * dy, total
    float sq = 0.0f, dot = 0.0f;
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * kSegment;
      const int valid = (int)min((int64_t)kSegment, a.cols - col);
      segment_load<T, VEC>(reinterpret_cast<const T*>(a.dy) + row * a.dy_pitch + col, valid, lane, g[s]);
      segment_load<T, VEC>(reinterpret_cast<const T*>(a.total) + row * a.total_pitch + col, valid, lane, t[s]);
    }
    float w[VPL][8];
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * kSegment;
      weight_load<VEC>(a.weight + col, (int)min((int64_t)kSegment, a.cols - col), lane, w_aligned, w[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sq = fmaf(t[s][i], t[s][i], sq);
        dot = fmaf(g[s][i] * w[s][i], t[s][i], dot);
      }
    }
    if constexpr (WPR == 1) {
      sq = warp_sum(sq);
      dot = warp_sum(dot);
    } else {
      sq = warp_sum(sq);
      dot = warp_sum(dot);
      if (lane == 0) { slots[flip][0][warp] = sq; slots[flip][1][warp] = dot; }
      __syncthreads();
      sq = dot = 0.0f;
#pragma unroll
      for (int q = 0; q < WPR; ++q) { sq += slots[flip][0][q]; dot += slots[flip][1][q]; }
      flip ^= 1;                                                       // the other set is written before the next barrier
    }
    const float r = 1.0f / sqrtf(fmaf(sq, a.inv_cols, a.eps));
    const float c = r * r * r * (dot * a.inv_cols);
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int seg = seg0 + s * WPR;
      const int64_t col = (int64_t)seg * kSegment;
      const int valid = (int)min((int64_t)kSegment, a.cols - col);
      if (valid <= 0) continue;
      float d[8];
      if (a.dtotal) segment_load<T, VEC>(reinterpret_cast<const T*>(a.dtotal) + row * a.dtotal_pitch + col, valid, lane, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dw[s][i] = fmaf(g[s][i] * t[s][i], r, dw[s][i]);
        const float v = r * (g[s][i] * w[s][i]) - t[s][i] * c;
        d[i] = a.dtotal ? d[i] + v : v;
      }
      segment_store<T, VEC>(reinterpret_cast<T*>(a.dresidual) + row * a.dresidual_pitch + col, valid, lane, d);
      if (a.dx) {
        if (m.threshold != 0) segment_dropout<VEC>(d, (uint32_t)seg * (kSegment / 8), (uint32_t)row, lane, m);
        segment_store<T, VEC>(reinterpret_cast<T*>(a.dx) + row * a.dx_pitch + col, valid, lane, d);
      }
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (int64_t)blockIdx.x * a.cols;
  if constexpr (WPR == 1) {
#pragma unroll
    for (int s = 0; s < VPL; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) parts[(warp * VPL + s) * kSegment + segment_column<VEC>(lane, i)] = dw[s][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += 128) {
      float v = parts[c];
#pragma unroll
      for (int q = 1; q < 4; ++q) v += parts[q * VPL * kSegment + c];
      out[c] = v;
    }
  } else {
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * kSegment;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = col + segment_column<VEC>(lane, i);
        if (c < a.cols) out[c] = dw[s][i];
      }
    }
  }
}

// dweight[c] = sum of the CTAs' parts: CTA = 32 columns x 32 runs of parts, the runs added in run order.
__global__ void __launch_bounds__(1024)
norm_dweight_kernel(const float* __restrict__ partial, int parts, int64_t cols, float* __restrict__ dweight) {
  __shared__ float runs[32][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float v = 0.0f;
  if (c < cols)
    for (int p = run; p < parts; p += 32) v += partial[(int64_t)p * cols + c];
  runs[run][lane] = v;
  __syncthreads();
  if (run == 0 && c < cols) {
    float sum = 0.0f;
#pragma unroll
    for (int q = 0; q < 32; ++q) sum += runs[q][lane];
    dweight[c] = sum;
  }
}

constexpr int kNormGradMaxCtas = 148 * 8;              // the workspace holds this many parts at most

// Runs CALL with WPR warps per row and VPL segments per warp for rows of `cols` columns.
#define SWARM_NORM_SHAPES(cols, CALL)                      \
  do {                                                     \
    const int64_t segs_ = ((cols) + kSegment - 1) / kSegment; \
    if (segs_ <= 1) CALL(1, 1)                             \
    else if (segs_ <= 2) CALL(1, 2)                        \
    else if (segs_ <= 4) CALL(1, 4)                        \
    else if (segs_ <= 8) CALL(4, 2)                        \
    else if (segs_ <= 16) CALL(8, 2)                       \
    else if (segs_ <= 32) CALL(16, 2)                      \
    else if (segs_ <= 64) CALL(16, 4)                      \
    else CALL(32, 4)                                       \
  } while (0)

template <typename T, bool VEC, bool CODES>
cudaError_t launch_norm(const NormArgs& a, const DropoutMask& m, cudaStream_t st) {
#define SWARM_CALL(W, V)                                                                                  \
  {                                                                                                       \
    const unsigned grid_ = (unsigned)(W == 1 ? (a.rows + 3) / 4 : a.rows);                                \
    add_rms_norm_kernel<T, VEC, W, V, CODES><<<grid_, W == 1 ? 128 : W * 32, 0, st>>>(a, m);              \
  }
  SWARM_NORM_SHAPES(a.cols, SWARM_CALL);
#undef SWARM_CALL
  return cudaGetLastError();
}

// CTAs of the gradient kernel for these sizes.
int64_t norm_grad_ctas(int64_t rows, int64_t cols) {
  const int64_t groups = cols <= 4 * kSegment ? (rows + 3) / 4 : rows;
  const int64_t most = cols <= 4 * kSegment ? 148 * 4 : cols <= 16 * kSegment ? 148 * 2 : 148;
  const int64_t ctas = groups < most ? groups : most;
  return ctas < kNormGradMaxCtas ? ctas : kNormGradMaxCtas;
}

template <typename T, bool VEC>
cudaError_t launch_norm_grad(const NormGradArgs& a, const DropoutMask& m, cudaStream_t st) {
#define SWARM_CALL(W, V) add_rms_norm_grad_kernel<T, VEC, W, V><<<(unsigned)norm_grad_ctas(a.rows, a.cols), W == 1 ? 128 : W * 32, 0, st>>>(a, m);
  SWARM_NORM_SHAPES(a.cols, SWARM_CALL);
#undef SWARM_CALL
  return cudaGetLastError();
}

// ---- argument checks ------------------------------------------------------------------------
bool rows_ok(int64_t rows, int64_t cols, int32_t dtype, double rate) {
  return rows >= 0 && cols >= 0 && rows < (int64_t)1 << 31 && cols < (int64_t)1 << 31 &&
         (dtype == SWARM_F32 || dtype == SWARM_BF16 || dtype == SWARM_F16) && rate >= 0.0 && rate <= 1.0;
}
// A tensor of the call: present or optional, its pitch and its address.
bool tensor_ok(const void* p, int64_t pitch, int64_t cols, size_t size, bool optional) {
  if (!p) return optional;
  return pitch >= cols && ((uintptr_t)p & (size - 1)) == 0;
}
bool on16(const void* p, int64_t pitch, size_t size) {
  return !p || (((uintptr_t)p & 15) == 0 && ((pitch * (int64_t)size) & 15) == 0);
}

}  // namespace
}  // namespace swarm

using namespace swarm;

extern "C" {

int swarm_dropout(const void* x_dev, const void* residual_dev, void* out_dev, int64_t rows, int64_t cols,
                  int64_t x_pitch, int64_t residual_pitch, int64_t out_pitch, int32_t dtype, double rate,
                  uint64_t seed, uint32_t event, void* cuda_stream) {
  if (!rows_ok(rows, cols, dtype, rate)) return SWARM_EINVAL;
  if (rows == 0 || cols == 0) return SWARM_OK;
  const size_t size = element_size(dtype);
  if (!tensor_ok(x_dev, x_pitch, cols, size, false) || !tensor_ok(residual_dev, residual_pitch, cols, size, true) ||
      !tensor_ok(out_dev, out_pitch, cols, size, false))
    return SWARM_EINVAL;
  DropoutArgs a{};
  a.x = x_dev; a.residual = residual_dev; a.out = out_dev;
  a.x_pitch = x_pitch; a.residual_pitch = residual_pitch; a.out_pitch = out_pitch;
  a.rows = rows; a.cols = cols;
  a.segments = (uint32_t)((cols + kSegment - 1) / kSegment);
  const DropoutMask m = make_dropout_mask(rate, seed, event);
  const bool vec = on16(x_dev, x_pitch, size) && on16(residual_dev, residual_pitch, size) && on16(out_dev, out_pitch, size);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == SWARM_F32) return operator_result(launch_dropout<float>(a, m, vec, st));
  if (dtype == SWARM_BF16) return operator_result(launch_dropout<__nv_bfloat16>(a, m, vec, st));
  return operator_result(launch_dropout<__half>(a, m, vec, st));
}

int swarm_add_rms_norm(const void* x_dev, const void* residual_dev, const float* weight_dev, void* total_dev,
                       void* y_dev, uint8_t* codes_dev, float* scales_dev, int64_t rows, int64_t cols,
                       int64_t x_pitch, int64_t residual_pitch, int64_t total_pitch, int64_t y_pitch, int32_t dtype,
                       float eps, double rate, uint64_t seed, uint32_t event, void* cuda_stream) {
  if (!rows_ok(rows, cols, dtype, rate) || cols > SWARM_NORM_MAX_COLS) return SWARM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return SWARM_EINVAL;
  if (rows == 0 || cols == 0) return SWARM_OK;
  const size_t size = element_size(dtype);
  if ((y_dev != nullptr) == (codes_dev != nullptr) || (codes_dev && !scales_dev)) return SWARM_EINVAL;
  if (!tensor_ok(x_dev, x_pitch, cols, size, false) || !tensor_ok(residual_dev, residual_pitch, cols, size, true) ||
      !tensor_ok(total_dev, total_pitch, cols, size, true) || !tensor_ok(weight_dev, cols, cols, 4, false) ||
      !tensor_ok(scales_dev, 0, 0, 4, true))
    return SWARM_EINVAL;
  if (y_dev ? !tensor_ok(y_dev, y_pitch, cols, size, false) : y_pitch < cols) return SWARM_EINVAL;
  NormArgs a{};
  a.x = x_dev; a.residual = residual_dev; a.weight = weight_dev; a.total = total_dev; a.y = y_dev; a.codes = codes_dev;
  a.scales = scales_dev;
  a.x_pitch = x_pitch; a.residual_pitch = residual_pitch; a.total_pitch = total_pitch; a.y_pitch = y_pitch;
  a.rows = rows; a.cols = cols; a.blocks = (cols + kNormBlock - 1) / kNormBlock;
  a.eps = eps; a.inv_cols = (float)(1.0 / (double)cols);
  const DropoutMask m = make_dropout_mask(rate, seed, event);
  // the 8-bit rows are stored 8 bytes at a time
  const bool vec = on16(x_dev, x_pitch, size) && on16(residual_dev, residual_pitch, size) && on16(total_dev, total_pitch, size) &&
                   (y_dev ? on16(y_dev, y_pitch, size) : (((uintptr_t)codes_dev | (uintptr_t)y_pitch) & 7) == 0);
  cudaStream_t st = (cudaStream_t)cuda_stream;
#define SWARM_NORM_TYPED(T)                                                                                        \
  operator_result(vec ? (codes_dev ? launch_norm<T, true, true>(a, m, st) : launch_norm<T, true, false>(a, m, st)) \
                      : (codes_dev ? launch_norm<T, false, true>(a, m, st) : launch_norm<T, false, false>(a, m, st)))
  if (dtype == SWARM_F32) return SWARM_NORM_TYPED(float);
  if (dtype == SWARM_BF16) return SWARM_NORM_TYPED(__nv_bfloat16);
  return SWARM_NORM_TYPED(__half);
#undef SWARM_NORM_TYPED
}

size_t swarm_add_rms_norm_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > SWARM_NORM_MAX_COLS) return 0;
  return (size_t)(norm_grad_ctas(rows, cols) * cols) * sizeof(float);
}

int swarm_add_rms_norm_backward(const void* dy_dev, const void* dtotal_dev, const void* total_dev,
                                const float* weight_dev, void* dresidual_dev, void* dx_dev, float* dweight_dev,
                                int64_t rows, int64_t cols, int64_t dy_pitch, int64_t dtotal_pitch, int64_t total_pitch,
                                int64_t dresidual_pitch, int64_t dx_pitch, int32_t dtype, float eps, double rate,
                                uint64_t seed, uint32_t event, void* workspace_dev, size_t workspace_bytes,
                                void* cuda_stream) {
  if (!rows_ok(rows, cols, dtype, rate) || cols > SWARM_NORM_MAX_COLS) return SWARM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return SWARM_EINVAL;
  if (cols == 0) return SWARM_OK;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (!tensor_ok(dweight_dev, cols, cols, 4, true)) return SWARM_EINVAL;
  if (rows == 0) return dweight_dev ? operator_result(cudaMemsetAsync(dweight_dev, 0, (size_t)cols * 4, st)) : SWARM_OK;
  const size_t size = element_size(dtype);
  if (!tensor_ok(dy_dev, dy_pitch, cols, size, false) || !tensor_ok(dtotal_dev, dtotal_pitch, cols, size, true) ||
      !tensor_ok(total_dev, total_pitch, cols, size, false) || !tensor_ok(dresidual_dev, dresidual_pitch, cols, size, false) ||
      !tensor_ok(dx_dev, dx_pitch, cols, size, true) || !tensor_ok(weight_dev, cols, cols, 4, false))
    return SWARM_EINVAL;
  if (dweight_dev && (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < swarm_add_rms_norm_workspace(rows, cols)))
    return SWARM_EINVAL;
  NormGradArgs a{};
  a.dy = dy_dev; a.dtotal = dtotal_dev; a.total = total_dev; a.weight = weight_dev; a.dresidual = dresidual_dev; a.dx = dx_dev;
  a.partial = dweight_dev ? reinterpret_cast<float*>(workspace_dev) : nullptr;
  a.dy_pitch = dy_pitch; a.dtotal_pitch = dtotal_pitch; a.total_pitch = total_pitch; a.dresidual_pitch = dresidual_pitch;
  a.dx_pitch = dx_pitch;
  a.rows = rows; a.cols = cols; a.eps = eps; a.inv_cols = (float)(1.0 / (double)cols);
  const DropoutMask m = make_dropout_mask(rate, seed, event);
  const bool vec = on16(dy_dev, dy_pitch, size) && on16(dtotal_dev, dtotal_pitch, size) && on16(total_dev, total_pitch, size) &&
                   on16(dresidual_dev, dresidual_pitch, size) && on16(dx_dev, dx_pitch, size);
  cudaError_t e;
  if (dtype == SWARM_F32) e = vec ? launch_norm_grad<float, true>(a, m, st) : launch_norm_grad<float, false>(a, m, st);
  else if (dtype == SWARM_BF16) e = vec ? launch_norm_grad<__nv_bfloat16, true>(a, m, st) : launch_norm_grad<__nv_bfloat16, false>(a, m, st);
  else e = vec ? launch_norm_grad<__half, true>(a, m, st) : launch_norm_grad<__half, false>(a, m, st);
  if (e == cudaSuccess && dweight_dev) {
    norm_dweight_kernel<<<(unsigned)((cols + 31) / 32), 1024, 0, st>>>(a.partial, (int)norm_grad_ctas(rows, cols), cols, dweight_dev);
    e = cudaGetLastError();
  }
  return operator_result(e);
}

int swarm_operator_error(void) { return g_operator_error; }

}  // extern "C"
