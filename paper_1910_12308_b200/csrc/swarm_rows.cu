// Row operators of the models that the nodes train: dropout with a residual addition, and the root-mean-square norm
// with the residual's addition (dropout included), its 8-bit output and its gradient.
//
// All of them are one pass over their tensors: every element is read once and written once, a row stays in registers
// between its reduction and its output, and HBM bandwidth is the bound where tensors are many; the generator's ~60 integer
// instructions per eight elements run beside the loads.
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

// CTAs of a kernel that the device holds at once, looked up once per kernel and device.
template <auto Kernel>
cudaError_t resident_ctas(int threads, int64_t* out) {
  static int per_device[64] = {};
  static std::mutex mutex;
  int sms = 0, dev = 0;
  cudaError_t e = operator_sm_count(&sms);
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lock(mutex);
  if (!per_device[dev]) {
    int n = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, threads, 0);
    if (e != cudaSuccess) return e;
    per_device[dev] = n < 1 ? 1 : n;
  }
  *out = (int64_t)per_device[dev] * sms;
  return cudaSuccess;
}

// =================================================================================================
// Dropout. A warp takes one segment of 32 / LPR rows at a time, two such items in flight; the warps of the grid walk the
// (rows, segment) list with a fixed stride, whose quotient and remainder by the segments of a row come from the host,
// so that the walk needs no division.
// Measured, 32768 x 1024 bf16: with a residual 39 us, 5.1 TB/s (a device copy of as many bytes takes 37); without one 34 us,
// 4.0 TB/s, where no unit is near its end: integer pipe 45 % of its rate, issue 47 %, with 39 % of the warps there can be. As
// many bytes of fp32, half the elements, take 26 us; four items in flight, or the next pair fetched ahead, changed nothing.
// =================================================================================================
constexpr int kRowThreads = 256;

struct DropoutArgs {
  const void* x;
  const void* residual;
  void* out;
  int64_t x_pitch, residual_pitch, out_pitch;
  int64_t rows, cols, row_groups;     // groups of 32 / LPR rows
  uint32_t segments;                  // per row
  int64_t row_step;                   // the stride of the walk: this many groups
  uint32_t segment_step;              // and this many segments
};

template <typename T, bool VEC, int LPR, bool RES>
__global__ void __launch_bounds__(kRowThreads)
dropout_kernel(DropoutArgs a, DropoutMask m) {
  constexpr int kItems = 2;
  const int lane = threadIdx.x & 31, l = lane % LPR, sub = lane / LPR;
  const int64_t first = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  int64_t group = first / a.segments;
  uint32_t seg = (uint32_t)(first - group * a.segments);
  while (group < a.row_groups) {
    Segment<T, VEC, LPR> x[kItems], r[kItems];
    int64_t row[kItems], col[kItems];
    int valid[kItems];
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      row[u] = group * (32 / LPR) + sub;
      col[u] = (int64_t)seg * (LPR * 8);
      valid[u] = group < a.row_groups && row[u] < a.rows ? (int)min((int64_t)LPR * 8, a.cols - col[u]) : 0;
      if (valid[u] > 0) {
        x[u].load(reinterpret_cast<const T*>(a.x) + row[u] * a.x_pitch + col[u], valid[u], l);
        if constexpr (RES) r[u].load(reinterpret_cast<const T*>(a.residual) + row[u] * a.residual_pitch + col[u], valid[u], l);
      }
      group += a.row_step;
      seg += a.segment_step;
      if (seg >= a.segments) { seg -= a.segments; ++group; }
    }
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      float v[8], w[8];
      x[u].get(v);
      if (m.active) segment_drop<VEC, LPR>(v, (uint32_t)(col[u] >> 3), (uint32_t)row[u], l, m);
      if constexpr (RES) {
        r[u].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], m.factor, w[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * m.factor;
      }
      if (valid[u] > 0) segment_store<T, VEC, LPR>(reinterpret_cast<T*>(a.out) + row[u] * a.out_pitch + col[u], valid[u], l, v);
    }
  }
}

template <typename T, bool VEC, int LPR, bool RES>
cudaError_t launch_dropout_as(DropoutArgs a, const DropoutMask& m, cudaStream_t st) {
  int64_t most = 0;
  const cudaError_t e = resident_ctas<dropout_kernel<T, VEC, LPR, RES>>(kRowThreads, &most);
  if (e != cudaSuccess) return e;
  a.segments = (uint32_t)((a.cols + LPR * 8 - 1) / (LPR * 8));
  a.row_groups = (a.rows + 32 / LPR - 1) / (32 / LPR);
  const int64_t items = a.row_groups * (int64_t)a.segments, per_cta = kRowThreads / 32;
  const int64_t ctas = items < most * per_cta ? (items + per_cta - 1) / per_cta : most;
  a.row_step = ctas * per_cta / a.segments;
  a.segment_step = (uint32_t)(ctas * per_cta % a.segments);
  dropout_kernel<T, VEC, LPR, RES><<<(unsigned)ctas, kRowThreads, 0, st>>>(a, m);
  return cudaGetLastError();
}

template <typename T, bool VEC>
cudaError_t launch_dropout(const DropoutArgs& a, const DropoutMask& m, cudaStream_t st) {
#define SWARM_DROPOUT_LPR(L) (a.residual ? launch_dropout_as<T, VEC, L, true>(a, m, st) : launch_dropout_as<T, VEC, L, false>(a, m, st))
  return a.cols <= 64 ? SWARM_DROPOUT_LPR(8) : a.cols <= 128 ? SWARM_DROPOUT_LPR(16) : SWARM_DROPOUT_LPR(32);
#undef SWARM_DROPOUT_LPR
}

// =================================================================================================
// Norm. A row belongs to LPR lanes of a warp (rows of up to 256 columns) or to WPR whole warps, each lane with VPL times
// eight of its elements in registers: segment v of warp w is segment w + v * WPR of the row. The warps of a CTA form
// groups of WPR that walk the rows with a fixed stride and fetch their next row before they reduce this one; a group of
// several warps meets once per row in shared memory at a barrier of its own.
// Few registers and many warps carry it: with a whole row of 1024 in each warp (four segments, 88 registers) 16384
// rows took 44 us forward and, with 225 registers, 69 us backward; now 25 and 35 (bf16, residual, 5.3 TB/s and 3.8 TB/s with
// the addition of dweight; 32768 rows 46 us, 5.8 TB/s, and 60 us). HBM is the bound; of the gradient about 5 us are the
// second kernel.
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

template <int LPR, int WPR> struct NormShape {
  static constexpr int kThreads = WPR <= 8 ? 256 : WPR * 32;
  static constexpr int kGroups = kThreads / (32 * WPR);                // of a CTA
  static constexpr int kRows = kGroups * (32 / LPR);                   // rows of a CTA at a time
};

template <bool VEC, int LPR>
__device__ __forceinline__ void weight_load(const float* w, int valid, int l, bool aligned, float v[8]) {
  if (VEC && aligned && l * 8 + 8 <= valid) {
    unpack8<float>(load_raw8<float>(w + l * 8), v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = segment_column<VEC, LPR>(l, i);
      v[i] = c < valid ? w[c] : 0.0f;
    }
  }
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

template <int LPR> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Sums of two values over the lanes and warps of a row, the warps added in order: the same in every thread. `slots`: two
// sets of [WPR][2] floats of the group, taken in turn (a set is written again two barriers later).
template <int LPR, int WPR>
__device__ __forceinline__ void row_sums(float& u, float& v, float (*slots)[WPR][2], int& turn, int warp_of_row, int group) {
  u = lanes_sum<LPR>(u);
  v = lanes_sum<LPR>(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 31) == 0) { slots[turn][warp_of_row][0] = u; slots[turn][warp_of_row][1] = v; }
    asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "n"(WPR * 32) : "memory");
    u = v = 0.0f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) { u += slots[turn][w][0]; v += slots[turn][w][1]; }
    turn ^= 1;
  }
}

template <typename T, bool VEC, int LPR, int WPR, int VPL, bool RES, bool CODES>
__global__ void __launch_bounds__(NormShape<LPR, WPR>::kThreads)
add_rms_norm_kernel(NormArgs a, DropoutMask m) {
  using Shape = NormShape<LPR, WPR>;
  __shared__ float slots[Shape::kGroups][2][WPR][2];
  const int lane = threadIdx.x & 31, l = lane % LPR, warp = threadIdx.x >> 5, group = warp / WPR, seg0 = warp % WPR;
  const bool w_aligned = (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0;
  int64_t row = (int64_t)blockIdx.x * Shape::kRows + group * (32 / LPR) + lane / LPR;
  // narrow rows: a warp goes on while any of its rows exists
  int64_t lead = (int64_t)blockIdx.x * Shape::kRows + group * (32 / LPR);
  Segment<T, VEC, LPR> x[VPL], r[VPL];
  auto columns = [&](int s) { return (int)min((int64_t)LPR * 8, a.cols - (int64_t)(seg0 + s * WPR) * (LPR * 8)); };
  auto fetch = [&]() {
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * (LPR * 8);
      const int valid = row < a.rows ? columns(s) : 0;
      x[s].load(reinterpret_cast<const T*>(a.x) + row * a.x_pitch + col, valid, l);
      if constexpr (RES) r[s].load(reinterpret_cast<const T*>(a.residual) + row * a.residual_pitch + col, valid, l);
    }
  };
  fetch();
  int turn = 0;
  while (lead < a.rows) {
    float t[VPL][8], sq = 0.0f, none = 0.0f;
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      x[s].get(t[s]);
      if (m.active) segment_drop<VEC, LPR>(t[s], (uint32_t)(seg0 + s * WPR) * LPR, (uint32_t)row, l, m);
      float w[8];
      if constexpr (RES) r[s].get(w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        t[s][i] = t[s][i] * m.factor;
        if constexpr (RES) t[s][i] += w[i];
        sq = fmaf(t[s][i], t[s][i], sq);
      }
    }
    const int64_t here = row;
    row += (int64_t)gridDim.x * Shape::kRows;
    lead += (int64_t)gridDim.x * Shape::kRows;
    if (lead < a.rows) fetch();
    row_sums<LPR, WPR>(sq, none, slots[group], turn, seg0, group);
    const float rstd = 1.0f / sqrtf(fmaf(sq, a.inv_cols, a.eps));
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int seg = seg0 + s * WPR;
      const int64_t col = (int64_t)seg * (LPR * 8);
      const int valid = here < a.rows ? columns(s) : 0;
      if (LPR == 32 && valid <= 0) continue;                           // the same for the whole warp
      if (a.total) segment_store<T, VEC, LPR>(reinterpret_cast<T*>(a.total) + here * a.total_pitch + col, valid, l, t[s]);
      float w[8];
      weight_load<VEC, LPR>(a.weight + col, valid, l, w_aligned, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[s][i] = t[s][i] * rstd * w[i];
      if constexpr (!CODES) {
        segment_store<T, VEC, LPR>(reinterpret_cast<T*>(a.y) + here * a.y_pitch + col, valid, l, t[s]);
      } else {
        // largest magnitude of each 128-column block, as bit patterns, so that a NaN is the largest. Consecutive elements:
        // a block is 16 lanes (or a narrow row's 8); else elements 0..3 of all lanes, and 4..7
        constexpr bool kConsecutive = VEC || LPR < 32;
        constexpr int kParts = kConsecutive ? 1 : 2;                   // blocks that a lane has elements of
        uint32_t top[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t mag = segment_column<VEC, LPR>(l, i) < valid ? __float_as_uint(t[s][i]) & 0x7FFFFFFFu : 0u;
          top[kConsecutive ? 0 : i >> 2] = max(top[kConsecutive ? 0 : i >> 2], mag);
        }
        float scale[2], inv[2];
#pragma unroll
        for (int b = 0; b < kParts; ++b) {
          if constexpr (kConsecutive) {
#pragma unroll
            for (int o = (LPR < 16 ? LPR : 16) / 2; o > 0; o >>= 1) top[b] = max(top[b], __shfl_xor_sync(0xFFFFFFFFu, top[b], o));
          } else {
            top[b] = __reduce_max_sync(0xFFFFFFFFu, top[b]);
          }
          scale[b] = __uint_as_float(top[b]) * (1.0f / 448.0f);
          if (scale[b] < 0x1p-126f) scale[b] = 0.0f;                   // its reciprocal could overflow
          inv[b] = scale[b] == 0.0f ? 0.0f : 1.0f / scale[b];
          const int64_t block = kConsecutive ? (col >> 7) + (l >> 4) : (col >> 7) + b;
          if ((kConsecutive ? (l & 15) == 0 : l == 0) && block < a.blocks && valid > 0) a.scales[here * a.blocks + block] = scale[b];
        }
        uint8_t* out = a.codes + here * a.y_pitch + col;
        if constexpr (kConsecutive) {
          const float f = inv[0];
          const uint32_t lo = e4m3x2(t[s][0] * f, t[s][1] * f) | e4m3x2(t[s][2] * f, t[s][3] * f) << 16;
          const uint32_t hi = e4m3x2(t[s][4] * f, t[s][5] * f) | e4m3x2(t[s][6] * f, t[s][7] * f) << 16;
          if (VEC && l * 8 + 8 <= valid) *reinterpret_cast<uint2*>(out + l * 8) = make_uint2(lo, hi);
          else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (l * 8 + i < valid) out[l * 8 + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int c = i * 32 + l;
            if (c < valid) out[c] = (uint8_t)e4m3x2(t[s][i] * inv[i >> 2], 0.0f);
          }
        }
      }
    }
  }
}

// =================================================================================================
// Gradient of the norm: the same walk. The weights and the lanes' parts of dweight stay in registers; the parts of a CTA
// meet in shared memory in group order, those of the CTAs in a second kernel in CTA order, so the sum over rows has one
// fixed association.
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

template <typename T, bool VEC, int LPR, int WPR, int VPL, bool PAST>
__global__ void __launch_bounds__(NormShape<LPR, WPR>::kThreads)
add_rms_norm_grad_kernel(NormGradArgs a, DropoutMask m) {
  using Shape = NormShape<LPR, WPR>;
  constexpr int kCols = LPR * 8 * WPR * VPL;                           // columns that the registers of a group cover
  constexpr int kParts = Shape::kGroups * (32 / LPR);                  // parts of dweight in a CTA
  __shared__ float slots[Shape::kGroups][2][WPR][2];
  __shared__ float parts[kParts > 1 ? kParts * kCols : 1];
  const int lane = threadIdx.x & 31, l = lane % LPR, warp = threadIdx.x >> 5, group = warp / WPR, seg0 = warp % WPR;
  const bool w_aligned = (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0;
  int64_t row = (int64_t)blockIdx.x * Shape::kRows + group * (32 / LPR) + lane / LPR;
  int64_t lead = (int64_t)blockIdx.x * Shape::kRows + group * (32 / LPR);
  auto columns = [&](int s) { return (int)min((int64_t)LPR * 8, a.cols - (int64_t)(seg0 + s * WPR) * (LPR * 8)); };
  float dw[VPL][8], w[VPL][8];
  Segment<T, VEC, LPR> dy[VPL], tot[VPL], past[VPL];
  auto fetch = [&]() {
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * (LPR * 8);
      const int valid = row < a.rows ? columns(s) : 0;
      dy[s].load(reinterpret_cast<const T*>(a.dy) + row * a.dy_pitch + col, valid, l);
      tot[s].load(reinterpret_cast<const T*>(a.total) + row * a.total_pitch + col, valid, l);
      if constexpr (PAST) past[s].load(reinterpret_cast<const T*>(a.dtotal) + row * a.dtotal_pitch + col, valid, l);
    }
  };
  fetch();
#pragma unroll
  for (int s = 0; s < VPL; ++s) {
    weight_load<VEC, LPR>(a.weight + (int64_t)(seg0 + s * WPR) * (LPR * 8), columns(s), l, w_aligned, w[s]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[s][i] = 0.0f;
  }
  int turn = 0;
  while (lead < a.rows) {
    float g[VPL][8], t[VPL][8], d[VPL][8], sq = 0.0f, dot = 0.0f;
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      dy[s].get(g[s]);
      tot[s].get(t[s]);
      if constexpr (PAST) past[s].get(d[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sq = fmaf(t[s][i], t[s][i], sq);
        dot = fmaf(g[s][i] * w[s][i], t[s][i], dot);
      }
    }
    const int64_t here = row;
    row += (int64_t)gridDim.x * Shape::kRows;
    lead += (int64_t)gridDim.x * Shape::kRows;
    if (lead < a.rows) fetch();
    row_sums<LPR, WPR>(sq, dot, slots[group], turn, seg0, group);
    const float r = 1.0f / sqrtf(fmaf(sq, a.inv_cols, a.eps));
    const float c = r * r * r * (dot * a.inv_cols);
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int seg = seg0 + s * WPR;
      const int64_t col = (int64_t)seg * (LPR * 8);
      const int valid = here < a.rows ? columns(s) : 0;
      if (LPR == 32 && valid <= 0) continue;                           // the same for the whole warp
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (here < a.rows) dw[s][i] = fmaf(g[s][i] * t[s][i], r, dw[s][i]);
        const float v = r * (g[s][i] * w[s][i]) - t[s][i] * c;
        d[s][i] = PAST ? d[s][i] + v : v;
      }
      segment_store<T, VEC, LPR>(reinterpret_cast<T*>(a.dresidual) + here * a.dresidual_pitch + col, valid, l, d[s]);
      if (a.dx) {
        if (m.active) segment_drop<VEC, LPR>(d[s], (uint32_t)seg * LPR, (uint32_t)here, l, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[s][i] = d[s][i] * m.factor;
        segment_store<T, VEC, LPR>(reinterpret_cast<T*>(a.dx) + here * a.dx_pitch + col, valid, l, d[s]);
      }
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (int64_t)blockIdx.x * a.cols;
  if constexpr (kParts > 1) {
    float* mine = parts + (group * (32 / LPR) + lane / LPR) * kCols;
#pragma unroll
    for (int s = 0; s < VPL; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) mine[(seg0 + s * WPR) * (LPR * 8) + segment_column<VEC, LPR>(l, i)] = dw[s][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += Shape::kThreads) {
      float v = parts[c];
#pragma unroll
      for (int q = 1; q < kParts; ++q) v += parts[q * kCols + c];
      out[c] = v;
    }
  } else {
#pragma unroll
    for (int s = 0; s < VPL; ++s) {
      const int64_t col = (int64_t)(seg0 + s * WPR) * (LPR * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = col + segment_column<VEC, LPR>(l, i);
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
  if (c < cols) {
#pragma unroll 8
    for (int p = run; p < parts; p += 32) v += partial[(int64_t)p * cols + c];
  }
  runs[run][lane] = v;
  __syncthreads();
  if (run == 0 && c < cols) {
    float sum = 0.0f;
#pragma unroll
    for (int q = 0; q < 32; ++q) sum += runs[q][lane];
    dweight[c] = sum;
  }
}

// Runs CALL(lanes per row, warps per row, segments per warp) for rows of `cols` columns; WIDE: the call for 2049 to 4096.
#define SWARM_NORM_SHAPES(cols, CALL, WIDE)       \
  ((cols) <= 64 ? CALL(8, 1, 1)                   \
   : (cols) <= 128 ? CALL(16, 1, 1)               \
   : (cols) <= 256 ? CALL(32, 1, 1)               \
   : (cols) <= 512 ? CALL(32, 2, 1)               \
   : (cols) <= 1024 ? CALL(32, 4, 1)              \
   : (cols) <= 2048 ? CALL(32, 8, 1)              \
   : (cols) <= 4096 ? WIDE                        \
   : (cols) <= 8192 ? CALL(32, 16, 2)             \
   : (cols) <= 16384 ? CALL(32, 16, 4)            \
                     : CALL(32, 32, 4))

template <typename T, bool VEC, int LPR, int WPR, int VPL, bool RES, bool CODES>
cudaError_t launch_norm_as(const NormArgs& a, const DropoutMask& m, cudaStream_t st) {
  using Shape = NormShape<LPR, WPR>;
  int64_t most = 0;
  const cudaError_t e = resident_ctas<add_rms_norm_kernel<T, VEC, LPR, WPR, VPL, RES, CODES>>(Shape::kThreads, &most);
  if (e != cudaSuccess) return e;
  const int64_t ctas = (a.rows + Shape::kRows - 1) / Shape::kRows;
  add_rms_norm_kernel<T, VEC, LPR, WPR, VPL, RES, CODES><<<(unsigned)(ctas < most ? ctas : most), Shape::kThreads, 0, st>>>(a, m);
  return cudaGetLastError();
}

template <typename T, bool VEC, bool CODES>
cudaError_t launch_norm(const NormArgs& a, const DropoutMask& m, cudaStream_t st) {
#define SWARM_CALL(L, W, V) (a.residual ? launch_norm_as<T, VEC, L, W, V, true, CODES>(a, m, st) : launch_norm_as<T, VEC, L, W, V, false, CODES>(a, m, st))
  // measured on 16384 x 4096 bf16: 85 us with eight warps of two segments against 90 with sixteen of one, and for the 8-bit
  // output, whose blocks' maxima want more warps at work, 103 against 100
  return SWARM_NORM_SHAPES(a.cols, SWARM_CALL, (CODES ? SWARM_CALL(32, 16, 1) : SWARM_CALL(32, 8, 2)));
#undef SWARM_CALL
}

// Parts of dweight that the workspace has room for: no gradient kernel runs with more CTAs.
constexpr int64_t kNormGradCtas = 148 * 4;

template <typename T, bool VEC, int LPR, int WPR, int VPL, bool PAST>
cudaError_t launch_norm_grad_as(const NormGradArgs& a, const DropoutMask& m, int64_t* ctas, cudaStream_t st) {
  using Shape = NormShape<LPR, WPR>;
  int64_t most = 0;
  const cudaError_t e = resident_ctas<add_rms_norm_grad_kernel<T, VEC, LPR, WPR, VPL, PAST>>(Shape::kThreads, &most);
  if (e != cudaSuccess) return e;
  if (most > kNormGradCtas) most = kNormGradCtas;
  *ctas = (a.rows + Shape::kRows - 1) / Shape::kRows;
  if (*ctas > most) *ctas = most;
  add_rms_norm_grad_kernel<T, VEC, LPR, WPR, VPL, PAST><<<(unsigned)*ctas, Shape::kThreads, 0, st>>>(a, m);
  return cudaGetLastError();
}

template <typename T, bool VEC>
cudaError_t launch_norm_grad(const NormGradArgs& a, const DropoutMask& m, int64_t* ctas, cudaStream_t st) {
#define SWARM_CALL(L, W, V) (a.dtotal ? launch_norm_grad_as<T, VEC, L, W, V, true>(a, m, ctas, st) : launch_norm_grad_as<T, VEC, L, W, V, false>(a, m, ctas, st))
  return SWARM_NORM_SHAPES(a.cols, SWARM_CALL, SWARM_CALL(32, 16, 1));               // 117 us there, 122 with eight warps
#undef SWARM_CALL
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
  const DropoutMask m = make_dropout_mask(rate, seed, event);
  const bool vec = on16(x_dev, x_pitch, size) && on16(residual_dev, residual_pitch, size) && on16(out_dev, out_pitch, size);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == SWARM_F32) return operator_result(vec ? launch_dropout<float, true>(a, m, st) : launch_dropout<float, false>(a, m, st));
  if (dtype == SWARM_BF16)
    return operator_result(vec ? launch_dropout<__nv_bfloat16, true>(a, m, st) : launch_dropout<__nv_bfloat16, false>(a, m, st));
  return operator_result(vec ? launch_dropout<__half, true>(a, m, st) : launch_dropout<__half, false>(a, m, st));
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
  return (size_t)((rows < kNormGradCtas ? rows : kNormGradCtas) * cols) * sizeof(float);
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
  int64_t ctas = 0;
  cudaError_t e;
  if (dtype == SWARM_F32) e = vec ? launch_norm_grad<float, true>(a, m, &ctas, st) : launch_norm_grad<float, false>(a, m, &ctas, st);
  else if (dtype == SWARM_BF16) e = vec ? launch_norm_grad<__nv_bfloat16, true>(a, m, &ctas, st) : launch_norm_grad<__nv_bfloat16, false>(a, m, &ctas, st);
  else e = vec ? launch_norm_grad<__half, true>(a, m, &ctas, st) : launch_norm_grad<__half, false>(a, m, &ctas, st);
  if (e == cudaSuccess && dweight_dev) {
    norm_dweight_kernel<<<(unsigned)((cols + 31) / 32), 1024, 0, st>>>(a.partial, (int)ctas, cols, dweight_dev);
    e = cudaGetLastError();
  }
  return operator_result(e);
}

int swarm_operator_error(void) { return g_operator_error; }

}  // extern "C"
