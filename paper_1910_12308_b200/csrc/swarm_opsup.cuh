// Shared by the operators of the models that the nodes train: host-side checks and error record, and the row
// segments in which dropout and the norm walk their tensors.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/swarm.h"
#include "swarm_dev.cuh"

namespace swarm {

// cudaError_t of this thread's last SWARM_ECUDA from an operator (defined in swarm_rows.cu).
extern thread_local int g_operator_error;

// The result of a launch sequence as a return code.
inline int operator_result(cudaError_t e) {
  if (e == cudaSuccess) return SWARM_OK;
  g_operator_error = (int)e;
  return SWARM_ECUDA;
}

// Multiprocessors of the current device (looked up once per device).
cudaError_t operator_sm_count(int* out);

inline size_t element_size(int32_t dtype) { return dtype == SWARM_F32 ? 4 : 2; }

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Two floats rounded to T and packed, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float& lo, float& hi);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& lo, float& hi) {
  lo = __uint_as_float(w << 16);
  hi = __uint_as_float(w & 0xFFFF0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& lo, float& hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  lo = f.x;
  hi = f.y;
}

// Eight consecutive elements of a row whose addresses are multiples of 16 bytes.
template <typename T> struct Raw8 { uint4 w[sizeof(T) == 4 ? 2 : 1]; };
template <typename T> __device__ __forceinline__ Raw8<T> load_raw8(const T* p) {
  Raw8<T> r;
  r.w[0] = *reinterpret_cast<const uint4*>(p);
  if constexpr (sizeof(T) == 4) r.w[1] = *reinterpret_cast<const uint4*>(p + 4);
  return r;
}
template <typename T> __device__ __forceinline__ void unpack8(const Raw8<T>& r, float v[8]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(r.w[0].x); v[1] = __uint_as_float(r.w[0].y); v[2] = __uint_as_float(r.w[0].z); v[3] = __uint_as_float(r.w[0].w);
    v[4] = __uint_as_float(r.w[1].x); v[5] = __uint_as_float(r.w[1].y); v[6] = __uint_as_float(r.w[1].z); v[7] = __uint_as_float(r.w[1].w);
  } else {
    unpack2<T>(r.w[0].x, v[0], v[1]); unpack2<T>(r.w[0].y, v[2], v[3]);
    unpack2<T>(r.w[0].z, v[4], v[5]); unpack2<T>(r.w[0].w, v[6], v[7]);
  }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float v[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
  }
}

// A segment is 8 LPR consecutive columns of a row, taken by LPR lanes (8, 16 or 32) of a warp, l = lane % LPR; narrow rows
// put 32 / LPR rows into a warp. Element i (0..7) of a lane is column
//   l * 8 + i    if the rows start on 16-byte boundaries (VEC): one 128-bit access per lane (two in fp32); also of narrow
//                rows that do not, element by element
//   i * 32 + l   of wide rows with any other base, pitch or width: one coalesced access per element
// `valid` counts the segment's columns that exist (<= 0: none).
template <bool VEC, int LPR> __device__ __forceinline__ int segment_column(int l, int i) { return VEC || LPR < 32 ? l * 8 + i : i * 32 + l; }

// Elements as they are stored: 128 bits where that is possible, so that a prefetched row takes few registers.
template <typename T, bool VEC, int LPR> struct Segment {
  Raw8<T> raw;
  __device__ __forceinline__ void load(const T* p, int valid, int l) {
    if (VEC && l * 8 + 8 <= valid) {
      raw = load_raw8<T>(p + l * 8);
    } else {
      T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = segment_column<VEC, LPR>(l, i);
        e[i] = c < valid ? p[c] : from_float<T>(0.0f);
      }
    }
  }
  __device__ __forceinline__ void get(float v[8]) const { unpack8<T>(raw, v); }
};
template <typename T, bool VEC, int LPR>
__device__ __forceinline__ void segment_store(T* p, int valid, int l, const float v[8]) {
  if (VEC && l * 8 + 8 <= valid) {
    store8<T>(p + l * 8, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = segment_column<VEC, LPR>(l, i);
      if (c < valid) p[c] = from_float<T>(v[i]);
    }
  }
}

// Mask of a dropout call with threshold T: a 16-bit draw below T drops the element. `limit` = T * 2^16 - 1, so that a draw in
// the high half of a word is kept iff word > limit, whatever its low half holds (T = 2^16 keeps nothing).
struct DropoutMask {
  PhiloxRoundKeys rk;
  uint32_t event, limit;
  float factor;
  int32_t active;                     // 0: T = 0, nothing is dropped
};

inline DropoutMask make_dropout_mask(double rate, uint64_t seed, uint32_t event) {
  DropoutMask m;
  m.rk = philox_round_keys((uint32_t)seed, (uint32_t)(seed >> 32));
  m.event = event;
  const uint32_t threshold = (uint32_t)(rate * 65536.0 + 0.5);
  m.active = threshold != 0;
  m.limit = (threshold << 16) - 1u;
  m.factor = threshold >= 65536 ? 0.0f : (float)(65536.0 / (double)(65536 - threshold));
  return m;
}

// Zeroes the dropped elements of a segment (the factor is left to the caller): one generator call per lane and segment
// covers the lane's eight consecutive columns; where the lane's elements are others, the keep bits of a column come from
// the lane that drew them. group0: the segment's first column div 8. All lanes of the warp call it.
template <bool VEC, int LPR>
__device__ __forceinline__ void segment_drop(float v[8], uint32_t group0, uint32_t row, int l, const DropoutMask& m) {
  const uint4 w = philox4x32_10(group0 + (uint32_t)l, row, m.event, kStreamDropout, m.rk);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
  if constexpr (VEC || LPR < 32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = (word[i] << 16) > m.limit ? v[2 * i] : 0.0f;                  // low half
      v[2 * i + 1] = word[i] > m.limit ? v[2 * i + 1] : 0.0f;                  // high half
    }
  } else {
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) keep |= ((word[i] << 16) > m.limit ? 1u << (2 * i) : 0u) | (word[i] > m.limit ? 2u << (2 * i) : 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = __shfl_sync(0xFFFFFFFFu, keep, i * 4 + (l >> 3));
      v[i] = (bits >> (l & 7)) & 1u ? v[i] : 0.0f;
    }
  }
}

}  // namespace swarm
