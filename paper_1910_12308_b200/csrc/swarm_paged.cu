// The paged cache of keys and values: argument checks, entry points, and the kernel that appends to it.
#include <cmath>

#include "swarm_paged.h"

namespace swarm {
namespace {

// Keys and values of new tokens into their pages, keys and queries rotated on the way: each value is read and written once, HBM is
// the bound. A warp takes a token (or, where tokens are few, some heads of it). Its angles are computed once and wait in shared
// memory for all heads; a lane then takes W pairs of a head at a time, as two vectors of W values half a rotation apart, or as one
// of 2 W neighbours. Values that do not turn go the same way.
//
// The angle p f is taken in 64 bits as half turns, t = p (f / pi), brought to [-1, 1] by an exact subtraction and only then rounded
// to fp32: a rotation at position 2^31 is as good as one at the start, but for the 22 bits that t has left behind the point there.
//
// Measured on the device: 16 prompts of 512 to 1024 tokens, 32 heads of 128 on 8, 302 MB, 56 us, 5.4 TB/s (all of 1024 tokens, 403 MB,
// 69 us, 5.9); neighbouring pairs 61 us; one token of 4 sentences 2.9 us. More units of a lane at a time cost warps: two 65 us, four 90.
// Reading a unit before the sentence's length is known reads padded rows too: 69.
constexpr int kAppendWarps = 4, kAppendSms = 148;

struct AppendPlan {
  int32_t heads, units, parts;                          // heads of q, k and v together; units of a head; warps for a token
  uint32_t unit_multiplier;                             // x / units = high word of x * multiplier, for x below 2^26 and units above 1
};

template <int BYTES> struct VectorOf;
struct __align__(16) Two16 { uint4 a, b; };
template <> struct VectorOf<32> { using Type = Two16; };
template <> struct VectorOf<16> { using Type = uint4; };
template <> struct VectorOf<8> { using Type = uint2; };
template <> struct VectorOf<4> { using Type = uint32_t; };
template <> struct VectorOf<2> { using Type = uint16_t; };

template <typename T, int N> struct Pieces {            // N consecutive values, N * 2 bytes aligned (16 at most)
  using Raw = typename VectorOf<N * 2>::Type;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ float get(int i) const { return to_float<T>(reinterpret_cast<const T*>(&raw)[i]); }
  __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T*>(&raw)[i] = from_float<T>(v); }
};

template <typename T, int W, bool INTERLEAVED>
__global__ void __launch_bounds__(kAppendWarps * 32)
cache_append_kernel(PagedArgs a, AppendPlan plan) {
  __shared__ __align__(16) float2 s_turn[kAppendWarps][kMaxDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = a.rotated / 2, pairs = a.head_dim / 2;
  const int q_heads = plan.heads - 2 * a.kv_heads;
  float2* turn = s_turn[warp];
  const int64_t items = (int64_t)a.batch * a.tokens * plan.parts, all = (int64_t)gridDim.x * kAppendWarps;
  for (int64_t item = (int64_t)blockIdx.x * kAppendWarps + warp; item < items; item += all) {
    const int part = (int)(item % plan.parts), t = (int)(item / plan.parts % a.tokens), b = (int)(item / plan.parts / a.tokens);
    const int units = plan.heads * plan.units;
    const int begin = (int)((int64_t)units * part / plan.parts) + lane, end = (int)((int64_t)units * (part + 1) / plan.parts);
    const int length = length_in(a, b), n = rows_in(a, b, length), at = length - n + t;
    const bool live = t < n;
    int page = -1;
    if (live) page = page_of(a, b, at / a.page_size);
    const int slot = live ? at % a.page_size : 0;
    if (live && page < 0 && lane == 0) atomicOr(a.status, kStatusPage);
    __syncwarp();                                       // the last token's angles have been read
    for (int i = lane; i < half; i += 32) {
      const double v = (double)at * ((double)a.frequencies[i] * 0.31830988618379067154);
      float s, c;
      sincospif((float)(v - 2.0 * rint(0.5 * v)), &s, &c);
      turn[i] = make_float2(c, s);
    }
    __syncwarp();
    for (int i = begin; i < end; i += 32) {
      // head h of q (0), k (1) or v (2), the unit's first pair, and where that lies: pairs of the rotated values, then those of
      // the others, which lie half of what is left apart
      const int head = plan.units == 1 ? i : (int)__umulhi((uint32_t)i, plan.unit_multiplier);
      const int of = head < q_heads ? 0 : head < q_heads + a.kv_heads ? 1 : 2, h = of == 0 ? head : of == 1 ? head - q_heads : head - q_heads - a.kv_heads;
      const int pair = (i - head * plan.units) * W, first = INTERLEAVED ? 2 * pair : pair < half ? pair : pair + half, apart = pair < half ? half : pairs - half;
      Pieces<T, INTERLEAVED ? 2 * W : W> x{}, y{};
      if (live) {
        const T* from = reinterpret_cast<const T*>(of == 0 ? a.q : of == 1 ? a.k : a.v) + offset_of(of == 0 ? a.qs : of == 1 ? a.ks : a.vs, b, t, h) + first;
        x.load(from);
        if (!INTERLEAVED) y.load(from + apart);
      }
      T* to = nullptr;
      if (of == 0) to = reinterpret_cast<T*>(a.out) + offset_of(a.os, b, t, h) + first;
      else if (page >= 0) to = reinterpret_cast<T*>(of == 1 ? a.k_pages : a.v_pages) + offset_of(of == 1 ? a.kps : a.vps, page, slot, h) + first;
      if (!to) continue;
      if (live && of != 2 && pair < half) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          float2 cs;
          if (W == 1) {
            cs = turn[pair];
          } else {                                      // two pairs' at a time
            const float4 two = *reinterpret_cast<const float4*>(turn + pair + (e & ~1));
            cs = e & 1 ? make_float2(two.z, two.w) : make_float2(two.x, two.y);
          }
          if (INTERLEAVED) {
            const float u = x.get(2 * e), v = x.get(2 * e + 1);
            x.set(2 * e, fmaf(u, cs.x, -(v * cs.y)));
            x.set(2 * e + 1, fmaf(v, cs.x, u * cs.y));
          } else {
            const float u = x.get(e), v = y.get(e);
            x.set(e, fmaf(u, cs.x, -(v * cs.y)));
            y.set(e, fmaf(v, cs.x, u * cs.y));
          }
        }
      }
      x.store(to);
      if (!INTERLEAVED) y.store(to + apart);
    }
  }
}

template <typename T, int W, bool INTERLEAVED>
cudaError_t launch_append_as(const PagedArgs& a, cudaStream_t st) {
  AppendPlan p{};
  p.heads = (a.out ? a.heads : 0) + 2 * a.kv_heads;
  p.units = a.head_dim / (2 * W);
  p.unit_multiplier = (uint32_t)((((uint64_t)1 << 32) + p.units - 1) / p.units);
  // as many warps to a token as have a unit for each lane, while the device has room for them
  const int64_t tokens = (int64_t)a.batch * a.tokens, most = ((int64_t)p.heads * p.units + 31) / 32, room = (int64_t)kAppendSms * 16 / (tokens > 0 ? tokens : 1);
  p.parts = (int32_t)(room < 1 ? 1 : room < most ? room : most);
  const int64_t ctas = (tokens * p.parts + kAppendWarps - 1) / kAppendWarps, cap = (int64_t)kAppendSms * 64;
  cache_append_kernel<T, W, INTERLEAVED><<<(unsigned)(ctas < cap ? ctas : cap), kAppendWarps * 32, 0, st>>>(a, p);
  return cudaGetLastError();
}

// The widest vectors that the pairs of a head allow.
template <typename T>
cudaError_t launch_append(const PagedArgs& a, cudaStream_t st) {
  const int half = a.rotated / 2, rest = (a.head_dim - a.rotated) / 2;
  if (a.interleaved && a.rotated > 0) {
    if (half % 8 == 0 && rest % 8 == 0) return launch_append_as<T, 8, true>(a, st);
    return half % 4 == 0 ? launch_append_as<T, 4, true>(a, st) : half % 2 == 0 ? launch_append_as<T, 2, true>(a, st) : launch_append_as<T, 1, true>(a, st);
  }
  if (half % 8 == 0 && rest % 8 == 0) return launch_append_as<T, 8, false>(a, st);
  return half % 4 == 0 && rest % 4 == 0 ? launch_append_as<T, 4, false>(a, st) : half % 2 == 0 && rest % 2 == 0 ? launch_append_as<T, 2, false>(a, st)
                                                                             : launch_append_as<T, 1, false>(a, st);
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
  const int64_t room = (int64_t)d->table_columns * d->page_size;
  a.capacity = (int32_t)(room < 0x7FFFFFFF ? room : 0x7FFFFFFF);
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
