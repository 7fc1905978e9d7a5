// The attention kernels as the C entry points launch them.
#pragma once
#include <cuda.h>

#include "swarm_opsup.cuh"

namespace swarm {

constexpr int kMaxDim = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kAttentionWaitLimit = 1u << 22;     // default polls of a device-side wait

struct AttentionArgs {
  const void *q, *k, *v, *o, *dout;
  const float* lse_in;
  void *out, *dq, *dk, *dv;
  float* lse;
  // backward, per (sentence, head) padded to whole row tiles: lse and rowsum(dout * o) as factors of a product (see the
  // backward kernels), 32 bytes a row each
  uint8_t *stat_lse, *stat_delta;
  const int32_t *query_lengths, *key_lengths;
  swarm_strides qs, ks, vs, os, dos, dqs, dks, dvs;
  int32_t batch, heads, kv_heads, group, queries, keys, head_dim;
  float scale;
  uint32_t wait_limit;
  int* status;                        // raised when a device-side wait gives up
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int b, int most) {
  return lengths ? min(max(lengths[b], 0), most) : most;
}

__device__ __forceinline__ int64_t offset_of(const swarm_strides& s, int b, int t, int h) {
  return b * s.batch + t * s.token + h * s.head;
}

// A strided tensor as tiles of `rows` rows x 64 values of one head: coordinates (value, token, head, sentence), rows and
// values past the ends read as zero and are not written. A broadcast dimension (stride 0) has extent 1 in the map and
// its coordinate is multiplied by 0.
struct TileMap {
  CUtensorMap map;
  int32_t token_step, head_step, batch_step;
};
cudaError_t make_tile_map(TileMap* out, const void* p, const swarm_strides& s, int dtype, int batch, int tokens, int heads,
                          int head_dim, int rows);

cudaError_t launch_attention_forward_tc(const AttentionArgs& a, int dtype, cudaStream_t st);
// Few query rows; the workspace holds the parts of split states.
size_t attention_rows_workspace(const AttentionArgs& a);
cudaError_t launch_attention_rows(const AttentionArgs& a, int dtype, void* workspace, cudaStream_t st);
size_t attention_backward_workspace(const AttentionArgs& a);
cudaError_t launch_attention_backward_tc(AttentionArgs a, int dtype, void* workspace, cudaStream_t st);

}  // namespace swarm
