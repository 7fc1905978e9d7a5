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
  // fp16: the largest |ds| (without the factor scale; 2^-7 sum |dout| at least) of 32 rows, [batch][heads][row tiles][4][parts of dq]
  float* stat_peak;
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

// A call whose states are split over CTAs: their parts of every row (query token x query head of a key head), joined by a
// kernel of their own.
constexpr int kMaxSplits = 32;                          // a lane of the joining warp each
struct SplitPlan {
  int32_t rows;                       // of a key head: queries * group
  int32_t splits;
  float* part_o;                      // [batch][kv_heads][rows][splits][head_dim] weighted sums
  float* part_ml;                     // [batch][kv_heads][rows][splits][2] their maximum and the sum of the weights
};
inline size_t split_parts(const AttentionArgs& a, const SplitPlan& p) { return (size_t)a.batch * a.kv_heads * p.rows * p.splits; }
inline size_t split_bytes(const AttentionArgs& a, const SplitPlan& p) {
  return p.splits == 1 ? 0 : split_parts(a, p) * (a.head_dim + 2) * sizeof(float) + 16;
}
inline void place_parts(const AttentionArgs& a, SplitPlan* p, void* workspace) {
  p->part_o = reinterpret_cast<float*>(workspace);
  p->part_ml = p->part_o + split_parts(a, *p) * a.head_dim;
}
// Device address of the current device's word that swarm_operator_check reads (defined in swarm_attention.cu): bit 0, a
// device-side wait gave up; bit 1, a table named a page that does not exist.
cudaError_t status_word(int** out);
constexpr int kStatusWait = 1, kStatusPage = 2;

cudaError_t launch_attention_join(const AttentionArgs& a, const SplitPlan& p, int dtype, cudaStream_t st);

size_t attention_forward_workspace(const AttentionArgs& a);
cudaError_t launch_attention_forward_tc(const AttentionArgs& a, int dtype, void* workspace, cudaStream_t st);
// Few query rows; the workspace holds the parts of split states.
size_t attention_rows_workspace(const AttentionArgs& a);
cudaError_t launch_attention_rows(const AttentionArgs& a, int dtype, void* workspace, cudaStream_t st);
size_t attention_backward_workspace(const AttentionArgs& a);
cudaError_t launch_attention_backward_tc(AttentionArgs a, int dtype, void* workspace, cudaStream_t st);

}  // namespace swarm
