// The paged cache of keys and values as its kernels see it.
#pragma once
#include "swarm_attention.h"

namespace swarm {

struct PagedArgs {
  const void *q, *k, *v;
  void *k_pages, *v_pages, *out;
  float* lse;
  const float* frequencies;
  const int32_t *table, *lengths, *counts;
  int64_t table_pitch;
  swarm_strides kps, vps, qs, os, ks, vs;               // of the pages: .batch is the page's
  int32_t batch, heads, kv_heads, group, tokens, head_dim, pages, page_size, table_columns;
  int32_t capacity;                                     // positions that a row of the table has room for
  int32_t rotated, interleaved, window, sinks;
  float scale;
  int* status;                                          // kStatusPage is raised for pages that do not exist
};

// The sentence's tokens, and how many of them are rows of the call.
__device__ __forceinline__ int length_in(const PagedArgs& a, int b) { return max(a.lengths[b], 0); }
__device__ __forceinline__ int rows_in(const PagedArgs& a, int b, int length) {
  return min(a.counts ? min(max(a.counts[b], 0), a.tokens) : a.tokens, length);
}
// The page of a column of a sentence's table, -1 where there is none.
__device__ __forceinline__ int page_of(const PagedArgs& a, int b, int column) {
  if (column >= a.table_columns) return -1;
  const int page = a.table[b * a.table_pitch + column];
  return (uint32_t)page < (uint32_t)a.pages ? page : -1;
}

// How many CTAs, from CTA `first` on, hold parts of an item that `first` begins and `last` ends. What a CTA says of the last one
// is a number in memory: whatever it is, no part outside the `ctas` that the workspace has is read.
__host__ __device__ inline int parts_between(int first, int last, int ctas) {
  return (last < first ? first : last < ctas ? last : ctas - 1) - first + 1;
}

size_t paged_attention_workspace(const PagedArgs& a);
cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, void* workspace, cudaStream_t st);

}  // namespace swarm
