// The cache operators as the decoder's own steps launch them (bpd.hip; the kernels are built with bpd_cache.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/bpd.h"

// Self-attention of one layer: T rows of each of B sequences (or slots: seq, as length indexed by slot), queries in fp32 [B * T][heads * head_dim], results
// in the cache's type, as rows or (packed) as packed_at() of that many columns.  tree: the rows' tree in a word (0: a chain).  blocks (null: all of the prefix is seen): chosen
// ones, with `added` rows at most since the call before.
struct BlockAttention {
  bpd_cache cache;                               // of the layer
  const float* q; void* out; int packed;
  const int *length, *seq;
  unsigned long long tree;
  int B, T, heads; float scale;
  const bpd_blocks* blocks; int added;
  void* scratch; size_t scratch_bytes;           // partial results (blocks: all that bpd_attention_workspace_bytes() counts)
  int cus;
};
void launch_block_attention(const BlockAttention& a, hipStream_t stream);
// Summaries of the complete blocks of B sequences of `length` rows, of one layer
void launch_summaries(const bpd_cache& cache, const int* length, int B, int block, void* summaries, hipStream_t stream);
// Rows of accepted nodes to the end of the prefix, in all layers: accepted[b] nodes path[b * ld ..], of a prefix that has them already in length[b]
void launch_tree_move(const bpd_cache& cache, const int* path, int ld, const int* accepted, const int* length, int B, hipStream_t stream);
