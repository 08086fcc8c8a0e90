// Accumulated attention weight of the paged cache's rows, and the eviction by it.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"
#include "paged_batch.cuh"

namespace ilre {

struct PagedWeightParams {
  PagedBatch batch;
  const void* q;                                 // read by the row kernel without a map
  long long q_stride;
  const float* lse;                              // [n_tokens][n_q]
  float* w;                                      // [n_pages][n_kv][page_size]
  int n_q, n_kv, group;
  float c2;
  float* part;                                   // [CTA][2][256]: sums of the pieces of cut items
  uint32_t* arrived;                             // [CTA][2], 0 between launches
};

struct EvictParams {
  PagedBatch batch;
  int n_kv, budget, n_sink, n_recent, per_head;
  const int32_t* dst_table;                      // null: in place
  int dst_blocks;
  void* k;
  void* v;
  float* w;
  long long k_page_stride, v_page_stride;        // elements
  int32_t* kept;                                 // [n_seqs][rows][budget]
  int32_t* new_len;                              // [n_seqs]
  int32_t* n_keep;                               // workspace [max_seqs]: rows that stay, -1: sequence left out
};

// Shared memory of the kernels, once per device.
cudaError_t init_paged_weights();
cudaError_t init_paged_weight_rows();
cudaError_t init_evict();

// Query tokens of a row tile: up to 64 rows (one token of a larger group), or all that any sequence has.
int weight_tile_tokens(int group, int max_q_len);
// map_q: {channel, head, token}, boxes of 64 channels x group x weight_tile_tokens; map_k: the pool as {channel, kv head,
// row, page}, boxes of 64 channels x min(page_size, 128) rows.
cudaError_t launch_paged_weights(const CUtensorMap& map_q, const CUtensorMap& map_k, const PagedWeightParams& p, bool f16,
                                 int n_sm, cudaStream_t st);
// Sequences of at most 16 rows (new tokens x heads of a group).
cudaError_t launch_paged_weight_rows(const CUtensorMap& map_k, const PagedWeightParams& p, bool f16, int n_sm,
                                     cudaStream_t st);
long long evict_copy_blocks(const EvictParams& p);     // CTAs per sequence of the copy to other pages, < 2^31
cudaError_t launch_evict(const EvictParams& p, int n_sm, cudaStream_t st);

}  // namespace ilre
