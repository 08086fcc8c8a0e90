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
  const void* q;
  long long q_stride;
  const void* k;                                 // pool
  long long k_page_stride;
  const float* lse;                              // [n_tokens][n_q]
  float* w;                                      // [n_pages][n_kv][page_size]
  int n_q, n_kv, group;
  float c2;
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

cudaError_t launch_paged_weights(const PagedWeightParams& p, bool f16, cudaStream_t st);
cudaError_t launch_evict(const EvictParams& p, int n_sm, cudaStream_t st);

}  // namespace ilre
