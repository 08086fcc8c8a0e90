// Rotary positions of whole tensors, and of new rows on their way into the paged cache.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"
#include "paged_batch.cuh"

namespace ilre {

static constexpr int kRopeMaxPairs = 128;        // rotary_dim <= 256

struct RopeFreqs {
  double turns[kRopeMaxPairs];                   // full turns per position of each channel pair
  float scale;                                   // attention factor
  int rotary_dim;                                // 0: nothing turns
  int interleaved;
};

// One kind of rows of the launch: `heads` heads of each token, in and out.
struct RopeRows {
  const void* in;
  void* out;
  long long in_stride, out_stride;               // elements from token to token
  int heads;
};

struct RopeParams {
  RopeRows rows;
  const int32_t* pos;
  long long n_tokens;
  int head_dim;
  float sign;                                    // -1: transposed
};

struct AppendParams {
  RopeRows q;                                    // heads = 0: none
  RopeRows k, v;                                 // out: the pools
  long long k_page_stride, v_page_stride;
  float* w;
  const int32_t* pos;
  int n_kv;
  PagedBatch batch;
};

cudaError_t launch_rope(const RopeFreqs& f, const RopeParams& p, bool f16, int n_sm, cudaStream_t st);
cudaError_t launch_append(const RopeFreqs& f, const AppendParams& p, bool f16, int n_sm, cudaStream_t st);

}  // namespace ilre
