// Attention of new tokens over the paged cache.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"
#include "paged_batch.cuh"

namespace ilre {

static constexpr int kRowTile = 16;              // query rows of a work item of the row kernel
static constexpr int kRowKeys = 64;              // keys of a stage
static constexpr int kRowCtasPerSm = 2;
static constexpr int kChunkRows = 256;           // query rows of a work item of the chunk kernel

// The probabilities are rounded to the cache's type for their product with the values, which the tensor cores take no
// other way at this rate: half a step each (bf16 2^-8, fp16 2^-11), as the output; their sum is of the unrounded ones.
// Against 64 bits the output's error is 1.4 times the 32-bit form's (bf16 0.0023 against 0.0017 of its norm).
// fp16 ends at 2^-24, and in a long cache most of a row's weight may lie in probabilities below that times the largest
// (2^17 of 2^-26 each came out as nothing), so there they are held 2^kRowShift or 2^kChunkShift times as large, sum and output
// alike: the quotient does not change, and the logarithm takes it off again.  The largest is then 2^15.
static constexpr float kRowShift = 15.f;         // the row kernel's reference is the maximum itself
static constexpr float kChunkSlack = 8.f;        // the chunk kernel's may lag behind it by 2^8: the output is rescaled less often
static constexpr float kChunkShift = 7.f;

// The cut item that begins in a CTA's share: its last CTA (-1: there is none), first token, tokens, kv head.
struct ChunkJoin {
  int c_last, token, n_tok, head;
};

struct PagedAttnParams {
  PagedBatch batch;
  const void* q;
  long long q_stride;                            // elements from token to token
  void* out;                                     // [n_tokens][n_q][128]
  float* lse;                                    // [n_tokens][n_q] or null
  int n_q, n_kv, group;
  float c2;                                      // log2(e) / sqrt(d)
  float* part_o;                                 // [CTA][2][rows][128]
  float2* part_ml;                               // [CTA][2][rows]: (maximum in log2 units, sum)
  uint32_t* arrived;                             // [CTA], 0 between launches
  float* chunk_o;                                // the chunk kernel's: [CTA][2][32][kChunkRows][4]
  float2* chunk_ml;                              // [CTA][2][kChunkRows]
  ChunkJoin* join;                               // [CTA]
};

// Shared memory of the kernels, once per device.
cudaError_t init_paged_rows();
cudaError_t init_paged_chunk();

// map_k, map_v: the pools as {channel, kv head, row, page}, boxes of 64 channels x min(page_size, kRowKeys) rows.
cudaError_t launch_paged_rows(const CUtensorMap& map_k, const CUtensorMap& map_v, const PagedAttnParams& p, bool f16,
                              int n_sm, cudaStream_t st);

// map_q: {channel, head, token}, boxes of 64 channels x group x 128 / group; map_k, map_v: as above with boxes of
// min(page_size, 128) rows.
cudaError_t launch_paged_chunk(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                               const PagedAttnParams& p, bool f16, int n_sm, cudaStream_t st);

}  // namespace ilre
