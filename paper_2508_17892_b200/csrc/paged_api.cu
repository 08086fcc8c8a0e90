// C ABI of the paged cache: handle, argument validation, launches; and the rotary positions without a handle.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>

#include "../../include/ilre_recall.h"
#include "api_common.cuh"
#include "launch.cuh"
#include "paged_attn_kernels.cuh"
#include "paged_weight_kernels.cuh"
#include "rope_kernels.cuh"
#include "sm100_ptx.cuh"

using namespace ilre;

struct ilre_paged {
  ilre_paged_config_t cfg;
  int n_sm;
  EncodeTiledFn encode;
  const uint8_t* guard[kMaxGuards];
  int n_guards;
  float* part_o;                        // partial results of cut items
  float2* part_ml;
  uint32_t* arrived;
  float* chunk_o;
  float2* chunk_ml;
  ChunkJoin* join;
  float* w_part;
  int32_t* n_keep;                      // rows that an eviction keeps of each sequence
  int* status;
  int last_launches;
};

namespace {

constexpr int kDim = 128;
constexpr double kPi = 3.14159265358979323846;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }    // int32 and fp32 arrays; null passes

void free_all(ilre_paged* h) {
  cudaFree(h->part_o); cudaFree(h->part_ml); cudaFree(h->arrived); cudaFree(h->n_keep); cudaFree(h->chunk_o);
  cudaFree(h->chunk_ml); cudaFree(h->join); cudaFree(h->w_part); cudaFree(h->status);
}

// Full turns per position of every channel pair.  The last spec's are kept per thread: their powers take longer than a
// small call's launch.
int make_freqs(const ilre_rope_spec_t* s, int head_dim, RopeFreqs* f) {
  struct Last {
    ilre_rope_spec_t spec;
    RopeFreqs freqs;
  };
  thread_local Last last;                                // rotary_dim 0 before the first
  if (!s) {                                              // nothing turns
    std::memset(f, 0, sizeof(*f));
    return ILRE_OK;
  }
  if (!(s->theta > 1.0) || !std::isfinite(s->theta) || s->rotary_dim < 1 || s->layout < ILRE_ROPE_HALF ||
      s->layout > ILRE_ROPE_INTERLEAVED || s->scaling < ILRE_ROPE_PLAIN || s->scaling > ILRE_ROPE_YARN ||
      !(s->attn_factor >= 0.0) || !std::isfinite(s->attn_factor))
    return ILRE_ERR_INVALID_ARG;
  if (s->scaling != ILRE_ROPE_PLAIN && (!(s->factor >= 1.0) || !std::isfinite(s->factor))) return ILRE_ERR_INVALID_ARG;
  if (s->scaling >= ILRE_ROPE_BANDED &&
      (!(s->orig_len >= 1.0) || !std::isfinite(s->orig_len) || !(s->low > 0.0) || !(s->high > s->low) ||
       !std::isfinite(s->high)))
    return ILRE_ERR_INVALID_ARG;
  if (s->rotary_dim % 16 != 0 || s->rotary_dim > head_dim || s->rotary_dim > 2 * kRopeMaxPairs)
    return ILRE_ERR_UNSUPPORTED;
  const ilre_rope_spec_t& o = last.spec;
  if (last.freqs.rotary_dim != 0 && o.theta == s->theta && o.rotary_dim == s->rotary_dim && o.layout == s->layout &&
      o.scaling == s->scaling && o.factor == s->factor && o.orig_len == s->orig_len && o.low == s->low &&
      o.high == s->high && o.attn_factor == s->attn_factor) {
    *f = last.freqs;
    return ILRE_OK;
  }
  std::memset(f, 0, sizeof(*f));
  const int R = s->rotary_dim;
  double lo = 0.0, hi = 0.0;
  if (s->scaling == ILRE_ROPE_YARN) {
    const auto d = [&](double n) { return R * std::log(s->orig_len / (2.0 * kPi * n)) / (2.0 * std::log(s->theta)); };
    lo = std::fmax(std::floor(d(s->high)), 0.0);
    hi = std::fmin(std::ceil(d(s->low)), R - 1.0);
  }
  for (int i = 0; i < R / 2; ++i) {
    const double b = std::pow(s->theta, -2.0 * i / R);
    double x = b;
    if (s->scaling == ILRE_ROPE_LINEAR) x = b / s->factor;
    if (s->scaling == ILRE_ROPE_BANDED) {
      const double t = std::fmin(1.0, std::fmax(0.0, (s->orig_len * b / (2.0 * kPi) - s->low) / (s->high - s->low)));
      x = (1.0 - t) * b / s->factor + t * b;
    }
    if (s->scaling == ILRE_ROPE_YARN) {
      const double r = std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 0.001)));
      x = r * b / s->factor + (1.0 - r) * b;
    }
    f->turns[i] = x / (2.0 * kPi);
  }
  const double own = s->scaling == ILRE_ROPE_YARN ? 0.1 * std::log(s->factor) + 1.0 : 1.0;
  f->scale = static_cast<float>(s->attn_factor > 0.0 ? s->attn_factor : own);
  f->rotary_dim = R;
  f->interleaved = s->layout == ILRE_ROPE_INTERLEAVED;
  last.spec = *s;
  last.freqs = *f;
  return ILRE_OK;
}

// The batch's and the pool's numbers and pointers; fills the kernels' form.  with_q: q_start is read.
int validate_batch(const ilre_paged* h, const ilre_paged_batch_t* b, const ilre_paged_pool_t* pool, bool with_q,
                   PagedBatch* out) {
  if (!h || !b || !pool) return ILRE_ERR_INVALID_ARG;
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_q_len < 0 || b->max_blocks < 0 || pool->n_pages < 0)
    return ILRE_ERR_INVALID_ARG;
  if (b->n_seqs > 0 && ((with_q && !b->q_start_dev) || !b->kv_len_dev || (b->max_blocks > 0 && !b->block_table_dev)))
    return ILRE_ERR_INVALID_ARG;
  if (b->n_seqs > h->cfg.max_seqs ||
      static_cast<long long>(b->max_blocks) * h->cfg.page_size >= 2147483647LL - 2048)
    return ILRE_ERR_CAPACITY;
  if (!aligned4(b->q_start_dev) || !aligned4(b->kv_len_dev) || !aligned4(b->block_table_dev) || !aligned4(pool->w_dev))
    return ILRE_ERR_ALIGNMENT;
  int shift = 0;
  while ((1 << shift) < h->cfg.page_size) ++shift;
  *out = PagedBatch{b->n_seqs, b->n_tokens, b->max_q_len, b->max_blocks, shift, pool->n_pages, 0, 2147483647, b->q_start_dev,
                    b->kv_len_dev, b->block_table_dev, h->status};
  return ILRE_OK;
}

int validate_pool(const ilre_paged* h, const void* base, int64_t* stride) {
  if (!base) return ILRE_ERR_INVALID_ARG;
  const int64_t least = static_cast<int64_t>(h->cfg.page_size) * h->cfg.n_kv_heads * kDim;
  if (*stride == 0) *stride = least;
  if (*stride < least || *stride > (1ll << 38)) return ILRE_ERR_INVALID_ARG;
  if (!aligned16(base) || *stride % 8 != 0) return ILRE_ERR_ALIGNMENT;
  return ILRE_OK;
}

// Rows of `heads` heads with `stride` elements from token to token.
int validate_rows(const void* base, int64_t stride, int64_t heads, int head_dim) {
  if (!base || stride < heads * head_dim || stride > (1ll << 38)) return ILRE_ERR_INVALID_ARG;
  if (!aligned16(base) || stride % 8 != 0) return ILRE_ERR_ALIGNMENT;
  return ILRE_OK;
}

// Do n rows of a (a_row elements, a_stride from one to the next) and n rows of b share memory?  Rows of one stride are told
// apart even where they alternate (slices of one tensor); with two strides the spans count.
bool rows_overlap(const void* a, int64_t a_stride, int64_t a_row, const void* b, int64_t b_stride, int64_t b_row, int64_t n) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  const auto bytes = [n](int64_t stride, int64_t row) -> uintptr_t {       // no memory is as long as would wrap
    return (static_cast<uintptr_t>(n - 1) * static_cast<uintptr_t>(stride) + static_cast<uintptr_t>(row)) * 2;
  };
  if (a0 >= b0 + bytes(b_stride, b_row) || b0 >= a0 + bytes(a_stride, a_row)) return false;
  if (n == 1 || a_stride != b_stride) return true;
  const int64_t step = a_stride * 2, apart = static_cast<int64_t>(b0 - a0) % step;
  const int64_t behind = apart < 0 ? apart + step : apart;     // from a row of a to the next one of b
  return behind < a_row * 2 || behind + b_row * 2 > step;
}

// Rows turned in place: every thread writes what it read, so the strides must agree; other rows must not be written.
int validate_in_place(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t row, int64_t n) {
  if (in == out) return in_stride != out_stride && n > 1 ? ILRE_ERR_INVALID_ARG : ILRE_OK;
  return rows_overlap(in, in_stride, row, out, out_stride, row, n) ? ILRE_ERR_INVALID_ARG : ILRE_OK;
}

// Query rows are read by many CTAs while others write their output.
bool overlap(const void* q, int64_t q_stride, const void* out, int64_t n_tokens, int64_t row) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(q), b = reinterpret_cast<uintptr_t>(out);
  return a < b + static_cast<uintptr_t>(n_tokens * row) * 2 && b < a + static_cast<uintptr_t>((n_tokens - 1) * q_stride + row) * 2;
}

// A pool as {channel, kv head, row of the page, page}, boxes of 64 channels of one head by box_rows rows.
bool encode_pool(const ilre_paged* h, CUtensorMap* map, const void* base, int64_t page_stride, int n_pages,
                 int box_rows) {
  const cuuint64_t n_kv = h->cfg.n_kv_heads, ps = h->cfg.page_size;
  const cuuint64_t gdim[4] = {kDim, n_kv, ps, static_cast<cuuint64_t>(n_pages)};
  const cuuint64_t gstride[3] = {kDim * 2, n_kv * kDim * 2, static_cast<cuuint64_t>(page_stride) * 2};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t estride[4] = {1, 1, 1, 1};
  const CUtensorMapDataType t = h->cfg.dtype == ILRE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return h->encode(map, t, 4, const_cast<void*>(base), gdim, gstride, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Query rows as {channel, head, token}, boxes of 64 channels of one group's heads by box_tokens tokens.
bool encode_rows(const ilre_paged* h, CUtensorMap* map, const void* base, int64_t stride, int n_tokens, int group,
                 int box_tokens) {
  const cuuint64_t gdim[3] = {kDim, static_cast<cuuint64_t>(h->cfg.n_q_heads), static_cast<cuuint64_t>(n_tokens)};
  const cuuint64_t gstride[2] = {kDim * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(box_tokens)};
  const cuuint32_t estride[3] = {1, 1, 1};
  const CUtensorMapDataType t = h->cfg.dtype == ILRE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return h->encode(map, t, 3, const_cast<void*>(base), gdim, gstride, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

float softmax_scale() { return static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(kDim))); }

// Sequences whose rows (new tokens x heads of a group) fit one tile of 16 are bound by the reading of the cache and
// go to the row kernels; the others' rows share a key tile in the tensor-core kernels.  The launches follow from what
// the host knows: one sequence has one kind, and max_q_len may rule out the second.  (32 / 8 heads, us by the chunk kernel
// / by rows in tiles of 16: 5 new tokens behind 500 rows 17.0 / 17.2, behind 4096 18.4 / 21.9, 16000 25.6 / 30.5; 16
// sequences of them 21.5 / 22.3, 70 / 65, 194 / 210; of 16 new tokens 24 / 33, 72 / 122, 196 / 411.  Up to 4 new tokens,
// one tile: 8 sequences of 16000 rows 95 by rows, 111 in the chunk kernel.)
struct KernelChoice {
  int row_tokens;                                        // most new tokens of the first kind; 0: more than 16 heads
  bool rows, chunks;
};
KernelChoice choose_kernels(const ilre_paged_batch_t& b, int group) {
  KernelChoice c;
  c.row_tokens = kRowTile / group;
  c.chunks = b.max_q_len > c.row_tokens || c.row_tokens == 0;
  c.rows = c.row_tokens > 0 && (!c.chunks || b.n_seqs > 1);
  return c;
}

#define ILRE_CHECK(expr)                \
  do {                                  \
    const int rc_ = (expr);             \
    if (rc_ != ILRE_OK) return rc_;     \
  } while (0)

}  // namespace

extern "C" {

int ilre_rope(const ilre_rope_spec_t* spec, const void* x_dev, int64_t x_stride, void* out_dev, int64_t out_stride,
              const int32_t* pos_dev, int64_t n_tokens, int32_t n_heads, int32_t head_dim, int32_t dtype,
              int32_t transposed, void* cuda_stream) {
  TraceRange trace("ilre: rotary positions (Eq. 3)");
  if (!spec || n_tokens < 0 || n_heads < 1 || head_dim < 1 || dtype < ILRE_BF16 || dtype > ILRE_F16)
    return ILRE_ERR_INVALID_ARG;
  if (head_dim % 16 != 0 || head_dim > 1024) return ILRE_ERR_UNSUPPORTED;
  if (n_heads > 65535 || n_tokens > 2147483647LL) return ILRE_ERR_CAPACITY;
  RopeFreqs f;
  ILRE_CHECK(make_freqs(spec, head_dim, &f));
  if (n_tokens == 0) return ILRE_OK;
  if (!pos_dev) return ILRE_ERR_INVALID_ARG;
  if (!aligned4(pos_dev)) return ILRE_ERR_ALIGNMENT;
  ILRE_CHECK(validate_rows(x_dev, x_stride, n_heads, head_dim));
  ILRE_CHECK(validate_rows(out_dev, out_stride, n_heads, head_dim));
  ILRE_CHECK(validate_in_place(x_dev, x_stride, out_dev, out_stride, static_cast<int64_t>(n_heads) * head_dim, n_tokens));
  int dev = 0, n_sm = 0;
  ILRE_CUDA(cudaGetDevice(&dev));
  ILRE_CUDA(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
  RopeParams p;
  p.rows = RopeRows{x_dev, out_dev, x_stride, out_stride, n_heads};
  p.pos = pos_dev; p.n_tokens = n_tokens; p.head_dim = head_dim;
  p.sign = transposed ? -1.f : 1.f;
  ILRE_CUDA(launch_rope(f, p, dtype == ILRE_F16, n_sm, static_cast<cudaStream_t>(cuda_stream)));
  return ILRE_OK;
}

int ilre_paged_create(const ilre_paged_config_t* cfg, ilre_paged_t** out) {
  if (!cfg || !out) return ILRE_ERR_INVALID_ARG;
  if (cfg->n_kv_heads < 1 || cfg->n_q_heads < 1 || cfg->max_seqs < 1 || cfg->device < 0 || cfg->dtype < ILRE_BF16 ||
      cfg->dtype > ILRE_F16 || cfg->page_size < 1)
    return ILRE_ERR_INVALID_ARG;
  if (cfg->head_dim != kDim || cfg->n_q_heads % cfg->n_kv_heads != 0 || cfg->n_q_heads / cfg->n_kv_heads > 128 ||
      cfg->page_size < 16 || cfg->page_size > 1024 || (cfg->page_size & (cfg->page_size - 1)) != 0)
    return ILRE_ERR_UNSUPPORTED;
  if (cfg->max_seqs > 65535 || cfg->n_kv_heads > 1024) return ILRE_ERR_CAPACITY;
  int n_dev = 0;
  if (cudaGetDeviceCount(&n_dev) != cudaSuccess || cfg->device >= n_dev) return ILRE_ERR_CUDA;
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaDeviceProp prop;
  ILRE_CUDA(cudaGetDeviceProperties(&prop, cfg->device));
  if (prop.major != 10) return ILRE_ERR_UNSUPPORTED;
  ilre_paged* h = new (std::nothrow) ilre_paged();
  if (!h) return ILRE_ERR_NOMEM;
  std::memset(h, 0, sizeof(*h));
  h->cfg = *cfg;
  h->n_sm = prop.multiProcessorCount;
  h->encode = tensor_map_encoder();
  if (!h->encode) {
    delete h;
    return ILRE_ERR_CUDA;
  }
  if (init_paged_rows() != cudaSuccess || init_paged_chunk() != cudaSuccess || init_paged_weights() != cudaSuccess ||
      init_paged_weight_rows() != cudaSuccess || init_evict() != cudaSuccess) {
    delete h;
    return ILRE_ERR_CUDA;
  }
  const size_t ctas = static_cast<size_t>(h->n_sm) * kRowCtasPerSm;
  bool ok = dev_alloc(h, &h->part_o, ctas * 2 * kRowTile * kDim);
  ok = ok && dev_alloc(h, &h->part_ml, ctas * 2 * kRowTile);
  ok = ok && dev_alloc(h, &h->arrived, ctas);
  ok = ok && dev_alloc(h, &h->chunk_o, static_cast<size_t>(h->n_sm) * 2 * kChunkRows * kDim);
  ok = ok && dev_alloc(h, &h->chunk_ml, static_cast<size_t>(h->n_sm) * 2 * kChunkRows);
  ok = ok && dev_alloc(h, &h->join, h->n_sm);
  ok = ok && dev_alloc(h, &h->w_part, static_cast<size_t>(h->n_sm) * 2 * 256);
  ok = ok && dev_alloc(h, &h->n_keep, cfg->max_seqs);
  ok = ok && dev_alloc(h, &h->status, 1);
  if (ok) ok = cudaMemset(h->status, 0, sizeof(int)) == cudaSuccess;
  if (ok) ok = cudaMemset(h->arrived, 0, ctas * sizeof(uint32_t)) == cudaSuccess;
  if (ok) ok = cudaDeviceSynchronize() == cudaSuccess;
  if (!ok) {
    cudaGetLastError();
    free_all(h);
    delete h;
    return ILRE_ERR_NOMEM;
  }
  *out = h;
  return ILRE_OK;
}

int ilre_paged_append(ilre_paged_t* h, const ilre_paged_batch_t* batch, const ilre_rope_spec_t* spec,
                      const int32_t* pos_dev, const void* q_dev, int64_t q_stride, void* q_out_dev,
                      int64_t q_out_stride, const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                      const ilre_paged_pool_t* pool, void* cuda_stream) {
  TraceRange trace("ilre: new rows of the paged cache");
  AppendParams p;
  std::memset(&p, 0, sizeof(p));
  ILRE_CHECK(validate_batch(h, batch, pool, true, &p.batch));
  RopeFreqs f;
  ILRE_CHECK(make_freqs(spec, kDim, &f));
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return ILRE_OK;
  if ((spec && !pos_dev) || (q_dev == nullptr) != (q_out_dev == nullptr)) return ILRE_ERR_INVALID_ARG;
  if (!aligned4(pos_dev)) return ILRE_ERR_ALIGNMENT;
  int64_t ks = pool->k_page_stride, vs = pool->v_page_stride;
  ILRE_CHECK(validate_pool(h, pool->k_dev, &ks));
  ILRE_CHECK(validate_pool(h, pool->v_dev, &vs));
  ILRE_CHECK(validate_rows(k_dev, k_stride, h->cfg.n_kv_heads, kDim));
  ILRE_CHECK(validate_rows(v_dev, v_stride, h->cfg.n_kv_heads, kDim));
  if (q_dev) {
    ILRE_CHECK(validate_rows(q_dev, q_stride, h->cfg.n_q_heads, kDim));
    ILRE_CHECK(validate_rows(q_out_dev, q_out_stride, h->cfg.n_q_heads, kDim));
    const int64_t q_row = static_cast<int64_t>(h->cfg.n_q_heads) * kDim, kv_row = static_cast<int64_t>(h->cfg.n_kv_heads) * kDim;
    ILRE_CHECK(validate_in_place(q_dev, q_stride, q_out_dev, q_out_stride, q_row, batch->n_tokens));
    if (rows_overlap(k_dev, k_stride, kv_row, q_out_dev, q_out_stride, q_row, batch->n_tokens) ||
        rows_overlap(v_dev, v_stride, kv_row, q_out_dev, q_out_stride, q_row, batch->n_tokens))
      return ILRE_ERR_INVALID_ARG;
  }
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  p.q = RopeRows{q_dev, q_out_dev, q_stride, q_out_stride, q_dev ? h->cfg.n_q_heads : 0};
  p.k = RopeRows{k_dev, pool->k_dev, k_stride, 0, h->cfg.n_kv_heads};
  p.v = RopeRows{v_dev, pool->v_dev, v_stride, 0, h->cfg.n_kv_heads};
  p.k_page_stride = ks; p.v_page_stride = vs;
  p.w = pool->w_dev; p.pos = pos_dev; p.n_kv = h->cfg.n_kv_heads;
  ILRE_CUDA(launch_append(f, p, h->cfg.dtype == ILRE_F16, h->n_sm, st));
  h->last_launches = 1;
  return ILRE_OK;
}

int ilre_paged_attention(ilre_paged_t* h, const ilre_paged_batch_t* batch, const void* q_dev, int64_t q_stride,
                         const ilre_paged_pool_t* pool, void* out_dev, float* lse_out_dev, void* cuda_stream) {
  TraceRange trace("ilre: attention over the paged cache");
  PagedAttnParams p;
  std::memset(&p, 0, sizeof(p));
  ILRE_CHECK(validate_batch(h, batch, pool, true, &p.batch));
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return ILRE_OK;
  if (pool->n_pages < 1) return ILRE_ERR_INVALID_ARG;
  int64_t ks = pool->k_page_stride, vs = pool->v_page_stride;
  ILRE_CHECK(validate_pool(h, pool->k_dev, &ks));
  ILRE_CHECK(validate_pool(h, pool->v_dev, &vs));
  ILRE_CHECK(validate_rows(q_dev, q_stride, h->cfg.n_q_heads, kDim));
  if (!out_dev) return ILRE_ERR_INVALID_ARG;
  if (!aligned16(out_dev) || !aligned4(lse_out_dev)) return ILRE_ERR_ALIGNMENT;
  if (overlap(q_dev, q_stride, out_dev, batch->n_tokens, static_cast<int64_t>(h->cfg.n_q_heads) * kDim))
    return ILRE_ERR_INVALID_ARG;
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  p.q = q_dev; p.q_stride = q_stride; p.out = out_dev; p.lse = lse_out_dev;
  p.n_q = h->cfg.n_q_heads; p.n_kv = h->cfg.n_kv_heads; p.group = p.n_q / p.n_kv;
  p.c2 = softmax_scale();
  p.part_o = h->part_o; p.part_ml = h->part_ml; p.arrived = h->arrived;
  p.chunk_o = h->chunk_o; p.chunk_ml = h->chunk_ml; p.join = h->join;
  const bool f16 = h->cfg.dtype == ILRE_F16;
  const KernelChoice use = choose_kernels(*batch, p.group);
  h->last_launches = 0;
  CUtensorMap map_q, map_k, map_v;
  auto maps = [&](int tile_rows) {
    const int box = h->cfg.page_size < tile_rows ? h->cfg.page_size : tile_rows;
    return encode_pool(h, &map_k, pool->k_dev, ks, pool->n_pages, box) &&
           encode_pool(h, &map_v, pool->v_dev, vs, pool->n_pages, box);
  };
  if (use.rows) {
    if (!maps(kRowKeys)) return ILRE_ERR_CUDA;
    if (use.chunks) p.batch.q_to = use.row_tokens;
    ILRE_CUDA(launch_paged_rows(map_k, map_v, p, f16, h->n_sm, st));
    ++h->last_launches;
  }
  if (use.chunks) {
    if (!maps(128) || !encode_rows(h, &map_q, q_dev, q_stride, batch->n_tokens, p.group, 128 / p.group))
      return ILRE_ERR_CUDA;
    p.batch.q_from = use.rows ? use.row_tokens + 1 : 0;
    p.batch.q_to = 2147483647;
    ILRE_CUDA(launch_paged_chunk(map_q, map_k, map_v, p, f16, h->n_sm, st));
    h->last_launches += 2;
  }
  return ILRE_OK;
}

int ilre_paged_accumulate(ilre_paged_t* h, const ilre_paged_batch_t* batch, const void* q_dev, int64_t q_stride,
                          const float* lse_dev, const ilre_paged_pool_t* pool, void* cuda_stream) {
  TraceRange trace("ilre: accumulated attention weight");
  PagedWeightParams p;
  std::memset(&p, 0, sizeof(p));
  ILRE_CHECK(validate_batch(h, batch, pool, true, &p.batch));
  if (batch->n_tokens == 0 || batch->n_seqs == 0 || batch->max_blocks == 0) return ILRE_OK;
  if (pool->n_pages < 1 || !lse_dev || !pool->w_dev) return ILRE_ERR_INVALID_ARG;
  if (!aligned4(lse_dev)) return ILRE_ERR_ALIGNMENT;
  int64_t ks = pool->k_page_stride;
  ILRE_CHECK(validate_pool(h, pool->k_dev, &ks));
  ILRE_CHECK(validate_rows(q_dev, q_stride, h->cfg.n_q_heads, kDim));
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  p.lse = lse_dev; p.w = pool->w_dev;
  p.n_q = h->cfg.n_q_heads; p.n_kv = h->cfg.n_kv_heads; p.group = p.n_q / p.n_kv;
  p.c2 = softmax_scale();
  p.part = h->w_part; p.arrived = h->arrived;
  p.q = q_dev; p.q_stride = q_stride;
  const bool f16 = h->cfg.dtype == ILRE_F16;
  const KernelChoice use = choose_kernels(*batch, p.group);
  h->last_launches = 0;
  CUtensorMap map_q, map_k;
  if (!encode_pool(h, &map_k, pool->k_dev, ks, pool->n_pages, h->cfg.page_size < 128 ? h->cfg.page_size : 128))
    return ILRE_ERR_CUDA;
  if (use.rows) {
    if (use.chunks) p.batch.q_to = use.row_tokens;
    ILRE_CUDA(launch_paged_weight_rows(map_k, p, f16, h->n_sm, st));
    ++h->last_launches;
  }
  if (use.chunks) {
    if (!encode_rows(h, &map_q, q_dev, q_stride, batch->n_tokens, p.group, weight_tile_tokens(p.group, batch->max_q_len)))
      return ILRE_ERR_CUDA;
    p.batch.q_from = use.rows ? use.row_tokens + 1 : 0;
    p.batch.q_to = 2147483647;
    ILRE_CUDA(launch_paged_weights(map_q, map_k, p, f16, h->n_sm, st));
    ++h->last_launches;
  }
  return ILRE_OK;
}

int ilre_paged_evict(ilre_paged_t* h, const ilre_paged_batch_t* batch, int32_t budget, int32_t n_sink,
                     int32_t n_recent, int32_t per_head, const ilre_paged_pool_t* pool, const int32_t* dst_table_dev,
                     int32_t dst_blocks, int32_t* kept_out_dev, int32_t* new_len_out_dev, void* cuda_stream) {
  TraceRange trace("ilre: eviction by accumulated weight");
  EvictParams p;
  std::memset(&p, 0, sizeof(p));
  ILRE_CHECK(validate_batch(h, batch, pool, false, &p.batch));
  if (budget < 1 || n_sink < 0 || n_recent < 0) return ILRE_ERR_INVALID_ARG;
  if (static_cast<long long>(n_sink) + n_recent > budget) return ILRE_ERR_BUDGET;
  if (budget >= 2147483647 - 4096) return ILRE_ERR_CAPACITY;       // the kernels step over it by up to 4096 at a time
  if (dst_table_dev && (dst_blocks < 1 || static_cast<long long>(dst_blocks) * h->cfg.page_size < budget))
    return ILRE_ERR_INVALID_ARG;
  if (batch->n_seqs == 0) return ILRE_OK;
  if (!pool->w_dev || !kept_out_dev || !new_len_out_dev) return ILRE_ERR_INVALID_ARG;
  if (!aligned4(dst_table_dev) || !aligned4(kept_out_dev) || !aligned4(new_len_out_dev)) return ILRE_ERR_ALIGNMENT;
  int64_t ks = pool->k_page_stride, vs = pool->v_page_stride;
  ILRE_CHECK(validate_pool(h, pool->k_dev, &ks));
  ILRE_CHECK(validate_pool(h, pool->v_dev, &vs));
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  p.k = pool->k_dev; p.v = pool->v_dev; p.w = pool->w_dev; p.k_page_stride = ks; p.v_page_stride = vs;
  p.n_kv = h->cfg.n_kv_heads; p.budget = budget; p.n_sink = n_sink; p.n_recent = n_recent;
  p.per_head = per_head != 0; p.dst_table = dst_table_dev; p.dst_blocks = dst_blocks;
  p.kept = kept_out_dev; p.new_len = new_len_out_dev; p.n_keep = h->n_keep;
  if (dst_table_dev && evict_copy_blocks(p) > 2147483647LL) return ILRE_ERR_CAPACITY;
  ILRE_CUDA(launch_evict(p, h->n_sm, st));
  h->last_launches = 2;
  return ILRE_OK;
}

int ilre_paged_status(ilre_paged_t* h) {
  if (!h) return ILRE_ERR_INVALID_ARG;
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  ILRE_CUDA(cudaDeviceSynchronize());                    // the device: graphs with the handle's calls run on any stream
  int word = 0;
  ILRE_CUDA(cudaMemcpy(&word, h->status, sizeof(int), cudaMemcpyDeviceToHost));
  if (word == 0) return ILRE_OK;
  ILRE_CUDA(cudaMemset(h->status, 0, sizeof(int)));
  // a kernel that gave up (now or behind another fault) may not have counted all arrivals
  ILRE_CUDA(cudaMemset(h->arrived, 0, static_cast<size_t>(h->n_sm) * kRowCtasPerSm * sizeof(uint32_t)));
  ILRE_CUDA(cudaDeviceSynchronize());                    // before a later call, whose stream may not wait for this one
  return (word == kDevBadLengths || word == kDevBadPage) ? ILRE_ERR_BATCH : ILRE_ERR_DEVICE_WAIT;
}

int ilre_paged_last_launch_count(ilre_paged_t* h) { return h ? h->last_launches : ILRE_ERR_INVALID_ARG; }

int ilre_paged_check_guards(ilre_paged_t* h) {
  if (!h) return ILRE_ERR_INVALID_ARG;
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  ILRE_CUDA(cudaDeviceSynchronize());
  return damaged_guards(h->guard, h->n_guards);
}

int ilre_paged_destroy(ilre_paged_t* h) {
  if (!h) return ILRE_ERR_INVALID_ARG;
  DeviceGuard guard(h->cfg.device);
  if (!guard.ok) return ILRE_ERR_CUDA;
  cudaDeviceSynchronize();
  free_all(h);
  delete h;
  return ILRE_OK;
}

}  // extern "C"
