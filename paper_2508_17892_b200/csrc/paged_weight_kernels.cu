// Accumulated attention weight: w[t, g] += sum over the rows (token, head of g) that see t of 2^(s c2 - lse2).
// One CTA per (64 keys, kv head, sequence); each of its four warps has 16 keys as the N of mma.m16n8k16 and walks
// over the query rows 16 at a time.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "launch.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

template <bool kF16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (kF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool kF16>
__global__ void __launch_bounds__(128)
paged_weights_kernel(const PagedWeightParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = blockIdx.y, seq = blockIdx.z;
  const PagedBatch& b = p.batch;
  grid_dep_wait();
  const SeqSpan span = load_span(b, seq);
  const int key0 = blockIdx.x * 64 + warp * 16;
  if (span.n == 0 || key0 >= span.kv) return;
  const int r0 = lane >> 2, c0 = (lane & 3) * 2;
  uint32_t kb[2][8][2];                                  // [8-key half][16-channel step]
  const int ps = 1 << b.page_shift;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int key = key0 + 8 * x + r0;
    const int page = key < span.kv ? page_of(b, seq, key) : b.n_pages;
    const bool ok = page < b.n_pages;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(
        static_cast<const uint16_t*>(p.k) + (ok ? page * p.k_page_stride + (static_cast<long long>(key & (ps - 1)) * p.n_kv + g) * 128 : 0));
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      kb[x][ks][0] = ok ? src[ks * 8 + (c0 >> 1)] : 0u;
      kb[x][ks][1] = ok ? src[ks * 8 + 4 + (c0 >> 1)] : 0u;
    }
  }
  const int pre = span.kv - span.n, n_rows = span.n * p.group;
  const int first_tok = key0 > pre ? key0 - pre : 0;     // earlier tokens see none of these keys
  float acc[4] = {};
  for (int row0 = first_tok * p.group / 16 * 16; row0 < n_rows; row0 += 16) {
    uint32_t qa[8][4];
    float lse2[2];
    int lim[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = row0 + r0 + 8 * x;
      const bool ok = r < n_rows;
      const long long tok = span.q0 + (ok ? r / p.group : 0);
      const int head = g * p.group + (ok ? r % p.group : 0);
      const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.q) + tok * p.q_stride + head * 128);
      lse2[x] = p.lse[tok * p.n_q + head] * 1.44269504f;
      lim[x] = ok ? pre + r / p.group : -1;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        qa[ks][x] = ok ? src[ks * 8 + (c0 >> 1)] : 0u;
        qa[ks][2 + x] = ok ? src[ks * 8 + 4 + (c0 >> 1)] : 0u;
      }
    }
    float s[2][4] = {};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      mma16816<kF16>(s[0], qa[ks], kb[0][ks][0], kb[0][ks][1]);
      mma16816<kF16>(s[1], qa[ks], kb[1][ks][0], kb[1][ks][1]);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 8 * y + c0 + (i & 1);
        acc[2 * y + (i & 1)] += key <= lim[i >> 1] ? ex2_approx(fmaf(s[y][i], p.c2, -lse2[i >> 1])) : 0.f;
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], 4);
    acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], 8);
    acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], 16);
  }
  if (r0 == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + 8 * (i >> 1) + c0 + (i & 1);
      if (key >= span.kv) continue;
      const int page = page_of(b, seq, key);
      if (page < b.n_pages)
        atomicAdd(&p.w[((static_cast<long long>(page) * p.n_kv + g) << b.page_shift) + (key & (ps - 1))], acc[i]);
    }
}

}  // namespace

cudaError_t launch_paged_weights(const PagedWeightParams& p, bool f16, cudaStream_t st) {
  const long long rows = static_cast<long long>(p.batch.max_blocks) << p.batch.page_shift;
  const dim3 grid(static_cast<unsigned>((rows + 63) / 64), p.n_kv, p.batch.n_seqs);
  if (f16) paged_weights_kernel<true><<<grid, 128, 0, st>>>(p);
  else paged_weights_kernel<false><<<grid, 128, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace ilre
