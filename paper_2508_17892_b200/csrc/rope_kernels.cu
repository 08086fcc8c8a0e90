// Rotary positions: pair (a, b) of channels turns by position * f_i,
//   a' = m (a cos - b sin),  b' = m (b cos + a sin),
// pairs (i, i + R/2) or (2i, 2i + 1) of the first R channels, the rest copied.
//
// Bound by HBM: every element is read once and written once.  What could bound it instead is the trigonometry,
// 64 angles per token, so a CTA takes a few tokens, computes their angles once into shared memory and turns all of
// their heads with them.  An angle is formed in turns: position * f_i / (2 pi) in double, less its nearest
// integer, then sine and cosine of pi times twice the remainder in single precision.  So a position of 10^6 loses
// nothing against a small one (in single precision its angle would be off by 0.06 radians).
//
// One thread moves 2 x 16 bytes at a time: the two halves of eight pairs (or 16 channels next to each other), two
// such items in flight, 24 warps per SM.
#include "launch.cuh"
#include "paged_mma.cuh"
#include "rope_kernels.cuh"

namespace ilre {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTok = 4;                   // tokens of a CTA
constexpr int kRopeFlight = 2;                   // items of a thread in flight (four prompts appended: 2 61.7 us, 4 67.7)

template <bool kF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if (kF16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
// (cos, sin) of the CTA's tokens: [token][vector 0..3][segment], two pairs per float4, so that the eight threads of a
// head read 16 bytes each without bank conflicts.
struct Angles {
  float4 cs[kRopeMaxTok][4][kRopeMaxPairs / 8];
};

__device__ __forceinline__ void fill_angles(Angles& a, const RopeFreqs& f, const int32_t* pos, long long t0, int n_tok,
                                            float sign) {
  const int half = f.rotary_dim >> 1;
  for (int i = threadIdx.x; i < n_tok * half; i += blockDim.x) {
    const int tok = i / half, pair = i - tok * half;
    const double turns = static_cast<double>(pos[t0 + tok]) * f.turns[pair];
    const float r = static_cast<float>(turns - rint(turns));
    float sn, cs;
    sincospif(2.f * r, &sn, &cs);
    float* dst = reinterpret_cast<float*>(&a.cs[tok][(pair & 7) >> 1][pair >> 3]) + (pair & 1) * 2;
    dst[0] = f.scale * cs;
    dst[1] = sign * f.scale * sn;
  }
}

// Eight pairs: `lo` and `hi` are the first and second channels of the pairs (half layout) or the first and
// second eight of 16 channels (interleaved).
template <bool kF16, bool kInter>
__device__ __forceinline__ void turn8(uint4& lo, uint4& hi, const Angles& a, int tok, int seg) {
  uint32_t* l = reinterpret_cast<uint32_t*>(&lo);
  uint32_t* h = reinterpret_cast<uint32_t*>(&hi);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float4 c = a.cs[tok][v][seg];
    if (kInter) {                                // words 2v and 2v + 1 of the 16 channels hold a pair each
      uint32_t* w0 = (v < 2) ? l + 2 * v : h + 2 * v - 4;
      const float2 x = unpack2<kF16>(w0[0]), y = unpack2<kF16>(w0[1]);
      w0[0] = pack2<kF16>(fmaf(x.x, c.x, -x.y * c.y), fmaf(x.y, c.x, x.x * c.y));
      w0[1] = pack2<kF16>(fmaf(y.x, c.z, -y.y * c.w), fmaf(y.y, c.z, y.x * c.w));
    } else {
      const float2 x = unpack2<kF16>(l[v]), y = unpack2<kF16>(h[v]);
      l[v] = pack2<kF16>(fmaf(x.x, c.x, -y.x * c.y), fmaf(x.y, c.z, -y.y * c.w));
      h[v] = pack2<kF16>(fmaf(y.x, c.x, x.x * c.y), fmaf(y.y, c.z, x.y * c.w));
    }
  }
}

// Vectors (of 16 bytes) of item `seg` inside a head: rotated items first, then the copied channels.
template <bool kInter>
__device__ __forceinline__ int2 item_vectors(int seg, int rotary_dim) {
  if (kInter || seg * 16 >= rotary_dim) return make_int2(2 * seg, 2 * seg + 1);
  return make_int2(seg, seg + rotary_dim / 16);
}

template <bool kF16, bool kInter>
__global__ void __launch_bounds__(kRopeThreads)
rope_kernel(const __grid_constant__ RopeFreqs f, const RopeParams p, int tok_per_cta) {
  __shared__ Angles ang;
  grid_dep_wait();
  grid_dep_launch();
  const long long t0 = static_cast<long long>(blockIdx.x) * tok_per_cta;
  const int n_tok = static_cast<int>(min(static_cast<long long>(tok_per_cta), p.n_tokens - t0));
  fill_angles(ang, f, p.pos, t0, n_tok, p.sign);
  __syncthreads();
  const int per_head = p.head_dim >> 4, rot = f.rotary_dim >> 4;
  const int lanes = kRopeThreads / per_head;                        // heads at a time
  const int seg = threadIdx.x % per_head, first = threadIdx.x / per_head;
  if (first >= lanes) return;
  const int2 vec = item_vectors<kInter>(seg, f.rotary_dim);
  const int n_rows = n_tok * p.rows.heads;
  const uint4* in = static_cast<const uint4*>(p.rows.in);
  uint4* out = static_cast<uint4*>(p.rows.out);
  for (int r0 = first; r0 < n_rows; r0 += lanes * kRopeFlight) {
    uint4 lo[kRopeFlight], hi[kRopeFlight];
    int tok[kRopeFlight];
    long long at[kRopeFlight];
#pragma unroll
    for (int i = 0; i < kRopeFlight; ++i) {
      const int r = r0 + i * lanes;
      if (r < n_rows) {
        tok[i] = r / p.rows.heads;
        const int head = r - tok[i] * p.rows.heads;
        const long long off = ((t0 + tok[i]) * p.rows.in_stride + static_cast<long long>(head) * p.head_dim) >> 3;
        at[i] = ((t0 + tok[i]) * p.rows.out_stride + static_cast<long long>(head) * p.head_dim) >> 3;
        lo[i] = in[off + vec.x];
        hi[i] = in[off + vec.y];
      }
    }
#pragma unroll
    for (int i = 0; i < kRopeFlight; ++i) {
      if (r0 + i * lanes < n_rows) {
        if (seg < rot) turn8<kF16, kInter>(lo[i], hi[i], ang, tok[i], seg);
        out[at[i] + vec.x] = lo[i];
        out[at[i] + vec.y] = hi[i];
      }
    }
  }
}

// New rows of the paged cache: q and k turned, v copied, the rows' weights cleared.  A thread finds the sequence of
// each of the CTA's tokens by bisection of q_start; its row in the cache follows from the sequence's lengths.
template <bool kF16, bool kInter>
__global__ void __launch_bounds__(kRopeThreads)
append_kernel(const __grid_constant__ RopeFreqs f, const __grid_constant__ AppendParams p, int tok_per_cta) {
  __shared__ Angles ang;
  __shared__ int s_page[kRopeMaxTok], s_row[kRopeMaxTok];           // page -1: not written; row -1: no sequence
  grid_dep_wait();
  grid_dep_launch();
  const PagedBatch& b = p.batch;
  const long long t0 = static_cast<long long>(blockIdx.x) * tok_per_cta;
  const int n_tok = static_cast<int>(min(static_cast<long long>(tok_per_cta), b.n_tokens - t0));
  if (blockIdx.x == 0)                                              // every sequence's lengths looked at once
    for (int i = threadIdx.x; i < b.n_seqs; i += kRopeThreads) {
      const SeqSpan s = load_span(b, i);
      if (s.kv < s.n) report(b.status, kDevBadLengths);
    }
  if (threadIdx.x < n_tok) {
    const int t = static_cast<int>(t0) + threadIdx.x;
    int lo = 0, hi = b.n_seqs;                                      // first i with q_start[i + 1] > t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (b.q_start[mid + 1] > t) hi = mid; else lo = mid + 1;
    }
    int page = -1, row = -1;
    if (lo < b.n_seqs) {
      const SeqSpan s = load_span(b, lo);
      if (s.n > 0 && t >= s.q0 && s.kv >= s.n) {
        const int slot = s.kv - s.n + (t - s.q0);
        const int pg = page_of(b, lo, slot);
        row = slot & ((1 << b.page_shift) - 1);
        page = pg < b.n_pages ? pg : -1;
      }
    }
    s_page[threadIdx.x] = page;
    s_row[threadIdx.x] = row;
  }
  if (f.rotary_dim) fill_angles(ang, f, p.pos, t0, n_tok, 1.f);
  __syncthreads();
  constexpr int kDim = 128, kPerHead = kDim / 16, kLanes = kRopeThreads / kPerHead;
  const int seg = threadIdx.x % kPerHead, rot = f.rotary_dim >> 4;
  const int2 vec = item_vectors<kInter>(seg, f.rotary_dim);
  const int heads = p.q.heads + 2 * p.n_kv, n_rows = n_tok * heads;
  for (int r0 = threadIdx.x / kPerHead; r0 < n_rows; r0 += kLanes * kRopeFlight) {
    uint4 lo[kRopeFlight], hi[kRopeFlight];
    int tok[kRopeFlight];
    uint4* dst[kRopeFlight];
    bool turn[kRopeFlight];
#pragma unroll
    for (int i = 0; i < kRopeFlight; ++i) {
      const int r = r0 + i * kLanes;
      dst[i] = nullptr;
      if (r < n_rows) {
        tok[i] = r / heads;
        int h = r - tok[i] * heads;
        const int page = s_page[tok[i]], row = s_row[tok[i]];
        const long long t = t0 + tok[i];
        const uint4* src;
        turn[i] = rot > seg;
        if (h < p.q.heads) {
          src = static_cast<const uint4*>(p.q.in) + ((t * p.q.in_stride + h * kDim) >> 3);
          if (row >= 0) dst[i] = static_cast<uint4*>(p.q.out) + ((t * p.q.out_stride + h * kDim) >> 3);
        } else {
          h -= p.q.heads;
          const bool is_v = h >= p.n_kv;
          if (is_v) { h -= p.n_kv; turn[i] = false; }
          const RopeRows& rr = is_v ? p.v : p.k;
          src = static_cast<const uint4*>(rr.in) + ((t * rr.in_stride + h * kDim) >> 3);
          if (page >= 0)
            dst[i] = static_cast<uint4*>(rr.out) + ((page * (is_v ? p.v_page_stride : p.k_page_stride) +
                                                     (static_cast<long long>(row) * p.n_kv + h) * kDim) >> 3);
        }
        if (dst[i]) {
          lo[i] = src[vec.x];
          hi[i] = src[vec.y];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kRopeFlight; ++i) {
      if (dst[i]) {
        if (turn[i]) turn8<kF16, kInter>(lo[i], hi[i], ang, tok[i], seg);
        dst[i][vec.x] = lo[i];
        dst[i][vec.y] = hi[i];
      }
    }
  }
  if (p.w)
    for (int i = threadIdx.x; i < n_tok * p.n_kv; i += kRopeThreads) {
      const int tok = i / p.n_kv, g = i - tok * p.n_kv;
      if (s_page[tok] >= 0)
        p.w[((static_cast<long long>(s_page[tok]) * p.n_kv + g) << b.page_shift) + s_row[tok]] = 0.f;
    }
}

// Tokens of a CTA: four share their angles' latency where that leaves 1.5 CTAs per SM, else one for more CTAs (32 heads, 1
// against 4: 256 tokens 2.5 / 3.4 us, 1024 4.5 / 4.3, 4096 12.3 / 10.3, 16384 57 / 42; 2: 50, 8: 44).
int rope_tokens(long long n_tokens, int n_sm) { return n_tokens >= 6ll * n_sm ? kRopeMaxTok : 1; }

}  // namespace

cudaError_t launch_rope(const RopeFreqs& f, const RopeParams& p, bool f16, int n_sm, cudaStream_t st) {
  const int tok = rope_tokens(p.n_tokens, n_sm);
  const int grid = static_cast<int>((p.n_tokens + tok - 1) / tok);
  auto k = f16 ? (f.interleaved ? rope_kernel<true, true> : rope_kernel<true, false>)
               : (f.interleaved ? rope_kernel<false, true> : rope_kernel<false, false>);
  return launch_after_previous(k, grid, kRopeThreads, 0, st, f, p, tok);
}

cudaError_t launch_append(const RopeFreqs& f, const AppendParams& p, bool f16, int n_sm, cudaStream_t st) {
  const int tok = rope_tokens(p.batch.n_tokens, n_sm);
  const int grid = (p.batch.n_tokens + tok - 1) / tok;
  auto k = f16 ? (f.interleaved ? append_kernel<true, true> : append_kernel<true, false>)
               : (f.interleaved ? append_kernel<false, true> : append_kernel<false, false>);
  return launch_after_previous(k, grid, kRopeThreads, 0, st, f, p, tok);
}

}  // namespace ilre
