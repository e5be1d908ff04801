// Attention over packed sequences (include/moeca_attention.h): the call, its
// choice of kernel, the CUDA-core kernel and the join of key chunks.
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "moeca_probe.h"
#include "packed_attn.cuh"

namespace moeca {
namespace {

// ---------------------------------------------------------------------------
// The CUDA-core kernel: fp32 values (the debug path), and bf16 rows that the
// tensor-core kernels do not take (heads above 128 values, rows that do not
// start at 16 bytes).  A block works on BQ queries of one head; 16 x 16 threads,
// BQ / 16 rows and two keys each for the scores, BQ / 16 rows and four channels
// in every 64 for the sums.  One pass over the keys, 32 at a time, with a running
// maximum m and sum l per row:
//   m' = max(m, max_j s_j), o <- o 2^((m - m') c) + sum_j 2^((s_j - m') c) v_j,
// s = q . k, c = scale log2(e).  The difference comes before the product: of s c - m c
// the compiler would make a fused multiply-add, whose exponent at s = m is the rounding of
// m c, a power of two of its own for scores of 2^31.  Bound by FFMA and the shared-memory reads beside it (24.3 ms for
// prompts of 16384 tokens, 32 heads of 128, bf16: 24 TFLOP/s); four texts of 16 to 121 tokens,
// 12 heads of 64 in fp32, take 22 us, the latency of four blocks of keys.
// ---------------------------------------------------------------------------
constexpr int kSimtThreads = 256, kSimtKeys = 32;
constexpr int kSimtPitch = kSimtKeys + 4;  // floats from row to row of p

// Floats from row to row of q, k and v: the next multiple of 4 that is an odd
// number of 16-byte pieces, so that eight rows' pieces fall in distinct banks.
__host__ __device__ constexpr int simt_pitch(int dim) { return (dim + 3) / 4 % 2 ? (dim + 3) / 4 * 4 : (dim + 3) / 4 * 4 + 4; }
constexpr size_t simt_smem(int rows, int dim) {
  return (static_cast<size_t>(rows + 2 * kSimtKeys) * simt_pitch(dim) + rows * kSimtPitch) * 4;
}

// `rows` rows of one head into shared memory as floats, zeros from row `n` on and past dim.
template <typename T>
__device__ __forceinline__ void load_rows(float* dst, int pitch, const T* src, int64_t stride, int rows, int n, int dim,
                                          bool vec) {
  constexpr int V = Elem<T>::kVec;
  if (vec) {
    const int units = dim / V;
    for (int i = threadIdx.x; i < rows * units; i += kSimtThreads) {
      const int r = i / units, u = i - r * units;
      float f[V] = {};
      if (r < n) load_vec(src + r * stride + u * V, f);
#pragma unroll
      for (int j = 0; j < V; j += 4) store_vec(dst + r * pitch + u * V + j, f + j);
    }
  } else {
    const int width = (dim + 3) / 4 * 4;
    for (int i = threadIdx.x; i < rows * width; i += kSimtThreads) {
      const int r = i / width, c = i - r * width;
      dst[r * pitch + c] = r < n && c < dim ? Elem<T>::to_f(src[r * stride + c]) : 0.f;
    }
  }
}

__device__ __forceinline__ float group16_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float group16_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T, int BQ, int DC>  // DC: channels in 64s
__global__ void __launch_bounds__(kSimtThreads) attn_simt_kernel(const __grid_constant__ PackedAttnArgs a, const bool vec) {
  constexpr int R = BQ / 16;
  extern __shared__ float4 smem4[];
  pdl_entry();
  const int index = blockIdx.x / static_cast<uint32_t>(a.q.heads), h = blockIdx.x - index * a.q.heads;
  const AttnWork w = attn_work(a, index);
  clear_rest<T>(a, w, index, h, a.q.heads, threadIdx.x, kSimtThreads);
  if (!w.any) return;
  const int dim = a.dim, pitch = simt_pitch(dim);
  float* sq = reinterpret_cast<float*>(smem4);
  float* sk = sq + BQ * pitch;
  float* sv = sk + kSimtKeys * pitch;
  float* sp = sv + kSimtKeys * pitch;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int rows = min(BQ, min(w.nq, a.max_q) - w.row0);
  const T* q = static_cast<const T*>(a.q.data) + static_cast<int64_t>(w.q0 + w.row0) * a.q.token_stride + h * a.q.head_stride;
  const T* k = static_cast<const T*>(a.k.data) + static_cast<int64_t>(w.k0) * a.k.token_stride + h / a.group * a.k.head_stride;
  const T* v = static_cast<const T*>(a.v.data) + static_cast<int64_t>(w.k0) * a.v.token_stride + h / a.group * a.v.head_stride;
  load_rows(sq, pitch, q, a.q.token_stride, BQ, rows, dim, vec);
  float m[R], l[R], o[R][DC][4];
  int see[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    see[r] = visible_keys(a, w, w.row0 + ty * R + r);
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[r][c][j] = 0.f;
  }
  // The last row of the tile sees the most.
  const int end = min(w.key_hi, visible_keys(a, w, w.row0 + rows - 1));
  const int d4 = (dim + 3) / 4;
  for (int key0 = w.key_lo; key0 < end; key0 += kSimtKeys) {
    const int n = min(kSimtKeys, w.key_hi - key0);
    __syncthreads();
    load_rows(sk, pitch, k + key0 * a.k.token_stride, a.k.token_stride, kSimtKeys, n, dim, vec);
    load_rows(sv, pitch, v + key0 * a.v.token_stride, a.v.token_stride, kSimtKeys, n, dim, vec);
    __syncthreads();
    float s[R][2] = {};
    for (int c = 0; c < d4; ++c) {
      const float4 k0 = *reinterpret_cast<const float4*>(sk + tx * pitch + 4 * c);
      const float4 k1 = *reinterpret_cast<const float4*>(sk + (tx + 16) * pitch + 4 * c);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(sq + (ty * R + r) * pitch + 4 * c);
        s[r][0] = fmaf(x.x, k0.x, fmaf(x.y, k0.y, fmaf(x.z, k0.z, fmaf(x.w, k0.w, s[r][0]))));
        s[r][1] = fmaf(x.x, k1.x, fmaf(x.y, k1.y, fmaf(x.z, k1.z, fmaf(x.w, k1.w, s[r][1]))));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int limit = min(see[r], w.key_hi) - key0;
      if (tx >= limit) s[r][0] = -INFINITY;
      if (tx + 16 >= limit) s[r][1] = -INFINITY;
      // A score that is not a number reaches p through s, not through the maximum.
      const float top = fmaxf(m[r], group16_max(fmaxf(s[r][0], s[r][1])));
      const float ref = top == -INFINITY ? 0.f : top;
      const float keep = exp2f((m[r] - ref) * a.scale_log2);
      s[r][0] = exp2f((s[r][0] - ref) * a.scale_log2);
      s[r][1] = exp2f((s[r][1] - ref) * a.scale_log2);
      l[r] = l[r] * keep + group16_sum(s[r][0] + s[r][1]);
      m[r] = top;
      sp[(ty * R + r) * kSimtPitch + tx] = s[r][0];
      sp[(ty * R + r) * kSimtPitch + tx + 16] = s[r][1];
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[r][c][j] *= keep;
    }
    __syncwarp();  // a row's p is written and read by the same half warp
    for (int j = 0; j < n; j += 4) {
      float4 p[R];
#pragma unroll
      for (int r = 0; r < R; ++r) p[r] = *reinterpret_cast<const float4*>(sp + (ty * R + r) * kSimtPitch + j);
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        const int at = c * 64 + tx * 4;
        if (at >= dim) continue;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const float4 x = *reinterpret_cast<const float4*>(sv + (j + jj) * pitch + at);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float pr = jj == 0 ? p[r].x : jj == 1 ? p[r].y : jj == 2 ? p[r].z : p[r].w;
            o[r][c][0] = fmaf(pr, x.x, o[r][c][0]);
            o[r][c][1] = fmaf(pr, x.y, o[r][c][1]);
            o[r][c][2] = fmaf(pr, x.z, o[r][c][2]);
            o[r][c][3] = fmaf(pr, x.w, o[r][c][3]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = w.row0 + ty * R + r;
    if (ty * R + r >= rows) continue;
    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
    const float lse2 = l[r] == 0.f ? -INFINITY : m[r] * a.scale_log2 + log2f(l[r]);
    if (a.ks.unit && w.nk > a.ks.unit) {
      const int64_t at = (static_cast<int64_t>(w.piece) * a.max_q + i) * a.q.heads + h;
      if (tx == 0) a.part_ml[at] = make_float2(m[r], l[r]);
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c * 64 + tx * 4 + j < dim) a.part_o[at * dim + c * 64 + tx * 4 + j] = o[r][c][j] * inv;
    } else {
      if (tx == 0 && a.lse) a.lse[static_cast<int64_t>(w.q0 + i) * a.q.heads + h] = lse2 * kLn2;
      T* out = static_cast<T*>(a.out.data) + static_cast<int64_t>(w.q0 + i) * a.out.token_stride + h * a.out.head_stride;
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c * 64 + tx * 4 + j < dim) out[c * 64 + tx * 4 + j] = Elem<T>::from_f(o[r][c][j] * inv);
    }
  }
}

// ---------------------------------------------------------------------------
// Join of a (query, head)'s chunks.  With m_j and l_j the chunks' maxima and sums, m the
// largest maximum, c = scale log2(e) and w_j = 2^((m_j - m) c) l_j:
//   o = sum_j w_j o_j / sum_j w_j.
// W warps share a row: each adds every W-th chunk, and the W sums are added in
// their order.  Few rows with many chunks take a block of eight, so that the loads of
// many chunks are in flight at once (171 chunks of 32 rows took one warp a row 80 us);
// many rows, whose chunks are few, a warp each (2048 tokens, 8 heads of 128 in two
// chunks: 29 us with the kernel before it, 66 with a block each).
// ---------------------------------------------------------------------------
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
constexpr int64_t kJoinFewRows = 2048;  // up to here a block per row

template <typename T, int C, int W>  // C: channels of a lane, 32 apart
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const PackedAttnArgs a) {
  __shared__ float sh[W > 1 ? W : 1][32 * C];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t row = W > 1 ? blockIdx.x : blockIdx.x * kJoinWarps + warp;
  const int t = row / static_cast<uint32_t>(a.q.heads), h = row - t * a.q.heads;
  pdl_entry();
  const bool some = t < a.qs.total;
  const int b = some ? a.qs.owner(t) : 0, i = some ? t - a.qs.start(b) : -1;
  const bool mine = i >= 0 && i < min(a.qs.length(b), a.max_q);
  const int chunks = static_cast<int>((static_cast<uint32_t>(a.ks.length(b)) + a.ks.unit - 1) / a.ks.unit);
  if (!mine || chunks == 1) return;  // one chunk: the kernel before this one wrote it
  const int first = a.ks.chunk(b, 0), others = a.ks.chunk(b, 1) - 1;
  const auto at = [&](int j) { return (static_cast<int64_t>(j == 0 ? first : others + j) * a.max_q + i) * a.q.heads + h; };
  float m = -INFINITY;
  for (int j = lane; j < chunks; j += 32) m = fmaxf(m, a.part_ml[at(j)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float ref = m == -INFINITY ? 0.f : m;
  // A lane forms the weight of one chunk in 32, and all lanes take it from there.
  float sum = 0.f, o[C] = {};
  for (int j0 = 0; j0 < chunks; j0 += 32) {
    float own = 0.f;
    if (j0 + lane < chunks) {
      const float2 ml = a.part_ml[at(j0 + lane)];
      own = exp2f((ml.x - ref) * a.scale_log2) * ml.y;
    }
    sum += own;
    const int n = min(32, chunks - j0);
#pragma unroll W > 1 ? 4 : 2
    for (int j = W > 1 ? warp : 0; j < n; j += W) {
      const float w = __shfl_sync(0xffffffffu, own, j);
      const float* part = a.part_o + at(j0 + j) * a.dim;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (c * 32 + lane < a.dim) o[c] = fmaf(w, part[c * 32 + lane], o[c]);
    }
  }
  sum = warp_sum(sum);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.out.data) + t * a.out.token_stride + h * a.out.head_stride;
  if (lane == 0 && (W == 1 || warp == 0) && a.lse)
    a.lse[static_cast<int64_t>(t) * a.q.heads + h] = sum == 0.f ? -INFINITY : (ref * a.scale_log2 + log2f(sum)) * kLn2;
  if constexpr (W == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c * 32 + lane < a.dim) out[c * 32 + lane] = Elem<T>::from_f(o[c] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) sh[warp][c * 32 + lane] = o[c];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += kJoinThreads) {
      float v = 0.f;
#pragma unroll
      for (int u = 0; u < W; ++u) v += sh[u][c];
      out[c] = Elem<T>::from_f(v * inv);
    }
  }
}

template <typename T, int BQ>
cudaError_t simt(const PackedAttnArgs& a, bool vec, int64_t blocks, cudaStream_t s) {
  const size_t smem = simt_smem(BQ, a.dim);
  const auto run = [&](auto kernel) {
    if (smem > 48 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(simt_smem(BQ, 256)));
      if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kSimtThreads), smem, s, a, vec);
  };
  if (a.dim <= 64) return run(attn_simt_kernel<T, BQ, 1>);
  if (a.dim <= 128) return run(attn_simt_kernel<T, BQ, 2>);
  return run(attn_simt_kernel<T, BQ, 4>);
}

}  // namespace

cudaError_t launch_attn_simt(const PackedAttnArgs& a, int dtype, int tile, cudaStream_t s) {
  const int64_t es = elem_size(dtype), n = 16 / es;
  const auto fits = [&](const Heads& h) { return addr(h.data) % 16 == 0 && h.token_stride % n == 0 && h.head_stride % n == 0; };
  const bool vec = a.dim % n == 0 && fits(a.q) && fits(a.k) && fits(a.v);
  const int64_t blocks = (a.ks.unit ? a.k_pieces * a.tiles : a.q_pieces) * a.q.heads;
  if (dtype == MOECA_BF16)
    return tile == 16 ? simt<__nv_bfloat16, 16>(a, vec, blocks, s) : simt<__nv_bfloat16, 32>(a, vec, blocks, s);
  return tile == 16 ? simt<float, 16>(a, vec, blocks, s) : simt<float, 32>(a, vec, blocks, s);
}

cudaError_t launch_attn_join(const PackedAttnArgs& a, int dtype, cudaStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.qs.total) * a.q.heads;
  const auto run = [&](auto kernel, int64_t blocks) {
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kJoinThreads), 0, s, a);
  };
  const auto pick = [&](auto* t, auto c) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (rows <= kJoinFewRows) return run(attn_join_kernel<T, c.value, kJoinWarps>, rows);
    return run(attn_join_kernel<T, c.value, 1>, (rows + kJoinWarps - 1) / kJoinWarps);
  };
  using Four = std::integral_constant<int, 4>;
  using Eight = std::integral_constant<int, 8>;
  if (dtype == MOECA_BF16) {
    __nv_bfloat16* t = nullptr;
    return a.dim <= 128 ? pick(t, Four()) : pick(t, Eight());
  }
  float* t = nullptr;
  return a.dim <= 128 ? pick(t, Four()) : pick(t, Eight());
}

namespace {

constexpr unsigned long long kWaitNs = 1000000000ull;  // a wait gives up after a second
thread_local unsigned long long g_wait_ns = kWaitNs;
thread_local int g_stall = MOECA_ATTENTION_NONE;

constexpr int64_t kMaxTokens = 1 << 30;
constexpr int kMaxHeadDim = 256, kMaxSeqs = 1 << 20;
constexpr int64_t kMaxWorkspace = int64_t(1) << 30;  // beyond, the key axis is not cut

struct Plan {
  int rows;           // tiles of 128 rows per block of the tensor-core kernel; 0: the CUDA-core kernel, -1: the one for few rows
  int tile;           // query tokens of a tile
  int chunk;          // keys of a chunk, 0: not cut
  int max_q, tiles;
  int64_t q_pieces, k_pieces;
  int q_per, k_per;
  int firsts;         // chunks are numbered with every sequence's first in front
  int64_t blocks;
  int64_t ml_bytes, bytes;  // workspace: the maxima and sums, all of it
};

int64_t pieces(const int32_t* off, int64_t total, int n, int unit, int most, int* per) {
  // Sequences of known or bounded length have the same number of pieces, or the
  // pieces follow the offsets, whichever are fewer.
  const int64_t each = ((off ? std::min<int64_t>(most, total) : total / n) + unit - 1) / unit;
  const int64_t packed = total / unit + n;
  *per = 0;
  if (!off || each * n <= packed) {
    *per = static_cast<int>(std::max<int64_t>(each, 1));
    return each * n;
  }
  return packed;
}

// Whether the tensor-core kernels can take the heads: pieces of 16 bytes everywhere, and
// strides that a tensor map takes (one value for several tokens or heads, stride 0, is none).
bool fits_tc(const moeca_heads& h, int64_t tokens) {
  const auto stride = [](int64_t s, int64_t n) { return n == 1 || (s > 0 && s % 8 == 0 && s < (int64_t(1) << 38)); };
  return tokens == 0 || (addr(h.data) % 16 == 0 && stride(h.token_stride, tokens) && stride(h.head_stride, h.heads));
}

// A GB300's, not the current device's: the plan follows from the arguments alone, so that a workspace asked for with
// another device current is the one that the call needs.
constexpr int kSms = 152;
constexpr int64_t kLongKeys = 4096, kKeysSaved = 1536, kKeysUneven = 8192;

// How a call is carried out: a function of its sizes, type and alignment.
Plan plan_attention(const moeca_attention_args& a) {
  Plan p{};
  const int64_t most = a.q_offsets ? a.n_queries : a.n_queries / a.n_seqs;
  p.max_q = static_cast<int>(a.max_q > 0 ? std::min<int64_t>(a.max_q, most) : most);
  const int group = a.q.heads / a.k.heads;
  int heads, fill, least;  // blocks of a tile, blocks that fill the GPU, keys of a chunk at least
  if (a.dtype == MOECA_BF16 && a.dim % 8 == 0 && a.dim <= 128 && group <= 128 && fits_tc(a.q, a.n_queries) &&
      fits_tc(a.k, a.n_keys) && fits_tc(a.v, a.n_keys) && fits_tc(a.out, a.n_queries)) {
    heads = a.k.heads;
    if (static_cast<int64_t>(p.max_q) * group <= 16) {
      p.rows = -1;
      p.tile = std::max(p.max_q, 1);
      fill = 0;
      least = 512;
    } else {
      const int each = 128 / group;
      // One tile a block where all blocks then run at once, two an SM, and keys are too few to be cut (2 x 1024
      // tokens, 8 heads of 64: 12.9 us, with two tiles 14.2; 2048 tokens, 8 heads of 128: 26.7 and 28.7).
      int per;
      const bool at_once = pieces(a.q_offsets, a.n_queries, a.n_seqs, each, p.max_q, &per) * heads <= 2 * kSms;
      p.rows = p.max_q <= each || (at_once && a.n_keys < a.n_seqs * kLongKeys) ? 1 : 2;
      p.tile = p.rows * each;
      fill = p.rows == 1 ? 2 * kSms : kSms;
      least = 512;
    }
  } else {
    p.tile = p.max_q <= 16 ? 16 : 32;
    heads = a.q.heads;
    fill = 4 * kSms;
    least = 256;
  }
  p.q_pieces = pieces(a.q_offsets, a.n_queries, a.n_seqs, p.tile, p.max_q, &p.q_per);
  p.tiles = (p.max_q + p.tile - 1) / p.tile;
  p.blocks = p.q_pieces * heads;
  // Few blocks with many keys each: the key axis is cut so that the chunks' blocks fill the GPU once.
  // For few rows, whose blocks are small, it is cut wherever a chunk is shorter than a sequence may be: into
  // two blocks an SM (as many as run at once; four sequences of 131072 keys in all, 8 x 128, take 94 us so and with six
  // blocks an SM), and six of up to 64 channels (four run at once, and sequences of different lengths share
  // the GPU more evenly: 64 sequences of 131072 keys in all, 8 x 64, take 51 us, with two 57).
  if (p.blocks > 0 && (p.rows < 0 || 2 * p.blocks <= fill)) {
    const int64_t mean = a.n_keys / a.n_seqs;
    int64_t chunk;
    if (p.rows < 0) {
      chunk = a.n_keys * heads / ((a.dim <= 64 ? 6 : 2) * kSms);
    } else {
      const int64_t cuts = fill / p.blocks;
      chunk = (mean + cuts - 1) / cuts;
    }
    chunk = std::max<int64_t>(least, (chunk + 127) / 128 * 128);
    const int64_t longest = a.k_offsets ? a.n_keys : mean;
    bool uneven = false;
    // Writing and joining the tiles' partial results costs what some 1500 keys do: 2048 tokens, 8 heads of 128, cut
    // in two 34.5 us, whole 26.7; 4096 tokens, 4 heads, 41.6 and 50.9.
    if (p.rows > 0 && mean - chunk < kKeysSaved) {
      // Where one sequence may hold most of the keys, those far above the mean are cut all the same, the others being
      // one chunk each: 32 queries of 32 heads on 2 (64 channels) in each of 16 sequences, one of 32768 keys among ones of
      // 512, take 50 us, whole 263; of 2528 keys each 29.6, whole 25.5.
      chunk = (mean + kKeysSaved + 127) / 128 * 128;
      uneven = longest - chunk >= kKeysUneven;
      if (!uneven) chunk = kMaxTokens;
    }
    if (chunk < longest) {
      const int64_t n = pieces(a.k_offsets, a.n_keys, a.n_seqs, static_cast<int>(chunk), 0x7fffffff, &p.k_per);
      const int64_t rows = n * p.max_q * a.q.heads;
      const int64_t ml = (rows * 8 + 15) / 16 * 16, bytes = ml + rows * a.dim * 4;
      if (rows < kMaxWorkspace && bytes <= kMaxWorkspace) {
        p.chunk = static_cast<int>(chunk);
        p.k_pieces = n;
        p.firsts = uneven && p.k_per == 0;
        p.blocks = n * p.tiles * heads;
        p.ml_bytes = ml;
        p.bytes = bytes;
      }
    }
  }
  return p;
}

// What is wrong with a call but for its buffers (null: nothing).
const char* bad_attention(const moeca_attention_args& a) {
  if (!is_dtype(a.dtype)) return "dtype must be MOECA_F32 or MOECA_BF16";
  if (a.dim < 1 || a.dim > kMaxHeadDim) return "1 <= dim <= 256";
  if (a.n_seqs < 1 || a.n_seqs > kMaxSeqs) return "1 <= n_seqs <= 2^20";
  if (a.n_queries < 0 || a.n_keys < 0 || a.max_q < 0) return "n_queries, n_keys and max_q must not be negative";
  if (!a.q_offsets && a.n_queries % a.n_seqs) return "n_queries must be a multiple of n_seqs without q_offsets";
  if (!a.k_offsets && a.n_keys % a.n_seqs) return "n_keys must be a multiple of n_seqs without k_offsets";
  if (a.q.heads < 1 || a.k.heads < 1 || a.q.heads % a.k.heads || a.v.heads != a.k.heads || a.out.heads != a.q.heads)
    return "q.heads must be a multiple of k.heads = v.heads, and out.heads = q.heads";
  if (a.causal < 0 || a.causal > 1) return "causal must be 0 or 1";
  if (a.clear < 0 || a.clear > 2) return "clear must be 0, 1 or 2";
  // The kernels take it in base 2, where an infinite one would make NaN of a score of 0.
  if (!(a.scale > 0) || !std::isfinite(a.scale * kLog2e)) return "scale must be positive, and scale log2(e) finite";
  if (const char* why = bad_heads(a.q, a.n_queries, a.dim, a.dtype, false)) return why;
  if (const char* why = bad_heads(a.k, a.n_keys, a.dim, a.dtype, false)) return why;
  if (const char* why = bad_heads(a.v, a.n_keys, a.dim, a.dtype, false)) return why;
  if (const char* why = bad_heads(a.out, a.n_queries, a.dim, a.dtype, true)) return why;
  return nullptr;
}

}  // namespace
}  // namespace moeca

extern "C" {

int64_t moeca_attention_workspace(const moeca_attention_args* a) {
  using namespace moeca;
  if (!a || bad_attention(*a) || a->n_queries > kMaxTokens || a->n_keys > kMaxTokens) return -1;
  return a->n_queries == 0 ? 0 : plan_attention(*a).bytes;
}

moeca_status moeca_attention(const moeca_attention_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_attention(*a)) return refuse(why);
  if (addr(a->q_offsets) % 4 || addr(a->k_offsets) % 4 || addr(a->lse) % 4 || addr(a->status) % 4)
    return refuse("offsets, lse or status is not 4-byte aligned");
  if (a->n_queries > kMaxTokens || a->n_keys > kMaxTokens) {
    keep_call_error("more than 2^30 tokens");
    return MOECA_ERR_UNSUPPORTED;
  }
  const int64_t es = elem_size(a->dtype), nq = a->n_queries, nk = a->n_keys;
  const int dim = a->dim;
  const Plan p = nq > 0 ? plan_attention(*a) : Plan{};
  if (p.bytes > 0 && (!a->workspace || addr(a->workspace) % 16)) return refuse("workspace is NULL or not 16-byte aligned");
  const Range q_list = {a->q_offsets, 4ll * (a->n_seqs + 1)}, k_list = {a->k_offsets, 4ll * (a->n_seqs + 1)};
  const Range lse = {a->lse, 4 * nq * a->q.heads}, work = {p.bytes ? a->workspace : nullptr, p.bytes}, status = {a->status, 8};
  const Range written[] = {lse, work, status};
  const Range read[] = {q_list, k_list};
  if (any_overlap(written, read)) return refuse("lse, workspace or status overlaps another buffer of the call");
  for (const Range& r : {lse, work, status, q_list, k_list})
    if (heads_overlap(a->out, nq, r, dim, es)) return refuse("out overlaps another buffer of the call");
  for (const Range& r : written)
    if (heads_overlap(a->q, nq, r, dim, es) || heads_overlap(a->k, nk, r, dim, es) || heads_overlap(a->v, nk, r, dim, es))
      return refuse("lse, workspace or status overlaps another buffer of the call");
  if ((!same_heads(a->out, a->q) && heads_overlap(a->out, nq, a->q, nq, dim, es)) ||
      heads_overlap(a->out, nq, a->k, nk, dim, es) || heads_overlap(a->out, nq, a->v, nk, dim, es))
    return refuse("out overlaps another buffer of the call");
  if (nq == 0 || p.max_q == 0) return MOECA_OK;
  if (p.blocks > kMaxRows || nq * a->q.heads > kMaxRows) {
    keep_call_error("too many tiles for one launch");
    return MOECA_ERR_UNSUPPORTED;
  }
  PackedAttnArgs d{};
  d.q = device_heads(a->q); d.k = device_heads(a->k); d.v = device_heads(a->v); d.out = device_heads(a->out);
  d.qs = {a->q_offsets, static_cast<int>(nq), a->n_seqs, static_cast<int>(nq / a->n_seqs), p.tile, p.q_per, 0};
  d.ks = {a->k_offsets, static_cast<int>(nk), a->n_seqs, static_cast<int>(nk / a->n_seqs), p.chunk, p.k_per, p.firsts};
  d.q_pieces = p.q_pieces; d.k_pieces = p.k_pieces;
  d.lse = a->lse;
  d.part_ml = static_cast<float2*>(a->workspace);
  d.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(a->workspace) + p.ml_bytes);
  d.max_q = p.max_q; d.tiles = p.tiles;
  d.group = a->q.heads / a->k.heads;
  d.dim = dim; d.causal = a->causal; d.clear = a->clear;
  d.scale_log2 = a->scale * kLog2e;
  d.status = a->status;
  d.wait_ns = g_wait_ns;
  d.stall = g_stall;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched([&] {
    cudaError_t e = p.rows > 0    ? launch_attn_packed_tc(d, p.rows, s)
                    : p.rows < 0 ? launch_attn_rows(d, s)
                                 : launch_attn_simt(d, a->dtype, p.tile, s);
    if (e == cudaSuccess && p.chunk) e = launch_attn_join(d, a->dtype, s);
    return e;
  });
}

int32_t moeca_probe_attention_form(const moeca_attention_args* a, int32_t* chunk) {
  using namespace moeca;
  if (chunk) *chunk = 0;
  if (!a || bad_attention(*a) || a->n_queries > kMaxTokens || a->n_keys > kMaxTokens || a->n_queries == 0) return -1;
  const Plan p = plan_attention(*a);
  if (chunk) *chunk = p.chunk;
  return p.rows == 2 ? MOECA_ATTENTION_FORM_TILES : p.rows == 1 ? MOECA_ATTENTION_FORM_TILE
                     : p.rows < 0 ? MOECA_ATTENTION_FORM_ROWS : MOECA_ATTENTION_FORM_CORES;
}

int32_t moeca_probe_attention_stall(int32_t barrier, int64_t wait_ns) {
  using namespace moeca;
  if (barrier < MOECA_ATTENTION_NONE || barrier > MOECA_ATTENTION_SLOTS || wait_ns < 1000000 || wait_ns > 1000000000) return -1;
  g_wait_ns = barrier == MOECA_ATTENTION_NONE ? kWaitNs : static_cast<unsigned long long>(wait_ns);
  g_stall = barrier;
  return 0;
}

}  // extern "C"
