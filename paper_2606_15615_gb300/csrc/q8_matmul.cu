// Grouped product of 8-bit rows (include/moeca_q8.h).
//   c[m, n] = act(sum_k a[m, k] b[g(m) N + n, k] + bias[g(m), n])
#include <algorithm>

#include "common.cuh"
#include "q8.cuh"

namespace moeca {
namespace {

constexpr int kM = 64, kN = 128, kK = 32, kThreads = 256;

template <bool E5>
__device__ __forceinline__ float value_at(const Q8Rows& r, int64_t row, int k) {
  const float f = scale_value(r.scale[row * r.scale_stride + k / kQ8Block]);
  return decode2<E5>(r.q[row * r.q_stride + k]).x * f;
}

// A block per 64 x 128 tile: 4 x 8 sums per thread, operands decoded into
// shared memory as fp32.  The 16 threads of a row of the tile hold its 128
// columns, which are one block of an 8-bit output row.
__global__ void __launch_bounds__(kThreads) q8_matmul_kernel(const Q8MatmulArgs p) {
  __shared__ float as[kM][kK + 1], bs[kN][kK + 1];
  __shared__ int sh_g, sh_lo, sh_hi;
  pdl_entry();
  if (threadIdx.x == 0) {
    const int M = static_cast<int>(p.a.rows);
    int tile = blockIdx.y, g = 0, lo = 0, hi = 0;
    for (; g < p.n_groups; ++g) {
      lo = p.offsets ? min(max(p.offsets[g], 0), M) : 0;
      hi = p.offsets ? min(max(p.offsets[g + 1], 0), M) : M;
      const int tiles = (max(hi - lo, 0) + kM - 1) / kM;
      if (tile < tiles) break;
      tile -= tiles;
    }
    sh_g = g;
    sh_lo = lo + tile * kM;
    sh_hi = hi;
  }
  __syncthreads();
  const int g = sh_g, m0 = sh_lo, m1 = sh_hi, n0 = blockIdx.x * kN;
  if (g >= p.n_groups) return;
  const int N = p.n_cols, K = p.a.width, tn = threadIdx.x & 15, tm = threadIdx.x >> 4;
  float c[4][8] = {};
  for (int k0 = 0; k0 < K; k0 += kK) {
    for (int e = threadIdx.x; e < kM * kK; e += kThreads) {
      const int r = e / kK, k = k0 + e % kK, m = m0 + r;
      as[r][e % kK] = m < m1 && k < K ? (p.a_e5 ? value_at<true>(p.a, m, k) : value_at<false>(p.a, m, k)) : 0.f;
    }
    for (int e = threadIdx.x; e < kN * kK; e += kThreads) {
      const int r = e / kK, k = k0 + e % kK, n = n0 + r;
      const int64_t row = static_cast<int64_t>(g) * N + n;
      bs[r][e % kK] = n < N && k < K ? (p.b_e5 ? value_at<true>(p.b, row, k) : value_at<false>(p.b, row, k)) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < kK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) c[i][j] = fmaf(as[tm * 4 + i][k], bs[tn + 16 * j][k], c[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + tm * 4 + i;
    int row = -1;
    if (m < m1) row = p.dst ? p.dst[m] : m;
    const bool live = row >= 0 && row < p.out.rows;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = n0 + tn + 16 * j;
      float v = n < N && live ? c[i][j] + (p.bias ? p.bias[static_cast<int64_t>(g) * N + n] : 0.f) : 0.f;
      if (p.act != MOECA_ACT_NONE) v = gelu_f(v, p.act == MOECA_ACT_GELU_TANH);
      c[i][j] = v;
      if (abs_bits(v) < kNonFinite) top = max(top, abs_bits(v));
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (!live) continue;
    uint8_t* out = p.out.q + row * p.out.q_stride;
    const bool e5 = p.out_format == MOECA_E5M2;
    const int byte = e5 ? scale_byte<true>(top) : scale_byte<false>(top);
    if (tn == 0 && (e5 || p.out_format == MOECA_E4M3))
      p.out.scale[row * p.out.scale_stride + blockIdx.x] = static_cast<uint8_t>(byte);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = n0 + tn + 16 * j;
      if (n >= N) continue;
      const float q = c[i][j] * scale_inverse(byte);
      if (p.out_format == MOECA_F32) reinterpret_cast<float*>(out)[n] = c[i][j];
      else if (p.out_format == MOECA_BF16) reinterpret_cast<__nv_bfloat16*>(out)[n] = __float2bfloat16_rn(c[i][j]);
      else out[n] = static_cast<uint8_t>(e5 ? encode_any<true>(q) : encode_any<false>(q));
    }
  }
}

}  // namespace

cudaError_t launch_q8_matmul(const Q8MatmulArgs& a, cudaStream_t s) {
  const int64_t tiles = (a.a.rows + kM - 1) / kM + a.n_groups - 1;
  const dim3 grid((a.n_cols + kN - 1) / kN, static_cast<unsigned>(tiles));
  return launch_pdl(q8_matmul_kernel, grid, dim3(kThreads), 0, s, a);
}

}  // namespace moeca
