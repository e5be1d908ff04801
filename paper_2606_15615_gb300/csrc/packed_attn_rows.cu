// Attention over packed sequences for a few query rows (include/moeca_attention.h):
// bf16, heads of up to 128 values, at most 16 (query, head) rows per key head,
// as one new token after a long prompt has.
//
// Every key and value is read once for a handful of rows: HBM bounds it, and a
// tensor-core tile of 128 rows would be mostly empty.  A block of four warps works
// on one key head and a sequence's keys or a chunk of them; each warp takes every
// fourth tile of 16 keys through a ring of its own (cp.async, two tiles in flight,
// no barrier between warps), so that two to four blocks an SM keep HBM
// busy.  A warp's 16 rows are one m16n8k16 fragment: S = Q K^T, the
// running maximum m and sum per row in registers, P = 2^((s - m) scale) in bf16 straight
// from the scores' fragment into the product with V (the difference first: 1 at s = m,
// however large the scores).  The four warps' results meet in shared
// memory at the end.
// Four tokens over 131072 keys in all, 32 heads of 128 on 8 (537 MB): 92 us with the
// join, 5.8 TB/s, 0.86 of the measured copy rate; one over 65536 keys on 4 key heads (134
// MB) 30 us, a fifth of it the join's launch and its dependent loads; one over 300 keys 6 us.
// The exponential is ex2.approx (2 ulp), far below the bf16 rounding of P.
#include <algorithm>

#include "attn_tc.cuh"
#include "packed_attn.cuh"

namespace moeca {
namespace {

constexpr int kRowsWarps = 4, kRowsThreads = 32 * kRowsWarps;
constexpr int kRowsKeys = 16;   // keys of a warp's tile
constexpr int kRowsStages = 3;

template <int DK>  // 16-channel steps of a head
struct RowsShape {
  static constexpr int DP = DK * 16;
  // An odd number of 16-byte pieces from row to row: eight rows' pieces fall in distinct banks.
  static constexpr int PITCH = DP * 2 + 16;
  static constexpr int TILE = kRowsKeys * PITCH;       // bytes of a tile's keys, or values
  static constexpr int RING = kRowsStages * 2 * TILE;  // per warp; holds the warp's 16 x DP fp32 sums in the end
  static constexpr int SMEM = kRowsWarps * RING;
  static_assert(RING >= 16 * DP * 4);
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}

template <int DK>
__global__ void __launch_bounds__(kRowsThreads, DK <= 4 ? 4 : 2) attn_rows_kernel(const __grid_constant__ PackedAttnArgs a) {
  using Sh = RowsShape<DK>;
  extern __shared__ __align__(16) uint8_t rows_smem[];
  __shared__ float sh_m[kRowsWarps][16], sh_l[kRowsWarps][16];
  pdl_entry();
  const int index = blockIdx.x / static_cast<uint32_t>(a.k.heads), kvh = blockIdx.x - index * a.k.heads;
  const AttnWork w = attn_work(a, index);
  clear_rest<__nv_bfloat16>(a, w, index, kvh, a.k.heads, threadIdx.x, kRowsThreads);
  if (!w.any) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.group, n_q = min(w.nq, a.max_q), rows = n_q * G;
  uint8_t* ring = rows_smem + warp * Sh::RING;
  const uint32_t ring_at = smem_u32(ring);
  const int chunks = a.dim / 8;  // 16-byte pieces of a row
  // Channels past dim are never copied: zero in keys (their products must vanish) and values.
  for (int i = lane; i < kRowsStages * 2 * kRowsKeys * (2 * DK - chunks); i += 32) {
    const int row = i / (2 * DK - chunks), c = chunks + i - row * (2 * DK - chunks);
    *reinterpret_cast<uint4*>(ring + row * Sh::PITCH + c * 16) = make_uint4(0, 0, 0, 0);
  }
  const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(a.k.data) + static_cast<int64_t>(w.k0) * a.k.token_stride + kvh * a.k.head_stride;
  const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v.data) + static_cast<int64_t>(w.k0) * a.v.token_stride + kvh * a.v.head_stride;
  // The last query sees the most.
  const int end = min(w.key_hi, visible_keys(a, w, n_q - 1));
  const int tiles = (max(end - w.key_lo, 0) + kRowsKeys - 1) / kRowsKeys;
  const auto fetch = [&](int t, int stage) {  // tile t of the block; rows behind the end become zeros
    if (t < tiles) {
      const int key0 = w.key_lo + t * kRowsKeys, n = min(kRowsKeys, w.key_hi - key0);
      const uint32_t dst = ring_at + stage * 2 * Sh::TILE;
#pragma unroll
      for (int i = 0; i < kRowsKeys * 2 * DK / 32; ++i) {
        const int at = i * 32 + lane, r = at / (2 * DK), c = at - r * (2 * DK);
        if (c < chunks) {
          const int64_t key = key0 + min(r, n - 1);
          cp_async16(dst + r * Sh::PITCH + c * 16, k + key * a.k.token_stride + c * 8, r < n);
          cp_async16(dst + Sh::TILE + r * Sh::PITCH + c * 16, v + key * a.v.token_stride + c * 8, r < n);
        }
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int s = 0; s < kRowsStages - 1; ++s) fetch(warp + s * kRowsWarps, s);
  // This lane's rows of the fragments: lane / 4 and lane / 4 + 8.
  int see[2];
  uint32_t q[DK][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = lane / 4 + 8 * h, i = min(r, rows - 1) / G, g = min(r, rows - 1) - i * G;
    see[h] = min(visible_keys(a, w, i), w.key_hi);
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q.data) + static_cast<int64_t>(w.q0 + i) * a.q.token_stride + (kvh * G + g) * a.q.head_stride;
#pragma unroll
    for (int kk = 0; kk < DK; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = kk * 16 + e * 8 + (lane & 3) * 2;
        q[kk][e * 2 + h] = r < rows && c < a.dim ? *reinterpret_cast<const uint32_t*>(src + c) : 0u;
      }
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[2 * DK][4];
#pragma unroll
  for (int c = 0; c < 2 * DK; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[c][j] = 0.f;
  // Where a lane's row of each 8 x 8 matrix lies: keys by channels for S, and the same transposed for the second product.
  const uint32_t k_row = ((lane >> 4) * 8 + (lane & 7)) * Sh::PITCH + ((lane >> 3) & 1) * 16;
  const uint32_t v_row = Sh::TILE + (((lane >> 3) & 1) * 8 + (lane & 7)) * Sh::PITCH + (lane >> 4) * 16;
  int stage = 0;
  for (int t = warp; t < tiles; t += kRowsWarps) {
    cp_wait<kRowsStages - 2>();
    __syncwarp();
    const uint32_t at = ring_at + stage * 2 * Sh::TILE;
    float s[2][4] = {};
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) {
      uint32_t b[4];
      ldsm_x4(at + k_row + kk * 32, b[0], b[1], b[2], b[3]);
      mma_16816(s[0], q[kk][0], q[kk][1], q[kk][2], q[kk][3], b[0], b[1]);
      mma_16816(s[1], q[kk][0], q[kk][1], q[kk][2], q[kk][3], b[2], b[3]);
    }
    const int key0 = w.key_lo + t * kRowsKeys + (lane & 3) * 2;
    float p[2][4], keep[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float& x = s[n][2 * h + e];
          if (key0 + n * 8 + e >= see[h]) x = -INFINITY;
          top = fmaxf(top, x);
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(m[h], fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
      const float ref = top == -INFINITY ? 0.f : top;
      keep[h] = ex2f_approx((m[h] - ref) * a.scale_log2);
      m[h] = top;
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          p[n][2 * h + e] = ex2f_approx((s[n][2 * h + e] - ref) * a.scale_log2);
          sum += p[n][2 * h + e];
        }
      l[h] = l[h] * keep[h] + sum;
    }
    if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
      for (int c = 0; c < 2 * DK; ++c) {
        o[c][0] *= keep[0];
        o[c][1] *= keep[0];
        o[c][2] *= keep[1];
        o[c][3] *= keep[1];
      }
    }
    const uint32_t pa[4] = {pack2(p[0][0], p[0][1]), pack2(p[0][2], p[0][3]), pack2(p[1][0], p[1][1]), pack2(p[1][2], p[1][3])};
#pragma unroll
    for (int c = 0; c < DK; ++c) {
      uint32_t b[4];
      ldsm_x4_trans(at + v_row + c * 32, b);
      mma_16816(o[2 * c], pa[0], pa[1], pa[2], pa[3], b[0], b[1]);
      mma_16816(o[2 * c + 1], pa[0], pa[1], pa[2], pa[3], b[2], b[3]);
    }
    __syncwarp();
    fetch(t + (kRowsStages - 1) * kRowsWarps, stage == 0 ? kRowsStages - 1 : stage - 1);
    stage = stage + 1 == kRowsStages ? 0 : stage + 1;
  }
  cp_wait<0>();
  __syncwarp();
  // The warps' sums meet.
  float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = lane / 4 + 8 * h;
    if ((lane & 3) == 0) {
      sh_m[warp][r] = m[h];
      sh_l[warp][r] = l[h];
    }
#pragma unroll
    for (int c = 0; c < 2 * DK; ++c)
      *reinterpret_cast<float2*>(mine + r * Sh::DP + c * 8 + (lane & 3) * 2) = make_float2(o[c][2 * h], o[c][2 * h + 1]);
  }
  __syncthreads();
  const int units = a.dim / 8;
  for (int i = threadIdx.x; i < rows * units; i += kRowsThreads) {
    const int r = i / units, c = (i - r * units) * 8;
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kRowsWarps; ++u) top = fmaxf(top, sh_m[u][r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, f[8] = {};
#pragma unroll
    for (int u = 0; u < kRowsWarps; ++u) {
      const float weight = ex2f_approx((sh_m[u][r] - ref) * a.scale_log2);
      sum += weight * sh_l[u][r];
      const float* part = reinterpret_cast<const float*>(rows_smem + u * Sh::RING) + r * Sh::DP + c;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = fmaf(weight, part[j], f[j]);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv;
    const int q_i = r / G, head = kvh * G + r - q_i * G;
    const float lse2 = sum == 0.f ? -INFINITY : top * a.scale_log2 + log2f(sum);
    if (a.ks.unit && w.nk > a.ks.unit) {
      const int64_t part = (static_cast<int64_t>(w.piece) * a.max_q + q_i) * a.q.heads + head;
      if (c == 0) a.part_ml[part] = make_float2(top, sum);
      store_vec(a.part_o + part * a.dim + c, f);
      store_vec(a.part_o + part * a.dim + c + 4, f + 4);
    } else {
      if (c == 0 && a.lse) a.lse[static_cast<int64_t>(w.q0 + q_i) * a.q.heads + head] = lse2 * kLn2;
      store_vec(static_cast<__nv_bfloat16*>(a.out.data) + static_cast<int64_t>(w.q0 + q_i) * a.out.token_stride + head * a.out.head_stride + c, f);
    }
  }
}

template <int DK>
cudaError_t run(const PackedAttnArgs& a, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(attn_rows_kernel<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsShape<DK>::SMEM);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (a.ks.unit ? a.k_pieces : a.q_pieces) * a.k.heads;
  return launch_pdl(attn_rows_kernel<DK>, dim3(static_cast<unsigned>(blocks)), dim3(kRowsThreads), RowsShape<DK>::SMEM, s, a);
}

}  // namespace

cudaError_t launch_attn_rows(const PackedAttnArgs& a, cudaStream_t s) {
  const int dk = (a.dim + 15) / 16;
  if (dk <= 4) return run<4>(a, s);
  if (dk == 5) return run<5>(a, s);
  if (dk == 6) return run<6>(a, s);
  return run<8>(a, s);
}

}  // namespace moeca
