// Grouped product of 8-bit rows (include/moeca_q8.h) for sm_103a:
//   c[m, n] = act(sum_k a[m, k] b[g(m) N + n, k] + bias[g(m), n])
// for the rows m of every group g, a group being an expert's rows.
//
// tcgen05.mma of kind mxf8f6f4 multiplies 8-bit values and applies the blocks'
// power-of-two scales itself: D += 2^(sa - 127) 2^(sb - 127) (A B) over 32
// values of K at a time, sums in fp32 in TMEM over all of K.  The scales are
// read from TMEM, one byte per row and MMA; a block of 128 values is four MMAs
// that name the same byte, so a 32-bit TMEM cell holds a row's scales of four
// blocks (512 values of K) just as they lie in memory.
//
// Persistent CTA pairs (clusters of two, cta_group::2): a tile is 256 weight
// rows (the MMA's M side, 128 per CTA) by n token rows (its N side, half per
// CTA; n a multiple of 16 up to 192, chosen per group so that its tiles are as
// even and as narrow as its rows allow), K in stages of two blocks of 128.
// The weights take the wide side because a group's rows are few and ragged,
// its weights neither.  Two accumulators of 192 TMEM columns, so that a tile's
// epilogue runs beside the next one's MMAs; the rest of TMEM holds the scales.
// 15 warps per CTA:
//   warp 0      TMA producer of the weight boxes (128 rows x 128 bytes);
//   warp 14     TMA producer of the token boxes (n / 2 rows x 128 bytes);
//   warps 10-13 scales: each loads the scale words of the tile's rows (weights'
//               own 128, all n tokens') and stores them to its lane quadrant of
//               TMEM: the MMA wants rows 32 c + l in lane l of column c, in all
//               four quadrants;
//   warp 1      TMEM allocation; in the leader one thread issues the MMAs;
//   warps 2-9   epilogue, two warps per lane quadrant, alternate chunks of 32
//               token columns: a lane is a feature (weight row), a register a
//               token.  The 128 features of a CTA are one block of an 8-bit
//               output row: each warp takes its 32 features' maxima, the four
//               quadrants exchange them through shared memory, and 4 x 4 byte
//               transposes among lanes make words of four features.
// Every wait is bounded as in the other tensor-core kernels; a wait that runs
// out writes the caller's status word.
#include <cuda.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "q8.cuh"
#include "tc_common.cuh"

namespace moeca {
namespace {

constexpr int kBM = 128;                  // weight rows per CTA (half of the MMA's M)
constexpr int kSub = 2;                   // K blocks of 128 per stage
constexpr int kMaxN = 192;                // token rows per tile
constexpr int kBoxes = kMaxN / 16;        // token boxes of 8, 16, .., 96 rows
constexpr int kMaxStages = 5;
constexpr int kRingBytes = 200 * 1024;    // weight slots first, then token slots
constexpr int kWBytes = kBM * kQ8Block;   // 16 KB: one weight block
constexpr int kWSlot = kSub * kWBytes;
constexpr int kSfStages = 4;              // scale words of 4 K blocks each
constexpr int kSfCols = 16;               // TMEM columns of one: 4 for the weights, from 8 on the tokens
constexpr int kSfBase = 2 * kMaxN;
constexpr int kEpiWarps = 8;              // warps 2-9
constexpr int kSfWarp = 2 + kEpiWarps;    // warps 10-13
constexpr int kTokWarp = kSfWarp + 4;
constexpr int kThreads = 32 * (kTokWarp + 1);
constexpr int kTmemCols = 512;
constexpr int kMaxGroups = 1024;
static_assert(kSfBase + kSfStages * kSfCols <= kTmemCols, "TMEM");

// Behind the ring: what the warps share.
struct Shared {
  int units[kMaxGroups + 1];              // first unit of each group
  int lo[kMaxGroups], rows[kMaxGroups];   // first row, rows
  uint32_t top[2][2][4][32];              // [part][buffer][quadrant][token]: largest |z| bits
  alignas(16) float inv[kEpiWarps][32];   // 1 / scale of the chunk's tokens, read four at a time
  uint64_t full[kMaxStages], empty[kMaxStages], sf_full[kSfStages], sf_empty[kSfStages], tfull[2], tempty[2], drain;
  uint32_t tmem;
  int max_n;
  volatile int abort_flag;
};
constexpr int kSmem = kRingBytes + sizeof(Shared) + 1024;
static_assert(kSmem <= 227 * 1024, "shared memory");

struct Maps {
  CUtensorMap w;             // weights, box 128 rows
  CUtensorMap act[kBoxes];   // token rows, boxes of 8 .. 96 rows
};

// Token tiles of a group of `rows` rows, and their width.
__device__ __forceinline__ int token_tiles(int rows) { return (rows + kMaxN - 1) / kMaxN; }
__device__ __forceinline__ int token_width(int rows) {
  const int t = token_tiles(rows), w = (rows + t - 1) / t;
  return (w + 15) / 16 * 16;
}

// What a unit (tile) works on.
struct Unit {
  int g, m0, m_end, n, w;  // group, first row, end of the group's rows in the tile, token columns, weight tile
};
// Units are numbered group by group, token tile by token tile, weight tile by
// weight tile; every role walks them in ascending order, so that g only grows.
__device__ __forceinline__ Unit unit_at(const Shared& sh, int u, int g, int nw) {
  while (u >= sh.units[g + 1]) ++g;
  Unit r;
  r.g = g;
  const int at = u - sh.units[g], tt = at / nw;
  r.w = at - tt * nw;
  r.n = token_width(sh.rows[g]);
  r.m0 = sh.lo[g] + tt * r.n;
  r.m_end = min(r.m0 + r.n, sh.lo[g] + sh.rows[g]);
  return r;
}

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
      "[%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// Instruction descriptor of kind::mxf8f6f4 without its scale bytes' numbers
// (bits 4-5: B, 29-30: A): A and B K-major e4m3 (0) or e5m2 (1), E8M0 scales.
__device__ __forceinline__ uint32_t mx_desc(int n, bool a_e5, bool b_e5) {
  return (a_e5 ? 1u << 7 : 0u) | (b_e5 ? 1u << 10 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) |
         (static_cast<uint32_t>(2 * kBM >> 4) << 24);
}

__device__ __forceinline__ void mma_mx_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                            uint32_t sf_a, uint32_t sf_b, uint32_t acc) {
  constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);  // smem_desc's bits 32-63
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n"
      " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a, b, %3, [%6], [%7], p;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kHi), "r"(sf_a), "r"(sf_b)
      : "memory");
}

// GELU of an epilogue value (Eq. 5).  tanh form: z sigmoid(2 u), u = sqrt(2/pi) (z + 0.044715 z^3).
// erf form: Phi(-|z|) = erfc(|z| / sqrt 2) / 2 by Abramowitz and Stegun's
// formula 7.1.26, P(t) exp(-z^2 / 2) / 2 with t = 1 / (1 + p |z| / sqrt 2), within
// 0.75e-7; z Phi(z) is z - z Phi(-z) or z Phi(-|z|), so that nothing cancels.
// Both cost two special-function evaluations and about ten others; the library
// functions' longer forms would bound the products with short K.
template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  if constexpr (ACT == MOECA_ACT_GELU_TANH) {
    const float v = z * fmaf(0.0713548163f, z * z, 1.5957691216f);  // 2 u
    return __fdividef(z, 1.f + __expf(-v));
  } else if constexpr (ACT == MOECA_ACT_GELU) {
    const float x = fabsf(z);
    const float t = __fdividef(1.f, fmaf(0.3275911f * 0.70710678f, x, 1.f));
    float s = fmaf(1.061405429f, t, -1.453152027f);
    s = fmaf(s, t, 1.421413741f);
    s = fmaf(s, t, -0.284496736f);
    s = fmaf(s, t, 0.254829592f);
    const float tail = 0.5f * s * t * __expf(-0.5f * z * z) * x;  // |z| Phi(-|z|)
    return fmaxf(z, 0.f) - tail;
  } else {
    return z;
  }
}

// Four features' bytes of one token per lane from four tokens' bytes of one
// feature: lane j of each four lanes gets token j's.
__device__ __forceinline__ uint32_t transpose4(uint32_t own, int lane) {
  const uint32_t p1 = __shfl_xor_sync(0xffffffffu, own, 1);
  const uint32_t a = lane & 1 ? __byte_perm(p1, own, 0x7351) : __byte_perm(own, p1, 0x6240);
  const uint32_t p2 = __shfl_xor_sync(0xffffffffu, a, 2);
  return lane & 2 ? __byte_perm(p2, a, 0x7632) : __byte_perm(a, p2, 0x5410);
}

// Barrier over the four epilogue warps of a part (ids 1 and 2); true if `ok` in all.
__device__ __forceinline__ bool part_sync(int part, bool ok) {
  uint32_t all;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred.aligned q, %2, 128, p;\n"
      " selp.u32 %0, 1, 0, q;\n}"
      : "=r"(all)
      : "r"(static_cast<uint32_t>(ok)), "r"(part + 1)
      : "memory");
  return all != 0;
}

struct MatmulParams {
  const uint8_t *w_scale, *t_scale;
  int64_t w_stride, t_stride;  // scale rows
  int64_t w_rows;
  int M, N, K, G;
  const int32_t *offsets, *dst;
  const float* bias;
  uint8_t* out;
  uint8_t* out_scale;
  int64_t out_rows, out_stride, os_stride;
  bool w_e5, t_e5, wide;       // wide: 4-byte stores of bf16 pairs
  int32_t* status;
};

// Epilogue of one chunk: 32 features (lanes) x 32 tokens (z), all four
// quadrants of the part together.  row: lane t's output row of token t, or -1.
template <int OUT>
__device__ __forceinline__ void store_chunk(const MatmulParams& p, Shared& sh, float (&z)[32], int row, int feat0,
                                            int block, int lane, int warp, int part, int quad, int buf) {
  if constexpr (OUT == MOECA_F32) {
    if (feat0 >= p.N) return;
#pragma unroll
    for (int t = 0; t < 32; ++t) {
      const int r = __shfl_sync(0xffffffffu, row, t);
      if (r >= 0 && feat0 + lane < p.N) reinterpret_cast<float*>(p.out + r * p.out_stride)[feat0 + lane] = z[t];
    }
  } else if constexpr (OUT == MOECA_BF16) {
    if (feat0 >= p.N) return;
    if (p.wide) {
      // Lanes 2i and 2i + 1 swap halves: each holds the feature pair of every other token.
      const int odd = lane & 1, f = feat0 + (lane & ~1);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const uint32_t own = pack_bf16(z[2 * t], z[2 * t + 1]);
        const uint32_t got = __shfl_xor_sync(0xffffffffu, own, 1);
        const uint32_t word = odd ? __byte_perm(got, own, 0x7632) : __byte_perm(own, got, 0x5410);
        const int r = __shfl_sync(0xffffffffu, row, 2 * t + odd);
        if (r < 0 || f >= p.N) continue;
        uint8_t* at = p.out + r * p.out_stride + f * 2;
        if (f + 1 < p.N) *reinterpret_cast<uint32_t*>(at) = word;
        else *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(word);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 32; ++t) {
        const int r = __shfl_sync(0xffffffffu, row, t);
        if (r >= 0 && feat0 + lane < p.N)
          reinterpret_cast<__nv_bfloat16*>(p.out + r * p.out_stride)[feat0 + lane] = __float2bfloat16_rn(z[t]);
      }
    }
  } else {
    constexpr bool E5 = OUT == MOECA_E5M2;
    uint32_t mine = 0;  // lane t: the largest |z| of token t over the warp's features
#pragma unroll
    for (int t = 0; t < 32; ++t) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, abs_bits(z[t]));
      if (lane == t) mine = top;
    }
    const bool odd = __any_sync(0xffffffffu, row >= 0 && mine >= kNonFinite);
    if (odd) {
      mine = 0;
#pragma unroll
      for (int t = 0; t < 32; ++t) {
        const uint32_t b = abs_bits(z[t]), top = __reduce_max_sync(0xffffffffu, b < kNonFinite ? b : 0u);
        if (lane == t) mine = top;
      }
    }
    sh.top[part][buf][quad][lane] = mine;
    part_sync(part, true);
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) top = max(top, sh.top[part][buf][q][lane]);
    const int byte = scale_byte<E5>(top);
    float* inv = sh.inv[warp - 2];
    __syncwarp();
    inv[lane] = scale_inverse(byte);
    __syncwarp();
    if (quad == 0 && row >= 0) p.out_scale[row * p.os_stride + block] = static_cast<uint8_t>(byte);
    if (feat0 >= p.N) return;
    const int f = feat0 + (lane >> 2) * 4, left = p.N - f;
#pragma unroll
    for (int t = 0; t < 32; t += 4) {
      const float4 s = *reinterpret_cast<const float4*>(inv + t);
      uint32_t word = encode2<E5>(z[t] * s.x, z[t + 1] * s.y) | encode2<E5>(z[t + 2] * s.z, z[t + 3] * s.w) << 16;
      if (odd)
        word = encode_any<E5>(z[t] * s.x) | encode_any<E5>(z[t + 1] * s.y) << 8 | encode_any<E5>(z[t + 2] * s.z) << 16 |
               encode_any<E5>(z[t + 3] * s.w) << 24;
      word = transpose4(word, lane);
      const int r = __shfl_sync(0xffffffffu, row, t + (lane & 3));
      if (r < 0 || left <= 0) continue;
      uint8_t* at = p.out + r * p.out_stride + f;
      if (left >= 4) {
        *reinterpret_cast<uint32_t*>(at) = word;
      } else {
        for (int i = 0; i < left; ++i) at[i] = static_cast<uint8_t>(word >> 8 * i);
      }
    }
  }
}

template <int OUT, int ACT>
__global__ void __launch_bounds__(kThreads, 1) q8_matmul_kernel(const __grid_constant__ Maps maps, const MatmulParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Shared& sh = *reinterpret_cast<Shared*>(smem + kRingBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  volatile int* abort_flag = &sh.abort_flag;

  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(smem_u32(&sh.full[s]), 1);
      mbar_init(smem_u32(&sh.empty[s]), 1);
    }
    for (int s = 0; s < kSfStages; ++s) {
      mbar_init(smem_u32(&sh.sf_full[s]), 8);
      mbar_init(smem_u32(&sh.sf_empty[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&sh.tfull[s]), 1);
      mbar_init(smem_u32(&sh.tempty[s]), 2 * kEpiWarps);
    }
    mbar_init(smem_u32(&sh.drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  if (warp == 2 && lane <= kBoxes) {
    const CUtensorMap* t = lane ? &maps.act[lane - 1] : &maps.w;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(t)) : "memory");
  }
  pdl_entry();
  const int nw = (p.N + 2 * kBM - 1) / (2 * kBM);
  if (warp == 0) {
    // The groups' rows and units, 32 groups at a time.
    int units = 0, max_n = 16;
    for (int g0 = 0; g0 < p.G; g0 += 32) {
      const int g = g0 + lane;
      int lo = 0, rows = 0;
      if (g < p.G) {
        lo = p.offsets ? min(max(__ldg(p.offsets + g), 0), p.M) : 0;
        const int hi = p.offsets ? min(max(__ldg(p.offsets + g + 1), 0), p.M) : p.M;
        rows = max(hi - lo, 0);
      }
      const int own = token_tiles(rows) * nw;
      int sum = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      if (g < p.G) {
        sh.lo[g] = lo;
        sh.rows[g] = rows;
        sh.units[g] = units + sum - own;
      }
      units += __shfl_sync(0xffffffffu, sum, 31);
      max_n = max(max_n, static_cast<int>(__reduce_max_sync(0xffffffffu, rows ? token_width(rows) : 0)));
    }
    if (lane == 0) {
      sh.units[p.G] = units;
      sh.max_n = max_n;
    }
  }
  __syncthreads();
  cluster_arrive();
  cluster_wait();  // both CTAs' barriers are initialised, TMEM is allocated
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  const int units = sh.units[p.G];
  const int kb = (p.K + kQ8Block - 1) / kQ8Block, ks = (kb + kSub - 1) / kSub, kc = (kb + 3) / 4;
  const int t_slot = kSub * (sh.max_n >> 1) * kQ8Block;
  const int nst = min(kMaxStages, kRingBytes / (kWSlot + t_slot));
  const uint32_t ring = smem_u32(smem), ring_t = ring + nst * kWSlot;
  const uint32_t empty0 = smem_u32(&sh.empty[0]);

  if (warp == 0 || warp == kTokWarp) {
    if (lane == 0) {
      // ---------------- TMA producers: weights (warp 0), tokens ----------------
      const bool wts = warp == 0;
      const int slot_bytes = wts ? kWSlot : t_slot;
      const uint32_t first = wts ? ring : ring_t, end = first + nst * slot_bytes;
      const uint32_t full0 = cluster_addr(smem_u32(&sh.full[0]), 0);
      uint32_t dst = first, eb = empty0, fb = full0, par = 1u;
      int issued = 0, g = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += n_pairs) {
        const Unit t = unit_at(sh, u, g, nw);
        g = t.g;
        const int half = t.n >> 1;
        const CUtensorMap* map = wts ? &maps.w : &maps.act[(t.n >> 4) - 1];
        // Weight rows past the group's (another group's, or none) meet no stored result.
        const int row = wts ? g * p.N + t.w * 2 * kBM + static_cast<int>(rank) * kBM : t.m0 + static_cast<int>(rank) * half;
        const int box = wts ? kWBytes : half * kQ8Block;
        const uint32_t tx = 2 * kWSlot + kSub * t.n * kQ8Block;  // both CTAs' bytes; outside the rows or K: zeros
        for (int k = 0; k < ks; ++k) {
          if (!(ok = mbar_wait_hot(eb, par, abort_flag))) break;
          if (wts && rank == 0) mbar_expect_tx(fb, tx);
#pragma unroll
          for (int q = 0; q < kSub; ++q) tma_load_pair(dst + q * box, map, (k * kSub + q) * kQ8Block, row, fb);
          ++issued;
          dst += slot_bytes;
          eb += 8;
          fb += 8;
          if (dst == end) {
            dst = first;
            eb = empty0;
            fb = full0;
            par ^= 1u;
          }
        }
      }
      if (!ok) {
        if (!sh.abort_flag) report_status(p.status, MOECA_ERR_TIMEOUT, wts ? 700 : 703);
        sh.abort_flag = 1;
        // Copies already issued land before the CTAs can exit: the newest use
        // of every slot (the leader's barriers see both CTAs').
        for (int q = 0; wts && rank == 0 && q < nst && q < issued; ++q) {
          const int last = issued - 1 - (issued - 1 - q) % nst;
          const unsigned long long t0 = globaltimer();
          while (!mbar_try(smem_u32(&sh.full[q]), (last / nst) & 1) && globaltimer() - t0 < kTcWaitNs) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // ---------------- MMA issuer (the leader, for both CTAs) ----------------
      const uint32_t w_lo0 = ((ring & 0x3FFFFu) >> 4) | (1u << 16), x_lo0 = ((ring_t & 0x3FFFFu) >> 4) | (1u << 16);
      const uint32_t full0 = smem_u32(&sh.full[0]);
      const uint32_t x_end = x_lo0 + nst * (static_cast<uint32_t>(t_slot) >> 4);
      const int last_steps = (p.K - (kb - 1) * kQ8Block + 31) / 32;  // MMAs of the last K block
      uint32_t w_lo = w_lo0, x_lo = x_lo0, fb = full0, eb = empty0, par = 0u, acc_phase = 0, sf_par = 0;
      int acc = 0, sfs = 0, g = 0;
      bool ok = true;
      for (int u = pair; u < units; u += n_pairs) {
        const Unit t = unit_at(sh, u, g, nw);
        g = t.g;
        if (!(ok = mbar_wait_cluster(smem_u32(&sh.tempty[acc]), acc_phase ^ 1u, abort_flag))) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem + static_cast<uint32_t>(acc * kMaxN);
        const uint32_t idesc = mx_desc(t.n, p.w_e5, p.t_e5), x_sub = static_cast<uint32_t>(t.n >> 1) * kQ8Block >> 4;
        for (int k = 0; k < ks; ++k) {
          if ((k & 1) == 0 && !(ok = mbar_wait_cluster(smem_u32(&sh.sf_full[sfs]), sf_par, abort_flag))) break;
          if (!(ok = mbar_wait_hot(fb, par, abort_flag))) break;
          tc_fence_after();
          const uint32_t sf = tmem + kSfBase + sfs * kSfCols;
#pragma unroll
          for (int q = 0; q < kSub; ++q) {
            const int b = k * kSub + q;
            if (b >= kb) break;
            const uint32_t wq = w_lo + q * (kWBytes >> 4), xq = x_lo + q * x_sub;
            const uint32_t id = static_cast<uint32_t>(b & 3), desc = idesc | id << 4 | id << 29;
            const int steps = b == kb - 1 ? last_steps : 4;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              if (kk < steps) mma_mx_pair(d_tmem, wq + kk * 2, xq + kk * 2, desc, sf, sf + 8, b != 0 || kk != 0);
          }
          mma_commit_pair(eb);
          if ((k & 1) || k == ks - 1) {
            mma_commit_pair(smem_u32(&sh.sf_empty[sfs]));
            if (++sfs == kSfStages) {
              sfs = 0;
              sf_par ^= 1u;
            }
          }
          w_lo += kWSlot >> 4;
          x_lo += static_cast<uint32_t>(t_slot) >> 4;
          fb += 8;
          eb += 8;
          if (x_lo == x_end) {
            w_lo = w_lo0;
            x_lo = x_lo0;
            fb = full0;
            eb = empty0;
            par ^= 1u;
          }
        }
        if (!ok) break;
        mma_commit_pair(smem_u32(&sh.tfull[acc]));
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
      if (!ok) {
        if (!sh.abort_flag) report_status(p.status, MOECA_ERR_TIMEOUT, 701);
        sh.abort_flag = 1;
      }
      // Every MMA issued so far has completed once the drain barrier fires.
      mma_commit_pair(smem_u32(&sh.drain), 1);
      const unsigned long long t0 = globaltimer();
      while (!mbar_try(smem_u32(&sh.drain), 0) && globaltimer() - t0 < kTcWaitNs) {
      }
    }
  } else if (warp >= kSfWarp) {
    // ---------------- Scales ----------------
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t full0 = cluster_addr(smem_u32(&sh.sf_full[0]), 0);
    int g = 0, sfs = 0;
    uint32_t par = 1u;
    bool ok = true;
    for (int u = pair; u < units && ok; u += n_pairs) {
      const Unit t = unit_at(sh, u, g, nw);
      g = t.g;
      const int cols = (t.n + 31) >> 5;
      const uint8_t *wp[4], *tp[8];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int64_t r = static_cast<int64_t>(g) * p.N + t.w * 2 * kBM + static_cast<int>(rank) * kBM + c * 32 + lane;
        wp[c] = p.w_scale + min(r, p.w_rows - 1) * p.w_stride;
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) tp[c] = p.t_scale + static_cast<int64_t>(min(t.m0 + c * 32 + lane, p.M - 1)) * p.t_stride;
      uint32_t ws[4], ts[8];
      auto load = [&](int k) {
#pragma unroll
        for (int c = 0; c < 4; ++c) ws[c] = __ldg(reinterpret_cast<const uint32_t*>(wp[c]) + k);
#pragma unroll
        for (int c = 0; c < 8; ++c) ts[c] = c < cols ? __ldg(reinterpret_cast<const uint32_t*>(tp[c]) + k) : 0u;
      };
      load(0);
      for (int k = 0; k < kc; ++k) {
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.sf_empty[sfs]), par, abort_flag)))) break;
        tc_fence_after();
        const uint32_t at = tmem + lanes + kSfBase + sfs * kSfCols;
        asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(ws[0]), "r"(ws[1]),
                     "r"(ws[2]), "r"(ws[3])
                     : "memory");
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at + 8),
                     "r"(ts[0]), "r"(ts[1]), "r"(ts[2]), "r"(ts[3]), "r"(ts[4]), "r"(ts[5]), "r"(ts[6]), "r"(ts[7])
                     : "memory");
        if (k + 1 < kc) load(k + 1);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(full0 + sfs * 8);
        if (++sfs == kSfStages) {
          sfs = 0;
          par ^= 1u;
        }
      }
    }
    if (!ok) {
      if (lane == 0 && !sh.abort_flag) report_status(p.status, MOECA_ERR_TIMEOUT, 704);
      sh.abort_flag = 1;
    }
  } else {
    // ---------------- Epilogue ----------------
    const int quad = warp & 3, part = (warp - 2) >> 2;
    const uint32_t tempty0 = cluster_addr(smem_u32(&sh.tempty[0]), 0);
    int acc = 0, g = 0, buf = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int u = pair; u < units; u += n_pairs) {
      const Unit t = unit_at(sh, u, g, nw);
      g = t.g;
      const int block = t.w * 2 + static_cast<int>(rank), feat0 = block * kBM + quad * 32;
      const float bias = p.bias && feat0 + lane < p.N ? __ldg(p.bias + static_cast<int64_t>(g) * p.N + feat0 + lane) : 0.f;
      const bool live = feat0 + lane < p.N;
      ok = mbar_wait(smem_u32(&sh.tfull[acc]), acc_phase, abort_flag);
      if (!(ok = part_sync(part, ok))) break;  // all warps of the part, or none: the chunks' exchanges need all
      tc_fence_after();
      const uint32_t tb = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(acc * kMaxN);
      // A CTA whose features lie past N has no block: it only keeps in step.
      const int cols = block * kBM < p.N ? t.m_end - t.m0 : 0;
      int c = part * 32;
      if (c >= cols) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty0 + acc * 8);
      }
#pragma unroll 1
      for (; c < cols; c += 64) {
        const int m = t.m0 + c + lane;
        int row = -1;
        if (m < t.m_end) {
          row = p.dst ? __ldg(p.dst + m) : m;
          if (row >= p.out_rows) row = -1;
        }
        uint32_t v[32];
        tmem_ld32_async(tb + c, v);
        tmem_wait32(v);
        if (c + 64 >= cols) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(tempty0 + acc * 8);
        }
        float z[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] = live ? act_f<ACT>(__uint_as_float(v[i]) + bias) : 0.f;
        store_chunk<OUT>(p, sh, z, row, feat0, block, lane, warp, part, quad, buf);
        buf ^= 1;
      }
      if (++acc == 2) {
        acc = 0;
        acc_phase ^= 1u;
      }
    }
    if (!ok) {
      if (lane == 0 && !sh.abort_flag) report_status(p.status, MOECA_ERR_TIMEOUT, 702);
      sh.abort_flag = 1;
    }
  }
  // Neither CTA leaves (or frees TMEM) while the other may still reach its
  // shared memory or the pair's MMAs run.
  tc_fence_before();
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Bytes [rows, cols] with a row stride, box {128, box_rows}, 128-byte swizzle; outside: zeros.
bool encode_rows(CUtensorMap* m, const Q8Rows& r, uint32_t box_rows) {
  EncodeTiledFn enc = get_encoder();
  if (!enc) return false;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(r.width), static_cast<cuuint64_t>(r.rows)};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(r.q_stride)};
  cuuint32_t box[2] = {kQ8Block, box_rows};
  cuuint32_t estr[2] = {1, 1};
  g_maps_encoded.fetch_add(1, std::memory_order_relaxed);
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, r.q, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_q8_matmul(const Q8MatmulArgs& a, cudaStream_t s) {
  Maps maps;
  bool ok = encode_rows(&maps.w, a.b, kBM);
  for (int i = 0; i < kBoxes && ok; ++i) ok = encode_rows(&maps.act[i], a.a, 8 * (i + 1));
  if (!ok) return cudaErrorInvalidValue;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  MatmulParams p{};
  p.w_scale = a.b.scale; p.w_stride = a.b.scale_stride; p.w_rows = a.b.rows;
  p.t_scale = a.a.scale; p.t_stride = a.a.scale_stride;
  p.M = static_cast<int>(a.a.rows); p.N = a.n_cols; p.K = a.a.width; p.G = a.n_groups;
  p.offsets = a.offsets; p.dst = a.dst; p.bias = a.bias;
  p.out = a.out.q; p.out_scale = a.out.scale;
  p.out_rows = a.out.rows; p.out_stride = a.out.q_stride; p.os_stride = a.out.scale_stride;
  p.w_e5 = a.b_e5; p.t_e5 = a.a_e5;
  p.wide = reinterpret_cast<uintptr_t>(a.out.q) % 4 == 0 && a.out.q_stride % 4 == 0;
  p.status = a.status;
  // At most one pair per tile there can be.
  const int64_t nw = (a.n_cols + 2 * kBM - 1) / (2 * kBM);
  const int64_t most = nw * ((a.a.rows + kMaxN - 1) / kMaxN + std::min<int64_t>(a.n_groups, a.a.rows) - 1);
  const int pairs = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(sms / 2, most)));
  auto run = [&](auto kern) -> cudaError_t {
    const cudaError_t err = set_dyn_smem_on_device(reinterpret_cast<const void*>(kern), kSmem);
    if (err != cudaSuccess) return err;
    return launch_pdl<2>(kern, dim3(2 * pairs), dim3(kThreads), kSmem, s, maps, p);
  };
  auto with_act = [&](auto out) -> cudaError_t {
    constexpr int OUT = decltype(out)::value;
    switch (a.act) {
      case MOECA_ACT_GELU: return run(q8_matmul_kernel<OUT, MOECA_ACT_GELU>);
      case MOECA_ACT_GELU_TANH: return run(q8_matmul_kernel<OUT, MOECA_ACT_GELU_TANH>);
      default: return run(q8_matmul_kernel<OUT, MOECA_ACT_NONE>);
    }
  };
  switch (a.out_format) {
    case MOECA_F32: return with_act(std::integral_constant<int, MOECA_F32>());
    case MOECA_BF16: return with_act(std::integral_constant<int, MOECA_BF16>());
    case MOECA_E4M3: return with_act(std::integral_constant<int, MOECA_E4M3>());
    default: return with_act(std::integral_constant<int, MOECA_E5M2>());
  }
}

}  // namespace moeca
