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
// CTA; n a multiple of 16 up to 224, chosen per group so that its tiles are as
// even and as narrow as its rows allow), K in stages of two blocks of 128.
// The weights take the wide side because a group's rows are few and ragged,
// its weights neither.  Two accumulators of 224 TMEM columns, so that a tile's
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
// One launch after a flush of L2: 16384 x 6912 x 2560 to bf16 172 us (3.4 PFLOP/s, the
// tensor pipe 0.90 active under the power cap; 201 where launch follows launch and the
// clock falls); 8192 x 4608 x 1152 in 16 groups 50 us to bf16, 54 to e4m3, 64 and 66 with
// the tanh and erf GELU, where the epilogue's chains bound it; 8192 x 1152 x 4608 to
// e4m3 52 us (240 tiles are four rounds of 76 pairs).  Launch to launch in a graph,
// three sets of buffers in turn: 42, 46, 60, 63 and 40 us; two rows of 16 experts'
// 4608 x 1152 6.3 us.  224 tokens, not 192: a stage's fills and hand-overs cost the
// same for fewer MMAs (dense 195 -> 175 us); 256 leave TMEM no room for two accumulators
// and the scales.
// The tensor core's fp32 accumulator truncates where it adds: relative errors of sums
// 6.6e-8 at K 1152 and 2.6e-7 at 4608, for 4.4e-8 and 6.1e-8 with rounding.
// Every wait is bounded as in the other tensor-core kernels; a wait that runs
// out writes the caller's status word.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "moeca_probe.h"
#include "q8.cuh"
#include "tc_common.cuh"

namespace moeca {
namespace {

constexpr int kBM = 128;                  // weight rows per CTA (half of the MMA's M)
constexpr int kSub = 2;                   // K blocks of 128 per stage
constexpr int kMaxN = kQ8TileRows;        // token rows per tile
constexpr int kBoxes = kMaxN / 16;        // token boxes of 8, 16, .., 112 rows
constexpr int kMaxStages = 5;
constexpr int kRingBytes = 192 * 1024;    // weight slots first, then token slots
constexpr int kWBytes = kBM * kQ8Block;   // 16 KB: one weight block
constexpr int kWSlot = kSub * kWBytes;
constexpr int kSfStages = 4;              // scale words of 4 K blocks each
constexpr int kSfCols = 16;               // TMEM columns of one: 4 for the weights, from 8 on the tokens
constexpr int kSfBase = 2 * kMaxN;
constexpr int kEpiWarps = 8;              // warps 2-9
constexpr int kParts = kEpiWarps / 4;     // warps per lane quadrant
constexpr int kChunks = (kMaxN / 32 + kParts - 1) / kParts;  // chunks of 32 tokens a part has in a tile, at most
constexpr int kSfWarp = 2 + kEpiWarps;    // warps 10-13
constexpr int kTokWarp = kSfWarp + 4;
constexpr int kThreads = 32 * (kTokWarp + 1);
constexpr int kTmemCols = 512;
constexpr int kMaxGroups = 512;
static_assert(kSfBase + kSfStages * kSfCols <= kTmemCols, "TMEM");
static_assert(kMaxN <= 256, "eight scale columns");
static_assert(2 * kBM == kQ8TileCols, "tile width");

// Behind the ring: what the warps share.
struct Shared {
  int units[kMaxGroups + 1];              // first unit of each group
  int lo[kMaxGroups], rows[kMaxGroups];   // first row, rows
  alignas(16) uint32_t top[kParts][2][4][32];         // [part][buffer][quadrant][token]: largest |z| bits
  alignas(16) uint32_t stage[kEpiWarps][256];  // a chunk on its way out: 32 x 32 bytes, or 16 x 32 bf16
  alignas(16) float inv[kEpiWarps][32];   // 1 / scale of the chunk's tokens, read four at a time
  uint64_t full[kMaxStages], empty[kMaxStages], sf_full[kSfStages], sf_empty[kSfStages], tfull[2], tempty[2], drain;
  uint32_t tmem;
  int max_n;
  volatile int abort_flag;
  unsigned long long wait_ns;
};
constexpr int kSmem = kRingBytes + sizeof(Shared) + 1024;
static_assert(kSmem <= 227 * 1024, "shared memory");

struct Maps {
  CUtensorMap w;             // weights, box 128 rows
  CUtensorMap act[kBoxes];   // token rows, boxes of 8 .. 112 rows
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

// The four MMAs of one K block (128 values), issued by the lane whose `issue`
// is set; all lanes of the warp run it, so that the operands stay in uniform
// registers (one thread alone spent longer moving them there than the MMAs
// take).  acc: 0 where the block is the tile's first.
__device__ __forceinline__ void mma_mx_block(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                             uint32_t sf_a, uint32_t sf_b, uint32_t acc, uint32_t issue) {
  constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);  // smem_desc's bits 32-63
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %8, 0;\n"
      " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a, b, %3, [%6], [%7], p;\n"
      " add.s64 a, a, 2;\n add.s64 b, b, 2;\n setp.eq.b32 p, 0, 0;\n"
      " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a, b, %3, [%6], [%7], p;\n"
      " add.s64 a, a, 2;\n add.s64 b, b, 2;\n"
      " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a, b, %3, [%6], [%7], p;\n"
      " add.s64 a, a, 2;\n add.s64 b, b, 2;\n"
      " @e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a, b, %3, [%6], [%7], p;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kHi), "r"(sf_a), "r"(sf_b), "r"(issue)
      : "memory");
}
__device__ __forceinline__ void commit_pair_if(uint32_t bar, uint32_t issue, uint16_t ranks = 3) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %2, 0;\n"
      " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar),
      "h"(ranks), "r"(issue)
      : "memory");
}
// Arrive on a barrier of either CTA without a release: what is handed over lies
// in TMEM and is ordered by the tcgen05 fences; a release would wait for the
// warp's global accesses in flight (16 us of 50 in products with short K).
__device__ __forceinline__ void arrive_relaxed(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Bounded wait for phase `parity` of a barrier.  False when it has run out, or
// another of the CTA's has.
__device__ __noinline__ bool wait_bar(uint32_t bar, uint32_t parity, Shared* sh) {
  unsigned long long t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (mbar_try(bar, parity)) return true;
    if ((it & 255u) == 0) {
      if (sh->abort_flag) return false;
      const unsigned long long now = globaltimer();
      if (t0 == 0) t0 = now;
      else if (now - t0 > sh->wait_ns) return false;
    }
  }
}
// The same with the first try inline: one thread runs a ring's loop.
__device__ __forceinline__ bool wait_hot(uint32_t bar, uint32_t parity, Shared* sh) {
  return mbar_try(bar, parity) || wait_bar(bar, parity, sh);
}
// Every lane's bounded wait, the first try inline; the same answer in all lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, Shared* sh) {
  if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
  return __all_sync(0xffffffffu, wait_bar(bar, parity, sh));
}

// 2^x and 1 / x of the special-function unit (about 2^-22 relative).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// GELU of a chunk's values (Eq. 5), z (1 + h) / 2 with h rounded to fp32 as in
// gelu_f: where h is -1 the result is 0, so that an 8-bit block of nothing else has
// the scale of zeros.
// erf form: |h| = erf(|z| / sqrt 2) = 1 - 2^(-|z| Q(|z|)).  -log2 erfc(a / sqrt 2) / a is
// smooth, about 1.15 + 0.46 a + .., so that a polynomial Q of degree 8, fitted for
// the smallest largest error in h over 0 .. 5.8 (where 1 - h is below half a step of
// fp32), is within 2.3e-9 of it, and 2^-g turns g's rounding into little of h.
// tanh form: |h| = 1 - 2 t, t = 1 / (1 + 2^w), w = 2 sqrt(2/pi) log2(e) (|z| + 0.044715 |z|^3):
// t is at most 1/2, and its error shrinks with it (h = 2 t - 1 of the signed w has
// twice the error at z > 1).  Two values share one reciprocal, 1/a = b / (ab): the
// special-function unit takes 8 clocks a warp for it.
// The minima take |z| where h is 1 in fp32 and keep one value's NaN out of the other.
// Largest and root mean square error over |z|, in units of 2^-24, in brackets that of
// the same formula in fp32 with erff and tanhf:
//   |z| < 1/2:     erf 1.3, 0.34 (1.4, 0.31)   tanh 2.2, 0.53 (1.5, 0.32)
//   z > 1/2:       erf 1.3, 0.40 (1.9, 0.51)   tanh 1.7, 0.40 (1.9, 0.50)
//   -1/2 .. -2:    erf 1.0, 0.21 (0.8, 0.20)   tanh 1.3, 0.26 (1.3, 0.28)
//   z < -2:        erf 0.4, 0.13 (0.5, 0.18)   tanh 0.4, 0.13 (0.4, 0.13)
// (a Newton step on t brings the tanh form's first line to 1.6, 0.44 and costs 1.9 us of 60).
template <int ACT>
__device__ __forceinline__ void activate(float (&z)[32]) {
  constexpr float kLog2e = 1.44269504f;
  const auto both = [](float v) { return make_float2(v, v); };
  if constexpr (ACT != MOECA_ACT_NONE) {
#pragma unroll
    for (int i0 = 0; i0 < 32; i0 += 8) {
      float2 v[4], h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = make_float2(z[i0 + 2 * i], z[i0 + 2 * i + 1]);
      if constexpr (ACT == MOECA_ACT_GELU_TANH) {
        float2 d[4], t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = make_float2(fminf(fabsf(v[i].x), 6.f), fminf(fabsf(v[i].y), 6.f));
          const float2 w = mul2(a, fma2(both(0.0713548163f * kLog2e), mul2(a, a), both(1.5957691216f * kLog2e)));
          d[i] = add2(both(1.f), make_float2(ex2(w.x), ex2(w.y)));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = mul2(both(rcp(d[i].x * d[i].y)), make_float2(d[i].y, d[i].x));
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = fma2(both(-2.f), t[i], both(1.f));
      } else {
        constexpr float kQ[9] = {-1.15110421f, -0.459221452f, -0.0524347648f, 0.0069311196f, 1.49909565e-05f, -0.000284347712f, 7.49738392e-05f, -9.56023268e-06f, 5.12861789e-07f};
        float2 a[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] = make_float2(fminf(fabsf(v[i].x), 5.8f), fminf(fabsf(v[i].y), 5.8f));
          q[i] = both(kQ[8]);
        }
#pragma unroll
        for (int c = 7; c >= 0; --c)
#pragma unroll
          for (int i = 0; i < 4; ++i) q[i] = fma2(q[i], a[i], both(kQ[c]));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 w = mul2(a[i], q[i]);
          h[i] = add2(both(1.f), make_float2(-ex2(w.x), -ex2(w.y)));
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 half = mul2(v[i], both(0.5f));
        const float2 r = fma2(make_float2(fabsf(half.x), fabsf(half.y)), h[i], half);
        z[i0 + 2 * i] = r.x;
        z[i0 + 2 * i + 1] = r.y;
      }
    }
  }
}

// Bits of the largest |v| over the warp's lanes; at least kNonFinite where one is NaN.
__device__ __forceinline__ uint32_t warp_top(float v) {
  float r;
  asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return abs_bits(r);
}

// Barrier over the four epilogue warps of a part (ids 1 to kParts); true if `ok` in all.
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
  bool w_e5, t_e5, wide;       // wide: 16-byte stores of bf16 rows
  int32_t* status;
  Q8Waits waits;
};

// Stores under a predicate, without a branch (a branch per store keeps the
// stores' address arithmetic from overlapping).
__device__ __forceinline__ void store_if(bool on, void* to, const uint4& v) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %5, 0;\n @p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n}" ::"l"(to), "r"(v.x),
               "r"(v.y), "r"(v.z), "r"(v.w), "r"(static_cast<uint32_t>(on))
               : "memory");
}
__device__ __forceinline__ void store_if(bool on, void* to, float v) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %2, 0;\n @p st.global.f32 [%0], %1;\n}" ::"l"(to), "f"(v),
               "r"(static_cast<uint32_t>(on))
               : "memory");
}
__device__ __forceinline__ void store_if(bool on, void* to, __nv_bfloat16 v) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %2, 0;\n @p st.global.b16 [%0], %1;\n}" ::"l"(to),
               "h"(__bfloat16_as_ushort(v)), "r"(static_cast<uint32_t>(on))
               : "memory");
}

// Epilogue of one chunk: 32 features (lanes) x 32 tokens (z), all four
// quadrants of the part together.  row: lane t's output row of token t, or -1.
// Rows go out through shared memory in 16-byte pieces; rows that are not
// aligned for them, and fp32 rows, straight from the registers, a token's 32
// features at a time.
template <int OUT>
__device__ __forceinline__ void store_chunk(const MatmulParams& p, Shared& sh, float (&z)[32], int row, int feat0,
                                            int block, int lane, int warp, int part, int quad, int buf) {
  uint32_t* stage = sh.stage[warp - 2];
  if constexpr (OUT == MOECA_F32 || OUT == MOECA_BF16) {
    if (feat0 >= p.N) return;
    if (OUT == MOECA_BF16 && p.wide) {
      // 16 tokens at a time; lanes 2i and 2i + 1 swap halves, so that each holds
      // the feature pair of every other token.
      const int f = feat0 + (lane & 3) * 8, left = p.N - f, odd = lane & 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i % 2 == 0) {
          __syncwarp();  // what was staged before has been read
          uint32_t own[8], got[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) own[t] = pack_bf16(z[8 * i + 2 * t], z[8 * i + 2 * t + 1]);
#pragma unroll
          for (int t = 0; t < 8; ++t) got[t] = __shfl_xor_sync(0xffffffffu, own[t], 1);
#pragma unroll
          for (int t = 0; t < 8; ++t)
            stage[(2 * t + odd) * 16 + (lane >> 1)] = __byte_perm(own[t], got[t], odd ? 0x3276 : 0x5410);
          __syncwarp();
        }
        const uint4 v = *reinterpret_cast<const uint4*>(stage + ((i & 1) * 8 + (lane >> 2)) * 16 + (lane & 3) * 4);
        const int r = __shfl_sync(0xffffffffu, row, i * 8 + (lane >> 2));
        uint8_t* at = p.out + r * p.out_stride + f * 2;
        store_if(r >= 0 && left >= 8, at, v);
        if (feat0 + 32 > p.N && r >= 0 && left > 0 && left < 8) {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int j = 0; j < 7; ++j)
            if (j < left) reinterpret_cast<uint16_t*>(at)[j] = static_cast<uint16_t>(w[j >> 1] >> 16 * (j & 1));
        }
      }
    } else {
      using T = std::conditional_t<OUT == MOECA_F32, float, __nv_bfloat16>;
      const uint32_t rows = __ballot_sync(0xffffffffu, row >= 0), live = feat0 + lane < p.N ? rows : 0u;
      uint8_t* base = p.out + static_cast<int64_t>(feat0 + lane) * sizeof(T);
      const int64_t mine = row * p.out_stride;
#pragma unroll
      for (int t = 0; t < 32; ++t) store_if(live >> t & 1, base + __shfl_sync(0xffffffffu, mine, t), Elem<T>::from_f(z[t]));
    }
  } else {
    constexpr bool E5 = OUT == MOECA_E5M2;
    if (feat0 + 32 > p.N && feat0 + lane >= p.N) {  // not a feature: another group's weights, or none
#pragma unroll
      for (int t = 0; t < 32; ++t) z[t] = 0.f;
    }
    // The tokens' largest |z| over the warp's features, then over the block's.
    const auto exchange = [&](auto magnitude) {
      uint32_t* mine = sh.top[part][buf][quad];
#pragma unroll
      for (int t = 0; t < 32; t += 4) {
        uint4 m;
        m.x = warp_top(magnitude(z[t]));
        m.y = warp_top(magnitude(z[t + 1]));
        m.z = warp_top(magnitude(z[t + 2]));
        m.w = warp_top(magnitude(z[t + 3]));
        if (lane == 0) *reinterpret_cast<uint4*>(mine + t) = m;
      }
      part_sync(part, true);
      uint32_t top = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) top = max(top, sh.top[part][buf][q][lane]);
      return top;
    };
    uint32_t top = exchange([](float v) { return v; });
    const bool odd = __any_sync(0xffffffffu, row >= 0 && top >= kNonFinite);  // the same in the part's four warps
    if (odd) {
      part_sync(part, true);  // all have read the first maxima
      top = exchange([](float v) { return abs_bits(v) < kNonFinite ? v : 0.f; });
    }
    const int byte = scale_byte<E5>(top);
    float* inv = sh.inv[warp - 2];
    __syncwarp();
    inv[lane] = scale_inverse(byte);
    __syncwarp();
    if (quad == 0 && row >= 0) p.out_scale[row * p.os_stride + block] = static_cast<uint8_t>(byte);
    if (feat0 >= p.N) return;
    // Step by step over all eight words, so that their chains interleave.
    uint32_t word[8], got[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const float4 s = *reinterpret_cast<const float4*>(inv + 4 * t);
      const float2 lo = mul2(make_float2(z[4 * t], z[4 * t + 1]), make_float2(s.x, s.y));
      const float2 hi = mul2(make_float2(z[4 * t + 2], z[4 * t + 3]), make_float2(s.z, s.w));
      z[4 * t] = lo.x; z[4 * t + 1] = lo.y; z[4 * t + 2] = hi.x; z[4 * t + 3] = hi.y;
      word[t] = encode2<E5>(z[4 * t], z[4 * t + 1]) | encode2<E5>(z[4 * t + 2], z[4 * t + 3]) << 16;
    }
    if (odd) {
      // Infinities (see encode2).
#pragma unroll
      for (int t = 0; t < 32; ++t) word[t >> 2] += abs_bits(z[t]) == kNonFinite ? 1u << 8 * (t & 3) : 0u;
    }
    // Four features' bytes of one token per lane from four tokens' bytes of one
    // feature: lane j of each four lanes gets token j's.
    const uint32_t sel1 = lane & 1 ? 0x3715 : 0x6240, sel2 = lane & 2 ? 0x3276 : 0x5410;
#pragma unroll
    for (int t = 0; t < 8; ++t) got[t] = __shfl_xor_sync(0xffffffffu, word[t], 1);
#pragma unroll
    for (int t = 0; t < 8; ++t) word[t] = __byte_perm(word[t], got[t], sel1);
#pragma unroll
    for (int t = 0; t < 8; ++t) got[t] = __shfl_xor_sync(0xffffffffu, word[t], 2);
#pragma unroll
    for (int t = 0; t < 8; ++t) stage[(4 * t + (lane & 3)) * 8 + (lane >> 2)] = __byte_perm(word[t], got[t], sel2);
    __syncwarp();
    const int f = feat0 + (lane & 1) * 16, left = p.N - f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(stage + (i * 16 + (lane >> 1)) * 8 + (lane & 1) * 4);
      const int r = __shfl_sync(0xffffffffu, row, i * 16 + (lane >> 1));
      uint8_t* at = p.out + r * p.out_stride + f;
      store_if(r >= 0 && left >= 16, at, v);
      if (feat0 + 32 > p.N && r >= 0 && left > 0 && left < 16) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 15; ++j)
          if (j < left) at[j] = static_cast<uint8_t>(w[j >> 2] >> 8 * (j & 3));
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

  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    sh.wait_ns = p.waits.ns;
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(smem_u32(&sh.full[s]), 1 + (p.waits.stall == MOECA_Q8_OPERANDS));
      mbar_init(smem_u32(&sh.empty[s]), 1);
    }
    for (int s = 0; s < kSfStages; ++s) {
      mbar_init(smem_u32(&sh.sf_full[s]), 8 + (p.waits.stall == MOECA_Q8_SCALES));
      mbar_init(smem_u32(&sh.sf_empty[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&sh.tfull[s]), 1 + (p.waits.stall == MOECA_Q8_ACCUMULATORS));
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
  cluster_arrive();
  cluster_wait();  // both CTAs' barriers are initialised, TMEM is allocated
  tc_fence_after();
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
          if (!(ok = wait_hot(eb, par, &sh))) break;
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
          while (!mbar_try(smem_u32(&sh.full[q]), (last / nst) & 1) && globaltimer() - t0 < sh.wait_ns) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------- MMA issuer (the leader, for both CTAs) ----------------
      uint32_t issue;
      asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n selp.u32 %0, 1, 0, e;\n}" : "=r"(issue));
      const uint32_t w_lo0 = ((ring & 0x3FFFFu) >> 4) | (1u << 16), x_lo0 = ((ring_t & 0x3FFFFu) >> 4) | (1u << 16);
      const uint32_t full0 = smem_u32(&sh.full[0]), sf_full0 = smem_u32(&sh.sf_full[0]), sf_empty0 = smem_u32(&sh.sf_empty[0]);
      int slot = 0, acc = 0, sfs = 0, g = 0;
      uint32_t par = 0u, acc_phase = 0, sf_par = 0;
      bool ok = true;
      for (int u = pair; u < units; u += n_pairs) {
        const Unit t = unit_at(sh, u, g, nw);
        g = t.g;
        if (!(ok = warp_wait(smem_u32(&sh.tempty[acc]), acc_phase ^ 1u, &sh))) break;
        const uint32_t d_tmem = tmem + static_cast<uint32_t>(acc * kMaxN);
        const uint32_t idesc = mx_desc(t.n, p.w_e5, p.t_e5), x_sub = static_cast<uint32_t>(t.n >> 1) * kQ8Block >> 4;
        for (int k = 0; k < ks; ++k) {
          if (k % (4 / kSub) == 0 && !(ok = warp_wait(sf_full0 + sfs * 8, sf_par, &sh))) break;
          if (!(ok = warp_wait(full0 + slot * 8, par, &sh))) break;
          tc_fence_after();
          const uint32_t sf = tmem + kSfBase + sfs * kSfCols;
          const uint32_t w_lo = w_lo0 + slot * (kWSlot >> 4), x_lo = x_lo0 + slot * (t_slot >> 4);
          // The values past K in the last block are zeros on both sides.
#pragma unroll
          for (int q = 0; q < kSub; ++q) {
            const int b = k * kSub + q;
            const uint32_t id = static_cast<uint32_t>(b & 3);
            if (q == 0 || b < kb)
              mma_mx_block(d_tmem, w_lo + q * (kWBytes >> 4), x_lo + q * x_sub, idesc | id << 4 | id << 29, sf, sf + 8,
                           b != 0, issue);
          }
          commit_pair_if(empty0 + slot * 8, issue);
          if (k % (4 / kSub) == 4 / kSub - 1 || k == ks - 1) {
            commit_pair_if(sf_empty0 + sfs * 8, issue);
            if (++sfs == kSfStages) {
              sfs = 0;
              sf_par ^= 1u;
            }
          }
          if (++slot == nst) {
            slot = 0;
            par ^= 1u;
          }
        }
        if (!ok) break;
        commit_pair_if(smem_u32(&sh.tfull[acc]), issue);
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
      if (lane == 0 && !ok) {
        if (!sh.abort_flag) report_status(p.status, MOECA_ERR_TIMEOUT, 701);
        sh.abort_flag = 1;
      }
      // Every MMA issued so far has completed once the drain barrier fires: a
      // commit covers what its own thread issued, so the issuing lane makes it.
      commit_pair_if(smem_u32(&sh.drain), issue, 1);
      if (issue) {
        const unsigned long long t0 = globaltimer();
        while (!mbar_try(smem_u32(&sh.drain), 0) && globaltimer() - t0 < sh.wait_ns) {
        }
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
        if (!(ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&sh.sf_empty[sfs]), par, &sh)))) break;
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
        if (lane == 0) arrive_relaxed(full0 + sfs * 8);
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
    int acc = 0, g = 0, buf = 0, first = part;  // the part's first chunk turns, so that the parts' shares even out
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int u = pair; u < units; u += n_pairs) {
      const Unit t = unit_at(sh, u, g, nw);
      g = t.g;
      const int block = t.w * 2 + static_cast<int>(rank), feat0 = block * kBM + quad * 32;
      const bool live = feat0 + lane < p.N;
      const float bias = p.bias && live ? __ldg(p.bias + static_cast<int64_t>(g) * p.N + feat0 + lane) : 0.f;
      // A CTA whose features lie past N has no block: it only keeps in step.
      const int cols = block * kBM < p.N ? t.m_end - t.m0 : 0;
      int rows[kChunks];  // this lane's output row in each of the part's chunks
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        const int m = t.m0 + (j * kParts + first) * 32 + lane;
        rows[j] = -1;
        if (m < t.m_end) rows[j] = p.dst ? __ldg(p.dst + m) : m;
        if (rows[j] >= p.out_rows) rows[j] = -1;
      }
      ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&sh.tfull[acc]), acc_phase, &sh));
      if (!(ok = part_sync(part, ok))) break;  // all warps of the part, or none: the chunks' exchanges need all
      tc_fence_after();
      const uint32_t tb = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(acc * kMaxN);
      int c = first * 32;
      first = (first + 1) % kParts;
      if (c >= cols) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_relaxed(tempty0 + acc * 8);
      }
#pragma unroll 1
      for (; c < cols; c += 32 * kParts) {
        float z[32];
        {
          uint32_t v[32];
          tmem_ld32_async(tb + c, v);
          tmem_wait32(v);
#pragma unroll
          for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(v[i]);
        }
        if (c + 32 * kParts >= cols) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_relaxed(tempty0 + acc * 8);
        }
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          const float2 v = add2(make_float2(z[i], z[i + 1]), make_float2(bias, bias));
          z[i] = v.x;
          z[i + 1] = v.y;
        }
        activate<ACT>(z);
        const int row = rows[0];
#pragma unroll
        for (int j = 0; j + 1 < kChunks; ++j) rows[j] = rows[j + 1];
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
  // No group has more than all rows: no wider boxes than theirs.
  const int boxes = static_cast<int>(std::min<int64_t>(kBoxes, (a.a.rows + 15) / 16));
  for (int i = 0; i < kBoxes && ok; ++i) {
    if (i < boxes) ok = encode_rows(&maps.act[i], a.a, 8 * (i + 1));
    else maps.act[i] = maps.act[0];
  }
  if (!ok) return cudaErrorInvalidValue;
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  MatmulParams p{};
  p.w_scale = a.b.scale; p.w_stride = a.b.scale_stride; p.w_rows = a.b.rows;
  p.t_scale = a.a.scale; p.t_stride = a.a.scale_stride;
  p.M = static_cast<int>(a.a.rows); p.N = a.n_cols; p.K = a.a.width; p.G = a.n_groups;
  p.offsets = a.offsets; p.dst = a.dst; p.bias = a.bias;
  p.out = a.out.q; p.out_scale = a.out.scale;
  p.out_rows = a.out.rows; p.out_stride = a.out.q_stride; p.os_stride = a.out.scale_stride;
  p.w_e5 = a.b_e5; p.t_e5 = a.a_e5;
  p.wide = reinterpret_cast<uintptr_t>(a.out.q) % 16 == 0 && a.out.q_stride % 16 == 0;
  p.status = a.status;
  p.waits = a.waits;
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
