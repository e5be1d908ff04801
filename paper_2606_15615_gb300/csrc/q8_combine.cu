// Eq. 8 over an 8-bit branch cache, and the cache read back as it is (one
// slot, no weights, no residual) (include/moeca_q8.h):
//   out_i = x_i + g * sum_p w_p h_p,   norm_p = ||h_p||
// A value h = f d is its byte times its block's power of two, exact in fp32 (but
// past its largest value, where it is an infinity, and below its least).  Where
// scales and weights are moderate w f is exact too, and one multiply-add does for
// both with the same result; elsewhere w f could pass fp32's range or fall among
// its subnormals where w h does neither, and make a NaN of a 0: there the value
// comes first.  Two values go through one packed fp32 instruction.  Compiled
// twice: bf16 rows here, fp32 rows in q8_combine_f32.cu.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "moeca_probe.h"
#include "q8.cuh"

namespace moeca {
namespace {

#ifdef MOECA_Q8_COMBINE_F32
using TI = float;
#else
using TI = __nv_bfloat16;
#endif

constexpr int W = 8;                      // values per lane and step
constexpr int V = Elem<TI>::kVec, NV = W / V;

// Eight cache bytes as floats, without their scale.  An e5m2 byte is the upper
// byte of an fp16 value.
template <bool E5>
__device__ __forceinline__ void decode8(const uint2& h, float2 (&d)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint32_t word = t < 2 ? h.x : h.y;
    if constexpr (E5) {
      const uint32_t two = __byte_perm(word, 0u, t & 1 ? 0x3424 : 0x1404);
      d[t] = __half22float2(*reinterpret_cast<const __half2*>(&two));
    } else {
      d[t] = decode2<E5>(t & 1 ? word >> 16 : word & 0xffffu);
    }
  }
}

// Scale bytes and weights between which w f d is exact up to its rounding in
// either order: 2^-63 .. 2^63 and 2^-60 .. 2^60, or a weight of 0.
__device__ __forceinline__ bool far_scale(uint32_t byte) { return byte - 64u > 126u; }
__device__ __forceinline__ bool far_weight(float w) { return w != 0.f && !(fabsf(w) >= 0x1p-60f && fabsf(w) <= 0x1p60f); }

// y (+)= w f d, and ss plus the square sum of the 8 values: that of d times f^2,
// which passes fp32's range only where the values' squares do.  FAR: any scale
// and weight.
template <bool FIRST, bool FAR>
__device__ __forceinline__ float slot_values(const float2 (&d)[4], float f, float w, float2 (&y)[4], float ss) {
  const float wf = FAR ? w : w * f;
  const float2 w2 = make_float2(wf, wf), f2 = make_float2(f, f);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const float2 h = FAR ? mul2(f2, d[t]) : d[t];
    y[t] = FIRST ? mul2(w2, h) : fma2(w2, h, y[t]);
  }
  float2 sq = mul2(d[0], d[0]);
#pragma unroll
  for (int t = 1; t < 4; ++t) sq = fma2(d[t], d[t], sq);
  return fmaf(f * (sq.x + sq.y), f, ss);
}

// The sum of K values over the warp's lanes, value p in lane p's result: each
// step hands over half of the values that a lane still holds.
template <int K>
__device__ __forceinline__ float warp_sums(const float (&s)[K], int lane) {
  constexpr int P = K <= 1 ? 1 : K <= 2 ? 2 : K <= 4 ? 4 : K <= 8 ? 8 : 16;
  float v[P];
#pragma unroll
  for (int p = 0; p < P; ++p) v[p] = p < K ? s[p] : 0.f;
#pragma unroll
  for (int n = P / 2; n > 0; n >>= 1) {  // lanes that differ in bit n of their number
    const bool up = lane & n;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float keep = up ? v[j + n] : v[j], give = up ? v[j] : v[j + n];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, n);
    }
  }
#pragma unroll
  for (int o = P; o < 32; o <<= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}

// A lane's gate values (zeros past the row's end).
struct Gate {
  float v[W];
};
__device__ __forceinline__ Gate load_gate(const float* gp, bool vec, int left) {
  Gate g;
  if (vec && left >= W) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(gp)), b = __ldg(reinterpret_cast<const float4*>(gp) + 1);
    g.v[0] = a.x; g.v[1] = a.y; g.v[2] = a.z; g.v[3] = a.w;
    g.v[4] = b.x; g.v[5] = b.y; g.v[6] = b.z; g.v[7] = b.w;
  } else {
#pragma unroll
    for (int t = 0; t < W; ++t) g.v[t] = t < left ? __ldg(gp + t) : 0.f;
  }
  return g;
}

// ---------------------------------------------------------------------------
// Direct form: a block per token, all slots' loads in flight before any
// arithmetic.  For few tokens, as long as all blocks run at once, and for rows
// too wide for the staged form.  Launch to launch, direct against staged: 2.2 and
// 3.0 us for 8 tokens of two slots and 1152 values, 2.8 and 3.2 for 608, 4.8 and 3.5
// for 1216; 3.8 and 4.3 for 304 tokens of eight slots, 6.7 and 4.3 for 608.
// ---------------------------------------------------------------------------
constexpr int kDirectWarps = 8;
// Blocks per SM that the registers allow.
constexpr int direct_blocks(int k) { return k <= 2 ? 4 : k <= 4 ? 3 : k <= 8 ? 2 : 1; }

template <bool E5, int KMAX>
__global__ void __launch_bounds__(kDirectWarps * 32, direct_blocks(KMAX)) q8_combine_kernel(const Q8CombineArgs a) {
  __shared__ float part[kDirectWarps][KMAX];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t i = blockIdx.x;
  const int k = a.k, width = a.c.width, chunks = (width + W - 1) / W;
  float w[KMAX], ss[KMAX];
  int row[KMAX];  // < 0: the slot holds nothing
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    w[p] = ss[p] = 0.f;
    row[p] = -1;
    if (p < k) {
      const int64_t at = i * k + p;
      const int r = a.rows ? __ldg(a.rows + at) : static_cast<int>(i);
      if (r >= 0 && r < a.c.rows) {
        row[p] = r;
        w[p] = a.weights ? __ldg(a.weights + at) : 1.f;
      }
    }
  }
  const TI* x = a.x ? static_cast<const TI*>(a.x) + i * a.x_stride : nullptr;
  TI* out = static_cast<TI*>(a.out) + i * a.out_stride;
  const float* gate = a.gate ? a.gate + (i / a.seq) * a.gate_stride : nullptr;
  for (int c = threadIdx.x; c < chunks; c += kDirectWarps * 32) {
    const int left = width - c * W;
    uint2 h[KMAX];
    float f[KMAX], xs[W];
    Gate g{};
    if (gate) g = load_gate(gate + c * W, a.gate_vec, left);
#pragma unroll
    for (int p = 0; p < KMAX; ++p) {
      h[p] = make_uint2(0u, 0u);
      f[p] = 1.f;
      if (row[p] >= 0) {
        h[p] = __ldg(reinterpret_cast<const uint2*>(a.c.q + row[p] * a.c.q_stride + c * W));
        f[p] = scale_value(__ldg(a.c.scale + row[p] * a.c.scale_stride + (c >> 4)));
      }
    }
    if (x) {
      if (a.vec && left >= W) {
#pragma unroll
        for (int j = 0; j < NV; ++j) load_vec(x + c * W + j * V, &xs[j * V]);
      } else {
#pragma unroll
        for (int t = 0; t < W; ++t) xs[t] = t < left ? Elem<TI>::to_f(x[c * W + t]) : 0.f;
      }
    }
    if (left < W) {  // the bytes past the row's width are anything
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        h[p].x &= left >= 4 ? 0xffffffffu : (1u << 8 * left) - 1;
        h[p].y &= left <= 4 ? 0u : (1u << 8 * (left - 4)) - 1;
      }
    }
    float2 y[4];
#pragma unroll
    for (int p = 0; p < KMAX; ++p) {
      float2 d[4];
      decode8<E5>(h[p], d);
      ss[p] = p == 0 ? slot_values<true, true>(d, f[p], w[p], y, ss[p]) : slot_values<false, true>(d, f[p], w[p], y, ss[p]);
    }
    float o[W] = {y[0].x, y[0].y, y[1].x, y[1].y, y[2].x, y[2].y, y[3].x, y[3].y};
    if (gate) {
#pragma unroll
      for (int t = 0; t < W; ++t) o[t] *= g.v[t];
    }
    if (x) {
#pragma unroll
      for (int t = 0; t < W; ++t) o[t] += xs[t];
    }
    if (a.vec && left >= W) {
#pragma unroll
      for (int j = 0; j < NV; ++j) store_vec(out + c * W + j * V, &o[j * V]);
    } else {
#pragma unroll
      for (int t = 0; t < W; ++t)
        if (t < left) out[c * W + t] = Elem<TI>::from_f(o[t]);
    }
  }
  if (!a.norms) return;
  const float s = warp_sums<KMAX>(ss, lane);
  if (lane < KMAX) part[warp][lane] = s;
  __syncthreads();
  if (threadIdx.x < k) {
    float t = 0.f;
    for (int q = 0; q < kDirectWarps; ++q) t += part[q][threadIdx.x];
    a.norms[i * k + threadIdx.x] = sqrtf(t);
  }
}

// ---------------------------------------------------------------------------
// Staged form: a warp walks its tokens i = w, w + W, ... (W the grid's warps),
// each brought into its buffer in shared memory by bulk copies, a lane per row
// (x's row is one more), so that the bytes in flight hang neither on registers
// nor on instructions, and the next token's copies start as soon as the last
// one's values are used.  The next token's row list is loaded a token ahead.
// One buffer per warp: twice the warps hide more of the arithmetic's latency
// than a second buffer does.
//
// Decoding is what costs next to HBM here: a conversion of two e4m3 values
// takes a scheduler 4 clocks, their widening 3; the loop over a token's values
// holds no branch and no select, so that the slots' chains interleave.  For that
// the buffer is prepared once per token: slots that hold nothing and the bytes
// past the row's width are zeros, and the scales are turned into floats by block.
// Tokens with a far scale or weight (see slot_values) have a loop of their own: one
// loop with the value first took 103 us for 95 at eight slots in e5m2.
//
// Rows of x and out that do not start at 16 bytes (VEC false): x is copied in
// the aligned pieces that hold it and shifted as it is read; out is put
// together in the buffer and leaves it in aligned pieces.
//
// One launch after a flush of L2: 32768 tokens x 8 slots x 1152 (e4m3, gated, bf16) 103 us
// (4.5 TB/s, bound by decoding and its latency; 172 us with loads to registers), 4096 x
// 3 x 2560 23 us, 20000 x 1 x 1152 40 us (5.3 TB/s), 60000 rows of 1152 read back 44 us, of
// 1153 62 us: a read's issue slots are 0.71 busy and HBM 0.44 (a token's fixed costs
// weigh most with one slot, and the square sums are formed for nobody).
// ---------------------------------------------------------------------------
constexpr int kStageWarps = 2;
constexpr int kStageSm = 227 * 1024, kStageMax = 112 * 1024;  // shared memory of an SM, and the most a block takes
// Blocks per SM that the registers allow (the grid is persistent: none may wait for another).
constexpr int stage_blocks(int k) { return k <= 2 ? 16 : k <= 4 ? 12 : k <= 9 ? 8 : 6; }
// The fewest slots that run with a kernel of `kmax` (see staged()).
__host__ __device__ constexpr int least_slots(int kmax) { return kmax == 6 ? 5 : kmax == 8 ? 7 : kmax == 16 ? 10 : kmax; }

// A warp's buffer: the slots' rows, x's, out's (VEC false), the scale words, the
// scales as floats.
struct StageLayout {
  int row, value, words, blocks, x_at, out_at, word_at, scale_at, bytes;
};
template <bool VEC>
__host__ __device__ inline StageLayout stage_layout(int k, int width, bool x) {
  StageLayout s;
  s.row = (width + 15) / 16 * 16;
  s.value = (width * static_cast<int>(sizeof(TI)) + 15) / 16 * 16 + (VEC ? 0 : 16);
  s.blocks = (width + kQ8Block - 1) / kQ8Block;
  s.words = (s.blocks + 3) / 4;
  s.x_at = k * s.row;
  s.out_at = s.x_at + (x ? s.value + 16 : 0);  // a last piece may be read past the copied ones
  s.word_at = s.out_at + (VEC ? 0 : s.value + 32);  // a piece before the first and one after the last may be read
  s.scale_at = (s.word_at + k * s.words * 4 + 15) / 16 * 16;
  s.bytes = (s.scale_at + k * s.blocks * 4 + 15) / 16 * 16;
  return s;
}

template <bool E5, int KMAX, bool VEC, bool GATED>
__global__ void __launch_bounds__(kStageWarps * 32, stage_blocks(KMAX)) q8_combine_staged_kernel(const Q8CombineArgs a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ __align__(8) uint64_t bars[kStageWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar = smem_u32(&bars[warp]);
  if (lane == 0) mbar_init(bar, 1 + (a.waits.stall == MOECA_Q8_COPIES));
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  pdl_entry();
  const int k = a.k, width = a.c.width, chunks = (width + W - 1) / W;
  const StageLayout L = stage_layout<VEC>(k, width, a.x != nullptr);
  uint8_t* const buf = dyn + static_cast<size_t>(warp) * L.bytes;
  const int64_t w0 = static_cast<int64_t>(blockIdx.x) * kStageWarps + warp, step = static_cast<int64_t>(gridDim.x) * kStageWarps;
  const TI* x = static_cast<const TI*>(a.x);

  // Lane p holds slot p's row (-1: nothing) and weight of the next token to fetch.
  int row = -1;
  float weight = 0.f;
  const auto look_up = [&](int64_t i) {
    row = -1;
    weight = 0.f;
    if (i < a.T && lane < k) {
      const int r = a.rows ? __ldg(a.rows + i * k + lane) : static_cast<int>(i);
      if (r >= 0 && r < a.c.rows) {
        row = r;
        weight = a.weights ? __ldg(a.weights + i * k + lane) : 1.f;
      }
    }
  };
  // Start token i's copies.  All lanes have left the buffer.
  const auto fetch = [&](int64_t i) {
    if (i >= a.T) return;
    const uint32_t slots = __ballot_sync(0xffffffffu, row >= 0);
    const uint8_t* xr = reinterpret_cast<const uint8_t*>(x + (x ? i * a.x_stride : 0));
    const uint32_t m = VEC ? 0u : static_cast<uint32_t>(reinterpret_cast<uintptr_t>(xr)) & 15u;
    const uint32_t x_bytes = x ? (m + static_cast<uint32_t>(width * sizeof(TI)) + 15) / 16 * 16 : 0u;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the copies: the lanes' own uses of the buffer
    if (lane == 0) mbar_expect_tx(bar, __popc(slots) * L.row + x_bytes);
    __syncwarp();
    if (row >= 0) bulk_g2s(smem_u32(buf + lane * L.row), a.c.q + row * a.c.q_stride, L.row, bar);
    if (lane == 31 && x) bulk_g2s(smem_u32(buf + L.x_at), xr - m, x_bytes, bar);
    for (int j0 = 0; j0 < k * L.words; j0 += 32) {  // the scales, four blocks at a time
      const int j = j0 + lane, p = min(j / L.words, k - 1), r = __shfl_sync(0xffffffffu, row, p);
      if (j < k * L.words && r >= 0)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(buf + L.word_at + j * 4)),
                     "l"(a.c.scale + r * a.c.scale_stride + (j - p * L.words) * 4)
                     : "memory");
    }
  };

  look_up(w0);
  uint32_t parity = 0;
  float w_now = weight;
  uint32_t slots = __ballot_sync(0xffffffffu, row >= 0);
  fetch(w0);
  look_up(w0 + step);
  for (int64_t i = w0; i < a.T; i += step) {
    // The gate's values are loaded a step ahead of their use.
    const float* gate = GATED ? a.gate + (i / a.seq) * a.gate_stride : nullptr;
    Gate next{};
    if (GATED && lane < chunks) next = load_gate(gate + lane * W, a.gate_vec, width - lane * W);
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!__all_sync(0xffffffffu, mbar_wait_for(bar, parity, a.waits.ns))) {
      if (lane == 0) report_status(a.status, MOECA_ERR_TIMEOUT, 710);
      mbar_wait_for(bar, parity, a.waits.ns);  // the copies still write this block's memory: as long again for them
      return;
    }
    parity ^= 1u;
    __syncwarp();
    // Prepare the buffer: zeros for what is not there, scales as floats.
    bool far = far_weight(w_now);
    float* scales = reinterpret_cast<float*>(buf + L.scale_at);
    for (int j = lane; j < k * L.blocks; j += 32) {
      const int p = j / L.blocks, b = j - p * L.blocks;
      const uint32_t byte = slots >> p & 1 ? buf[L.word_at + p * L.words * 4 + b] : 127u;
      scales[j] = scale_value(byte);
      far |= far_scale(byte);
    }
    if (lane < k && width < L.row) {
      for (int t = width; t < L.row; ++t) buf[lane * L.row + t] = 0;
    }
    for (int p = 0; p < k; ++p)
      if (!(slots >> p & 1))
        for (int c = lane * 16; c < L.row; c += 512) *reinterpret_cast<uint4*>(buf + p * L.row + c) = make_uint4(0u, 0u, 0u, 0u);
    float wp[KMAX];
#pragma unroll
    for (int p = 0; p < KMAX; ++p) wp[p] = __shfl_sync(0xffffffffu, w_now, p);
    far = __any_sync(0xffffffffu, far);
    __syncwarp();

    TI* out = static_cast<TI*>(a.out) + i * a.out_stride;
    const uint32_t mx = VEC || !x ? 0u : static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x + i * a.x_stride)) & 15u;
    const uint32_t mo = VEC ? 0u : static_cast<uint32_t>(reinterpret_cast<uintptr_t>(out)) & 15u;
    float ss[KMAX];
#pragma unroll
    for (int p = 0; p < KMAX; ++p) ss[p] = 0.f;
    const auto add_up = [&](auto any) {
      constexpr bool FAR = decltype(any)::value;
      for (int c = lane; c < chunks; c += 32) {
        const int left = width - c * W;
        const Gate now = next;
        if (GATED && c + 32 < chunks) next = load_gate(gate + (c + 32) * W, a.gate_vec, left - 32 * W);
        float2 y[4];
#pragma unroll
        for (int p = 0; p < KMAX; ++p) {
          // A slot past the last has the first one's bytes, cleared: an infinity times its weight of 0 would be NaN.
          const int at = p < k ? p : 0;
          uint2 h = *reinterpret_cast<const uint2*>(buf + at * L.row + c * W);
          if (p >= least_slots(KMAX)) {
            const uint32_t keep = p < k ? 0xffffffffu : 0u;
            h.x &= keep;
            h.y &= keep;
          }
          float2 d[4];
          decode8<E5>(h, d);
          const float f = scales[at * L.blocks + (c >> 4)];
          ss[p] = p == 0 ? slot_values<true, FAR>(d, f, wp[p], y, ss[p]) : slot_values<false, FAR>(d, f, wp[p], y, ss[p]);
        }
        float o[W] = {y[0].x, y[0].y, y[1].x, y[1].y, y[2].x, y[2].y, y[3].x, y[3].y};
        if constexpr (GATED) {
#pragma unroll
          for (int t = 0; t < W; ++t) o[t] *= now.v[t];
        }
        if (x) {
          float xs[W];
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            const uint4* piece = reinterpret_cast<const uint4*>(buf + L.x_at) + c * NV + j;
            if constexpr (VEC) unpack_vec(*piece, &xs[j * V], static_cast<TI*>(nullptr));
            else unpack_vec(shifted<TI>(piece[0], piece[1], mx), &xs[j * V], static_cast<TI*>(nullptr));
          }
#pragma unroll
          for (int t = 0; t < W; ++t) o[t] += xs[t];
        }
        if constexpr (VEC) {
          if (left >= W) {
#pragma unroll
            for (int j = 0; j < NV; ++j) store_vec(out + c * W + j * V, &o[j * V]);
          } else {
#pragma unroll
            for (int t = 0; t < W; ++t)
              if (t < left) out[c * W + t] = Elem<TI>::from_f(o[t]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < NV; ++j)
            store_vec(reinterpret_cast<TI*>(buf + L.out_at + 16) + c * W + j * V, &o[j * V]);
        }
      }
    };
    if (far) add_up(std::true_type());
    else add_up(std::false_type());
    __syncwarp();  // all have read the slots and x
    if constexpr (!VEC) {
      // out's aligned pieces, each from the two staged ones that it straddles; its
      // first and last values alone where a piece is another row's too.
      const uint32_t end = mo + width * sizeof(TI);
      uint8_t* base = reinterpret_cast<uint8_t*>(out) - mo;
      for (uint32_t t = lane * 16; t < end; t += 512) {
        const uint4* staged = reinterpret_cast<const uint4*>(buf + L.out_at + t + (mo ? 0 : 16));
        const uint4 v = shifted<TI>(staged[0], staged[1], mo ? 16 - mo : 0u);
        if (t >= mo && t + 16 <= end) {
          *reinterpret_cast<uint4*>(base + t) = v;
        } else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (uint32_t q = 0; q < 16; q += sizeof(TI)) {
            if (t + q < mo || t + q >= end) continue;
            if constexpr (sizeof(TI) == 2) *reinterpret_cast<uint16_t*>(base + t + q) = static_cast<uint16_t>(w[q / 4] >> 8 * (q & 3));
            else *reinterpret_cast<uint32_t*>(base + t + q) = w[q / 4];
          }
        }
      }
      __syncwarp();
    }
    w_now = weight;
    slots = __ballot_sync(0xffffffffu, row >= 0);
    fetch(i + step);
    look_up(i + 2 * step);
    if (a.norms) {
      const float s = warp_sums<KMAX>(ss, lane);
      if (lane < k) a.norms[i * k + lane] = sqrtf(s);
    }
  }
}

template <bool E5, bool VEC, int KMAX>
cudaError_t run_staged(const Q8CombineArgs& a, int smem, int sms, cudaStream_t s) {
  const auto kern = a.gate ? q8_combine_staged_kernel<E5, KMAX, VEC, true> : q8_combine_staged_kernel<E5, KMAX, VEC, false>;
  const cudaError_t e = set_dyn_smem_on_device(reinterpret_cast<const void*>(kern), kStageMax);
  if (e != cudaSuccess) return e;
  const int per_sm = std::max(1, std::min(kStageSm / (smem + 1088), stage_blocks(KMAX)));
  const int64_t blocks = std::min<int64_t>((static_cast<int64_t>(a.T) + kStageWarps - 1) / kStageWarps, sms * per_sm);
  return launch_pdl(kern, dim3(static_cast<unsigned>(blocks)), dim3(kStageWarps * 32), smem, s, a);
}

template <bool E5, bool VEC>
cudaError_t staged(const Q8CombineArgs& a, int smem, int sms, cudaStream_t s) {
  switch (a.k) {
    case 1: return run_staged<E5, VEC, 1>(a, smem, sms, s);
    case 2: return run_staged<E5, VEC, 2>(a, smem, sms, s);
    case 3: return run_staged<E5, VEC, 3>(a, smem, sms, s);
    case 4: return run_staged<E5, VEC, 4>(a, smem, sms, s);
    case 5:
    case 6: return run_staged<E5, VEC, 6>(a, smem, sms, s);
    case 7:
    case 8: return run_staged<E5, VEC, 8>(a, smem, sms, s);
    case 9: return run_staged<E5, VEC, 9>(a, smem, sms, s);
    default: return run_staged<E5, VEC, 16>(a, smem, sms, s);
  }
}

bool row_vec(const Q8CombineArgs& a) {
  constexpr int size = sizeof(TI);
  return q8_aligned16(a.out, a.out_stride * size) && (!a.x || q8_aligned16(a.x, a.x_stride * size));
}

// Shared memory of the staged form's blocks, 0 where the direct form is taken:
// staged where the tokens are more than direct blocks run at once and two
// blocks' buffers fit an SM (2000 tokens of 16 slots and 2560 values: 40 us for
// 111 direct; of four slots and 9000, whose buffers do not: 48 alone on an SM, 47 direct).
int staged_smem(const Q8CombineArgs& a, int sms) {
  const int64_t wide = static_cast<int64_t>(a.c.width) * (a.k + 2 * static_cast<int>(sizeof(TI)));
  if (a.T <= sms * direct_blocks(a.k) || wide >= kStageMax / kStageWarps) return 0;
  const StageLayout L = row_vec(a) ? stage_layout<true>(a.k, a.c.width, a.x != nullptr) : stage_layout<false>(a.k, a.c.width, a.x != nullptr);
  const int smem = kStageWarps * L.bytes;
  return smem <= kStageMax ? smem : 0;
}

template <bool E5>
cudaError_t combine(Q8CombineArgs a, cudaStream_t s) {
  a.vec = row_vec(a);
  a.gate_vec = a.gate && q8_aligned16(a.gate, a.gate_stride * 4);
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  const int smem = staged_smem(a, sms);
  if (smem > 0) return a.vec ? staged<E5, true>(a, smem, sms, s) : staged<E5, false>(a, smem, sms, s);
  const dim3 grid(a.T), block(kDirectWarps * 32);
  if (a.k == 1) return launch_pdl(q8_combine_kernel<E5, 1>, grid, block, 0, s, a);
  if (a.k == 2) return launch_pdl(q8_combine_kernel<E5, 2>, grid, block, 0, s, a);
  if (a.k <= 4) return launch_pdl(q8_combine_kernel<E5, 4>, grid, block, 0, s, a);
  if (a.k <= 8) return launch_pdl(q8_combine_kernel<E5, 8>, grid, block, 0, s, a);
  return launch_pdl(q8_combine_kernel<E5, 16>, grid, block, 0, s, a);
}

}  // namespace

#ifdef MOECA_Q8_COMBINE_F32
bool q8_combine_is_staged_f32(const Q8CombineArgs& a, int sms) { return staged_smem(a, sms) > 0; }
cudaError_t launch_q8_combine_f32(const Q8CombineArgs& a, bool e5, cudaStream_t s) {
#else
bool q8_combine_is_staged_bf16(const Q8CombineArgs& a, int sms) { return staged_smem(a, sms) > 0; }
cudaError_t launch_q8_combine_bf16(const Q8CombineArgs& a, bool e5, cudaStream_t s) {
#endif
  if (a.T <= 0) return cudaSuccess;
  return e5 ? combine<true>(a, s) : combine<false>(a, s);
}

}  // namespace moeca
