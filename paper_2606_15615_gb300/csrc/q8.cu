// 8-bit branch caches (include/moeca_q8.h): rows quantised as they are
// written, and read back by Eq. 8's combine or as they are.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "q8.cuh"

namespace moeca {
namespace {

// ---------------------------------------------------------------------------
// Write.  A block of 128 values (a unit) is the work of 8 lanes: each takes 16
// values in pieces of 16 bytes (piece l + 8 j of the block, so that 8 lanes
// cover 128 contiguous bytes), the block's largest magnitude is an integer
// maximum of |x|'s bits over the 8 lanes, and one byte per value goes out the
// same way.  One pass: b + 1 bytes a value (b = 2 or 4), nothing is read twice.
// Units are numbered over all rows, so that no lane idles at a row's end, and
// the next unit's loads are in flight while one is worked on.  Rows that do
// not start at 16 bytes are read in the aligned pieces that hold their values,
// shifted into place in registers.
// ---------------------------------------------------------------------------
constexpr int kWriteThreads = 256;
constexpr int kWriteBlocks = 3;  // per SM: 45.7 us for 60000 bf16 rows of 1152; 4 with fewer registers each: the same, but 164 us for 134 in fp32


// The 16 bytes from byte `m` (a multiple of the type's size, below 16) of two
// consecutive pieces.
template <typename TI>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t m) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = m & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = m & 4 ? w[i + 1] : w[i];
  if (sizeof(TI) == 2) {
    const uint32_t sel = m & 2 ? 0x5432 : 0x3210;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], w[i + 1], sel);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One unit on its way: where it goes and its raw values.
template <int J>
struct WriteUnit {
  uint4 raw[J];
  int row, block, left;  // cache row (< 0: nothing to write), block, values from the block's start to the row's end
};

template <typename TI, bool E5, bool ALIGNED>
__global__ void __launch_bounds__(kWriteThreads, kWriteBlocks) q8_write_kernel(const Q8WriteArgs a) {
  constexpr int V = Elem<TI>::kVec, J = 16 / V;
  pdl_entry();
  const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  const int width = a.c.width, nb = (width + kQ8Block - 1) / kQ8Block;
  const int64_t total = static_cast<int64_t>(n) * nb;
  const int lane = threadIdx.x & 31, l = lane & 7;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kWriteThreads / 8);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kWriteThreads / 8) + (threadIdx.x >> 5) * 4;
  const TI* x = static_cast<const TI*>(a.x);
  const auto fetch = [&](int64_t u) {
    WriteUnit<J> w;
    w.row = -1;
    w.block = w.left = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) w.raw[j] = make_uint4(0u, 0u, 0u, 0u);
    if (u >= total) return w;
    const int i = total <= 0xffffffffll ? static_cast<int>(static_cast<uint32_t>(u) / static_cast<uint32_t>(nb))
                                        : static_cast<int>(u / nb);
    w.block = static_cast<int>(u - static_cast<int64_t>(i) * nb);
    w.left = width - w.block * kQ8Block;
    const int r = a.src ? __ldg(a.src + i) : i, d = a.dst ? __ldg(a.dst + i) : i;
    if (r < 0 || r >= a.x_rows || d < 0 || d >= a.c.rows) return w;
    w.row = d;
    const TI* from = x + r * a.x_stride + w.block * kQ8Block;
    if constexpr (ALIGNED) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (V * (l + 8 * j) < w.left) w.raw[j] = __ldg(reinterpret_cast<const uint4*>(from) + l + 8 * j);
    } else {
      const uint32_t m = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(from)) & 15u;
      const uint4* base = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(from) - m);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int e = V * (l + 8 * j), head = V - static_cast<int>(m / sizeof(TI));  // values in the first piece
        uint4 p = make_uint4(0u, 0u, 0u, 0u), q = p;
        if (e < w.left) p = __ldg(base + l + 8 * j);
        if (m && e + head < w.left) q = __ldg(base + l + 8 * j + 1);
        w.raw[j] = shifted<TI>(p, q, m);
      }
    }
    return w;
  };
  const auto store = [&](const WriteUnit<J>& u) {
    float v[16];
#pragma unroll
    for (int j = 0; j < J; ++j) unpack_vec(u.raw[j], &v[V * j], static_cast<TI*>(nullptr));
    if (u.left < kQ8Block) {  // what lies past the row's end counts for nothing
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (V * (l + 8 * (t / V)) + t % V >= u.left) v[t] = 0.f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int t = 0; t < 16; ++t) top = max(top, abs_bits(v[t]));
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool odd = top >= kNonFinite;  // the same for the block's 8 lanes
    if (__any_sync(0xffffffffu, odd)) {
      uint32_t fin = 0;
#pragma unroll
      for (int t = 0; t < 16; ++t) fin = max(fin, abs_bits(v[t]) < kNonFinite ? abs_bits(v[t]) : 0u);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) fin = max(fin, __shfl_xor_sync(0xffffffffu, fin, o));
      top = fin;
    }
    if (u.row < 0) return;
    const int byte = scale_byte<E5>(top);
    const float inv = scale_inverse(byte);
    if (l == 0) a.c.scale[u.row * a.c.scale_stride + u.block] = static_cast<uint8_t>(byte);
    uint8_t* out = a.c.q + u.row * a.c.q_stride + u.block * kQ8Block;
    uint32_t w[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
      w[t] = encode2<E5>(v[4 * t] * inv, v[4 * t + 1] * inv) | encode2<E5>(v[4 * t + 2] * inv, v[4 * t + 3] * inv) << 16;
    if (odd) {
#pragma unroll
      for (int t = 0; t < 16; ++t) w[t >> 2] += abs_bits(v[t]) == kNonFinite ? 1u << 8 * (t & 3) : 0u;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = V * (l + 8 * j);
      if (e + V <= u.left) {
        if constexpr (V == 8) *reinterpret_cast<uint2*>(out + e) = make_uint2(w[2 * j], w[2 * j + 1]);
        else *reinterpret_cast<uint32_t*>(out + e) = w[j];
      } else {
#pragma unroll
        for (int t = 0; t < V; ++t)
          if (e + t < u.left) out[e + t] = static_cast<uint8_t>(w[(V * j + t) >> 2] >> 8 * (t & 3));
      }
    }
  };
  WriteUnit<J> next = fetch(first + (lane >> 3));
  for (int64_t base = first; base < total; base += step) {  // base: the warp's first unit
    const WriteUnit<J> now = next;
    next = fetch(base + step + (lane >> 3));
    store(now);
  }
}

// ---------------------------------------------------------------------------
// Combine (and read back: one slot, no weights, no residual).
//   out_i = x_i + g * sum_p w_p h_p,   norm_p = ||h_p||
// A warp per token, 8 values a lane and step: 8 cache bytes of each slot and
// their scale byte, all slots' loads in flight before any arithmetic.  Where
// the tokens are few, the 8 warps of a block share one token.  The scale is a
// power of two, so w x scale is exact and one multiply-add per value does for
// both; squares are summed over a lane's 8 values before their scale.
// ---------------------------------------------------------------------------
constexpr int kCombineWarps = 8;
constexpr int kLaneValues = 8;

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}

template <typename TI, bool E5, int KMAX, int CG>
__global__ void __launch_bounds__(kCombineWarps * 32) q8_combine_kernel(const Q8CombineArgs a) {
  constexpr int W = kLaneValues, NV = W / Elem<TI>::kVec;
  __shared__ float part[kCombineWarps][KMAX];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t i = a.split ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * kCombineWarps + warp;
  if (i >= a.T) return;  // whole warps; a shared token's block has all its warps
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
  const int c_step = (a.split ? kCombineWarps : 1) * 32 * CG;
  for (int c0 = (a.split ? warp * 32 * CG : 0) + lane; c0 < chunks; c0 += c_step) {
    uint2 h[CG][KMAX];
    uint8_t sc[CG][KMAX];
    uint4 xr[CG][NV];
    float xs[CG][W];
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const int c = c0 + g * 32;
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        h[g][p] = make_uint2(0u, 0u);
        sc[g][p] = 127;
        if (c < chunks && row[p] >= 0) {
          h[g][p] = __ldg(reinterpret_cast<const uint2*>(a.c.q + row[p] * a.c.q_stride + c * W));
          sc[g][p] = __ldg(a.c.scale + row[p] * a.c.scale_stride + (c >> 4));
        }
      }
      if (x && c < chunks) {
        if (a.vec && (c + 1) * W <= width) {
#pragma unroll
          for (int j = 0; j < NV; ++j) xr[g][j] = *(reinterpret_cast<const uint4*>(x + c * W) + j);
#pragma unroll
          for (int j = 0; j < NV; ++j) unpack_vec(xr[g][j], &xs[g][j * Elem<TI>::kVec], static_cast<TI*>(nullptr));
        } else {
#pragma unroll
          for (int t = 0; t < W; ++t) xs[g][t] = c * W + t < width ? Elem<TI>::to_f(x[c * W + t]) : 0.f;
        }
      }
    }
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const int c = c0 + g * 32, live = width - c * W;
      if (c >= chunks) continue;
      if (live < W) {  // the bytes past the row's width are anything
#pragma unroll
        for (int p = 0; p < KMAX; ++p) {
          h[g][p].x &= live >= 4 ? 0xffffffffu : (1u << 8 * live) - 1;
          h[g][p].y &= live <= 4 ? 0u : (1u << 8 * (live - 4)) - 1;
        }
      }
      float2 y[W / 2];
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        if (p >= k) continue;
        const float f = scale_value(sc[g][p]), wf = w[p] * f;
        float2 d[W / 2], sq;
#pragma unroll
        for (int t = 0; t < W / 2; ++t) d[t] = decode2<E5>((t < 2 ? h[g][p].x : h[g][p].y) >> (t & 1 ? 16 : 0) & 0xffffu);
        const float2 wf2 = make_float2(wf, wf);
#pragma unroll
        for (int t = 0; t < W / 2; ++t) y[t] = p == 0 ? mul2(wf2, d[t]) : fma2(wf2, d[t], y[t]);
        if (a.norms) {
          sq = mul2(d[0], d[0]);
#pragma unroll
          for (int t = 1; t < W / 2; ++t) sq = fma2(d[t], d[t], sq);
          ss[p] = fmaf(f * (sq.x + sq.y), f, ss[p]);
        }
      }
      float o[W];
#pragma unroll
      for (int t = 0; t < W / 2; ++t) {
        o[2 * t] = y[t].x;
        o[2 * t + 1] = y[t].y;
      }
      if (gate) {
        const float* gp = gate + c * W;
        if (a.gate_vec && live >= W) {
          const float4 g0 = __ldg(reinterpret_cast<const float4*>(gp)), g1 = __ldg(reinterpret_cast<const float4*>(gp) + 1);
          o[0] *= g0.x; o[1] *= g0.y; o[2] *= g0.z; o[3] *= g0.w;
          o[4] *= g1.x; o[5] *= g1.y; o[6] *= g1.z; o[7] *= g1.w;
        } else {
#pragma unroll
          for (int t = 0; t < W; ++t) o[t] *= t < live ? __ldg(gp + t) : 0.f;
        }
      }
      if (x) {
#pragma unroll
        for (int t = 0; t < W; ++t) o[t] += xs[g][t];
      }
      if (a.vec && live >= W) {
#pragma unroll
        for (int j = 0; j < NV; ++j) store_vec(out + c * W + j * Elem<TI>::kVec, &o[j * Elem<TI>::kVec]);
      } else {
#pragma unroll
        for (int t = 0; t < W; ++t)
          if (t < live) out[c * W + t] = Elem<TI>::from_f(o[t]);
      }
    }
  }
  if (!a.norms) return;
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    if (p >= k) continue;
    const float s = warp_sum(ss[p]);
    if (lane == 0) {
      if (a.split) part[warp][p] = s;
      else a.norms[i * k + p] = sqrtf(s);
    }
  }
  if (a.split) {
    __syncthreads();
    if (threadIdx.x < k) {
      float s = 0.f;
      for (int q = 0; q < kCombineWarps; ++q) s += part[q][threadIdx.x];
      a.norms[i * k + threadIdx.x] = sqrtf(s);
    }
  }
}

// ---------------------------------------------------------------------------
// The same for many tokens, staged: a warp walks its tokens i = w, w + W, ...
// (W the grid's warps), each brought into its buffer in shared memory by
// asynchronous copies (16 bytes at a time for the live cache rows and x, 4 for
// the scales), so that the bytes in flight do not hang on registers, and the
// next token's copies start as soon as the last one's values are used.  Its
// row list was loaded a token before.  One buffer per warp: twice the warps
// hide more of the arithmetic's latency than a second buffer (decoding costs
// 3.5 clocks a value and warp, as much as HBM takes for 8 slots).
// ---------------------------------------------------------------------------
constexpr int kStageWarps = 4;
constexpr int kStageBlocks = 8;            // per SM at most
constexpr int kStageSm = 227 * 1024, kStageMax = 112 * 1024;  // shared memory of an SM, and the most a block takes

// Bytes of a token's buffer: slots' rows, x, slots' scales, slots' weights.
struct StageLayout {
  int row, x, scale_words, x_at, scale_at, weight_at, bytes;
};
__host__ __device__ inline StageLayout stage_layout(int k, int width, int x_size) {
  StageLayout s;
  s.row = (width + 15) / 16 * 16;
  s.x = (width * x_size + 15) / 16 * 16;
  s.scale_words = ((width + kQ8Block - 1) / kQ8Block + 3) / 4;
  s.x_at = k * s.row;
  s.scale_at = s.x_at + s.x;
  s.weight_at = s.scale_at + k * s.scale_words * 4;
  s.bytes = (s.weight_at + k * 4 + 15) / 16 * 16;
  return s;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

template <typename TI, bool E5, int KMAX>
__global__ void __launch_bounds__(kStageWarps * 32) q8_combine_staged_kernel(const Q8CombineArgs a) {
  constexpr int W = kLaneValues, NV = W / Elem<TI>::kVec;
  extern __shared__ __align__(16) uint8_t dyn[];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k = a.k, width = a.c.width, chunks = (width + W - 1) / W;
  const StageLayout L = stage_layout(k, width, a.x ? sizeof(TI) : 0);
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
  // Start token i's copies.  A slot that holds nothing copies nothing.
  const auto fetch = [&](int64_t i) {
    const uint32_t to = smem_u32(buf);
    if (i < a.T) {
      for (int p = 0; p < k; ++p) {
        const int r = __shfl_sync(0xffffffffu, row, p);
        if (r < 0) continue;
        const uint8_t* q = a.c.q + r * a.c.q_stride;
        for (int c = lane * 16; c < L.row; c += 512) copy16(to + p * L.row + c, q + c);
        const uint8_t* sc = a.c.scale + r * a.c.scale_stride;
        for (int c = lane; c < L.scale_words; c += 32) copy4(to + L.scale_at + (p * L.scale_words + c) * 4, sc + c * 4);
      }
      if (x) {
        const uint8_t* xr = reinterpret_cast<const uint8_t*>(x + i * a.x_stride);
        for (int c = lane * 16; c < L.x; c += 512) copy16(to + L.x_at + c, xr + c);
      }
      if (lane < k) *reinterpret_cast<float*>(buf + L.weight_at + lane * 4) = weight;
    }
  };

  look_up(w0);
  uint32_t slots = __ballot_sync(0xffffffffu, row >= 0);  // bit p: slot p of the token in the buffer holds a row
  fetch(w0);
  look_up(w0 + step);
  for (int64_t i = w0; i < a.T; i += step) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    TI* out = static_cast<TI*>(a.out) + i * a.out_stride;
    const float* gate = a.gate ? a.gate + (i / a.seq) * a.gate_stride : nullptr;
    float ss[KMAX], w[KMAX];
#pragma unroll
    for (int p = 0; p < KMAX; ++p) {
      ss[p] = 0.f;
      w[p] = p < k ? *reinterpret_cast<const float*>(buf + L.weight_at + p * 4) : 0.f;
    }
    for (int c = lane; c < chunks; c += 32) {
      const int left = width - c * W;
      // Without branches, so that the slots' chains interleave: a slot that
      // holds nothing (or is not there) counts as zeros of scale 1.
      uint2 h[KMAX];
      float f[KMAX];
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        const bool on = slots >> p & 1;
        const uint2 raw = *reinterpret_cast<const uint2*>(buf + (p < k ? p : 0) * L.row + c * W);
        const uint32_t byte = buf[L.scale_at + (p < k ? p : 0) * L.scale_words * 4 + (c >> 4)];
        h[p] = make_uint2(on ? raw.x : 0u, on ? raw.y : 0u);
        f[p] = scale_value(on ? byte : 127u);
      }
      if (left < W) {  // the bytes past the row's width are anything
#pragma unroll
        for (int p = 0; p < KMAX; ++p) {
          h[p].x &= left >= 4 ? 0xffffffffu : (1u << 8 * left) - 1;
          h[p].y &= left <= 4 ? 0u : (1u << 8 * (left - 4)) - 1;
        }
      }
      float2 y[W / 2];
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        float2 d[W / 2];
#pragma unroll
        for (int t = 0; t < W / 2; ++t) d[t] = decode2<E5>((t < 2 ? h[p].x : h[p].y) >> (t & 1 ? 16 : 0) & 0xffffu);
        const float wf = w[p] * f[p];
        const float2 wf2 = make_float2(wf, wf);
#pragma unroll
        for (int t = 0; t < W / 2; ++t) y[t] = p == 0 ? mul2(wf2, d[t]) : fma2(wf2, d[t], y[t]);
        float2 sq = mul2(d[0], d[0]);
#pragma unroll
        for (int t = 1; t < W / 2; ++t) sq = fma2(d[t], d[t], sq);
        ss[p] = fmaf(f[p] * (sq.x + sq.y), f[p], ss[p]);
      }
      float o[W];
#pragma unroll
      for (int t = 0; t < W / 2; ++t) {
        o[2 * t] = y[t].x;
        o[2 * t + 1] = y[t].y;
      }
      if (gate) {
        const float* gp = gate + c * W;
        if (a.gate_vec && left >= W) {
          const float4 g0 = __ldg(reinterpret_cast<const float4*>(gp)), g1 = __ldg(reinterpret_cast<const float4*>(gp) + 1);
          o[0] *= g0.x; o[1] *= g0.y; o[2] *= g0.z; o[3] *= g0.w;
          o[4] *= g1.x; o[5] *= g1.y; o[6] *= g1.z; o[7] *= g1.w;
        } else {
#pragma unroll
          for (int t = 0; t < W; ++t) o[t] *= t < left ? __ldg(gp + t) : 0.f;
        }
      }
      if (x) {
        float xs[W];
#pragma unroll
        for (int j = 0; j < NV; ++j) load_vec(reinterpret_cast<const TI*>(buf + L.x_at) + c * W + j * Elem<TI>::kVec, &xs[j * Elem<TI>::kVec]);
#pragma unroll
        for (int t = 0; t < W; ++t) o[t] += xs[t];
      }
      if (left >= W) {
#pragma unroll
        for (int j = 0; j < NV; ++j) store_vec(out + c * W + j * Elem<TI>::kVec, &o[j * Elem<TI>::kVec]);
      } else {
#pragma unroll
        for (int t = 0; t < W; ++t)
          if (t < left) out[c * W + t] = Elem<TI>::from_f(o[t]);
      }
    }
    __syncwarp();  // all have read the buffer
    slots = __ballot_sync(0xffffffffu, row >= 0);
    fetch(i + step);
    look_up(i + 2 * step);
    if (a.norms) {
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        if (p >= k) continue;
        const float s = warp_sum(ss[p]);
        if (lane == 0) a.norms[i * k + p] = sqrtf(s);
      }
    }
  }
}

bool aligned16(const void* p, int64_t stride_bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride_bytes % 16 == 0;
}

}  // namespace

cudaError_t launch_q8_write(const Q8WriteArgs& a, bool bf16, bool e5, cudaStream_t s) {
  if (a.n <= 0) return cudaSuccess;
  const bool vec = aligned16(a.x, a.x_stride * (bf16 ? 2 : 4));
  const int64_t units = static_cast<int64_t>(a.n) * ((a.c.width + kQ8Block - 1) / kQ8Block);
  constexpr int64_t per_block = kWriteThreads / 8;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((units + per_block - 1) / per_block, 152 * kWriteBlocks)));
  auto run = [&](auto kern) { return launch_pdl(kern, grid, dim3(kWriteThreads), 0, s, a); };
  auto pick = [&](auto t) {
    using TI = decltype(t);
    if (e5) return vec ? run(q8_write_kernel<TI, true, true>) : run(q8_write_kernel<TI, true, false>);
    return vec ? run(q8_write_kernel<TI, false, true>) : run(q8_write_kernel<TI, false, false>);
  };
  return bf16 ? pick(__nv_bfloat16()) : pick(float());
}

namespace {

template <typename TI, bool E5>
cudaError_t combine_slots(Q8CombineArgs a, cudaStream_t s) {
  constexpr int size = sizeof(TI);
  a.vec = aligned16(a.out, a.out_stride * size) && (!a.x || aligned16(a.x, a.x_stride * size));
  a.gate_vec = a.gate && aligned16(a.gate, a.gate_stride * 4);
  a.split = a.T < 152 * 2;
  // Staged from two tokens per warp slot of the GPU on, where 16-byte copies can take the rows and four warps'
  // buffers fit a block.
  const int smem = kStageWarps * stage_layout(a.k, a.c.width, a.x ? size : 0).bytes;
  if (!a.split && a.vec && smem <= kStageMax) {
    const auto staged = [&](auto kern) {
      const cudaError_t e = set_dyn_smem_on_device(reinterpret_cast<const void*>(kern), kStageMax);
      if (e != cudaSuccess) return e;
      const int per_sm = std::max(1, std::min(kStageSm / (smem + 1024), kStageBlocks));
      return launch_pdl(kern, dim3(std::min((a.T + kStageWarps - 1) / kStageWarps, 152 * per_sm)), dim3(kStageWarps * 32), smem, s, a);
    };
    if (a.k == 1) return staged(q8_combine_staged_kernel<TI, E5, 1>);
    if (a.k == 2) return staged(q8_combine_staged_kernel<TI, E5, 2>);
    if (a.k == 3) return staged(q8_combine_staged_kernel<TI, E5, 3>);
    if (a.k == 4) return staged(q8_combine_staged_kernel<TI, E5, 4>);
    if (a.k <= 6) return staged(q8_combine_staged_kernel<TI, E5, 6>);
    if (a.k <= 9) return staged(q8_combine_staged_kernel<TI, E5, 9>);
    return staged(q8_combine_staged_kernel<TI, E5, 16>);
  }
  const dim3 grid(a.split ? a.T : (a.T + kCombineWarps - 1) / kCombineWarps), block(kCombineWarps * 32);
  if (a.k == 1) return launch_pdl(q8_combine_kernel<TI, E5, 1, 4>, grid, block, 0, s, a);
  if (a.k == 2) return launch_pdl(q8_combine_kernel<TI, E5, 2, 2>, grid, block, 0, s, a);
  if (a.k <= 4) return launch_pdl(q8_combine_kernel<TI, E5, 4, 2>, grid, block, 0, s, a);
  if (a.k <= 8) return launch_pdl(q8_combine_kernel<TI, E5, 8, 1>, grid, block, 0, s, a);
  return launch_pdl(q8_combine_kernel<TI, E5, 16, 1>, grid, block, 0, s, a);
}

}  // namespace

cudaError_t launch_q8_combine(const Q8CombineArgs& a, bool bf16, bool e5, cudaStream_t s) {
  if (a.T <= 0) return cudaSuccess;
  if (bf16) return e5 ? combine_slots<__nv_bfloat16, true>(a, s) : combine_slots<__nv_bfloat16, false>(a, s);
  return e5 ? combine_slots<float, true>(a, s) : combine_slots<float, false>(a, s);
}

// ---------------------------------------------------------------------------
// C calls: the arguments' checks.
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxWidth = 1 << 20, kMaxSlots = 16, kMaxGroups = 512;

bool is_format(int f) { return f == MOECA_E4M3 || f == MOECA_E5M2; }
bool is_dtype(int d) { return d == MOECA_F32 || d == MOECA_BF16; }
int64_t elem_size(int d) { return d == MOECA_BF16 ? 2 : 4; }
uintptr_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// A buffer's bytes: [from, from + bytes).
struct Range {
  const void* from;
  int64_t bytes;
};
Range rows_range(const void* p, int64_t rows, int64_t stride, int64_t row_bytes) {
  return {p, rows > 0 ? (rows - 1) * stride + row_bytes : 0};
}
bool overlap(const Range& a, const Range& b) {
  return a.from && b.from && a.bytes > 0 && b.bytes > 0 && addr(a.from) < addr(b.from) + b.bytes &&
         addr(b.from) < addr(a.from) + a.bytes;
}

// What is wrong with 8-bit rows (null: nothing).
const char* bad_rows(const moeca_q8_rows& r) {
  if (!is_format(r.format)) return "rows: format must be MOECA_E4M3 or MOECA_E5M2";
  if (r.width < 1 || r.width > kMaxWidth) return "rows: width out of range";
  if (r.rows < 0 || r.rows > kMaxRows) return "rows: row count out of range";
  if (r.rows > 0 && (!r.q || !r.scale)) return "rows: NULL q or scale";
  if (addr(r.q) % 16 || r.q_stride % 16 || r.q_stride < r.width)
    return "rows: q must be 16-byte aligned, q_stride a multiple of 16 and >= width";
  const int nb = (r.width + kQ8Block - 1) / kQ8Block;
  if (addr(r.scale) % 4 || r.scale_stride % 4 || r.scale_stride < nb)
    return "rows: scale must be 4-byte aligned, scale_stride a multiple of 4 and >= ceil(width / 128)";
  if (r.rows > 0 && (r.q_stride > INT64_MAX / 4 / r.rows || r.scale_stride > INT64_MAX / 4 / r.rows))
    return "rows: strides out of range";
  return nullptr;
}
const char* bad_values(const void* p, int64_t rows, int64_t stride, int width, int dtype, const char* what) {
  if (rows > 0 && !p) return what;
  if (addr(p) % elem_size(dtype)) return "a value buffer is not aligned to its type";
  if (stride < width || (rows > 0 && stride > INT64_MAX / 8 / rows)) return "a value stride is smaller than the width, or out of range";
  return nullptr;
}
Range q_range(const moeca_q8_rows& r) { return rows_range(r.q, r.rows, r.q_stride, r.q_stride); }
Range scale_range(const moeca_q8_rows& r) { return rows_range(r.scale, r.rows, r.scale_stride, r.scale_stride); }
Q8Rows device_rows(const moeca_q8_rows& r) {
  return {static_cast<uint8_t*>(r.q), r.scale, r.rows, r.q_stride, r.scale_stride, r.width};
}
moeca_status refuse(const char* why) {
  keep_call_error(why);
  return MOECA_ERR_INVALID_ARG;
}
moeca_status launched(cudaError_t e) {
  if (e == cudaSuccess) return MOECA_OK;
  cudaGetLastError();
  keep_call_error(cudaGetErrorString(e));
  return MOECA_ERR_CUDA;
}
// Whether any buffer of `written` overlaps one of `read` or another one written.
template <int NW, int NR>
bool any_overlap(const Range (&written)[NW], const Range (&read)[NR]) {
  for (int i = 0; i < NW; ++i) {
    for (const Range& r : read)
      if (overlap(written[i], r)) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return true;
  }
  return false;
}

}  // namespace
}  // namespace moeca

extern "C" {

moeca_status moeca_q8_write(const moeca_q8_write_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_rows(a->cache)) return refuse(why);
  if (!is_dtype(a->dtype)) return refuse("dtype must be MOECA_F32 or MOECA_BF16");
  if (a->x_rows < 0 || a->x_rows > kMaxRows) return refuse("x_rows out of range");
  const int width = a->cache.width;
  if (const char* why = bad_values(a->x, a->x_rows, a->x_stride, width, a->dtype, "x is NULL")) return refuse(why);
  if (a->n < 0 || (!a->src && a->n > a->x_rows) || (!a->dst && a->n > a->cache.rows))
    return refuse("n is negative, or larger than a side that has no list");
  if (addr(a->src) % 4 || addr(a->dst) % 4 || addr(a->count) % 4) return refuse("a list is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), list = 4 * static_cast<int64_t>(a->n);
  const Range written[] = {q_range(a->cache), scale_range(a->cache)};
  const Range read[] = {rows_range(a->x, a->x_rows, a->x_stride * es, width * es), {a->src, list}, {a->dst, list}, {a->count, 4}};
  if (any_overlap(written, read)) return refuse("the cache overlaps another buffer of the call");
  if (a->n == 0 || a->cache.rows == 0 || a->x_rows == 0) return MOECA_OK;
  const Q8WriteArgs d{device_rows(a->cache), a->x, a->x_rows, a->x_stride, a->n, a->src, a->dst, a->count};
  return launched(launch_q8_write(d, a->dtype == MOECA_BF16, a->cache.format == MOECA_E5M2, static_cast<cudaStream_t>(stream)));
}

moeca_status moeca_q8_read(const moeca_q8_read_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_rows(a->cache)) return refuse(why);
  if (!is_dtype(a->dtype)) return refuse("dtype must be MOECA_F32 or MOECA_BF16");
  if (a->n < 0 || (!a->rows && a->n > a->cache.rows)) return refuse("n is negative, or larger than the cache without a list");
  const int width = a->cache.width;
  if (const char* why = bad_values(a->out, a->n, a->out_stride, width, a->dtype, "out is NULL")) return refuse(why);
  if (addr(a->rows) % 4) return refuse("rows is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype);
  const Range written[] = {rows_range(a->out, a->n, a->out_stride * es, width * es)};
  const Range read[] = {q_range(a->cache), scale_range(a->cache), {a->rows, 4 * static_cast<int64_t>(a->n)}};
  if (any_overlap(written, read)) return refuse("out overlaps another buffer of the call");
  Q8CombineArgs d{};
  d.c = device_rows(a->cache);
  d.rows = a->rows;
  d.out = a->out;
  d.out_stride = a->out_stride;
  d.T = a->n;
  d.k = d.seq = 1;
  return launched(launch_q8_combine(d, a->dtype == MOECA_BF16, a->cache.format == MOECA_E5M2, static_cast<cudaStream_t>(stream)));
}

moeca_status moeca_q8_combine(const moeca_q8_combine_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_rows(a->cache)) return refuse(why);
  if (!is_dtype(a->dtype)) return refuse("dtype must be MOECA_F32 or MOECA_BF16");
  if (a->n_tokens < 0 || a->n_slots < 1 || a->n_slots > kMaxSlots) return refuse("n_tokens >= 0 and 1 <= n_slots <= 16");
  if (a->gate && a->seq < 1) return refuse("seq must be positive with a gate");
  const int T = a->n_tokens, width = a->cache.width;
  if (T > 0 && !a->rows) return refuse("rows is NULL");
  if (const char* why = bad_values(a->out, T, a->out_stride, width, a->dtype, "out is NULL")) return refuse(why);
  if (a->x)
    if (const char* why = bad_values(a->x, T, a->x_stride, width, a->dtype, "")) return refuse(why);
  const int64_t gates = a->gate ? (static_cast<int64_t>(T) + a->seq - 1) / a->seq : 0;
  if (a->gate)
    if (const char* why = bad_values(a->gate, gates, a->gate_stride, width, MOECA_F32, "")) return refuse(why);
  if (addr(a->rows) % 4 || addr(a->weights) % 4 || addr(a->norms) % 4) return refuse("rows, weights or norms is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), slots = 4 * static_cast<int64_t>(T) * a->n_slots;
  const Range out = rows_range(a->out, T, a->out_stride * es, width * es);
  const bool in_place = a->x == a->out && a->x_stride == a->out_stride;
  const Range written[] = {out, {a->norms, slots}};
  const Range read[] = {q_range(a->cache), scale_range(a->cache), {a->rows, slots}, {a->weights, slots},
                        rows_range(in_place ? nullptr : a->x, T, a->x_stride * es, width * es),
                        rows_range(a->gate, gates, a->gate_stride * 4, width * 4ll)};
  if (any_overlap(written, read)) return refuse("out or norms overlaps another buffer of the call");
  Q8CombineArgs d{};
  d.c = device_rows(a->cache);
  d.rows = a->rows; d.weights = a->weights;
  d.x = a->x; d.x_stride = a->x_stride;
  d.gate = a->gate; d.gate_stride = a->gate_stride;
  d.out = a->out; d.out_stride = a->out_stride;
  d.norms = a->norms;
  d.T = T; d.k = a->n_slots; d.seq = a->gate ? a->seq : 1;
  return launched(launch_q8_combine(d, a->dtype == MOECA_BF16, a->cache.format == MOECA_E5M2, static_cast<cudaStream_t>(stream)));
}

moeca_status moeca_q8_matmul(const moeca_q8_matmul_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_rows(a->a)) return refuse(why);
  if (const char* why = bad_rows(a->b)) return refuse(why);
  if (a->n_groups < 1 || a->n_groups > kMaxGroups || (!a->offsets && a->n_groups != 1))
    return refuse("1 <= n_groups <= 512, and offsets for more than one group");
  if (a->n_cols < 1 || a->n_cols > kMaxWidth || a->b.rows != static_cast<int64_t>(a->n_groups) * a->n_cols)
    return refuse("b must have n_groups x n_cols rows, n_cols in 1 .. 2^20");
  if (a->a.width != a->b.width) return refuse("a and b must have the same width");
  if (a->act < MOECA_ACT_NONE || a->act > MOECA_ACT_GELU_TANH) return refuse("unknown act");
  const moeca_q8_rows& o = a->out;
  if (o.width != a->n_cols) return refuse("out must be n_cols wide");
  if (is_format(o.format)) {
    if (const char* why = bad_rows(o)) return refuse(why);
  } else {
    if (!is_dtype(o.format)) return refuse("out: unknown format");
    if (o.rows < 0 || o.rows > kMaxRows || (o.rows > 0 && !o.q)) return refuse("out: NULL, or row count out of range");
    const int64_t es = elem_size(o.format);
    if (addr(o.q) % es || o.q_stride % es || o.q_stride < o.width * es || (o.rows > 0 && o.q_stride > INT64_MAX / 4 / o.rows))
      return refuse("out: base and row stride (bytes) aligned to the type, rows at least a row's bytes apart");
  }
  const int64_t M = a->a.rows;
  if (!a->dst && o.rows < M) return refuse("out has fewer rows than a, and there is no dst");
  if (addr(a->offsets) % 4 || addr(a->dst) % 4 || addr(a->bias) % 4 || addr(a->status) % 4)
    return refuse("offsets, dst, bias or status is not 4-byte aligned");
  const Range written[] = {rows_range(o.q, o.rows, o.q_stride, is_format(o.format) ? o.q_stride : o.width * elem_size(o.format)),
                           is_format(o.format) ? scale_range(o) : Range{nullptr, 0}, {a->status, 8}};
  const Range read[] = {q_range(a->a), scale_range(a->a), q_range(a->b), scale_range(a->b),
                        {a->offsets, 4ll * (a->n_groups + 1)}, {a->dst, 4 * M}, {a->bias, 4 * a->b.rows}};
  if (any_overlap(written, read)) return refuse("out or status overlaps another buffer of the call");
  if (M == 0 || o.rows == 0) return MOECA_OK;
  Q8MatmulArgs d{};
  d.a = device_rows(a->a); d.b = device_rows(a->b); d.out = device_rows(o);
  d.a_e5 = a->a.format == MOECA_E5M2; d.b_e5 = a->b.format == MOECA_E5M2;
  d.out_format = o.format; d.act = a->act; d.n_groups = a->n_groups; d.n_cols = a->n_cols;
  d.offsets = a->offsets; d.dst = a->dst; d.bias = a->bias; d.status = a->status;
  return launched(launch_q8_matmul(d, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
