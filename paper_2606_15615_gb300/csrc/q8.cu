// 8-bit branch caches (include/moeca_q8.h): rows quantised as they are
// written, and read back by Eq. 8's combine or as they are.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "q8.cuh"

namespace moeca {
namespace {

// ---------------------------------------------------------------------------
// Write.  A block of 128 values is the work of 8 lanes: each loads 16 values in
// 16-byte pieces (piece l + 8 j of the block, so that 8 lanes cover 128
// contiguous bytes), the block's largest magnitude is an integer maximum of
// |x|'s bits over the 8 lanes, and one byte per value goes out the same way.
// One pass: b + 1 bytes a value (b = 2 or 4), nothing is read twice.  Blocks
// are numbered over all rows, so that no lane idles at a row's end; kUnits of
// them are in flight per 8 lanes.
// ---------------------------------------------------------------------------
constexpr int kWriteThreads = 256;
constexpr int kUnits = 2;

// Where entry `u` (row, block) reads and writes; false: nothing to do.
struct WriteUnit {
  int64_t from, to;  // element of x, byte of q
  int row_to, block;
};

template <typename TI, bool E5, bool VEC>
__global__ void __launch_bounds__(kWriteThreads) q8_write_kernel(const Q8WriteArgs a) {
  constexpr int V = Elem<TI>::kVec, J = 16 / V;
  pdl_entry();
  const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  const int width = a.c.width, nb = (width + kQ8Block - 1) / kQ8Block;
  const int64_t total = static_cast<int64_t>(n) * nb;
  const int lane = threadIdx.x & 31, l = lane & 7;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kWriteThreads / 8);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kWriteThreads / 8) + (threadIdx.x >> 5) * 4;
  const TI* x = static_cast<const TI*>(a.x);
  for (int64_t base = first; base < total; base += step * kUnits) {  // base: the warp's first unit
    float v[kUnits][16];
    int block[kUnits], row[kUnits];  // row < 0: nothing to write
    bool whole[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int64_t u = base + q * step + (lane >> 3);
      row[q] = -1;
      block[q] = 0;
      int64_t from = 0;
      if (u < total) {
        const int i = total <= 0xffffffffll ? static_cast<int>(static_cast<uint32_t>(u) / static_cast<uint32_t>(nb))
                                            : static_cast<int>(u / nb);
        block[q] = static_cast<int>(u - static_cast<int64_t>(i) * nb);
        const int r = a.src ? __ldg(a.src + i) : i, d = a.dst ? __ldg(a.dst + i) : i;
        if (r >= 0 && r < a.x_rows && d >= 0 && d < a.c.rows) {
          row[q] = d;
          from = r * a.x_stride + block[q] * kQ8Block;
        }
      }
      whole[q] = VEC && (block[q] + 1) * kQ8Block <= width;
#pragma unroll
      for (int t = 0; t < 16; ++t) v[q][t] = 0.f;
      if (row[q] < 0) continue;
      if (whole[q]) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint4 raw = __ldg(reinterpret_cast<const uint4*>(x + from) + l + 8 * j);
          unpack_vec(raw, &v[q][V * j], static_cast<TI*>(nullptr));
        }
      } else {
        // The row's last block, or rows that 16-byte loads cannot take.
        const int left = width - block[q] * kQ8Block;
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (l + 8 * t < left) v[q][t] = Elem<TI>::to_f(x[from + l + 8 * t]);
      }
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      uint32_t top = 0;
#pragma unroll
      for (int t = 0; t < 16; ++t) top = max(top, abs_bits(v[q][t]));
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const bool odd = top >= kNonFinite;  // the same for the block's 8 lanes
      if (__any_sync(0xffffffffu, odd)) {
        uint32_t fin = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t) fin = max(fin, abs_bits(v[q][t]) < kNonFinite ? abs_bits(v[q][t]) : 0u);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) fin = max(fin, __shfl_xor_sync(0xffffffffu, fin, o));
        top = fin;
      }
      if (row[q] < 0) continue;
      const int byte = scale_byte<E5>(top);
      const float inv = scale_inverse(byte);
      if (l == 0) a.c.scale[row[q] * a.c.scale_stride + block[q]] = static_cast<uint8_t>(byte);
      uint8_t* out = a.c.q + row[q] * a.c.q_stride + block[q] * kQ8Block;
      uint32_t w[4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
        w[t] = encode2<E5>(v[q][4 * t] * inv, v[q][4 * t + 1] * inv) |
               encode2<E5>(v[q][4 * t + 2] * inv, v[q][4 * t + 3] * inv) << 16;
      if (odd) {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          w[t >> 2] = (w[t >> 2] & ~(0xffu << 8 * (t & 3))) | encode_any<E5>(v[q][t] * inv) << 8 * (t & 3);
      }
      if (whole[q]) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          if constexpr (V == 8)
            *reinterpret_cast<uint2*>(out + 8 * (l + 8 * j)) = make_uint2(w[2 * j], w[2 * j + 1]);
          else
            *reinterpret_cast<uint32_t*>(out + 4 * (l + 8 * j)) = w[j];
        }
      } else {
        const int left = width - block[q] * kQ8Block;
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (l + 8 * t < left) out[l + 8 * t] = static_cast<uint8_t>(w[t >> 2] >> 8 * (t & 3));
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Combine (and read back: one slot, no weights, no residual).
//   out_i = x_i + g * sum_p w_p h_p,   norm_p = ||h_p||
// A warp per token, 8 values a lane and step: 8 cache bytes of each slot and
// their scale byte, all slots' loads in flight before any arithmetic.  Where
// the tokens are few, a block of 8 warps shares one token (SPLIT).
// ---------------------------------------------------------------------------
constexpr int kCombineWarps = 8;

template <typename TI, bool E5, int KMAX, int CG, bool VEC, bool SPLIT>
__global__ void __launch_bounds__(kCombineWarps * 32) q8_combine_kernel(const Q8CombineArgs a) {
  constexpr int W = 8;  // values per lane and step
  __shared__ float part[SPLIT ? kCombineWarps : 1][KMAX];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = SPLIT ? blockIdx.x : blockIdx.x * kCombineWarps + warp;
  if (i >= a.T) return;  // whole warps; a split block has one token
  const int k = a.k, width = a.c.width, chunks = (width + W - 1) / W;
  float w[KMAX], ss[KMAX];
  const uint8_t *qp[KMAX], *sp[KMAX];  // null: the slot holds nothing
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    w[p] = ss[p] = 0.f;
    qp[p] = sp[p] = nullptr;
    if (p < k) {
      const int64_t at = static_cast<int64_t>(i) * k + p;
      const int r = a.rows ? __ldg(a.rows + at) : i;
      if (r >= 0 && r < a.c.rows) {
        w[p] = a.weights ? __ldg(a.weights + at) : 1.f;
        qp[p] = a.c.q + r * a.c.q_stride;
        sp[p] = a.c.scale + r * a.c.scale_stride;
      }
    }
  }
  const TI* x = a.x ? static_cast<const TI*>(a.x) + i * a.x_stride : nullptr;
  TI* out = static_cast<TI*>(a.out) + i * a.out_stride;
  const float* gate = a.gate ? a.gate + (i / a.seq) * a.gate_stride : nullptr;
  const int c_first = SPLIT ? warp * 32 * CG : 0, c_step = (SPLIT ? kCombineWarps : 1) * 32 * CG;
  for (int c0 = c_first; c0 < chunks; c0 += c_step) {
    uint2 h[CG][KMAX];
    uint8_t sc[CG][KMAX];
    float xv[CG][W];
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const int c = c0 + g * 32 + lane;
      if (c >= chunks) continue;
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        h[g][p] = make_uint2(0u, 0u);
        sc[g][p] = 127;
        if (qp[p]) {
          h[g][p] = *reinterpret_cast<const uint2*>(qp[p] + c * W);
          sc[g][p] = sp[p][c >> 4];
        }
      }
      if (x) {
        if (VEC && (c + 1) * W <= width) {
#pragma unroll
          for (int j = 0; j < W / Elem<TI>::kVec; ++j) load_vec(x + c * W + j * Elem<TI>::kVec, &xv[g][j * Elem<TI>::kVec]);
        } else {
#pragma unroll
          for (int t = 0; t < W; ++t) xv[g][t] = c * W + t < width ? Elem<TI>::to_f(x[c * W + t]) : 0.f;
        }
      }
    }
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const int c = c0 + g * 32 + lane;
      if (c >= chunks) continue;
      const int live = min(W, width - c * W);
      float y[W];
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        if (p >= k) continue;
        const float f = scale_value(sc[g][p]);
        float hv[W];
#pragma unroll
        for (int t = 0; t < W; t += 2) {
          const float2 d = decode2<E5>(((t < 4 ? h[g][p].x : h[g][p].y) >> (t & 2 ? 16 : 0)) & 0xffffu);
          hv[t] = t < live ? d.x * f : 0.f;
          hv[t + 1] = t + 1 < live ? d.y * f : 0.f;
        }
#pragma unroll
        for (int t = 0; t < W; ++t) {
          y[t] = p == 0 ? w[0] * hv[t] : fmaf(w[p], hv[t], y[t]);
          ss[p] = fmaf(hv[t], hv[t], ss[p]);
        }
      }
      if (gate) {
        const float* gp = gate + c * W;
#pragma unroll
        for (int t = 0; t < W; ++t) y[t] *= t < live ? __ldg(gp + t) : 0.f;
      }
      if (x) {
#pragma unroll
        for (int t = 0; t < W; ++t) y[t] += xv[g][t];
      }
      if (VEC && live == W) {
#pragma unroll
        for (int j = 0; j < W / Elem<TI>::kVec; ++j) store_vec(out + c * W + j * Elem<TI>::kVec, &y[j * Elem<TI>::kVec]);
      } else {
#pragma unroll
        for (int t = 0; t < W; ++t)
          if (t < live) out[c * W + t] = Elem<TI>::from_f(y[t]);
      }
    }
  }
  if (!a.norms) return;
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    if (p >= k) continue;
    const float s = warp_sum(ss[p]);
    if constexpr (SPLIT) {
      if (lane == 0) part[warp][p] = s;
    } else if (lane == 0) {
      a.norms[static_cast<int64_t>(i) * k + p] = sqrtf(s);
    }
  }
  if constexpr (SPLIT) {
    __syncthreads();
    if (threadIdx.x < k) {
      float s = 0.f;
      for (int q = 0; q < kCombineWarps; ++q) s += part[q][threadIdx.x];
      a.norms[static_cast<int64_t>(i) * k + threadIdx.x] = sqrtf(s);
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
  constexpr int64_t per_block = kWriteThreads / 8 * kUnits;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((units + per_block - 1) / per_block, 152 * 8)));
  auto run = [&](auto kern) { return launch_pdl(kern, grid, dim3(kWriteThreads), 0, s, a); };
  auto pick = [&](auto t) {
    using TI = decltype(t);
    if (e5) return vec ? run(q8_write_kernel<TI, true, true>) : run(q8_write_kernel<TI, true, false>);
    return vec ? run(q8_write_kernel<TI, false, true>) : run(q8_write_kernel<TI, false, false>);
  };
  return bf16 ? pick(__nv_bfloat16()) : pick(float());
}

namespace {

template <typename TI, bool E5, int KMAX, int CG>
cudaError_t run_combine(const Q8CombineArgs& a, bool vec, bool split, cudaStream_t s) {
  const dim3 grid(split ? a.T : (a.T + kCombineWarps - 1) / kCombineWarps), block(kCombineWarps * 32);
  if (split)
    return vec ? launch_pdl(q8_combine_kernel<TI, E5, KMAX, 1, true, true>, grid, block, 0, s, a)
               : launch_pdl(q8_combine_kernel<TI, E5, KMAX, 1, false, true>, grid, block, 0, s, a);
  return vec ? launch_pdl(q8_combine_kernel<TI, E5, KMAX, CG, true, false>, grid, block, 0, s, a)
             : launch_pdl(q8_combine_kernel<TI, E5, KMAX, CG, false, false>, grid, block, 0, s, a);
}

template <typename TI, bool E5>
cudaError_t combine_slots(const Q8CombineArgs& a, cudaStream_t s) {
  constexpr int size = sizeof(TI);
  const bool vec = aligned16(a.out, a.out_stride * size) && (!a.x || aligned16(a.x, a.x_stride * size));
  const bool split = a.T < 152 * 2;
  if (a.k == 1) return run_combine<TI, E5, 1, 4>(a, vec, split, s);
  if (a.k == 2) return run_combine<TI, E5, 2, 3>(a, vec, split, s);
  if (a.k <= 4) return run_combine<TI, E5, 4, 2>(a, vec, split, s);
  if (a.k <= 8) return run_combine<TI, E5, 8, 1>(a, vec, split, s);
  return run_combine<TI, E5, 16, 1>(a, vec, split, s);
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
