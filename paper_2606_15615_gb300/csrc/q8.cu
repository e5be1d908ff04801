// 8-bit branch caches (include/moeca_q8.h): rows quantised as they are
// written, and the checks of every call's arguments.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "moeca_probe.h"
#include "q8.cuh"

namespace moeca {
namespace {

constexpr Q8Waits kWaits{1000000000ull, 0};  // a wait gives up after a second
thread_local Q8Waits g_waits = kWaits;

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
// 65549 x 2568 fp32 rows take 130 us (6.5 TB/s, 0.95 of a plain copy's rate),
// 60000 x 1152 bf16 rows 42 us (5.0 TB/s with the launch: instruction issue and
// HBM share the bound), 60000 x 1153 unaligned ones 66 us (two 16-byte loads for
// each piece, and the shifts).
// ---------------------------------------------------------------------------
constexpr int kWriteThreads = 256;
// Per SM.  Four with fewer registers each: the same time in bf16, but 164 us for 134 in fp32.
constexpr int kWriteBlocks = 3;

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
  // The entry and block of the next unit to fetch; a step further without a division.
  int64_t entry = (first + (lane >> 3)) / nb;
  int block = static_cast<int>(first + (lane >> 3) - entry * nb);
  const int64_t step_entries = step / nb;
  const int step_blocks = static_cast<int>(step - step_entries * nb);
  const auto fetch = [&] {
    WriteUnit<J> w;
    w.row = -1;
    w.block = block;
    w.left = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) w.raw[j] = make_uint4(0u, 0u, 0u, 0u);
    if (entry >= n) return w;
    const int i = static_cast<int>(entry);
    entry += step_entries;
    block += step_blocks;
    if (block >= nb) {
      block -= nb;
      ++entry;
    }
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
    uint32_t raw[4 * J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      raw[4 * j] = u.raw[j].x; raw[4 * j + 1] = u.raw[j].y; raw[4 * j + 2] = u.raw[j].z; raw[4 * j + 3] = u.raw[j].w;
    }
    if (u.left < kQ8Block) {  // what lies past the row's end counts for nothing
#pragma unroll
      for (int t = 0; t < 4 * J; ++t) {
        const int past = V * (l + 8 * (t / 4)) + t % 4 * (V / 4) - u.left;  // >= 0: all of the word
        raw[t] &= past >= 0 ? 0u : V == 8 && past == -1 ? 0xffffu : 0xffffffffu;
      }
    }
    float v[16];
    uint32_t top = 0;
    if constexpr (V == 8) {  // two bf16 magnitudes at a time
#pragma unroll
      for (int t = 0; t < 4 * J; ++t) top = __vmaxu2(top, raw[t] & 0x7fff7fffu);
      top = max(top << 16, top & 0xffff0000u);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        v[2 * t] = __uint_as_float(raw[t] << 16);
        v[2 * t + 1] = __uint_as_float(raw[t] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        top = max(top, raw[t] & 0x7fffffffu);
        v[t] = __uint_as_float(raw[t]);
      }
    }
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
    for (int t = 0; t < 4; ++t) {
      const float2 lo = mul2(make_float2(v[4 * t], v[4 * t + 1]), make_float2(inv, inv));
      const float2 hi = mul2(make_float2(v[4 * t + 2], v[4 * t + 3]), make_float2(inv, inv));
      w[t] = __byte_perm(encode2<E5>(lo.x, lo.y), encode2<E5>(hi.x, hi.y), 0x5410);
    }
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
  WriteUnit<J> next = fetch();
  for (int64_t base = first; base < total; base += step) {  // base: the warp's first unit
    const WriteUnit<J> now = next;
    next = fetch();
    store(now);
  }
}

}  // namespace

Q8Waits q8_waits() { return g_waits; }

cudaError_t launch_q8_write(const Q8WriteArgs& a, bool bf16, bool e5, cudaStream_t s) {
  if (a.n <= 0) return cudaSuccess;
  const bool vec = q8_aligned16(a.x, a.x_stride * (bf16 ? 2 : 4));
  const int64_t units = static_cast<int64_t>(a.n) * ((a.c.width + kQ8Block - 1) / kQ8Block);
  constexpr int64_t per_block = kWriteThreads / 8;
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((units + per_block - 1) / per_block, sms * kWriteBlocks)));
  auto run = [&](auto kern) { return launch_pdl(kern, grid, dim3(kWriteThreads), 0, s, a); };
  auto pick = [&](auto t) {
    using TI = decltype(t);
    if (e5) return vec ? run(q8_write_kernel<TI, true, true>) : run(q8_write_kernel<TI, true, false>);
    return vec ? run(q8_write_kernel<TI, false, true>) : run(q8_write_kernel<TI, false, false>);
  };
  return bf16 ? pick(__nv_bfloat16()) : pick(float());
}

// ---------------------------------------------------------------------------
// C calls: the arguments' checks.
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int64_t kMaxProductRows = 1 << 30;
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
// What the kernels touch: rows in pieces of 16 bytes, their scales in words.
int64_t row_bytes(const moeca_q8_rows& r) { return (r.width + 15) / 16 * 16; }
int64_t scale_bytes(const moeca_q8_rows& r) { return ((r.width + kQ8Block - 1) / kQ8Block + 3) / 4 * 4; }
Range q_range(const moeca_q8_rows& r) { return rows_range(r.q, r.rows, r.q_stride, row_bytes(r)); }
Range scale_range(const moeca_q8_rows& r) { return rows_range(r.scale, r.rows, r.scale_stride, scale_bytes(r)); }
Q8Rows device_rows(const moeca_q8_rows& r) {
  return {static_cast<uint8_t*>(r.q), r.scale, r.rows, r.q_stride, r.scale_stride, r.width};
}
moeca_status refuse(const char* why) {
  keep_call_error(why);
  return MOECA_ERR_INVALID_ARG;
}
// Runs a launch; nothing is thrown to the caller.
template <typename F>
moeca_status launched(F launch) {
  try {
    const cudaError_t e = launch();
    if (e == cudaSuccess) return MOECA_OK;
    cudaGetLastError();
    keep_call_error(cudaGetErrorString(e));
    return MOECA_ERR_CUDA;
  } catch (...) {
    keep_call_error("out of host memory");
    return MOECA_ERR_OOM;
  }
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
  return launched([&] {
    return launch_q8_write(d, a->dtype == MOECA_BF16, a->cache.format == MOECA_E5M2, static_cast<cudaStream_t>(stream));
  });
}

moeca_status moeca_q8_read(const moeca_q8_read_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_rows(a->cache)) return refuse(why);
  if (!is_dtype(a->dtype)) return refuse("dtype must be MOECA_F32 or MOECA_BF16");
  if (a->n < 0 || (!a->rows && a->n > a->cache.rows)) return refuse("n is negative, or larger than the cache without a list");
  const int width = a->cache.width;
  if (const char* why = bad_values(a->out, a->n, a->out_stride, width, a->dtype, "out is NULL")) return refuse(why);
  if (addr(a->rows) % 4 || addr(a->status) % 4) return refuse("rows or status is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype);
  const Range written[] = {rows_range(a->out, a->n, a->out_stride * es, width * es), {a->status, 8}};
  const Range read[] = {q_range(a->cache), scale_range(a->cache), {a->rows, 4 * static_cast<int64_t>(a->n)}};
  if (any_overlap(written, read)) return refuse("out overlaps another buffer of the call");
  Q8CombineArgs d{};
  d.c = device_rows(a->cache);
  d.rows = a->rows;
  d.out = a->out;
  d.out_stride = a->out_stride;
  d.status = a->status;
  d.T = a->n;
  d.k = d.seq = 1;
  d.waits = q8_waits();
  return launched([&] {
    return (a->dtype == MOECA_BF16 ? launch_q8_combine_bf16 : launch_q8_combine_f32)(d, a->cache.format == MOECA_E5M2,
                                                                                     static_cast<cudaStream_t>(stream));
  });
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
  if (addr(a->rows) % 4 || addr(a->weights) % 4 || addr(a->norms) % 4 || addr(a->status) % 4)
    return refuse("rows, weights, norms or status is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), slots = 4 * static_cast<int64_t>(T) * a->n_slots;
  const Range out = rows_range(a->out, T, a->out_stride * es, width * es);
  const bool in_place = a->x == a->out && a->x_stride == a->out_stride;
  const Range written[] = {out, {a->norms, slots}, {a->status, 8}};
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
  d.status = a->status;
  d.T = T; d.k = a->n_slots; d.seq = a->gate ? a->seq : 1;
  d.waits = q8_waits();
  return launched([&] {
    return (a->dtype == MOECA_BF16 ? launch_q8_combine_bf16 : launch_q8_combine_f32)(d, a->cache.format == MOECA_E5M2,
                                                                                     static_cast<cudaStream_t>(stream));
  });
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
  // Rows and tiles are counted in 32 bits.  Offsets may step back, so that groups
  // claim the same rows: each step back is an empty group, after which all rows
  // may come again.
  const int64_t wide = (a->n_cols + kQ8TileCols - 1ll) / kQ8TileCols, passes = (a->n_groups + 1) / 2;
  if (M > kMaxProductRows || a->b.rows > kMaxProductRows || (M / 16 + a->n_groups) * wide > kMaxProductRows ||
      (passes * M / kQ8TileRows + a->n_groups) * wide > kMaxProductRows) {
    keep_call_error("a and b of at most 2^30 rows, (rows / 16 + n_groups) and (ceil(n_groups / 2) x rows / 224 + n_groups) "
                    "x ceil(n_cols / 256) at most 2^30");
    return MOECA_ERR_UNSUPPORTED;
  }
  if (!a->dst && o.rows < M) return refuse("out has fewer rows than a, and there is no dst");
  if (addr(a->offsets) % 4 || addr(a->dst) % 4 || addr(a->bias) % 4 || addr(a->status) % 4)
    return refuse("offsets, dst, bias or status is not 4-byte aligned");
  const Range written[] = {is_format(o.format) ? q_range(o) : rows_range(o.q, o.rows, o.q_stride, o.width * elem_size(o.format)),
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
  d.waits = q8_waits();
  return launched([&] { return launch_q8_matmul(d, static_cast<cudaStream_t>(stream)); });
}

int32_t moeca_probe_q8_staged(int32_t sms, int32_t n_tokens, int32_t n_slots, int32_t width, int32_t dtype, int32_t residual,
                              int32_t aligned) {
  using namespace moeca;
  if (sms < 1 || n_tokens < 0 || n_slots < 1 || n_slots > kMaxSlots || width < 1 || width > kMaxWidth || !is_dtype(dtype)) return -1;
  Q8CombineArgs a{};
  a.c.width = width;
  a.T = n_tokens;
  a.k = n_slots;
  a.out = reinterpret_cast<void*>(static_cast<uintptr_t>(aligned ? 16 : 20));  // looked at, not read
  a.x = residual ? a.out : nullptr;
  return dtype == MOECA_BF16 ? q8_combine_is_staged_bf16(a, sms) : q8_combine_is_staged_f32(a, sms);
}

int32_t moeca_probe_q8_stall(int32_t barrier, int64_t wait_ns) {
  using namespace moeca;
  if (barrier < MOECA_Q8_NONE || barrier > MOECA_Q8_ACCUMULATORS || wait_ns < 1000000 || wait_ns > 1000000000) return -1;
  g_waits = barrier == MOECA_Q8_NONE ? kWaits : Q8Waits{static_cast<unsigned long long>(wait_ns), barrier};
  return 0;
}

}  // extern "C"
