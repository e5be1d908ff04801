// Tokens sorted by expert and back, with the gradients (include/moeca_experts.h).
#include <algorithm>

#include "calls.h"
#include "common.cuh"
#include "moeca_experts.h"

namespace moeca {
namespace {

constexpr int kExpertsMost = 512;
constexpr int64_t kMaxBranches = 1 << 30;

// ---------------------------------------------------------------------------
// Sort: a stable counting sort.  A block's warps take consecutive pieces of the
// branches; a warp counts its piece 32 ids at a time (the lanes of one id find
// each other with a match, the first of them adds their number to the warp's
// count of that id).  A prefix sum over the warps and the experts turns counts
// into first rows, and a second walk over the same ids hands the rows out in
// order.  Few branches are one block's work; of many, a first launch counts each
// block's piece into the workspace, and every block of the second sums the
// counts of the blocks before it.  No atomic's order shows in a result.
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortOneBlock = 2048;  // branches that one block sorts
constexpr int kSortPiece = 1024;     // branches of a block otherwise, at least
constexpr int kSortBlocks = 128;     // at most
constexpr int kSortSteps = 8;

struct SortArgs {
  const int32_t* experts;
  int n, k, E;
  int piece;  // branches per block
  int32_t *offsets, *place, *slot, *token, *work;
};

int sort_blocks(int64_t n) {
  return n <= kSortOneBlock ? 1 : static_cast<int>(std::min<int64_t>(kSortBlocks, (n + kSortPiece - 1) / kSortPiece));
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
  extern __shared__ int32_t count[];  // [E]
  pdl_entry();
  for (int e = threadIdx.x; e < a.E; e += kSortThreads) count[e] = 0;
  __syncthreads();
  const int64_t lo = static_cast<int64_t>(blockIdx.x) * a.piece;
  const int hi = static_cast<int>(min(lo + a.piece, static_cast<int64_t>(a.n)));
  for (int i = static_cast<int>(min(lo, static_cast<int64_t>(hi))) + threadIdx.x; i < hi; i += kSortThreads) {
    const int e = a.experts[i];
    if (static_cast<unsigned>(e) < static_cast<unsigned>(a.E)) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kSortThreads) a.work[blockIdx.x * a.E + e] = count[e];
}

__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const SortArgs a) {
  extern __shared__ int32_t next[];  // [warps][E]: counts, then the next row of the warp's branches of expert e
  __shared__ int32_t warp_total[kSortWarps];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t before = (1u << lane) - 1;
  const int E = a.E;
  for (int i = threadIdx.x; i < kSortWarps * E; i += kSortThreads) next[i] = 0;
  __syncthreads();
  // This warp's piece, in steps of 32 branches.
  const int64_t lo = static_cast<int64_t>(blockIdx.x) * a.piece;
  const int64_t hi = min(lo + a.piece, static_cast<int64_t>(a.n));
  const int each = (a.piece + kSortThreads - 1) / kSortThreads * 32;
  const int64_t wlo = lo + static_cast<int64_t>(warp) * each, whi = min(wlo + each, hi);
  int32_t* mine = next + warp * E;
  // kSortSteps steps' ids are loaded at once, and kept for the second walk where that is all of the piece.
  int ids[kSortSteps];
  const auto load = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      const int64_t i = i0 + u * 32 + lane;
      ids[u] = i < whi ? a.experts[i] : -1;
      if (static_cast<unsigned>(ids[u]) >= static_cast<unsigned>(E)) ids[u] = -1;
    }
  };
  for (int64_t i0 = wlo; i0 < whi; i0 += 32 * kSortSteps) {
    load(i0);
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      if (i0 + u * 32 >= whi) break;
      const uint32_t same = __match_any_sync(0xffffffffu, ids[u]);
      if (ids[u] >= 0 && (same & before) == 0) mine[ids[u]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  // Thread e < E: the warps' counts become offsets within the block, and the
  // experts' totals offsets over all branches.
  const int e = threadIdx.x;
  int total = 0, earlier = 0;
  if (e < E) {
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = next[w * E + e];
      next[w * E + e] = total;
      total += c;
    }
    if (gridDim.x > 1) {
      total = 0;
      for (int b = 0; b < gridDim.x; ++b) {
        const int c = a.work[b * E + e];
        earlier += b < blockIdx.x ? c : 0;
        total += c;
      }
    }
  }
  int sum = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) warp_total[warp] = sum;
  __syncthreads();
  int first = sum - total, all = 0;
  for (int w = 0; w < kSortWarps; ++w) {
    if (w < warp) first += warp_total[w];
    all += warp_total[w];
  }
  if (e < E) {
    for (int w = 0; w < kSortWarps; ++w) next[w * E + e] += first + earlier;
    if (blockIdx.x == 0) a.offsets[e] = first;
  }
  if (blockIdx.x == 0 && e == 0) a.offsets[E] = all;
  __syncthreads();
  const bool kept = whi - wlo <= 32 * kSortSteps;
  for (int64_t i0 = wlo; i0 < whi; i0 += 32 * kSortSteps) {
    if (!kept) load(i0);
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      if (i0 + u * 32 >= whi) break;
      const int64_t i = i0 + u * 32 + lane;
      const int x = ids[u];
      const uint32_t same = __match_any_sync(0xffffffffu, x);
      int row = -1;
      if (x >= 0) row = mine[x] + __popc(same & before);
      __syncwarp();
      if (x >= 0 && (same & before) == 0) mine[x] += __popc(same);
      __syncwarp();
      if (i < whi) a.place[i] = row;
      if (row >= 0) {
        if (a.slot) a.slot[row] = static_cast<int>(i);
        if (a.token) a.token[row] = static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(a.k));
      }
    }
  }
  // Behind the last row.
  for (int64_t r = all + static_cast<int64_t>(blockIdx.x) * kSortThreads + threadIdx.x; r < a.n;
       r += static_cast<int64_t>(gridDim.x) * kSortThreads) {
    if (a.slot) a.slot[r] = -1;
    if (a.token) a.token[r] = -1;
  }
}

cudaError_t launch_sort(SortArgs a, cudaStream_t s) {
  const int blocks = sort_blocks(a.n);
  // A multiple of 32 ids for every warp.
  a.piece = static_cast<int>((static_cast<int64_t>(a.n) + blocks - 1) / blocks);
  a.piece = std::max((a.piece + kSortThreads - 1) / kSortThreads, 1) * kSortThreads;
  if (blocks > 1) {
    const cudaError_t e = launch_pdl(sort_count_kernel, dim3(blocks), dim3(kSortThreads), a.E * 4, s, a);
    if (e != cudaSuccess) return e;
  }
  const size_t smem = static_cast<size_t>(kSortWarps) * a.E * 4;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(sort_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               kSortWarps * kExpertsMost * 4);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(sort_place_kernel, dim3(blocks), dim3(kSortThreads), smem, s, a);
}

// ---------------------------------------------------------------------------
// Rows.  All three kernels move rows in units of 16 bytes; the written row's own
// 16-byte boundaries cut the units, so that rows of any alignment go out in whole
// sectors (the first and last unit of an unaligned row may be partial: value by
// value).  What is read is shifted into place from the aligned pieces that hold it.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;

template <typename T>
__device__ __forceinline__ int misalign(const T* p) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
}

// The V values from p on, of which lo .. hi - 1 are inside their row; the others
// are anything.  Unaligned ones are shifted into place from the aligned pieces
// that hold values of the row (no other piece is read).
template <typename T, bool ALIGNED>
__device__ __forceinline__ uint4 load_unit(const T* p, int lo, int hi) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (ALIGNED) return *reinterpret_cast<const uint4*>(p);
  const int m = static_cast<int>(at & 15);
  const uint4* piece = reinterpret_cast<const uint4*>(at - m);
  uint4 a = make_uint4(0, 0, 0, 0), b = a;
  if (m + lo * static_cast<int>(sizeof(T)) < 16) a = piece[0];
  if (m + hi * static_cast<int>(sizeof(T)) > 16) b = piece[1];
  return shifted<T>(a, b, m);
}
template <typename T>
__device__ __forceinline__ uint4 pack_unit(const float* f) {
  uint4 raw;
  store_vec(reinterpret_cast<T*>(&raw), f);
  return raw;
}

// A unit of a written row: values [lo, hi) of the V from `at` on.
template <typename T, bool ALIGNED>
struct Unit {
  int at, lo, hi;
  bool whole;
  __device__ __forceinline__ Unit(int u, const T* row, int width) {
    constexpr int V = Elem<T>::kVec;
    at = u * V - (ALIGNED ? 0 : misalign(row));
    lo = max(-at, 0);
    hi = min(width - at, V);
    whole = lo == 0 && hi == V;
  }
  __device__ __forceinline__ bool any() const { return lo < hi; }
  __device__ __forceinline__ uint4 load(const T* row) const {
    return load_unit<T, ALIGNED>(row + at, lo, hi);
  }
  __device__ __forceinline__ void store(T* row, const uint4& raw) const {
    if (whole) {
      *reinterpret_cast<uint4*>(row + at) = raw;
      return;
    }
    const T* v = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec; ++i)
      if (i >= lo && i < hi) row[at + i] = v[i];
  }
};

// Units that a row of any alignment needs.
template <typename T>
__host__ __device__ constexpr int row_units(int width, bool aligned) {
  constexpr int V = Elem<T>::kVec;
  return aligned ? (width + V - 1) / V : (width + 2 * V - 2) / V;
}

// The row and unit of the calling thread, the threads of all blocks numbered through.
struct Item {
  int64_t row;
  int u;
  __device__ __forceinline__ Item(int64_t block, int units) {
    const int64_t start = block * kRowThreads;
    int64_t row0;
    if (start < 0x7fffffff) row0 = static_cast<uint32_t>(start) / static_cast<uint32_t>(units);
    else row0 = start / units;
    const uint32_t t = static_cast<uint32_t>(start - row0 * units) + threadIdx.x;
    const uint32_t q = t / static_cast<uint32_t>(units);
    row = row0 + q;
    u = static_cast<int>(t - q * units);
  }
};

// Rows from *count on become zeros.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void clear_tail(T* rows, int64_t stride, int64_t n_rows, const int32_t* count, int units,
                                           int width) {
  if (!count) return;
  const int64_t used = min(max(static_cast<int64_t>(*count), int64_t(0)), n_rows);
  const int64_t blocks = ((n_rows - used) * units + kRowThreads - 1) / kRowThreads;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const Item it(b, units);
    const int64_t r = used + it.row;
    if (r >= n_rows) break;
    T* row = rows + r * stride;
    const Unit<T, ALIGNED> unit(it.u, row, width);
    if (unit.any()) unit.store(row, make_uint4(0, 0, 0, 0));
  }
}

// Work of a group of L lanes: a token and a segment of its units, J of them a lane.  A lane below k holds the place (and weight) of the token's branch;
// branches without a row are passed over by the whole group.
struct Segments {
  int units, segs, per;  // units of a row, its segments, units of a segment
};
Segments segments(int units, int lanes, int j) {
  const int segs = (units + j * lanes - 1) / (j * lanes);
  return {units, segs, (units + segs - 1) / segs};
}

template <int L>
struct Group {
  uint32_t mask, live;  // lanes of the group; branches that have a row
  int lane, place;
  __device__ __forceinline__ Group() {
    lane = threadIdx.x & (L - 1);
    mask = L == 32 ? 0xffffffffu : ((1u << (L & 31)) - 1) << (threadIdx.x & 31 & ~(L - 1));
  }
  __device__ __forceinline__ void load(const int32_t* places, int k, int64_t n_rows) {
    place = lane < k ? places[lane] : -1;
    if (place >= n_rows) place = -1;
    live = __ballot_sync(mask, place >= 0) >> (threadIdx.x & 31 & ~(L - 1));
    if (L < 32) live &= (1u << (L & 31)) - 1;
  }
  template <typename V>
  __device__ __forceinline__ V from(V v, int p) const {
    return __shfl_sync(mask, v, p, L);
  }
};

struct RowsArgs {
  const void* x;
  int64_t x_stride;
  void* rows;
  int64_t rows_stride, n_rows;
  const int32_t *place, *count;
  int T, k, width;
  Segments seg;
};

// x is read once and written to its rows (unaligned rows start at boundaries of
// their own: x then comes from L1 again for each).  HBM bounds it: 32768 tokens of
// 1152 (bf16) into 8 slots, the sort before it included, 120 us (5.7 TB/s, 0.84 of
// measured); 20011 tokens of 1001 into 3, unaligned, 44 us (3.7 TB/s).
constexpr int kRowsUnits = 2;

template <typename T, bool ALIGNED, int L>
__global__ void __launch_bounds__(kRowThreads) expert_rows_kernel(const RowsArgs a) {
  constexpr int J = kRowsUnits;
  pdl_entry();
  Group<L> g;
  const int64_t tasks = static_cast<int64_t>(a.T) * a.seg.segs, step = static_cast<int64_t>(gridDim.x) * (kRowThreads / L);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kRowThreads / L) + threadIdx.x / L; i < tasks; i += step) {
    const int64_t t = i < 0x7fffffff ? static_cast<uint32_t>(i) / static_cast<uint32_t>(a.seg.segs) : i / a.seg.segs;
    const int u0 = static_cast<int>(i - t * a.seg.segs) * a.seg.per, end = min(u0 + a.seg.per, a.seg.units);
    const T* x = static_cast<const T*>(a.x) + t * a.x_stride;
    uint4 raw[J];
    if (ALIGNED) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (u0 + g.lane + j * L < end) raw[j] = Unit<T, true>(u0 + g.lane + j * L, x, a.width).load(x);
    }
    g.load(a.place + t * a.k, a.k, a.n_rows);
    for (uint32_t live = g.live; live; live &= live - 1) {
      T* row = static_cast<T*>(a.rows) + static_cast<int64_t>(g.from(g.place, __ffs(live) - 1)) * a.rows_stride;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Unit<T, ALIGNED> unit(u0 + g.lane + j * L, row, a.width);
        if (u0 + g.lane + j * L < end && unit.any()) unit.store(row, ALIGNED ? raw[j] : unit.load(x));
      }
    }
  }
  clear_tail<T, ALIGNED>(static_cast<T*>(a.rows), a.rows_stride, a.n_rows, a.count, a.seg.units, a.width);
}

struct BackArgs {
  const void* rows;
  int64_t rows_stride, n_rows;
  const int32_t* place;
  const float* weights;
  const void* x;
  int64_t x_stride;
  void* out;
  int64_t out_stride;
  int T, k, width;
  Segments seg;
};

// A lane's loads in flight are those of CH branches for its J units; the rest of
// what HBM needs is other warps', so registers are held down.  32768 tokens with
// 8 slots of 1152 (bf16): four branches of one unit and five blocks an SM 128 us, with
// what the compiler takes (three blocks, two units) 232, eight branches of one unit on four blocks 145.  4096
// tokens with two of 2560: two branches of two units on four blocks 11.9 us, of one unit on six 13.0.
template <typename T, bool ALIGNED, int L, int CH, int J>
__global__ void __launch_bounds__(kRowThreads, CH == 2 ? 4 : ALIGNED ? 5 : 6) expert_combine_kernel(const BackArgs a) {
  constexpr int V = Elem<T>::kVec;
  pdl_entry();
  Group<L> g;
  const int64_t tasks = static_cast<int64_t>(a.T) * a.seg.segs, step = static_cast<int64_t>(gridDim.x) * (kRowThreads / L);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kRowThreads / L) + threadIdx.x / L; i < tasks; i += step) {
    const int64_t t = i < 0x7fffffff ? static_cast<uint32_t>(i) / static_cast<uint32_t>(a.seg.segs) : i / a.seg.segs;
    const int u0 = static_cast<int>(i - t * a.seg.segs) * a.seg.per, end = min(u0 + a.seg.per, a.seg.units);
    T* out = static_cast<T*>(a.out) + t * a.out_stride;
    g.load(a.place + t * a.k, a.k, a.n_rows);
    const float weight = a.weights && g.lane < a.k ? a.weights[t * a.k + g.lane] : 1.f;
    bool on[J];
    uint4 own[J];
    float sum[J][V];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Unit<T, ALIGNED> unit(u0 + g.lane + j * L, out, a.width);
      on[j] = u0 + g.lane + j * L < end && unit.any();
      if (a.x && on[j]) own[j] = unit.load(static_cast<const T*>(a.x) + t * a.x_stride);
#pragma unroll
      for (int v = 0; v < V; ++v) sum[j][v] = 0.f;
    }
    for (uint32_t live = g.live; live;) {
      uint4 raw[CH][J];
      float w[CH];
      int r[CH];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        r[c] = -1;
        if (live) {
          const int p = __ffs(live) - 1;
          live &= live - 1;
          r[c] = g.from(g.place, p);
          w[c] = g.from(weight, p);
          const T* row = static_cast<const T*>(a.rows) + r[c] * a.rows_stride;
#pragma unroll
          for (int j = 0; j < J; ++j)
            if (on[j]) raw[c][j] = Unit<T, ALIGNED>(u0 + g.lane + j * L, out, a.width).load(row);
        }
      }
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (r[c] >= 0) {
#pragma unroll
          for (int j = 0; j < J; ++j) {
            if (!on[j]) continue;
            float h[V];
            unpack_vec(raw[c][j], h, static_cast<T*>(nullptr));
#pragma unroll
            for (int v = 0; v < V; ++v) sum[j][v] = fmaf(w[c], h[v], sum[j][v]);
          }
        }
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (!on[j]) continue;
      if (a.x) {
        float f[V];
        unpack_vec(own[j], f, static_cast<T*>(nullptr));
#pragma unroll
        for (int v = 0; v < V; ++v) sum[j][v] += f[v];
      }
      Unit<T, ALIGNED>(u0 + g.lane + j * L, out, a.width).store(out, pack_unit<T>(sum[j]));
    }
  }
}

struct GradArgs {
  const void* dout;
  int64_t dout_stride;
  const void* rows;
  int64_t rows_stride, n_rows;
  const int32_t* place;
  const float* weights;
  const int32_t* count;
  void* drows;
  int64_t drows_stride;
  float* dweights;
  int T, k, width, units;
};

// A warp per branch: dout's row (from L1 or L2 but for the token's first branch)
// scaled into the gradient's row, and multiplied with the branch's row.
// As in the combine, warps are worth more than registers: 8191 tokens with 8
// slots of 768 (fp32) with two units a lane on five blocks an SM 106 us (both
// gradients), four on what the compiler takes 121; 20011 tokens with 3 unaligned slots of 1001
// (bf16) with one unit on six blocks 128 us, two on five 138, four 172.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads, ALIGNED ? 5 : 6) expert_grad_kernel(const GradArgs a) {
  constexpr int V = Elem<T>::kVec, J = ALIGNED ? 2 : 1;
  pdl_entry();
  const int lane = threadIdx.x & 31;
  const int64_t n = static_cast<int64_t>(a.T) * a.k, step = static_cast<int64_t>(gridDim.x) * (kRowThreads / 32);
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5); s < n; s += step) {
    const int r = a.place[s];
    float dot = 0.f;
    if (r >= 0 && r < a.n_rows) {
      const float w = a.weights ? a.weights[s] : 1.f;
      const T* dout = static_cast<const T*>(a.dout) + s / a.k * a.dout_stride;
      const T* row = static_cast<const T*>(a.rows) + r * a.rows_stride;
      T* drow = static_cast<T*>(a.drows) + r * a.drows_stride;
      const T* cut = a.drows ? drow : row;  // whose boundaries the units have
      for (int u0 = lane; u0 < a.units; u0 += 32 * J) {
        uint4 d[J], h[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Unit<T, ALIGNED> unit(u0 + 32 * j, cut, a.width);
          if (unit.any()) {
            d[j] = unit.load(dout);
            if (a.dweights) h[j] = unit.load(row);
          }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Unit<T, ALIGNED> unit(u0 + 32 * j, cut, a.width);
          if (!unit.any()) continue;
          float f[V], g[V];
          unpack_vec(d[j], f, static_cast<T*>(nullptr));
          if (a.dweights) {
            unpack_vec(h[j], g, static_cast<T*>(nullptr));
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (unit.whole || (i >= unit.lo && i < unit.hi)) dot = fmaf(f[i], g[i], dot);
          }
          if (a.drows) {
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] *= w;
            unit.store(drow, pack_unit<T>(f));
          }
        }
      }
    }
    if (a.dweights) {
      dot = warp_sum(dot);
      if (lane == 0) a.dweights[s] = dot;
    }
  }
  if (a.drows) clear_tail<T, ALIGNED>(static_cast<T*>(a.drows), a.drows_stride, a.n_rows, a.count, a.units, a.width);
}

constexpr int64_t kMaxBlocks = 1 << 30;  // beyond: blocks walk on

dim3 row_grid(int64_t threads) {
  return dim3(static_cast<unsigned>(std::max<int64_t>(1, std::min((threads + kRowThreads - 1) / kRowThreads, kMaxBlocks))));
}
bool aligned16(const void* p, int64_t stride, int dtype) {
  return addr(p) % 16 == 0 && stride * elem_size(dtype) % 16 == 0;
}
// f(T*, std::bool_constant<ALIGNED>)
template <typename F>
cudaError_t pick(int dtype, bool aligned, F f) {
  if (dtype == MOECA_BF16)
    return aligned ? f(static_cast<__nv_bfloat16*>(nullptr), std::true_type()) : f(static_cast<__nv_bfloat16*>(nullptr), std::false_type());
  return aligned ? f(static_cast<float*>(nullptr), std::true_type()) : f(static_cast<float*>(nullptr), std::false_type());
}

// f(std::integral_constant<lanes>): half a warp a token where a row has no more units.
template <typename F>
cudaError_t by_group(int units, F f) {
  return units <= 16 ? f(std::integral_constant<int, 16>()) : f(std::integral_constant<int, 32>());
}

const char* bad_branches(int n_tokens, int n_slots) {
  if (n_tokens < 0 || n_slots < 1 || n_slots > kMaxSlots) return "n_tokens >= 0 and 1 <= n_slots <= 16";
  if (static_cast<int64_t>(n_tokens) * n_slots > kMaxBranches) return "more than 2^30 branches";
  return nullptr;
}
const char* bad_shape(int dtype, int n_tokens, int n_slots, int width, int64_t n_rows, const int32_t* place) {
  if (!is_dtype(dtype)) return "dtype must be MOECA_F32 or MOECA_BF16";
  if (const char* why = bad_branches(n_tokens, n_slots)) return why;
  if (width < 1 || width > kMaxWidth) return "width out of range";
  if (n_rows < 0 || n_rows > kMaxRows) return "n_rows out of range";
  if (n_tokens > 0 && !place) return "place is NULL";
  if (addr(place) % 4) return "place is not 4-byte aligned";
  return nullptr;
}

}  // namespace
}  // namespace moeca

extern "C" {

int64_t moeca_expert_sort_workspace(int32_t n_tokens, int32_t n_slots, int32_t n_experts) {
  using namespace moeca;
  if (bad_branches(n_tokens, n_slots) || n_experts < 1 || n_experts > kExpertsMost) return -1;
  const int blocks = sort_blocks(static_cast<int64_t>(n_tokens) * n_slots);
  return blocks > 1 ? static_cast<int64_t>(blocks) * n_experts : 0;
}

moeca_status moeca_expert_sort(const moeca_expert_sort_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_branches(a->n_tokens, a->n_slots)) return refuse(why);
  if (a->n_experts < 1 || a->n_experts > kExpertsMost) return refuse("1 <= n_experts <= 512");
  const int64_t n = static_cast<int64_t>(a->n_tokens) * a->n_slots;
  const int64_t work = moeca_expert_sort_workspace(a->n_tokens, a->n_slots, a->n_experts);
  if (!a->offsets || (n > 0 && (!a->experts || !a->place)) || (work > 0 && !a->workspace))
    return refuse("experts, offsets, place or workspace is NULL");
  for (const void* p : {static_cast<const void*>(a->experts), static_cast<const void*>(a->offsets),
                        static_cast<const void*>(a->place), static_cast<const void*>(a->slot),
                        static_cast<const void*>(a->token), static_cast<const void*>(a->workspace)})
    if (addr(p) % 4) return refuse("a list is not 4-byte aligned");
  const Range written[] = {{a->offsets, 4ll * (a->n_experts + 1)}, {a->place, 4 * n}, {a->slot, 4 * n}, {a->token, 4 * n},
                           {work ? a->workspace : nullptr, 4 * work}};
  const Range read[] = {{a->experts, 4 * n}};
  if (any_overlap(written, read)) return refuse("lists overlap");
  SortArgs d{};
  d.experts = a->experts;
  d.n = static_cast<int>(n); d.k = a->n_slots; d.E = a->n_experts;
  d.offsets = a->offsets; d.place = a->place; d.slot = a->slot; d.token = a->token; d.work = a->workspace;
  return launched([&] { return launch_sort(d, static_cast<cudaStream_t>(stream)); });
}

moeca_status moeca_expert_rows(const moeca_expert_rows_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_shape(a->dtype, a->n_tokens, a->n_slots, a->width, a->n_rows, a->place)) return refuse(why);
  const int T = a->n_tokens, width = a->width;
  if (const char* why = bad_values(a->x, T, a->x_stride, width, a->dtype, "x is NULL")) return refuse(why);
  if (const char* why = bad_values(a->rows, a->n_rows, a->rows_stride, width, a->dtype, "rows is NULL")) return refuse(why);
  if (addr(a->count) % 4) return refuse("count is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), slots = static_cast<int64_t>(T) * a->n_slots;
  const Range written[] = {rows_range(a->rows, a->n_rows, a->rows_stride * es, width * es)};
  const Range read[] = {rows_range(a->x, T, a->x_stride * es, width * es), {a->place, 4 * slots}, {a->count, 4}};
  if (any_overlap(written, read)) return refuse("rows overlaps another buffer of the call");
  if (a->n_rows == 0 || (T == 0 && !a->count)) return MOECA_OK;
  const bool aligned = aligned16(a->x, a->x_stride, a->dtype) && aligned16(a->rows, a->rows_stride, a->dtype);
  return launched([&] {
    return pick(a->dtype, aligned, [&](auto* t, auto al) {
      using E = std::remove_pointer_t<decltype(t)>;
      const int units = row_units<E>(width, al.value);
      return by_group(units, [&](auto lanes) {
        const RowsArgs d{a->x, a->x_stride, a->rows, a->rows_stride, a->n_rows, a->place, a->count, T, a->n_slots, width,
                         segments(units, lanes.value, kRowsUnits)};
        // The tail of an empty batch is cleared by as many threads as its units need.
        const int64_t threads = T == 0 ? a->n_rows * units : static_cast<int64_t>(T) * d.seg.segs * lanes.value;
        return launch_pdl(expert_rows_kernel<E, al.value, lanes.value>, row_grid(threads), dim3(kRowThreads), 0,
                          static_cast<cudaStream_t>(stream), d);
      });
    });
  });
}

moeca_status moeca_expert_combine(const moeca_expert_combine_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_shape(a->dtype, a->n_tokens, a->n_slots, a->width, a->n_rows, a->place)) return refuse(why);
  const int T = a->n_tokens, width = a->width;
  if (const char* why = bad_values(a->rows, a->n_rows, a->rows_stride, width, a->dtype, "rows is NULL")) return refuse(why);
  if (const char* why = bad_values(a->out, T, a->out_stride, width, a->dtype, "out is NULL")) return refuse(why);
  if (a->x)
    if (const char* why = bad_values(a->x, T, a->x_stride, width, a->dtype, "")) return refuse(why);
  if (addr(a->weights) % 4) return refuse("weights is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), slots = static_cast<int64_t>(T) * a->n_slots;
  const bool in_place = a->x == a->out && a->x_stride == a->out_stride;
  const Range written[] = {rows_range(a->out, T, a->out_stride * es, width * es)};
  const Range read[] = {rows_range(a->rows, a->n_rows, a->rows_stride * es, width * es), {a->place, 4 * slots},
                        {a->weights, 4 * slots}, rows_range(in_place ? nullptr : a->x, T, a->x_stride * es, width * es)};
  if (any_overlap(written, read)) return refuse("out overlaps another buffer of the call");
  if (T == 0) return MOECA_OK;
  const bool aligned = aligned16(a->out, a->out_stride, a->dtype) &&
                       (a->n_rows == 0 || aligned16(a->rows, a->rows_stride, a->dtype)) &&
                       (!a->x || aligned16(a->x, a->x_stride, a->dtype));
  return launched([&] {
    return pick(a->dtype, aligned, [&](auto* t, auto al) {
      using E = std::remove_pointer_t<decltype(t)>;
      const int units = row_units<E>(width, al.value);
      return by_group(units, [&](auto lanes) {
        constexpr int L = lanes.value;
        const bool two = a->n_slots <= 2;
        const BackArgs d{a->rows, a->rows_stride, a->n_rows, a->place, a->weights, a->x, a->x_stride,
                         a->out, a->out_stride, T, a->n_slots, width, segments(units, L, two ? 2 : 1)};
        return launch_pdl(two ? expert_combine_kernel<E, al.value, L, 2, 2> : expert_combine_kernel<E, al.value, L, 4, 1>,
                          row_grid(static_cast<int64_t>(T) * d.seg.segs * L), dim3(kRowThreads), 0,
                          static_cast<cudaStream_t>(stream), d);
      });
    });
  });
}

moeca_status moeca_expert_combine_grad(const moeca_expert_combine_grad_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (const char* why = bad_shape(a->dtype, a->n_tokens, a->n_slots, a->width, a->n_rows, a->place)) return refuse(why);
  const int T = a->n_tokens, width = a->width;
  if (const char* why = bad_values(a->dout, T, a->dout_stride, width, a->dtype, "dout is NULL")) return refuse(why);
  if (a->dweights || a->rows)
    if (const char* why = bad_values(a->rows, a->n_rows, a->rows_stride, width, a->dtype, "rows is NULL")) return refuse(why);
  if (a->drows)
    if (const char* why = bad_values(a->drows, a->n_rows, a->drows_stride, width, a->dtype, "")) return refuse(why);
  if (addr(a->weights) % 4 || addr(a->dweights) % 4 || addr(a->count) % 4)
    return refuse("weights, dweights or count is not 4-byte aligned");
  const int64_t es = elem_size(a->dtype), slots = static_cast<int64_t>(T) * a->n_slots;
  const Range written[] = {rows_range(a->drows, a->n_rows, a->drows_stride * es, width * es), {a->dweights, 4 * slots}};
  const Range read[] = {rows_range(a->dout, T, a->dout_stride * es, width * es),
                        rows_range(a->rows, a->n_rows, a->rows_stride * es, width * es), {a->place, 4 * slots},
                        {a->weights, 4 * slots}, {a->count, 4}};
  if (any_overlap(written, read)) return refuse("drows or dweights overlaps another buffer of the call");
  const bool clears = a->drows && a->count && a->n_rows > 0;
  if ((!a->drows && !a->dweights) || (T == 0 && !clears)) return MOECA_OK;
  const GradArgs d{a->dout, a->dout_stride, a->rows, a->rows_stride, a->n_rows, a->place, a->weights, a->count,
                   a->drows, a->drows_stride, a->dweights, T, a->n_slots, width, 0};
  const bool aligned = aligned16(a->dout, a->dout_stride, a->dtype) &&
                       (!a->dweights || a->n_rows == 0 || aligned16(a->rows, a->rows_stride, a->dtype)) &&
                       (!a->drows || aligned16(a->drows, a->drows_stride, a->dtype));
  return launched([&] {
    return pick(a->dtype, aligned, [&](auto* t, auto al) {
      using E = std::remove_pointer_t<decltype(t)>;
      GradArgs k = d;
      k.units = row_units<E>(width, al.value);
      return launch_pdl(expert_grad_kernel<E, al.value>, row_grid((T == 0 ? a->n_rows : slots) * 32), dim3(kRowThreads), 0,
                        static_cast<cudaStream_t>(stream), k);
    });
  });
}

}  // extern "C"
