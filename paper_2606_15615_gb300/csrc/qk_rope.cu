// Norms of query and key heads with the position rotation (include/moeca_attention.h).
#include <algorithm>

#include "calls.h"
#include "common.cuh"
#include "heads.h"
#include "moeca_attention.h"

namespace moeca {
namespace {

constexpr int kQkThreads = 256;
constexpr int kMaxDim = 512;
constexpr int kQkGroups = 32768;   // groups of lanes from which on a group takes several heads
constexpr int kQkMostHeads = 8;

struct QkArgs {
  Heads q, k, q_out, k_out;
  const float *q_weight, *k_weight;
  const float2* table;
  const int32_t* pos;
  int64_t n_pos;
  int T, dim, rot;
  int lanes;   // lanes that share a head: its units, at most 32
  int per;     // heads that a group of lanes takes one after another
  int parts;   // groups per token
  float eps, inv_dim;
  int clear;   // results whose tokens without a position become 0: 1 of q, 2 of k
  bool table16, weight16;  // rows of the table, the weights' chunks can be read 16 bytes at a time
};

// W values of a head: as loaded, and in fp32.
template <typename T, int W>
struct Chunk {
  static constexpr int WORDS = (W * sizeof(T) + 3) / 4;
  uint32_t raw[WORDS];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) raw[i] = 0;
  }
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W * sizeof(T) == 16) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      raw[0] = v.x; raw[1] = v.y; raw[2] = v.z; raw[3] = v.w;
    } else if constexpr (W * sizeof(T) == 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      raw[0] = v.x; raw[1] = v.y;
    } else if constexpr (sizeof(T) == 4) {
      raw[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      raw[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < W; ++i)
      f[i] = sizeof(T) == 4 ? __uint_as_float(raw[i])
                            : __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);  // bf16: the upper half
  }
  __device__ __forceinline__ static void store(T* p, const float* f) {
    if constexpr (W * sizeof(T) == 16) {
      store_vec(p, f);
    } else if constexpr (W * sizeof(T) == 8) {
      uint2 v;
      if constexpr (sizeof(T) == 4) {
        v = make_uint2(__float_as_uint(f[0]), __float_as_uint(f[1]));
      } else {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        v = make_uint2(reinterpret_cast<const uint32_t&>(a), reinterpret_cast<const uint32_t&>(b));
      }
      *reinterpret_cast<uint2*>(p) = v;
    } else {
      p[0] = Elem<T>::from_f(f[0]);
    }
  }
};

// The sum over a group of n lanes, any n up to 32, the same in all of them.
// lane: the group's own number of this one; all lanes of the warp take part.
__device__ __forceinline__ float group_sum(float v, int lane, int n) {
  for (int o = 16; o > 0; o >>= 1) {
    const float w = __shfl_down_sync(0xffffffffu, v, o);
    if (lane + o < n) v += w;
  }
  return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31) - lane);
}

// A unit is two chunks of W values of a head: with PAIRS 2 W values side by side,
// else values i .. i + W - 1 and their partners rot / 2 further; what is not
// turned (rot .. dim - 1) is cut into units of neighbouring chunks either way.
// A group of `lanes` lanes takes the units of one head, U units a lane, and works
// through `per` heads of its token with the token's cosines and sines and the
// weights in registers: up to eight (16384 tokens of 20 + 4 heads of 128, rot 96
// in pairs: 47 us; with four 50, with two 69, as table and weights are loaded for
// each group).  The next head is loaded while one is worked on.  Blocks an SM: three
// with chunks of eight values (four spill: 55 us), five with four (16384 tokens
// of 32 heads of 72: 42 us; when this was chosen 44, with three 51).  One pass: every value is
// read and written once, the table comes from L1 / L2 but for the first token at a position.
template <typename T, int W, int U, bool PAIRS>
__global__ void __launch_bounds__(kQkThreads, U > 1 ? 1 : W == 8 ? 3 : 5) qk_norm_rope_kernel(const QkArgs a) {
  pdl_entry();
  const int warp_lane = threadIdx.x & 31, per_warp = 32 / a.lanes;
  const int in_warp = warp_lane / a.lanes, lane = warp_lane - in_warp * a.lanes;
  const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kQkThreads + threadIdx.x) >> 5;
  const int64_t group = warp * per_warp + in_warp;
  const int64_t t = group / a.parts;
  const int part = static_cast<int>(group - t * a.parts);
  bool on = in_warp < per_warp && t < a.T;
  int64_t row = 0;
  if (on && a.rot) {
    row = a.pos ? a.pos[t] : t;
    on = row >= 0 && row < a.n_pos;
  }
  const int turned = a.rot / (2 * W), units = turned + (a.dim - a.rot + 2 * W - 1) / (2 * W);
  int lo[U], hi[U];  // where the unit's chunks start; dim where there is none
  float2 turn[U][W];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = lane + u * a.lanes;
    lo[u] = hi[u] = a.dim;
    if (i < turned) {
      lo[u] = PAIRS ? 2 * W * i : W * i;
      hi[u] = lo[u] + (PAIRS ? W : a.rot / 2);
      if (on) {
        const float2* cs = a.table + row * (a.rot / 2) + W * i;
        if (W > 1 && a.table16) {
#pragma unroll
          for (int j = 0; j < W; j += 2) {
            const float4 v = *reinterpret_cast<const float4*>(cs + j);
            turn[u][j] = make_float2(v.x, v.y);
            turn[u][j + (W > 1)] = make_float2(v.z, v.w);
          }
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) turn[u][j] = cs[j];
        }
      }
    } else if (i < units) {
      lo[u] = a.rot + 2 * W * (i - turned);
      hi[u] = min(lo[u] + W, a.dim);
    }
  }
  if (a.clear && !on && in_warp < per_warp && t < a.T) {  // a token without a position
    const float zeros[W] = {};
    for (int h = part * a.per; h < min((part + 1) * a.per, a.q.heads + a.k.heads); ++h) {
      const bool is_q = h < a.q.heads;
      if (!(a.clear & (is_q ? 1 : 2))) continue;
      const Heads& out = is_q ? a.q_out : a.k_out;
      T* z = static_cast<T*>(out.data) + t * out.token_stride + (is_q ? h : h - a.q.heads) * out.head_stride;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (lo[u] < a.dim) Chunk<T, W>::store(z + lo[u], zeros);
        if (hi[u] < a.dim) Chunk<T, W>::store(z + hi[u], zeros);
      }
    }
  }
  float weight[U][2][W];
  const int heads = a.q.heads + a.k.heads;
  Chunk<T, W> next[U][2];
  // Where the next head to fetch and the one to write lie; the first key follows the last query.
  const int h0 = part * a.per;
  const bool from_q = h0 < a.q.heads;
  const int64_t hh = from_q ? h0 : h0 - a.q.heads;
  const T* x = static_cast<const T*>(from_q ? a.q.data : a.k.data) +
               (from_q ? t * a.q.token_stride + hh * a.q.head_stride : t * a.k.token_stride + hh * a.k.head_stride);
  T* y = static_cast<T*>(from_q ? a.q_out.data : a.k_out.data) +
         (from_q ? t * a.q_out.token_stride + hh * a.q_out.head_stride : t * a.k_out.token_stride + hh * a.k_out.head_stride);
  const auto fetch = [&](int h) {
    const bool live = on && h < heads;
    if (h > h0) x = h == a.q.heads ? static_cast<const T*>(a.k.data) + t * a.k.token_stride
                                   : x + (h < a.q.heads ? a.q.head_stride : a.k.head_stride);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      next[u][0].clear();
      next[u][1].clear();
      if (live && lo[u] < a.dim) next[u][0].load(x + lo[u]);
      if (live && hi[u] < a.dim) next[u][1].load(x + hi[u]);
    }
  };
  fetch(h0);
  // Every lane of the warp takes the same number of rounds: the sums are shuffles of whole warps.
  for (int i = 0; i < a.per; ++i) {
    const int h = h0 + i;
    const bool is_q = h < a.q.heads, live = on && h < heads;
    if (i > 0) y = h == a.q.heads ? static_cast<T*>(a.k_out.data) + t * a.k_out.token_stride
                                  : y + (is_q ? a.q_out.head_stride : a.k_out.head_stride);
    float c[U][2][W];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      next[u][0].get(c[u][0]);
      next[u][1].get(c[u][1]);
    }
    if (i + 1 < a.per) fetch(h + 1);  // in flight while this head is worked on
    if (i == 0 || h == a.q.heads) {
      const float* w = is_q ? a.q_weight : a.k_weight;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int at = e ? hi[u] : lo[u];
#pragma unroll
          for (int j = 0; j < W; ++j) weight[u][e][j] = 1.f;
          if (w && live && at < a.dim) {
            if (W >= 4 && a.weight16) {
#pragma unroll
              for (int j = 0; j + 3 < W; j += 4) load_vec(w + at + j, weight[u][e] + j);
            } else {
#pragma unroll
              for (int j = 0; j < W; ++j) weight[u][e][j] = w[at + j];
            }
          }
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < W; ++j) sum = fmaf(c[u][0][j], c[u][0][j], fmaf(c[u][1][j], c[u][1][j], sum));
    sum = group_sum(sum, lane, a.lanes);
    const float r = rsqrtf(fmaf(sum, a.inv_dim, a.eps));  // off by 2^-22 at most; the sum of squares by dim 2^-23
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < W; ++j) c[u][e][j] = c[u][e][j] * r * weight[u][e][j];
      if (lane + u * a.lanes < turned) {
        if (PAIRS && W > 1) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j + 1 < W; j += 2) {
              const float2 cs = turn[u][(e * W + j) / 2];
              const float p = c[u][e][j], q = c[u][e][j + 1];
              c[u][e][j] = p * cs.x - q * cs.y;
              c[u][e][j + 1] = q * cs.x + p * cs.y;
            }
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const float2 cs = turn[u][j];
            const float p = c[u][0][j], q = c[u][1][j];
            c[u][0][j] = p * cs.x - q * cs.y;
            c[u][1][j] = q * cs.x + p * cs.y;
          }
        }
      }
      if (live && lo[u] < a.dim) Chunk<T, W>::store(y + lo[u], c[u][0]);
      if (live && hi[u] < a.dim) Chunk<T, W>::store(y + hi[u], c[u][1]);
    }
  }
}

// Whether heads can be taken W values at a time.
bool by(const moeca_heads& h, int w, int64_t es) {
  return h.heads == 0 || (addr(h.data) % (w * es) == 0 && h.token_stride % w == 0 && h.head_stride % w == 0);
}

template <typename T>
cudaError_t launch_qk(QkArgs a, int width, int units, bool pairs, int blocks, cudaStream_t s) {
  constexpr int V = Elem<T>::kVec;
  const auto run = [&](auto kernel) { return launch_pdl(kernel, dim3(blocks), dim3(kQkThreads), 0, s, a); };
  const bool one = units <= 32;
  if (width == V) {
    if constexpr (V == 8) return run(pairs ? qk_norm_rope_kernel<T, 8, 1, true> : qk_norm_rope_kernel<T, 8, 1, false>);
    else if (one) return run(pairs ? qk_norm_rope_kernel<T, 4, 1, true> : qk_norm_rope_kernel<T, 4, 1, false>);
    else return run(pairs ? qk_norm_rope_kernel<T, 4, 2, true> : qk_norm_rope_kernel<T, 4, 2, false>);
  }
  if (width == V / 2) {
    if (one) return run(pairs ? qk_norm_rope_kernel<T, V / 2, 1, true> : qk_norm_rope_kernel<T, V / 2, 1, false>);
    return run(pairs ? qk_norm_rope_kernel<T, V / 2, 16 / V, true> : qk_norm_rope_kernel<T, V / 2, 16 / V, false>);
  }
  if (one) return run(pairs ? qk_norm_rope_kernel<T, 1, 1, true> : qk_norm_rope_kernel<T, 1, 1, false>);
  return run(pairs ? qk_norm_rope_kernel<T, 1, 8, true> : qk_norm_rope_kernel<T, 1, 8, false>);
}

}  // namespace
}  // namespace moeca

extern "C" moeca_status moeca_qk_norm_rope(const moeca_qk_norm_rope_args* a, void* stream) {
  using namespace moeca;
  if (!a) return refuse("NULL argument");
  if (!is_dtype(a->dtype)) return refuse("dtype must be MOECA_F32 or MOECA_BF16");
  if (a->n_tokens < 0) return refuse("n_tokens is negative");
  if (a->dim < 1 || a->dim > kMaxDim) return refuse("1 <= dim <= 512");
  if (a->rot < 0 || a->rot > a->dim || a->rot % 2) return refuse("rot must be even, 0 .. dim");
  if (!(a->eps >= 0)) return refuse("eps must not be negative");
  if (a->pairs < 0 || a->pairs > 1) return refuse("pairs must be 0 or 1");
  if (a->clear < 0 || a->clear > 3) return refuse("clear must be 0 .. 3");
  if (a->n_positions < 0 || a->n_positions > kMaxRows) return refuse("n_positions out of range");
  const int64_t T = a->n_tokens, es = elem_size(a->dtype);
  const int dim = a->dim;
  for (const moeca_heads* h : {&a->q, &a->k})
    if (const char* why = bad_heads(*h, T, dim, a->dtype, false)) return refuse(why);
  for (const moeca_heads* h : {&a->q_out, &a->k_out})
    if (const char* why = bad_heads(*h, T, dim, a->dtype, true)) return refuse(why);
  if (a->q.heads < 1 || a->q_out.heads != a->q.heads || a->k_out.heads != a->k.heads)
    return refuse("q has a head at least, and the results as many as what they come from");
  if (a->rot && a->n_positions > 0 && !a->table) return refuse("table is NULL");
  if (addr(a->table) % 8 || addr(a->pos) % 4 || addr(a->q_weight) % 4 || addr(a->k_weight) % 4)
    return refuse("table, pos or a weight is not aligned");
  const Range lists[] = {{a->table, a->n_positions * a->rot * 4}, {a->rot ? a->pos : nullptr, 4 * T},
                         {a->q_weight, 4ll * dim}, {a->k_weight, 4ll * dim}};
  const auto clash = [&](const moeca_heads& out, const moeca_heads& own, const moeca_heads& other) {
    for (const Range& r : lists)
      if (heads_overlap(out, T, r, dim, es)) return true;
    return (!same_heads(out, own) && heads_overlap(out, T, own, T, dim, es)) || heads_overlap(out, T, other, T, dim, es);
  };
  if (clash(a->q_out, a->q, a->k) || clash(a->k_out, a->k, a->q) || heads_overlap(a->q_out, T, a->k_out, T, dim, es))
    return refuse("q_out or k_out overlaps another buffer of the call");
  if (T == 0) return MOECA_OK;
  QkArgs d{};
  d.q = device_heads(a->q); d.k = device_heads(a->k);
  d.q_out = device_heads(a->q_out); d.k_out = device_heads(a->k_out);
  d.q_weight = a->q_weight; d.k_weight = a->k_weight;
  d.table = reinterpret_cast<const float2*>(a->table);
  d.pos = a->pos; d.n_pos = a->n_positions;
  d.T = a->n_tokens; d.dim = dim; d.rot = a->rot; d.eps = a->eps; d.clear = a->clear; d.inv_dim = 1.f / static_cast<float>(dim);
  // Chunks of 16 bytes, of 8, or single values.
  int w = static_cast<int>(16 / es);
  const auto fits = [&](int n) {
    return a->rot % (2 * n) == 0 && (dim - a->rot) % n == 0 && by(a->q, n, es) && by(a->k, n, es) && by(a->q_out, n, es) &&
           by(a->k_out, n, es);
  };
  if (!fits(w)) w = fits(w / 2) ? w / 2 : 1;
  d.table16 = addr(a->table) % 16 == 0 && a->rot % 4 == 0;
  d.weight16 = addr(a->q_weight) % 16 == 0 && addr(a->k_weight) % 16 == 0 && a->rot / 2 % 4 == 0 && a->rot % 4 == 0;
  const int units = a->rot / (2 * w) + (dim - a->rot + 2 * w - 1) / (2 * w), heads = a->q.heads + a->k.heads;
  d.lanes = std::min(units, 32);
  d.per = static_cast<int>(std::clamp<int64_t>(T * heads / kQkGroups, 1, kQkMostHeads));
  d.parts = (heads + d.per - 1) / d.per;
  const int64_t groups = T * d.parts, warps = (groups + 32 / d.lanes - 1) / (32 / d.lanes);
  const int64_t blocks = (warps * 32 + kQkThreads - 1) / kQkThreads;
  if (blocks > kMaxRows) {
    keep_call_error("too many heads for one launch");
    return MOECA_ERR_UNSUPPORTED;
  }
  return launched([&] {
    return (a->dtype == MOECA_BF16 ? launch_qk<__nv_bfloat16> : launch_qk<float>)(d, w, units, a->pairs != 0,
                                                                                  static_cast<int>(blocks),
                                                                                  static_cast<cudaStream_t>(stream));
  });
}
