// Attention over packed sequences (include/moeca_attention.h): what its kernels share.
//
// Every kernel works on (a tile of one sequence's query rows, a key head or query
// head, and either all of the sequence's keys or one chunk of them).  Where the
// key axis is cut into chunks, each chunk's kernel leaves its normalised result,
// its maximum and its sum in the workspace, and a last kernel joins
// the chunks of a row in their order.  (Maximum and sum apart: in a logarithm of
// the sum that holds both, a score of 2^20 leaves the sum three bits.)  A sequence
// whose keys are one chunk goes to its place at once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "heads.h"

namespace moeca {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The sequences' share of the tokens, and their pieces of `unit` tokens, numbered
// through.  Tokens and pieces are counted in 32 bits (the call takes 2^30 tokens at
// most): index arithmetic is a sizeable part of a short sequence's time.
struct Seqs {
  const int32_t* off;  // [n + 1], or null: `each` tokens each
  int total, n, each;
  int unit;
  int per;  // pieces of each sequence, or 0: sequence b's begin at off[b] / unit + b
  int firsts;  // how chunks are numbered, see below (with per 0)

  __device__ __forceinline__ int start(int b) const { return off ? min(max(off[b], 0), total) : b * each; }
  __device__ __forceinline__ int length(int b) const { return off ? max(start(b + 1) - start(b), 0) : each; }
  __device__ __forceinline__ int base(int b) const {
    return per ? b * per : static_cast<int>(static_cast<uint32_t>(start(b)) / static_cast<uint32_t>(unit)) + b;
  }
  // The last sequence with value(b) <= p, found 32 sequences at a time (all lanes of
  // a warp; the same answer in all).
  template <typename F>
  __device__ __forceinline__ int last(int p, F value) const {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, b = lo + static_cast<int>(threadIdx.x & 31) * step;
      const uint32_t ok = __ballot_sync(0xffffffffu, b < hi && value(b) <= p);
      const int count = __ffs(~ok) - 1;  // lanes 0 .. count - 1 hold; -1: all 32
      lo += max((count < 0 ? 32 : count) - 1, 0) * step;
      hi = min(lo + step, hi);
    }
    return lo;
  }
  // The sequence whose piece `p` is.  ceil(len / unit) pieces fit before the next
  // sequence's, wherever it begins.
  __device__ __forceinline__ int find(int p) const {
    if (per) return static_cast<int>(static_cast<uint32_t>(p) / static_cast<uint32_t>(per));
    return last(p, [this](int b) { return base(b); });
  }
  // The number of sequence b's chunk c: as pieces, or with `firsts` every sequence's first chunk, then the others, so
  // that where most sequences have one the blocks of these start at once and those without a chunk come last.
  // Sequence b's second is then n + off[b] / unit: floor((len - 1) / unit) others fit before the next sequence's.
  __device__ __forceinline__ int chunk(int b, int c) const {
    if (!firsts) return base(b) + c;
    return c == 0 ? b : n + second(b) + c - 1;
  }
  __device__ __forceinline__ int second(int b) const { return static_cast<int>(static_cast<uint32_t>(start(b)) / static_cast<uint32_t>(unit)); }
  // The sequence and its chunk (below 0: none) of number p.
  __device__ __forceinline__ int find_chunk(int p, int* c) const {
    if (!firsts || p < n) {
      const int b = firsts ? p : find(p);
      *c = firsts ? 0 : p - base(b);
      return b;
    }
    const int b = last(p - n, [this](int b) { return second(b); }), more = p - n - second(b);
    *c = more < 0 ? -1 : more + 1;
    return b;
  }
  // The sequence of a token.
  __device__ __forceinline__ int owner(int t) const {
    if (!off) return min(static_cast<int>(static_cast<uint32_t>(t) / static_cast<uint32_t>(max(each, 1))), n - 1);
    return last(t, [this](int b) { return start(b); });
  }
};

struct PackedAttnArgs {
  Heads q, k, v, out;
  Seqs qs;          // unit: query tokens of a tile
  Seqs ks;          // unit: keys of a chunk, 0 = no chunks
  int64_t q_pieces, k_pieces;
  float* lse;       // [queries, heads] or null
  float* part_o;    // [k_pieces, max_q, heads, dim]
  float2* part_ml;  // [k_pieces, max_q, heads]: the maximum of q . k, -infinity where no key is seen, and the sum
  int max_q;        // queries of a sequence that are computed
  int tiles;        // tiles of max_q queries
  int group;        // query heads per key head
  int dim;
  int causal;
  int clear;        // what becomes of query tokens that are not computed: 0 nothing, 1 out and lse, 2 lse
  float scale_log2; // scale log2(e)
  int32_t* status;
  // How long a bounded wait lasts, and the barrier whose wait is to run out (tests; see
  // moeca_probe_attention_stall): it is set up for one arrival more than comes.
  unsigned long long wait_ns;
  int stall;
};

// One block's work.
struct AttnWork {
  int q0, k0;            // first tokens of the sequence
  int nq, nk;            // its queries (of which the first max_q count) and keys
  int row0;              // first query of the tile
  int key_lo, key_hi;    // keys of the chunk
  int piece;             // the chunk's number
  bool any;              // whether the tile and the chunk exist
};
// index: the tile (no chunks), or chunk x tiles + tile.  All lanes of a warp.
__device__ __forceinline__ AttnWork attn_work(const PackedAttnArgs& a, int index) {
  AttnWork w;
  int b, tile, chunk = 0;
  if (a.ks.unit == 0) {
    b = a.qs.find(index);
    tile = index - a.qs.base(b);
    w.piece = 0;
  } else {
    w.piece = static_cast<int>(static_cast<uint32_t>(index) / static_cast<uint32_t>(a.tiles));
    b = a.ks.find_chunk(w.piece, &chunk);
    tile = index - w.piece * a.tiles;
  }
  w.q0 = a.qs.start(b);
  w.k0 = a.ks.start(b);
  w.nq = a.qs.length(b);
  w.nk = a.ks.length(b);
  const int64_t row0 = static_cast<int64_t>(tile) * a.qs.unit;
  w.any = row0 >= 0 && row0 < min(w.nq, a.max_q);
  w.row0 = w.any ? static_cast<int>(row0) : 0;
  w.key_lo = 0;
  w.key_hi = w.nk;
  if (a.ks.unit) {
    const int64_t lo = static_cast<int64_t>(chunk) * a.ks.unit;
    w.any = w.any && lo >= 0 && lo < w.nk;
    w.key_lo = w.any ? static_cast<int>(lo) : 0;
    w.key_hi = w.any ? min(w.key_lo + a.ks.unit, w.nk) : 0;
  }
  return w;
}
// Keys that query i of the sequence sees: 0 .. visible - 1.
__device__ __forceinline__ int visible_keys(const PackedAttnArgs& a, const AttnWork& w, int i) {
  return a.causal ? min(max(i + 1 - w.nq + w.nk, 0), w.nk) : w.nk;
}

// Query tokens that are not computed: their rows become 0 (clear 1), the logs of their sums -infinity.
// Those before the first and behind the last sequence: the blocks take them in turn.  A sequence's
// behind its first max_q: its own blocks do.  index: as for attn_work; head: of the `heads` that a tile has a block for;
// `threads` of the block's threads, whole warps, share a token.  A call: rare, and its loops would cost the kernels
// registers.
template <typename T>
__device__ __noinline__ void clear_tokens(const PackedAttnArgs& a, int index, int head, int heads, int thread, int threads) {
  const auto clear = [&](int64_t first, int64_t step, int64_t end) {
    for (int64_t t = first; t < end; t += step) {
      if (a.clear == 1) {
        T* out = static_cast<T*>(a.out.data) + t * a.out.token_stride;
        for (int h = 0; h < a.out.heads; ++h)
          for (int c = thread; c < a.dim; c += threads) out[h * a.out.head_stride + c] = T(0.f);
      }
      if (a.lse)
        for (int h = thread; h < a.out.heads; h += threads) a.lse[t * a.out.heads + h] = -INFINITY;
    }
  };
  if (a.qs.off) {
    const int lo = a.qs.start(0), hi = max(a.qs.start(a.qs.n), lo);
    clear(blockIdx.x, gridDim.x, lo);
    clear(static_cast<int64_t>(hi) + blockIdx.x, gridDim.x, a.qs.total);
  }
  int b, tile, chunk = 0, chunks = 1;
  if (a.ks.unit == 0) {
    b = a.qs.find(index);
    tile = index - a.qs.base(b);
  } else {
    const int piece = static_cast<int>(static_cast<uint32_t>(index) / static_cast<uint32_t>(a.tiles));
    b = a.ks.find_chunk(piece, &chunk);
    tile = index - piece * a.tiles;
    chunks = max((a.ks.length(b) - 1) / a.ks.unit + 1, 1);  // a sequence without keys still has its first chunk's block
  }
  if (tile < 0 || tile >= a.tiles || chunk < 0 || chunk >= chunks) return;
  const int64_t share = (static_cast<int64_t>(chunk) * a.tiles + tile) * heads + head, first = a.qs.start(b);
  clear(first + a.max_q + share, static_cast<int64_t>(chunks) * a.tiles * heads, first + a.qs.length(b));
}
template <typename T>
__device__ __forceinline__ void clear_rest(const PackedAttnArgs& a, const AttnWork& w, int index, int head, int heads, int thread,
                                           int threads) {
  if (a.clear && (w.nq > a.max_q || (a.qs.off && (a.qs.start(0) > 0 || a.qs.start(a.qs.n) < a.qs.total))))
    clear_tokens<T>(a, index, head, heads, thread, threads);
}

cudaError_t launch_attn_simt(const PackedAttnArgs& a, int dtype, int tile, cudaStream_t s);
// tiles: of 128 rows in a block, 1 or 2.
cudaError_t launch_attn_packed_tc(const PackedAttnArgs& a, int tiles, cudaStream_t s);
cudaError_t launch_attn_rows(const PackedAttnArgs& a, cudaStream_t s);
cudaError_t launch_attn_join(const PackedAttnArgs& a, int dtype, cudaStream_t s);

}  // namespace moeca
