// Attention over packed sequences on the tensor cores (include/moeca_attention.h):
// bf16, heads of up to 128 values.
//
// A CTA works on one key head and NT tiles of 128 rows, over the sequence's keys
// or one chunk of them.  A tile's rows are (query, head) pairs: 128 / G queries
// with the G query heads that share the key head, so that every key block that
// comes in serves all of them, and a single new token fills G rows instead of one.
//   warp 0      TMA: the tiles' queries once, then key and value blocks of 128 keys
//               through one ring of 32 KB (16 KB) slots, in the order of their use
//   warp 1      allocates TMEM and issues tcgen05.mma from one thread:
//               S_i = Q_i K_j^T (128 x 128, fp32), then O_i += P_i V_j
//   warps 2 ..  softmax: four warps per tile, a row per thread.  A thread takes its
//               row of S from TMEM, keeps the running maximum m and sum l, and
//               writes P = 2^((s - m) c), c = scale log2(e), in bf16 over S, where the
//               second product reads it as its A operand.
// With two tiles the tensor core works on one tile while the other's softmax
// runs; S, and O beside it, take 256 TMEM columns a tile.  V is taken as it lies in
// memory (keys x channels): the product reads it as an MN-major operand.
// The row's maximum moves only when it rises by more than 2^8 (O is then rescaled
// in TMEM; P stays below 2^8): after the first blocks that is rare.  S_{j+1}'s
// completion is committed after the product with P_j was issued, so a thread
// that sees S_{j+1} knows that O is quiet.
// P is rounded to bf16, the operand's type; l adds the unrounded values in fp32.
// Keys behind the sequence's end are masked; value rows there are zeroed in shared
// memory before the product, as they belong to another sequence and may hold
// infinities or NaN.
// 4 x 4096 tokens, 16 heads of 128: 366 us, 1.50 PFLOP/s (0.78 of the measured burst
// rate, 0.88 of the sustained one); of 64: 291 us (308 in some processes), 0.94 PFLOP/s: a
// tile's chain from its scores through its softmax and the hand-over to the next scores
// is longer there than the products of both tiles (1024 clocks a block). Causal, 8192
// tokens, 32 heads of 128 on 8: 357 us, 1.54 PFLOP/s. Short sequences are bound by a CTA's
// start and end (index, TMEM and first copies some 3 us): 16 of 256, 16 heads of 72, 17 us.
// Every wait is bounded (about one second); a wait that runs out records
// MOECA_ERR_TIMEOUT, raises the CTA's abort flag, lets what was issued finish,
// frees TMEM and returns.
#include <algorithm>

#include "attn_tc.cuh"
#include "moeca_probe.h"
#include "packed_attn.cuh"

namespace moeca {
namespace {

constexpr int kTileRows = 128;               // rows of a tile (MMA M)
constexpr int kBlockKeys = 128;              // keys of a block
constexpr int kPart = 128 * 128;             // bytes of 128 rows x 64 channels
constexpr int kMaxStages = 8;
constexpr float kFusedMost = 256.f;          // |m sc| up to which the exponent is one fused multiply-add
// Shared memory of a block less the static part: two blocks an SM with one tile, one with two.
constexpr size_t smem_most(int tiles) { return (tiles == 1 ? 110 : 225) * 1024; }

template <int DK, int NT>  // DK: 16-channel steps of a head
struct TcShape {
  static constexpr int DP = DK * 16;
  static constexpr int SUBS = (DP + 63) / 64;
  static constexpr int SLOT = SUBS * kPart;    // a tile of queries, a block of keys or of values
  static constexpr int STAGES_FIT = static_cast<int>((smem_most(NT) - 1024 - NT * SLOT) / SLOT);
  static constexpr int STAGES = STAGES_FIT < kMaxStages ? STAGES_FIT : kMaxStages;
  static constexpr size_t SMEM = static_cast<size_t>(NT + STAGES) * SLOT + 1024;
  static constexpr int COLUMNS = 256 * NT;     // TMEM
  // The result's rows on their way out: powers of two of 16-byte pieces are swizzled, others one piece further apart.
  static constexpr bool OUT_SWIZZLED = DP % 64 == 0;
  static constexpr int OUT_PITCH = DP * 2 + (OUT_SWIZZLED ? 0 : 16);
  static_assert(kTileRows * OUT_PITCH <= SLOT);
  static constexpr int THREADS = 64 + 128 * NT;
};

// Instruction descriptor: B with its N values side by side (MN-major), or with its K values (K-major).
__device__ __forceinline__ uint32_t instr_desc_b(int N, bool mn_major) {
  return instr_desc(kTileRows, 16) - (16u >> 3 << 17) + (static_cast<uint32_t>(N >> 3) << 17) + (mn_major ? 1u << 16 : 0u);
}
// Low word of a shared-memory matrix descriptor (128-byte swizzle, 8 rows 1024
// bytes on; the high word is the same for all).  K-major operands (queries, keys)
// do not use `lead`; for the MN-major values (64 channels a row, 8 keys 1024
// bytes on) it is the way to the next 64 channels.
__device__ __forceinline__ uint32_t desc_lo(uint32_t at, uint32_t lead) { return ((at & 0x3FFFFu) >> 4) | (lead >> 4 << 16); }
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
// One MMA, issued by the lane that has `issue` set.
__device__ __forceinline__ void mma_ss_if(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc, uint32_t issue) {
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %6, 0;\n"
      " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kDescHi), "r"(issue)
      : "memory");
}
__device__ __forceinline__ void mma_ts_if(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t acc, uint32_t issue) {
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %6, 0;\n"
      " mov.b64 b, {%2, %5};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kDescHi), "r"(issue)
      : "memory");
}
__device__ __forceinline__ void commit_if(uint32_t bar, uint32_t issue) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %1, 0;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(issue)
      : "memory");
}
__device__ __forceinline__ void tma_load_heads(uint32_t dst, const CUtensorMap* map, int channel, int head, int token, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(channel), "r"(head), "r"(token), "r"(bar)
      : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// mbar_wait without a call, the clock looked at every 256 tries (reading it takes longer than most waits).
__device__ __forceinline__ bool wait_here(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit) {
  if (mbar_try(bar, parity)) return true;
  unsigned long long t0 = 0;
#pragma unroll 1
  for (uint32_t it = 1; !mbar_try(bar, parity); ++it)
    if ((it & 255u) == 0) {
      const unsigned long long now = globaltimer();
      if (*abort_flag || (t0 != 0 && now - t0 > limit)) return false;
      if (t0 == 0) t0 = now;
    }
  return true;
}
__device__ __forceinline__ bool warp_wait_here(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit) {
  return __all_sync(0xffffffffu, wait_here(bar, parity, abort_flag, limit));
}

// Slots of the ring are filled and used in this order: K_0, K_1, V_0, K_2, V_1, ...
__device__ __forceinline__ int place_of_v(int j, int blocks) { return j + 1 < blocks ? 2 * j + 2 : 2 * j + 1; }

template <int DK, int NT>
__global__ void __launch_bounds__(64 + 128 * NT, NT == 1 ? 2 : 1)
    attn_packed_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                          const __grid_constant__ CUtensorMap vmap, const __grid_constant__ PackedAttnArgs a) {
  using Sh = TcShape<DK, NT>;
  constexpr int ST = Sh::STAGES;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full[NT], s_full[NT], p_full[NT][2], o_full[NT], full[ST], empty[ST], v_clean, drain;
  __shared__ int issued;          // slots that the producer filled (for the drain)
  __shared__ uint32_t tmem_sh;
  __shared__ volatile int abort_flag;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + NT * Sh::SLOT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    issued = 0;
    for (int i = 0; i < NT; ++i) {
      mbar_init(smem_u32(&q_full[i]), 1 + (a.stall == MOECA_ATTENTION_COPIES));
      mbar_init(smem_u32(&s_full[i]), 1 + (a.stall == MOECA_ATTENTION_SCORES));
      mbar_init(smem_u32(&p_full[i][0]), kTileRows);
      mbar_init(smem_u32(&p_full[i][1]), kTileRows + (a.stall == MOECA_ATTENTION_WEIGHTS));
      mbar_init(smem_u32(&o_full[i]), 1);
    }
    for (int i = 0; i < ST; ++i) {
      mbar_init(smem_u32(&full[i]), 1);
      mbar_init(smem_u32(&empty[i]), 1 + (a.stall == MOECA_ATTENTION_SLOTS));
    }
    mbar_init(smem_u32(&v_clean), 1);
    mbar_init(smem_u32(&drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&qmap)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&kmap)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&vmap)) : "memory");
  }
  __syncthreads();
  pdl_entry();
  // The heaviest tiles of a causal sequence are its last: they start first.
  const int turn = blockIdx.x / static_cast<uint32_t>(a.k.heads), kvh = blockIdx.x - turn * a.k.heads;
  const int index = a.causal && !a.ks.unit ? static_cast<int>(a.q_pieces) - 1 - turn : turn;
  const AttnWork w = attn_work(a, index);
  if (!w.any) {  // uniform over the CTA, before TMEM is taken
    clear_rest<__nv_bfloat16>(a, w, index, kvh, a.k.heads, threadIdx.x, blockDim.x);
    return;
  }
  const int G = a.group, per_tile = a.qs.unit / NT;  // queries of a tile
  const int n_q = min(w.nq, a.max_q);
  // Blocks of keys that each tile's rows see.
  int nb[NT], blocks = 0;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int first = w.row0 + i * per_tile, last = min(first + per_tile, n_q) - 1;
    nb[i] = first < n_q ? max(0, min(w.key_hi, visible_keys(a, w, last)) - w.key_lo + kBlockKeys - 1) / kBlockKeys : 0;
    blocks = max(blocks, nb[i]);
  }
  // Keys of the last block, in 16s, and whether foreign value rows are among them.
  const int last_keys = min(kBlockKeys, w.key_hi - (w.key_lo + (blocks - 1) * kBlockKeys));
  const bool dirty = blocks > 0 && last_keys % 16 != 0;
  // TMEM's address is waited for by the warps that use it; the copies start beside.
  uint32_t tmem = 0;
  if (warp != 0) {
    if (warp == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_sh)),
                   "r"(Sh::COLUMNS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      tc_fence_before();
    }
    asm volatile("bar.sync 1, %0;" ::"n"(Sh::THREADS - 32) : "memory");
    tc_fence_after();
    tmem = tmem_sh;
  }
  const auto give_up = [&](int where) {
    if (!abort_flag) report_status(a.status, MOECA_ERR_TIMEOUT, where);
    abort_flag = 1;
  };

  if (warp == 0) {
    if (lane == 0) {
      const int token = w.q0 + w.row0;
      const auto queries = [&](int i) {
        if (nb[i] == 0) return;
        mbar_expect_tx(smem_u32(&q_full[i]), Sh::SUBS * G * per_tile * 128);
        for (int s = 0; s < Sh::SUBS; ++s)
          tma_load_heads(smem_u32(smem + i * Sh::SLOT + s * kPart), &qmap, s * 64, kvh * G, token + i * per_tile, smem_u32(&q_full[i]));
      };
      int n = 0;
      bool ok = true;
      const auto fill = [&](const CUtensorMap* map, int block) {
        const int s = n % ST;
        if (n >= ST && !wait_here(smem_u32(&empty[s]), ((n / ST) - 1) & 1, &abort_flag, a.wait_ns)) {
          give_up(710);
          ok = false;
          return;
        }
        const uint32_t bar = smem_u32(&full[s]);
        mbar_expect_tx(bar, Sh::SLOT);
        for (int c = 0; c < Sh::SUBS; ++c)
          tma_load_heads(smem_u32(ring + s * Sh::SLOT + c * kPart), map, c * 64, kvh,
                         w.k0 + w.key_lo + block * kBlockKeys, bar);
        ++n;
      };
      queries(0);
      if (blocks > 0) fill(&kmap, 0);
      if constexpr (NT == 2) queries(1);
      for (int j = 0; ok && j < blocks; ++j) {
        if (j + 1 < blocks) fill(&kmap, j + 1);
        if (ok) fill(&vmap, j);
      }
      issued = n;
    }
    __syncwarp();
    // The lanes vote on the flag, which other warps may set meanwhile: what follows is a wait of the whole warp.
    if (dirty && !__any_sync(0xffffffffu, abort_flag != 0)) {
      // Value rows last_keys .. of the last block's 16s are another sequence's, or nobody's.
      const int n = place_of_v(blocks - 1, blocks), s = n % ST;
      if (warp_wait_here(smem_u32(&full[s]), (n / ST) & 1, &abort_flag, a.wait_ns)) {
        const int rows = (last_keys + 15) / 16 * 16 - last_keys;
        for (int i = lane; i < rows * 8 * Sh::SUBS; i += 32) {
          const int c = i / (rows * 8), at = i - c * rows * 8;
          *reinterpret_cast<uint4*>(ring + s * Sh::SLOT + c * kPart + last_keys * 128 + at * 16) = make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&v_clean));
      } else if (lane == 0) {
        give_up(711);
      }
    }
    clear_rest<__nv_bfloat16>(a, w, index, kvh, a.k.heads, lane, 32);
  } else if (warp == 1) {
    // All lanes run the loop and one issues; what the loop turns on is read from
    // lane 0, and so known to be the same in all (a block of two tiles of 64 channels
    // then took 2500 clocks; 3300 with each lane's own).
    const auto uniform = [](auto x) { return static_cast<decltype(x)>(__shfl_sync(0xffffffffu, x, 0)); };
    uint32_t issue;
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n selp.u32 %0, 1, 0, e;\n}" : "=r"(issue));
    const int n_blocks = uniform(blocks), n_last = uniform((last_keys + 15) / 16);
    int n_own[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) n_own[i] = uniform(nb[i]);
    const bool clean_first = uniform(static_cast<int>(dirty)) != 0;
    const uint32_t t = uniform(tmem);
    bool ok = true;
    const auto wait = [&](uint32_t bar, uint32_t phase) { return ok = warp_wait_here(bar, phase & 1, &abort_flag, a.wait_ns); };
    const uint32_t q_lo = desc_lo(smem_u32(smem), 16), ring_k = desc_lo(smem_u32(ring), 16), ring_v = desc_lo(smem_u32(ring), kPart);
    const uint32_t id_s = instr_desc_b(kBlockKeys, false), id_o = instr_desc_b(Sh::DP, true);
    const uint32_t full0 = smem_u32(&full[0]), empty0 = smem_u32(&empty[0]), p0 = smem_u32(&p_full[0][0]), s0 = smem_u32(&s_full[0]);
    // S_i, for the keys in slot `at`.
    const auto scores = [&](int i, uint32_t at, uint32_t id) {
      const uint32_t qa = q_lo + i * (Sh::SLOT >> 4), kb = ring_k + at * (Sh::SLOT >> 4);
#pragma unroll
      for (int kk = 0; kk < DK; ++kk) {
        const int off = ((kk >> 2) * kPart + (kk & 3) * 32) >> 4;
        mma_ss_if(t + i * 256, qa + off, kb + off, id, kk > 0, issue);
      }
      commit_if(s0 + i * 8, issue);
    };
    // The second product with 64 keys' P, `steps` of 16 keys of them.
    const auto values = [&](int i, int half, uint32_t vb, bool first, int steps) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        if (kk < steps)
          mma_ts_if(t + i * 256 + 128, t + i * 256 + (half * 4 + kk) * 8, vb + (half * 4 + kk) * (2048 >> 4), id_o,
                    !first || half > 0 || kk > 0, issue);
    };
    // Slots are used in the order in which they are filled.
    uint32_t at = 0, parity = 0;
    const auto next = [&] {
      if (++at == ST) {
        at = 0;
        parity ^= 1;
      }
    };
    const auto id_of = [&](int j) { return j + 1 < n_blocks ? id_s : instr_desc_b(n_last * 16, false); };
    if (n_blocks > 0 && wait(full0, 0)) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (ok && n_own[i] > 0 && wait(smem_u32(&q_full[i]), 0)) {
          tc_fence_after();
          scores(i, 0, id_of(0));
        }
      if (ok) commit_if(empty0, issue);
    }
    for (int j = 0; ok && j < n_blocks; ++j) {
      const bool last = j + 1 == n_blocks;
      const uint32_t id_next = id_of(j + 1);
      const int steps = last ? n_last : kBlockKeys / 16;
      // The next keys come before this block's values.
      uint32_t k_at = 0, k_parity = 0;
      if (!last) {
        next();
        k_at = at;
        k_parity = parity;
      }
      next();
      // Most often both are there: one vote for two barriers.
      const bool there = mbar_try(full0 + at * 8, parity) && (last || mbar_try(full0 + k_at * 8, k_parity));
      if (!__all_sync(0xffffffffu, there)) {
        if (!last && !wait(full0 + k_at * 8, k_parity)) break;
        if (!wait(full0 + at * 8, parity)) break;
      }
      if (last && clean_first && !wait(smem_u32(&v_clean), 0)) break;
      const uint32_t vb = ring_v + at * (Sh::SLOT >> 4);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        if (j >= n_own[i]) continue;
        // P comes in halves of 64 keys.
        if (!wait(p0 + i * 16, j)) break;
        tc_fence_after();
        values(i, 0, vb, j == 0, steps);
        if (!wait(p0 + i * 16 + 8, j)) break;
        tc_fence_after();
        values(i, 1, vb, j == 0, steps - 4);
        if (j + 1 == n_own[i]) commit_if(smem_u32(&o_full[i]), issue);
        else scores(i, k_at, id_next);
      }
      if (ok) {
        commit_if(empty0 + at * 8, issue);
        if (!last) commit_if(empty0 + k_at * 8, issue);
      }
    }
    if (!ok && lane == 0) give_up(712);
    // Every MMA issued so far has completed once this barrier fires: a commit
    // covers what its own thread issued, so the issuing lane makes it.
    commit_if(smem_u32(&drain), issue);
    if (issue) drain_wait(smem_u32(&drain), 0);
    __syncwarp();
  } else {
    const int tile = (warp - 2) >> 2, quad = warp & 3;
    const int r = quad * 32 + lane;
    const uint32_t t_s = tmem + (static_cast<uint32_t>(quad * 32) << 16) + tile * 256, t_o = t_s + 128;
    const int own_blocks = NT == 1 ? nb[0] : (tile == 0 ? nb[0] : nb[NT - 1]);
    const int query = w.row0 + tile * per_tile + r / G, head = kvh * G + r % G;
    const bool live = r < per_tile * G && query < n_q;
    const int see = min(live ? visible_keys(a, w, query) : w.nk, w.key_hi) - w.key_lo;
    const float sc = a.scale_log2;
    float m = -INFINITY, ref = 0.f, calm = -1.f;
    float2 l2[2] = {{0.f, 0.f}, {0.f, 0.f}};
    bool ok = true;
    for (int j = 0; j < own_blocks; ++j) {
      if (!warp_wait_here(smem_u32(&s_full[tile]), j & 1, &abort_flag, a.wait_ns)) {
        ok = false;
        break;
      }
      tc_fence_after();
      uint32_t sv[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_async(t_s + c * 32, sv + c * 32);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_wait32(sv + c * 32);
      const int limit = see - j * kBlockKeys;  // keys of the block that this row sees
      if (!__all_sync(0xffffffffu, limit >= kBlockKeys)) {
#pragma unroll
        for (int q = 0; q < 128; ++q)
          if (q >= limit) sv[q] = 0xff800000u;  // -infinity
      }
      float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int q = 0; q < 128; q += 8)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          top[u] = max3(top[u], __uint_as_float(sv[q + 2 * u]), __uint_as_float(sv[q + 2 * u + 1]));
      // Rows of no query hold other sequences' queries or what shared memory held: they have no say in the votes.
      const float cand = live ? fmaxf(m, max3(fmaxf(top[0], top[1]), top[2], top[3])) : 0.f;
      // P = 2^((s - m) sc).  Fused as s sc - fl(m sc), the rounding of m sc stays in every exponent and changes with m:
      // 2^-17 at most while |m sc| is below kFusedMost, but whole powers of two (P infinite, or 0 in every column) for
      // scores of 2^31.  Where a row of the warp is beyond the limit the difference is formed first, so that s = m
      // gives 1, and `calm` sends every later block this way.  One vote stands for that, a risen maximum and the first
      // block (the comparison is also taken where both maxima are infinite).
      if (__any_sync(0xffffffffu, !((cand - m) * sc <= calm))) {
        if (j == 0) {
          m = cand;
        } else if (__any_sync(0xffffffffu, (cand - m) * sc > 8.f)) {
          const float alpha = m == cand ? 1.f : ex2f_approx((m - cand) * sc);
#pragma unroll
          for (int c = 0; c < DK; ++c) {
            uint32_t v[16];
            tmem_ld16(t_o + c * 16, v);
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) * alpha);
            tmem_st16(t_o + c * 16, v);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) l2[u] = mul2(l2[u], make_float2(alpha, alpha));
          m = cand;
        }
        const float base = m == -INFINITY ? 0.f : m;
        ref = base * sc;
        const bool apart = __any_sync(0xffffffffu, fabsf(ref) > kFusedMost);
        calm = apart ? -1.f : 8.f;
        if (apart) {
          ref = 0.f;
#pragma unroll
          for (int q = 0; q < 128; q += 2) {
            const float2 d = add2(make_float2(__uint_as_float(sv[q]), __uint_as_float(sv[q + 1])), make_float2(-base, -base));
            sv[q] = __float_as_uint(d.x);
            sv[q + 1] = __float_as_uint(d.y);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t pk[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const int at = c * 32 + 2 * q;
          float2 p = fma2(make_float2(__uint_as_float(sv[at]), __uint_as_float(sv[at + 1])), make_float2(sc, sc), make_float2(-ref, -ref));
          p.x = ex2f_approx(p.x);
          p.y = ex2f_approx(p.y);
          l2[q & 1] = add2(l2[q & 1], p);
          pk[q] = pack2(p.x, p.y);
        }
        tmem_st16_async(t_s + c * 16, pk);
        if (c & 1) {
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(smem_u32(&p_full[tile][c >> 1]));
        }
      }
    }
    if (ok && own_blocks > 0) ok = warp_wait_here(smem_u32(&o_full[tile]), 0, &abort_flag, a.wait_ns);
    if (ok) {
      tc_fence_after();
      const float l = (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const float lse2 = l == 0.f ? -INFINITY : m * sc + log2f(l);
      const bool cut = a.ks.unit && w.nk > a.ks.unit;
      const int64_t part = (static_cast<int64_t>(w.piece) * a.max_q + query) * a.q.heads + head;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out.data) + static_cast<int64_t>(w.q0 + query) * a.out.token_stride + head * a.out.head_stride;
      float* part_o = a.part_o + part * a.dim;
      if (live) {
        if (cut) a.part_ml[part] = make_float2(m, l);
        else if (a.lse) a.lse[static_cast<int64_t>(w.q0 + query) * a.q.heads + head] = lse2 * kLn2;
      }
      uint32_t v[DK][16] = {};
      if (own_blocks > 0) {  // every lane: the loads are warp-collective
#pragma unroll
        for (int c = 0; c < DK; ++c) tmem_ld16_async(t_o + c * 16, v[c]);
#pragma unroll
        for (int c = 0; c < DK; ++c) tmem_wait16(v[c]);
      }
      if (cut) {
#pragma unroll
        for (int at = 0; at < Sh::DP; at += 8) {
          if (!live || at >= a.dim) continue;
          float f[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(v[at / 16][at % 16 + q]) * inv;
          store_vec(part_o + at, f);
          store_vec(part_o + at + 4, f + 4);
        }
      } else {
        // Through the tile's query slot, which the MMAs have done with: a warp's 32
        // rows then leave as whole rows, 32 pieces of 16 bytes side by side, not as one piece of each.
        uint8_t* stage = smem + tile * Sh::SLOT;
        const auto place = [&](int row, int piece) {
          return stage + row * Sh::OUT_PITCH + (Sh::OUT_SWIZZLED ? piece ^ (row & 7) : piece) * 16;
        };
#pragma unroll
        for (int at = 0; at < Sh::DP; at += 8) {
          if (at >= a.dim) continue;
          float f[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(v[at / 16][at % 16 + q]) * inv;
          store_vec(reinterpret_cast<__nv_bfloat16*>(place(r, at / 8)), f);
        }
        __syncwarp();
        const uint32_t rows = __ballot_sync(0xffffffffu, live);
        const int pieces = a.dim / 8, skip_rows = 32 / pieces, skip = 32 - skip_rows * pieces;
        int row = lane / pieces, piece = lane - row * pieces;
        const uint64_t own = reinterpret_cast<uint64_t>(out);
        for (int n = 0; n < pieces; ++n) {
          __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, own, row));
          if (rows >> row & 1) *reinterpret_cast<uint4*>(to + piece * 8) = *reinterpret_cast<const uint4*>(place(quad * 32 + row, piece));
          row += skip_rows;
          piece += skip;
          if (piece >= pieces) {
            piece -= pieces;
            ++row;
          }
        }
      }
    } else if (lane == 0) {
      give_up(713);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && abort_flag) {
    // Copies issued but never used still land in shared memory.
    for (int i = 0; i < NT; ++i)
      if (nb[i] > 0) drain_wait(smem_u32(&q_full[i]), 0);
    for (int s = 0; s < ST && s < issued; ++s) {
      const int last = issued - 1 - (issued - 1 - s) % ST;  // the newest copy into slot s
      drain_wait(smem_u32(&full[s]), (last / ST) & 1);
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Sh::COLUMNS) : "memory");
  }
}

// A map of heads: {channel, head, token}, boxes of 64 channels x `heads` x `tokens`, channels past dim zero-filled.
bool encode_heads(CUtensorMap* m, const Heads& h, int64_t tokens, int dim, int heads, int box_tokens) {
  EncodeTiledFn enc = get_encoder();
  if (!enc) return false;
  const auto stride = [&](int64_t s, int64_t n) { return static_cast<cuuint64_t>(n > 1 ? s * 2 : (dim * 2 + 15) / 16 * 16); };
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(h.heads), static_cast<cuuint64_t>(tokens)};
  cuuint64_t strides[2] = {stride(h.head_stride, h.heads), stride(h.token_stride, tokens)};
  cuuint32_t box[3] = {64, static_cast<cuuint32_t>(heads), static_cast<cuuint32_t>(box_tokens)};
  cuuint32_t estr[3] = {1, 1, 1};
  g_maps_encoded.fetch_add(1, std::memory_order_relaxed);
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, h.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK, int NT>
cudaError_t run(const PackedAttnArgs& a, cudaStream_t s) {
  using Sh = TcShape<DK, NT>;
  static_assert(Sh::STAGES >= 2, "keys of a block beside the values of the one before");
  CUtensorMap qm, km, vm;
  // Without keys nothing is loaded; the maps still want a tensor.
  const Heads& k = a.ks.total > 0 ? a.k : a.q;
  const Heads& v = a.ks.total > 0 ? a.v : a.q;
  const int64_t keys = a.ks.total > 0 ? a.ks.total : a.qs.total;
  if (!encode_heads(&qm, a.q, a.qs.total, a.dim, a.group, a.qs.unit / NT) || !encode_heads(&km, k, keys, a.dim, 1, kBlockKeys) ||
      !encode_heads(&vm, v, keys, a.dim, 1, kBlockKeys))
    return cudaErrorInvalidValue;
  const auto kernel = attn_packed_tc_kernel<DK, NT>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(Sh::SMEM));
  if (e != cudaSuccess) return e;
  const int64_t blocks = (a.ks.unit ? a.k_pieces * a.tiles : a.q_pieces) * a.k.heads;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(Sh::THREADS), Sh::SMEM, s, qm, km, vm, a);
}

}  // namespace

cudaError_t launch_attn_packed_tc(const PackedAttnArgs& a, int tiles, cudaStream_t s) {
  const int dk = (a.dim + 15) / 16;
  if (tiles == 2) {
    if (dk <= 4) return run<4, 2>(a, s);
    if (dk == 5) return run<5, 2>(a, s);
    if (dk == 6) return run<6, 2>(a, s);
    return run<8, 2>(a, s);
  }
  if (dk <= 4) return run<4, 1>(a, s);
  if (dk == 5) return run<5, 1>(a, s);
  if (dk == 6) return run<6, 1>(a, s);
  return run<8, 1>(a, s);
}

}  // namespace moeca
