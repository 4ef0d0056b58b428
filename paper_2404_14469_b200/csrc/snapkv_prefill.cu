// The prompt's own attention (the phase in front of the compression step): causal, grouped heads,
// sequences of different lengths.  Per query i of a sequence with Lq queries and Lk keys:
//   out_i = sum_j p_ij v_j / l_i,  p_ij = exp(s_ij - m_i),  s_ij = q_i.k_j / sqrt(d),  j <= Lk - Lq + i
// with m_i a reference near the running maximum and l_i the running sum; lse_i = m_i + ln l_i.
//
// One work unit: two tiles of 128 query rows that share their keys (one in the SPLIT form, see there).  Of a group's query heads the
// largest power of two that divides the group is packed into a tile, (token, head) with the head
// fastest: 32 tokens of 4 heads instead of 128 of one, so that a unit's two tiles need the same keys
// but for a few.  Both products run on tcgen05 over 128 keys at a time:
//   S = Q.K^T into TMEM; a warpgroup per tile reads it back, a query row per thread (no shuffles), and
//   writes P = exp2(S c - m) in bf16 over it; O += P.V with P as the operand in TMEM and O in TMEM to
//   the end.
// What bounds the kernel is a tile's chain: S, its weights, P.V, and no S before that as P lies over it.
// So the weights do not wait for a maximum, and none is taken: the reference m of a row is its maximum
// over the first 32 keys, with some room (PF_ROOM), and moves only when later weights pass it, which
// shows in their sum: to the maximum of those keys, wherever the old one was.  The
// row's thread then rescales what it has under the old reference, in TMEM too.  And P is handed over
// in two halves, so that the product with V runs while the second one is computed.
// Warps: 0-3 softmax of tile 0, 4-7 of tile 1, 8 TMA, 9 MMA.  The grid has a block per unit, longest
// sequences and their last queries first, and a running block takes over the next one that has not
// started (so the next unit's keys are on the way while the present one is written out, and blocks end
// together: with a fixed assignment eight prompts of 200 to 4000 tokens took 253 us, then 240).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "../../include/snapkv.h"
#include "launch.cuh"
#include "sm100_ptx.cuh"
#include "snapkv_internal.h"

namespace snapkv {
namespace {

constexpr int PF_MAX_SEQS = 32;   // sequences that share a launch
constexpr int PF_THREADS = 320;
constexpr int PF_UNITS = 4;       // units that the TMA thread may be ahead
constexpr int PF_KEYS = 128;      // keys per tile
// When a wait has given up, the block's other roles wait for the TMA thread to tell which units are left: it
// waits first for its queries, up to eight tiles, an answer and two units' places.  In wait limits.
constexpr int PF_PATIENCE = 16;
// A row's reference is 2^10 (PF_ROOM) above the keys that it was taken from, and the row takes a new one
// when 64 of its weights add up to more than 64 (PF_FAR).  So the sums are at most what a running maximum
// gives, (Lk + 64) and (Lk + 64) max|v|, and logits may rise by 2^10 to 2^16 without a new reference.  (The
// room costs nothing but the smallest 2^-10 of the number range.  With sums that may pass what the reference
// was taken from by 2^16, 2^10 and 2^7, mixed prompts of 64-wide heads took 156, 158 and 212 us, a 32K
// prompt 7.61, 7.63 and 8.43 ms.)
constexpr float PF_FAR = 64.f, PF_ROOM = 10.f;
constexpr float PF_WIDE = 16777216.f;  // 2^24
constexpr float PF_NONE = -3e38f;      // the reference of a row that has none yet: any finite score is far above it
constexpr int PF_BLOCK = 128 * 128;  // bytes of 128 rows of 64 elements, 128-byte swizzled

struct PrefillSeq {
  int lq, lk;
  int unit0;      // the sequence's first unit
  int batch;      // index in the caller's batch
  long long q0;   // first token
};
template <int MAPS>
struct PrefillSeqs {
  CUtensorMap k[MAPS], v[MAPS];  // a sequence's own rows: what lies behind them reads as zeros
  PrefillSeq s[MAPS];
};
struct PrefillArgs {
  int Hq, g, W, nseq, units;
  int pack_log2;       // query heads per tile
  int head_packs;      // Hq >> pack_log2
  float c2;            // log2(e) / sqrt(d)
  unsigned long long wait_ns;
  int lost;            // self-test: the unit whose first key tile never comes, else -1
  __nv_bfloat16* out;
  float *lse, *lse_obs;
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// Where `on`, which lanes may differ in: predicated instructions instead of branches, so that the warp stays
// whole for the .sync.aligned ones around them.
__device__ __forceinline__ void st_global_32_if(bool on, void* p, const uint32_t (&w)[8]) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %9, 0;\n\t"
      "@p st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n\t}" ::"l"(p),
      "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(static_cast<int>(on))
      : "memory");
}
__device__ __forceinline__ void mbar_arrive_if(bool on, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(static_cast<int>(on))
      : "memory");
}

// Wait for a copy or an MMA that is in flight, when the abort flag is set already.
__device__ __forceinline__ bool drain(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
  const unsigned long long t0 = globaltimer_ns();
  while (!mbar_try_wait(bar, parity))
    if (globaltimer_ns() - t0 > limit_ns) return false;
  return true;
}

// What a block knows of a unit.  The TMA thread works it out, ahead of the others, and leaves it in
// shared memory (each role for itself took 2000 clocks between two units).
struct __align__(16) Unit {
  int seq, lq, batch;
  int n0;         // keys in front of the first query (may be negative)
  int head0;      // first query head
  int token0;     // first token of tile 0
  int nk[2];      // key tiles of each query tile
  long long q0;
  int most;       // of nk; -1: there is no further unit
};

template <int D>
struct PfSmem {
  static constexpr int COLS = D / 64;
  static constexpr int TILE = COLS * PF_BLOCK;          // one tile of Q, K or V
  static constexpr int STAGES = D == 128 ? 5 : 8;       // ring of K and V tiles
  static constexpr int OFF_Q = 0, OFF_KV = 2 * TILE, OFF_BAR = OFF_KV + STAGES * TILE;
  // full[STAGES], empty[STAGES], q_full, q_empty, then per tile: S, the halves of P, the product with
  // the first of them, the whole product, O read out; drain; the answer about the next block; units
  // there and read
  static constexpr int NBAR = 2 * STAGES + 2 + 12 + 2 + 2 * PF_UNITS;
  static constexpr int OFF_MISC = OFF_BAR + ((NBAR * 8 + 15) & ~15);  // tensor memory, abort flag, wait limit
  static constexpr int OFF_UNIT = OFF_MISC + 16, OFF_ANSWER = OFF_UNIT + PF_UNITS * sizeof(Unit);
  static constexpr int OFF_CLOSED = OFF_ANSWER + 16;
  static constexpr int DYN_BYTES = OFF_CLOSED + 16 + 1024;
  static_assert(DYN_BYTES <= 227 * 1024, "shared memory of one block");
};

// SPLIT: for a few units.  A unit is one query tile, whose key tiles the two softmax warpgroups take in
// turn, each with a reference, a sum and an O of its own; in the end the second hands its results to the
// first through the ring's memory.  A block has one unit then.
template <int D, int MAPS, bool SPLIT>
__global__ void __launch_bounds__(PF_THREADS, 1)
prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const PrefillArgs a, const __grid_constant__ PrefillSeqs<MAPS> seqs) {
  using SM = PfSmem<D>;
  constexpr int COLS = SM::COLS, STAGES = SM::STAGES, TILE = SM::TILE;
  constexpr int TMEM_O = 256;   // S (and P over it) of tile t at 128 t, O at TMEM_O + D t
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  const uint32_t sbase = smem_u32(smem);
  const uint32_t q_s = sbase + SM::OFF_Q, kv_s = sbase + SM::OFF_KV, bar0 = sbase + SM::OFF_BAR;
  auto bar_full = [&](int s) { return bar0 + 8u * s; };
  auto bar_empty = [&](int s) { return bar0 + 8u * (STAGES + s); };
  const uint32_t bar_qf = bar0 + 8u * (2 * STAGES), bar_qe = bar_qf + 8u;
  auto bar_s = [&](int t) { return bar_qe + 8u * (1 + t); };
  auto bar_p = [&](int t, int h) { return bar_qe + 8u * (3 + 2 * t + h); };
  auto bar_ph = [&](int t) { return bar_qe + 8u * (7 + t); };
  auto bar_pv = [&](int t) { return bar_qe + 8u * (9 + t); };
  auto bar_of = [&](int t) { return bar_qe + 8u * (11 + t); };
  const uint32_t bar_drain = bar_qe + 8u * 13;
  const uint32_t bar_answer = bar_drain + 8u, answer = sbase + SM::OFF_ANSWER;
  auto bar_there = [&](int i) { return bar_answer + 8u * (1 + i); };
  auto bar_read = [&](int i) { return bar_answer + 8u * (1 + PF_UNITS + i); };
  Unit* units_s = reinterpret_cast<Unit*>(smem + SM::OFF_UNIT);
  volatile int* closed_s = reinterpret_cast<volatile int*>(smem + SM::OFF_CLOSED);  // -1, in the end the number of units
  volatile uint32_t* tmem_ptr_s = reinterpret_cast<volatile uint32_t*>(smem + SM::OFF_MISC);
  volatile int* abort_s = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmQ);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    mbar_init(bar_qf, 1);
    mbar_init(bar_qe, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar_s(t), 1);
      mbar_init(bar_p(t, 0), 4);
      mbar_init(bar_p(t, 1), 4);
      mbar_init(bar_ph(t), 1);
      mbar_init(bar_pv(t), 1);
      mbar_init(bar_of(t), 4);
    }
    mbar_init(bar_drain, 1);
    mbar_init(bar_answer, 1);
    for (int i = 0; i < PF_UNITS; ++i) {
      mbar_init(bar_there(i), 1);
      mbar_init(bar_read(i), 9);  // MMA and eight softmax warps
    }
    *closed_s = -1;
    *abort_s = 0;
    *reinterpret_cast<volatile unsigned long long*>(abort_s + 1) = a.wait_ns;
    mbar_fence_init();
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_s)), 512);
    tmem_relinquish();
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_ptr_s;

  const int tok_log2 = 7 - a.pack_log2, tile_tokens = 1 << tok_log2;
  auto unit_of = [&](int i, Unit* u) {
    int s = 0;
    while (s + 1 < a.nseq && i >= seqs.s[s + 1].unit0) ++s;
    const PrefillSeq& q = seqs.s[s];
    const int unit_log2 = tok_log2 + (SPLIT ? 0 : 1), blocks = (q.lq + (1 << unit_log2) - 1) >> unit_log2;
    const int at = i - q.unit0, from_end = at / a.head_packs;
    u->seq = s;
    u->lq = q.lq;
    u->batch = q.batch;
    u->q0 = q.q0;
    u->n0 = q.lk - q.lq;
    u->head0 = (at - from_end * a.head_packs) << a.pack_log2;
    u->token0 = (blocks - 1 - from_end) << unit_log2;
    for (int t = 0; t < 2; ++t) {
      const int first = u->token0 + (SPLIT ? 0 : t * tile_tokens), last = min(first + tile_tokens, q.lq) - 1;
      u->nk[t] = last < first ? 0 : (max(u->n0 + last + 1, 0) + PF_KEYS - 1) / PF_KEYS;
      if (SPLIT) u->nk[t] = (u->nk[t] + 1 - t) / 2;  // every other one
    }
    u->most = max(u->nk[0], u->nk[1]);
  };
  Unit u;

  if (warp == 8) {
    // ------------------------------------------------------------ TMA
    if (elect_one()) {
      int fill = 0, nq = 0;
      bool ok = true;
      // A unit for the others to see; its place is free once the unit PF_UNITS in front has been read.
      int shown = 0, asked = 0, pending = -1;  // units shown, blocks asked for, a unit taken but not shown
      bool ended = false;
      auto show = [&] {
        units_s[shown % PF_UNITS] = u;
        mbar_arrive(bar_there(shown % PF_UNITS));
        ++shown;
      };
      for (int i = static_cast<int>(blockIdx.x); i >= 0;) {
        if (SPLIT && shown) {
          i = -1;
        } else if (asked) {
          ok = mbar_wait_thread(bar_answer, (asked - 1) & 1, abort_s, 11);
          if (!ok) break;
          i = next_block_answer(answer);
        }
        ended = i < 0;
        pending = i;
        if (ended) {
          u.most = -1;
        } else if (SPLIT) {
          unit_of(i, &u);
        } else {
          fence_proxy_async();  // the last answer has been read
          mbar_expect_tx(bar_answer, 16);
          next_block_ask(answer, bar_answer);
          ++asked;
          unit_of(i, &u);
        }
        ok = mbar_wait_thread(bar_read(shown % PF_UNITS), (shown / PF_UNITS & 1) ^ 1, abort_s, 12);
        if (!ok) break;
        show();
        pending = -1;
        if (ended) break;
        if (u.most == 0) continue;
        const int kv = u.head0 / a.g;
        bool lost = i == a.lost;
        auto load = [&](const CUtensorMap* m, int j) {
          const int s = fill % STAGES;
          if (!mbar_wait_thread(bar_empty(s), (fill / STAGES & 1) ^ 1, abort_s, 1)) return false;
          if (!lost) {
            mbar_expect_tx(bar_full(s), TILE);
            for (int c = 0; c < COLS; ++c)
              tma_load_3d(kv_s + s * TILE + c * PF_BLOCK, m, bar_full(s), c * 64, j * PF_KEYS, kv);
          }
          lost = false;
          ++fill;
          return true;
        };
        ok = mbar_wait_thread(bar_qe, (nq & 1) ^ 1, abort_s, 2);
        if (!ok) break;
        constexpr int QT = SPLIT ? 1 : 2;
        mbar_expect_tx(bar_qf, QT * TILE);
        for (int t = 0; t < QT; ++t)
          for (int c = 0; c < COLS; ++c)
            tma_load_3d(q_s + t * TILE + c * PF_BLOCK, &tmQ, bar_qf, c * 64, u.head0,
                        static_cast<int>(u.q0) + u.token0 + t * tile_tokens);
        ++nq;
        for (int j = 0; ok && j < u.most; ++j) {
          if constexpr (SPLIT) {
            const bool two = j < u.nk[1];
            ok = load(&seqs.k[u.seq], 2 * j) && (!two || load(&seqs.k[u.seq], 2 * j + 1)) && load(&seqs.v[u.seq], 2 * j) &&
                 (!two || load(&seqs.v[u.seq], 2 * j + 1));
          } else {
            ok = load(&seqs.k[u.seq], j) && load(&seqs.v[u.seq], j);
          }
        }
        if (!ok) break;
      }
      if (*abort_s != 0) {  // never leave with copies in flight
        if (nq) drain(bar_qf, (nq - 1) & 1, a.wait_ns);
        for (int i = fill > STAGES ? fill - STAGES : 0; i < fill; ++i) drain(bar_full(i % STAGES), i / STAGES & 1, a.wait_ns);
        // blocks that this one has taken over, or asked for and got, are filled with NaN, too
        if (!ended && asked && drain(bar_answer, (asked - 1) & 1, a.wait_ns)) {
          const int last = next_block_answer(answer);
          for (int e = 0; e < 2; ++e) {
            const int i = e == 0 ? pending : last;
            if (i < 0) continue;
            unit_of(i, &u);
            drain(bar_read(shown % PF_UNITS), (shown / PF_UNITS & 1) ^ 1, a.wait_ns);
            show();
          }
        }
      }
      *closed_s = shown;
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------ MMA
    if (elect_one()) {
      constexpr uint32_t idesc_s = umma_idesc_bf16(128, 128), idesc_o = umma_idesc_bf16(128, D) | UMMA_B_MN_MAJOR;
      int use = 0, nq = 0, npv[2] = {0, 0}, no[2] = {0, 0};
      bool ok = true;
      auto full = [&](int i) { return mbar_wait_thread(bar_full(i % STAGES), i / STAGES & 1, abort_s, 3); };
      auto scores = [&](int t, int i) {  // S of tile t with the keys of ring entry i
        // P of the tile before lies over it: that product must be through
        if (npv[t] > 0 && !mbar_wait_thread(bar_pv(t), (npv[t] - 1) & 1, abort_s, 4)) return false;
        const uint64_t qd = umma_desc_k128(q_s + (SPLIT ? 0 : t * TILE)), kd = umma_desc_k128(kv_s + (i % STAGES) * TILE);
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t at = static_cast<uint64_t>((k >> 2) * (PF_BLOCK >> 4) + (k & 3) * 2);
          tc_mma_bf16(tmem + 128 * t, qd + at, kd + at, idesc_s, k != 0);
        }
        tc_commit(bar_s(t));
        return true;
      };
      auto values = [&](int t, int i, bool first) {
        // (a unit's first product overwrites O: the unit before must have been read out)
        if (first && !mbar_wait_thread(bar_of(t), (no[t]++ & 1) ^ 1, abort_s, 6)) return false;
        const uint64_t vd = umma_desc_mn128(kv_s + (i % STAGES) * TILE, PF_BLOCK);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!mbar_wait_thread(bar_p(t, h), npv[t] & 1, abort_s, 5)) return false;
          tc_fence_after();
#pragma unroll
          for (int k = 4 * h; k < 4 * h + 4; ++k)
            tc_mma_bf16_ts(tmem + TMEM_O + D * t, tmem + 128 * t + 8 * k, vd + static_cast<uint64_t>(k * (2048 >> 4)), idesc_o,
                           !first || k != 0);
          tc_commit(h ? bar_pv(t) : bar_ph(t));
        }
        ++npv[t];
        return true;
      };
      int r = 0;  // units read
      while (ok) {
        ok = mbar_wait_thread(bar_there(r % PF_UNITS), r / PF_UNITS & 1, abort_s, 11);
        if (!ok) break;
        u = units_s[r % PF_UNITS];
        mbar_arrive(bar_read(r++ % PF_UNITS));
        if (u.most < 0) break;
        if (u.most == 0) continue;
        ok = mbar_wait_thread(bar_qf, nq++ & 1, abort_s, 7);
        if constexpr (SPLIT) {
          // ring entries of step j: its one or two key tiles, then as many value tiles
          auto key = [&](int t, int j) { return use + 4 * j + t; };
          auto value = [&](int t, int j) { return use + 4 * j + (j < u.nk[1] ? 2 : 1) + t; };
          auto score = [&](int t, int j) {
            if (!full(key(t, j)) || !scores(t, key(t, j))) return false;
            tc_commit(bar_empty(key(t, j) % STAGES));
            return true;
          };
          for (int j = -1; ok && j < u.most; ++j)
            for (int t = 0; ok && t < 2; ++t) {
              if (j >= 0 && j < u.nk[t]) {
                ok = full(value(t, j)) && values(t, value(t, j), j == 0);
                if (ok) tc_commit(bar_empty(value(t, j) % STAGES));
              }
              if (ok && j + 1 < u.nk[t]) ok = score(t, j + 1);
            }
          use += 2 * (u.nk[0] + u.nk[1]);
          continue;
        }
        ok = ok && full(use);
        for (int t = 0; ok && t < 2; ++t)
          if (u.nk[t] > 0) ok = scores(t, use);
        if (!ok) break;
        tc_commit(bar_empty(use % STAGES));
        if (u.most == 1) tc_commit(bar_qe);
        for (int j = 0; ok && j < u.most; ++j, use += 2) {
          const bool more = j + 1 < u.most;
          for (int t = 0; ok && t < 2; ++t) {
            if (t == 0) ok = full(use + 1);
            if (ok && j < u.nk[t]) ok = values(t, use + 1, j == 0);
            if (ok && t == 0 && more) ok = full(use + 2);
            if (ok && j + 1 < u.nk[t]) ok = scores(t, use + 2);
          }
          if (!ok) break;
          tc_commit(bar_empty((use + 1) % STAGES));
          if (more) tc_commit(bar_empty((use + 2) % STAGES));
          if (j + 2 == u.most) tc_commit(bar_qe);  // the unit's last use of its queries
        }
      }
      if (*abort_s != 0) {
        tc_commit(bar_drain);
        drain(bar_drain, 0, a.wait_ns);
        // units that the softmax warps have still to fill: their places become free without this role
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < PF_PATIENCE * a.wait_ns) {
          if (mbar_try_wait(bar_there(r % PF_UNITS), r / PF_UNITS & 1)) mbar_arrive(bar_read(r++ % PF_UNITS));
          else if (*closed_s >= 0 && r >= *closed_s) break;
        }
      }
    }
  } else {
    // ------------------------------------------------------------ softmax
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + lanes + 128 * t, o_at = tmem + lanes + TMEM_O + D * t;
    const unsigned long long scale2 = pack2(a.c2, a.c2);
    int ns = 0;  // key tiles so far
    bool ok = true;
    for (int r = 0;; ++r) {
      const int at_unit = r % PF_UNITS;
      ok = ok && mbar_wait_warp(bar_there(at_unit), r / PF_UNITS & 1, abort_s, 11);
      if (!ok) {  // a wait gave up: what units there still are become NaN, once it is known how many
        const unsigned long long t0 = globaltimer_ns();
        bool there = false;
        while (!(there = __all_sync(0xffffffffu, mbar_try_wait(bar_there(at_unit), r / PF_UNITS & 1)))) {
          const int closed = *closed_s;
          if (__any_sync(0xffffffffu, (closed >= 0 && r >= closed) || globaltimer_ns() - t0 > PF_PATIENCE * a.wait_ns)) break;
        }
        if (!there) break;
      }
      u = units_s[at_unit];
      __syncwarp();
      mbar_arrive_if(lane == 0, bar_read(at_unit));
      if (u.most < 0) break;
      const int token = u.token0 + (SPLIT ? 0 : t * tile_tokens) + (row >> a.pack_log2);
      const int head = u.head0 + (row & ((1 << a.pack_log2) - 1));
      const int nk = u.nk[t];
      const int jmax = u.n0 + min(token, u.lq - 1);             // the last key that the row sees
      int jfree = u.n0 + u.token0 + (SPLIT ? 0 : t * tile_tokens);  // every row of the tile sees keys up to here
      // The row's reference in the log2 domain is m + far * c2, l the sum of exp2(. - reference).  m is a
      // whole number, so that a weight's exponent is rounded once (fma) and references differ by powers of
      // two.  From PF_WIDE on m would be coarser than one: there the score itself is the reference (far),
      // subtracted from the others before they are scaled, and m is the room.
      float m = PF_NONE, far = 0.f, l = 0.f;
      auto refer = [&](bool set, float top) {
        const float x = ceilf(top * a.c2);
        const bool is_far = fabsf(x) >= PF_WIDE;
        m = set ? (is_far ? PF_ROOM : x + PF_ROOM) : m;
        far = set ? (is_far ? top : 0.f) : far;
        if (__any_sync(0xffffffffu, far != 0.f)) jfree = INT_MIN;  // (the far rows' subtraction is with the masks)
      };
      for (int j = 0; ok && j < nk; ++j, ++ns) {
        ok = mbar_wait_warp(bar_s(t), ns & 1, abort_s, 8);
        if (!ok) break;
        tc_fence_after();
        const int key0 = (SPLIT ? 2 * j + t : j) * PF_KEYS;
        auto mask = [&](float (&x)[32], int c) {
          const int see = jmax - key0 - 32 * c;
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = i <= see ? x[i] : -INFINITY;
        };
        auto largest = [&](const float (&x)[32]) {
          float y = x[0];
#pragma unroll
          for (int i = 1; i < 32; ++i) y = fmaxf(y, x[i]);
          return y;
        };
        if (j == 0) {  // the reference: none yet where no key is in sight, or none that weighs anything
          float x[32];
          tmem_ld32(s_at, x);
          tmem_wait_ld();
          pin(x);
          if (key0 + PF_KEYS - 1 > jfree) mask(x, 0);
          const float top = largest(x);
          refer(top != -INFINITY, top);
        }
        // Half of the keys at a time: their scores are on the way while the first half is worked on.
        float v[2][32];
        tmem_ld32(s_at, v[0]);
        tmem_ld32(s_at + 32, v[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          tmem_wait_ld();
          pin(v[0]);
          pin(v[1]);
          if (key0 + PF_KEYS - 1 > jfree) {  // (with a branch for each a batch of 64-wide heads took 161 us, with one 158)
            mask(v[0], 2 * h);
            mask(v[1], 2 * h + 1);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[0][i] -= far, v[1][i] -= far;
          }
          uint32_t w[2][16];
          float sum[2];
          auto weights = [&](int c) {
            const unsigned long long negm = pack2(-m, -m);
            unsigned long long s2[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const unsigned long long p = ex2_approx2(fma2(pack2(v[c][i], v[c][i + 1]), scale2, negm));
              s2[i >> 1 & 1] = add2(s2[i >> 1 & 1], p);
              const float2 y = unpack2(p);
              // to bf16, half a step of 2^-8 of a probability whose fp32 value is in the sum
              const __nv_bfloat162 b = __floats2bfloat162_rn(y.x, y.y);
              w[c][i >> 1] = *reinterpret_cast<const uint32_t*>(&b);
            }
            const float2 y = unpack2(add2(s2[0], s2[1]));
            sum[c] = y.x + y.y;
          };
          weights(0);
          weights(1);
          if (__any_sync(0xffffffffu, sum[0] + sum[1] > PF_FAR)) {
            // A row passed its reference, or had none: a new one.
            const bool move = sum[0] + sum[1] > PF_FAR;
            if (__any_sync(0xffffffffu, far != 0.f)) {  // the scores themselves (this half's columns hold them until its weights are stored)
              tmem_ld32(s_at + 64 * h, v[0]);
              tmem_ld32(s_at + 64 * h + 32, v[1]);
              tmem_wait_ld();
              pin(v[0]);
              pin(v[1]);
              mask(v[0], 2 * h);
              mask(v[1], 2 * h + 1);
            }
            const float m_was = m, far_was = far;
            refer(move, fmaxf(largest(v[0]), largest(v[1])));
            const float f = move ? ex2_approx(fmaf(far_was - far, a.c2, m_was - m)) : 1.f;
            l *= f;
            if (h == 1) {  // the first half of P is handed over: its product must be through
              ok = mbar_wait_warp(bar_ph(t), ns & 1, abort_s, 9);
              tc_fence_after();
            }
            if (j > 0 || h == 1) {  // O is still: the product with this half waits for this warp
#pragma unroll 1
              for (int e = 0; e < D; e += 16) {
                uint32_t o[16];
                tmem_ld16(o_at + e, o);
                tmem_wait_ld();
                pin(o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_st16(o_at + e, o);
              }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[0][i] -= far, v[1][i] -= far;
            weights(0);
            weights(1);
          }
          l += sum[0] + sum[1];
          tmem_st16(s_at + 32 * h, w[0]);
          tmem_st16(s_at + 32 * h + 16, w[1]);
          if (h == 0) {
            tmem_ld32(s_at + 64, v[0]);
            tmem_ld32(s_at + 96, v[1]);
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          mbar_arrive_if(lane == 0, bar_p(t, h));
        }
      }
      // ---- the tile's result
      if (ok && nk > 0) ok = mbar_wait_warp(bar_pv(t), (ns - 1) & 1, abort_s, 9);
      tc_fence_after();
      // SPLIT: what the second warpgroup has, [element][row], a reference and a sum per row
      float* theirs = reinterpret_cast<float*>(smem + SM::OFF_KV) + row;
      float f_own = 1.f, f_their = 0.f;
      if constexpr (SPLIT) {
        if (t == 1) {
          if (nk == 0) continue;
          // (the ring is free when the first one's last product is through as well)
          ok = ok && mbar_wait_warp(bar_pv(0), (u.nk[0] - 1) & 1, abort_s, 9);
          if (!ok) continue;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t x[16];
            tmem_ld16(o_at + c, x);
            tmem_wait_ld();
            pin(x);
#pragma unroll
            for (int e = 0; e < 16; ++e) theirs[(c + e) * 128] = __uint_as_float(x[e]);
          }
          theirs[D * 128] = m;
          theirs[(D + 1) * 128] = far;
          theirs[(D + 2) * 128] = l;
          __syncwarp();
          mbar_arrive_if(lane == 0, bar_of(1));
          continue;
        }
        if (ok && u.nk[1] > 0) {
          ok = mbar_wait_warp(bar_of(1), 0, abort_s, 9);
          const float m1 = theirs[D * 128], far1 = theirs[(D + 1) * 128], l1 = theirs[(D + 2) * 128];
          if (ok && l1 != 0.f) {  // (a row that sees none of their keys has no reference there)
            const float above = fmaf(far - far1, a.c2, m - m1);  // of the own reference over theirs
            f_own = ex2_approx(fminf(above, 0.f));
            f_their = ex2_approx(fminf(-above, 0.f));
            l = l * f_own + l1 * f_their;
            if (above < 0.f) m = m1, far = far1;
          }
        }
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const bool mine = token < u.lq, bad = !ok || isnan(l);
      const long long at = (u.q0 + token) * a.Hq + head;
      if (mine) {
        const float e = bad ? NAN : (l > 0.f ? (fmaf(far, a.c2, m) + __log2f(l)) * 0.6931471805599453f : -INFINITY);
        if (a.lse) a.lse[at] = e;
        const int w = token - (u.lq - a.W);
        if (w >= 0) a.lse_obs[(static_cast<long long>(u.batch) * a.Hq + head) * a.W + w] = e;
      }
      __syncwarp();
      // (a row per lane: 32-byte stores write whole sectors and take half of the passes through the
      // load/store unit that 16-byte ones do)
      uint32_t o[16] = {}, ahead[16] = {};
      const bool there = ok && nk > 0;
      if (there) tmem_ld16(o_at, ahead);
#pragma unroll 1
      for (int c = 0; c < D; c += 16) {
        if (there) {
          tmem_wait_ld();
          pin(ahead);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = ahead[e];
          if (c + 16 < D) tmem_ld16(o_at + c + 16, ahead);
        }
        if constexpr (SPLIT) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = __uint_as_float(o[e]) * f_own + theirs[(c + e) * 128] * f_their;
            o[e] = f_their != 0.f ? __float_as_uint(x) : o[e];
          }
        }
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // (a row without keys has what another unit left in O)
          const float x = l > 0.f ? __uint_as_float(o[2 * e]) * inv : 0.f, y = l > 0.f ? __uint_as_float(o[2 * e + 1]) * inv : 0.f;
          const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
          w[e] = bad ? 0x7fff7fffu : *reinterpret_cast<const uint32_t*>(&h);
        }
        st_global_32_if(mine, a.out + at * D + c, w);
      }
      if (ok && nk > 0) {
        tc_fence_before();
        __syncwarp();
        mbar_arrive_if(lane == 0, bar_of(t));
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D, int MAPS, bool SPLIT>
cudaError_t launch_prefill(const CUtensorMap& tmQ, const PrefillArgs& a, const PrefillSeqs<MAPS>& seqs, cudaStream_t stream) {
  auto kernel = prefill_kernel<D, MAPS, SPLIT>;
  constexpr int SMEM = PfSmem<D>::DYN_BYTES;
  static DeviceOnce ready;
  if (!ready.done()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    ready.set();
  }
  return launch_pdl(kernel, dim3(a.units), dim3(PF_THREADS), SMEM, stream, tmQ, a, seqs);
}

bool strides_ok(const int64_t* s, int d) {
  for (int i = 0; i < 2; ++i)
    if (s[i] < d || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return true;
}

// What a call is about, apart from its sequences.
struct PrefillCall {
  const uint16_t *k, *v;
  const int64_t *ks, *vs;
  int Hkv, d;
};
struct SeqSpan {
  int lq, lk, batch;
  long long q0, k0;
};

template <int MAPS>
cudaError_t run_set(const PrefillCall& c, PrefillArgs a, const CUtensorMap& tmQ, const SeqSpan* span, int n, cudaStream_t stream) {
  using u64 = unsigned long long;
  PrefillSeqs<MAPS> seqs = {};
  // One tile per unit and its keys in two halves where that leaves every unit an SM of its own: the
  // chain is half as long (a 1K prompt of four heads of 64: 12.5 us; with two tiles per unit 17.9, with one 15.1).
  long long tiles = 0;
  for (int i = 0; i < n; ++i) tiles += (span[i].lq + (128ll >> a.pack_log2) - 1) / (128 >> a.pack_log2) * a.head_packs;
  const bool split = tiles <= sm_count();
  const int tok = (split ? 1 : 2) << (7 - a.pack_log2);
  long long units = 0;
  for (int i = 0; i < n; ++i) {
    const SeqSpan& p = span[i];
    seqs.s[i] = PrefillSeq{p.lq, p.lk, static_cast<int>(units), p.batch, p.q0};
    units += (static_cast<long long>(p.lq) + tok - 1) / tok * a.head_packs;
    const u64 dims[3] = {static_cast<u64>(c.d), static_cast<u64>(p.lk > 0 ? p.lk : 1), static_cast<u64>(c.Hkv)};
    const u64 ks[2] = {static_cast<u64>(c.ks[0]) * 2, static_cast<u64>(c.ks[1]) * 2},
              vs[2] = {static_cast<u64>(c.vs[0]) * 2, static_cast<u64>(c.vs[1]) * 2};
    const unsigned box[3] = {64, PF_KEYS, 1};
    if (!encode_tensor_map(&seqs.k[i], c.k + p.k0 * c.ks[0], 3, dims, ks, box) ||
        !encode_tensor_map(&seqs.v[i], c.v + p.k0 * c.vs[0], 3, dims, vs, box))
      return cudaErrorInvalidValue;
  }
  if (units > INT32_MAX / 2) return cudaErrorInvalidValue;
  a.nseq = n;
  a.units = static_cast<int>(units);
  if (units == 0) return cudaSuccess;
  auto f = c.d == 128 ? (split ? launch_prefill<128, MAPS, true> : launch_prefill<128, MAPS, false>)
                      : (split ? launch_prefill<64, MAPS, true> : launch_prefill<64, MAPS, false>);
  return f(tmQ, a, seqs, stream);
}

}  // namespace
}  // namespace snapkv

namespace snapkv {
namespace {

snapkv_status_t prefill_attention(const void* q, const void* k, const void* v, const int64_t* q_strides,
                                  const int64_t* k_strides, const int64_t* v_strides, const int32_t* q_lens,
                                  const int32_t* k_lens, const int64_t* q_starts, const int64_t* k_starts, int B, int Hq,
                                  int Hkv, int d, int W, void* out, float* out_lse, float* lse_obs, int lost,
                                  void* stream) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1 || W < 0 || !q_lens) return SNAPKV_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || W > 128 || Hq > 65535) return SNAPKV_ERR_UNSUPPORTED;
  if (!q || !k || !v || !out || (W > 0) != (lse_obs != nullptr)) return SNAPKV_ERR_INVALID_ARG;
  for (const void* p : {q, k, v})
    if (reinterpret_cast<uintptr_t>(p) & 15) return SNAPKV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(out) & 31) return SNAPKV_ERR_INVALID_ARG;  // (32-byte stores)
  if ((reinterpret_cast<uintptr_t>(out_lse) | reinterpret_cast<uintptr_t>(lse_obs)) & 3) return SNAPKV_ERR_INVALID_ARG;
  const int64_t dq[2] = {static_cast<int64_t>(Hq) * d, d}, dk[2] = {static_cast<int64_t>(Hkv) * d, d};
  const int64_t *qs = q_strides ? q_strides : dq, *ks = k_strides ? k_strides : dk, *vs = v_strides ? v_strides : dk;
  if (!strides_ok(qs, d) || !strides_ok(ks, d) || !strides_ok(vs, d)) return SNAPKV_ERR_INVALID_ARG;
  constexpr int64_t MAX_TOKENS = 1ll << 30;
  int64_t q_end = 0, k_end = 0, queries = 0;
  for (int b = 0; b < B; ++b) {
    const int lq = q_lens[b], lk = k_lens ? k_lens[b] : lq;
    if (lq < 0 || lk < 0 || lq < W) return SNAPKV_ERR_INVALID_ARG;
    const int64_t q0 = q_starts ? q_starts[b] : q_end, k0 = k_starts ? k_starts[b] : k_end;
    if (q0 < q_end || q0 > MAX_TOKENS || k0 < 0 || k0 > MAX_TOKENS) return SNAPKV_ERR_INVALID_ARG;
    queries += lq;
    q_end = q0 + lq;
    k_end = k0 + lk;
    if (q_end > MAX_TOKENS || k_end > MAX_TOKENS) return SNAPKV_ERR_INVALID_ARG;
  }
  PrefillArgs a = {};
  a.Hq = Hq, a.g = Hq / Hkv, a.W = W;
  while (a.pack_log2 < 6 && a.g % (2 << a.pack_log2) == 0) ++a.pack_log2;
  a.head_packs = Hq >> a.pack_log2;
  a.c2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(d)));
  a.wait_ns = wait_limit_setting();
  a.lost = lost;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = out_lse, a.lse_obs = lse_obs;
  if (queries == 0) return SNAPKV_OK;
  CUtensorMap tmQ;
  {
    using u64 = unsigned long long;
    const u64 dims[3] = {static_cast<u64>(d), static_cast<u64>(Hq), static_cast<u64>(q_end)};
    const u64 strides[2] = {static_cast<u64>(qs[1]) * 2, static_cast<u64>(qs[0]) * 2};
    const unsigned box[3] = {64, 1u << a.pack_log2, 128u >> a.pack_log2};
    if (!encode_tensor_map(&tmQ, q, 3, dims, strides, box)) return SNAPKV_ERR_CUDA;
  }
  const PrefillCall c = {static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), ks, vs, Hkv, d};
  int64_t q_at = 0, k_at = 0;
  for (int b0 = 0; b0 < B; b0 += PF_MAX_SEQS) {
    SeqSpan span[PF_MAX_SEQS];
    int n = 0;
    for (int b = b0; b < B && b < b0 + PF_MAX_SEQS; ++b) {
      SeqSpan p;
      p.lq = q_lens[b];
      p.lk = k_lens ? k_lens[b] : p.lq;
      p.batch = b;
      p.q0 = q_starts ? q_starts[b] : q_at;
      p.k0 = k_starts ? k_starts[b] : k_at;
      q_at = p.q0 + p.lq;
      k_at = p.k0 + p.lk;
      if (p.lq == 0) continue;
      int i = n++;  // the longest first
      for (; i > 0 && span[i - 1].lk < p.lk; --i) span[i] = span[i - 1];
      span[i] = p;
    }
    if (n == 0) continue;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = n == 1 ? run_set<1>(c, a, tmQ, span, n, st)
                                 : (n <= 8 ? run_set<8>(c, a, tmQ, span, n, st) : run_set<PF_MAX_SEQS>(c, a, tmQ, span, n, st));
    if (e != cudaSuccess) return SNAPKV_ERR_CUDA;
  }
  return SNAPKV_OK;
}

}  // namespace
}  // namespace snapkv

extern "C" snapkv_status_t snapkv_prefill_attention(const void* q, const void* k, const void* v,
                                                    const int64_t* q_strides, const int64_t* k_strides,
                                                    const int64_t* v_strides, const int32_t* q_lens,
                                                    const int32_t* k_lens, const int64_t* q_starts,
                                                    const int64_t* k_starts, int B, int Hq, int Hkv, int d, int W,
                                                    void* out, float* out_lse, float* lse_obs, void* stream) {
  return snapkv::prefill_attention(q, k, v, q_strides, k_strides, v_strides, q_lens, k_lens, q_starts, k_starts, B, Hq,
                                   Hkv, d, W, out, out_lse, lse_obs, -1, stream);
}

extern "C" snapkv_status_t snapkv_selftest_lost_keys(const void* q, const void* k, const void* v,
                                                     const int64_t* q_strides, const int64_t* k_strides,
                                                     const int64_t* v_strides, const int32_t* q_lens,
                                                     const int32_t* k_lens, const int64_t* q_starts,
                                                     const int64_t* k_starts, int B, int Hq, int Hkv, int d, int W,
                                                     void* out, float* out_lse, float* lse_obs, int unit, void* stream) {
  if (unit < 0) return SNAPKV_ERR_INVALID_ARG;
  return snapkv::prefill_attention(q, k, v, q_strides, k_strides, v_strides, q_lens, k_lens, q_starts, k_starts, B, Hq,
                                   Hkv, d, W, out, out_lse, lse_obs, unit, stream);
}
