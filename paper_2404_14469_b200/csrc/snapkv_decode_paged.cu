// One generation step's attention over a paged cache with a length per sequence:
// out = softmax(q . K^T / sqrt(d)) V over rows 0 .. seq_lens[b] - 1 of every sequence.
//
// Bound by HBM: the cache is read once per group of query heads.  The arithmetic is decode_kernel's
// (tiles of 16 rows of d = 128, or 32 of d = 64, through a TMA ring per warp; both products on
// warp-level matrix instructions with the cache as the 16-row operand; fp32 probabilities in three
// bf16 terms), the split another: the lengths are known on the device alone and differ, so all tiles
// of all (sequence, cache head) units are laid end to end and cut into one equal share per WARP.  A
// unit that lies inside a share is written by its warp, without any barrier: a batch of short
// sequences is many such units.  A unit that crosses shares leaves one partial (maximum, sum,
// unnormalised output) per share; the block folds those of its own warps once, at its end, and the
// block that has the unit's last share those of the blocks in front of it, in the order of the
// shares: same bits every run.  It waits (bounded) for a flag beside each partial.  The flags are the
// call's own 64-bit number, not a count, so that nothing has to be cleared in front of the call.  A replayed
// graph makes the same call again, so none may be left behind: who has read a flag clears it; who gives a
// flag up leaves the number's complement there, which tells the publisher, who comes later, to clear it.
// A block waits for blocks of lower numbers alone, which wait for nothing before they have published: they
// need not be resident together.
// What lies behind a sequence's last row may be anything: scores there are replaced and the values
// zeroed in registers, in a unit's last tile alone.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <unistd.h>

#include <atomic>
#include <chrono>

#include "../../include/snapkv.h"
#include "decode_mma.cuh"
#include "launch.cuh"
#include "sm100_ptx.cuh"
#include "snapkv_internal.h"

namespace snapkv {
namespace {

constexpr int DP_WARPS = 8, DP_STAGES = 2;
constexpr int DP_STAGE_BYTES = 8192;          // K and V of one row tile
constexpr int DP_BOX_ROWS = 16;               // rows per copy: a page holds a whole number of them
constexpr int DP_HEADS = 8;                   // query heads of a unit
constexpr int DP_THREADS = DP_WARPS * 32;
constexpr int DP_MAX_GRID = MAX_GRID;
// A block's last two threads publish, its first ones wait: up to one per block in front.
static_assert(DP_MAX_GRID <= DP_THREADS - 32, "a warp that publishes does not wait");
// What a unit costs a warp beside its tiles (queries to fetch, a result to reduce and write), in tiles:
// shares are equal in tiles and units.  (64 sequences of 20 to 300 rows: 14.9 us with 1, 14.0 with 2,
// 13.8 with 3; of 30 to 8000 rows 62.7, 61.9, 62.1.)
constexpr int DP_UNIT_COST = 2;
// References are at least this: below any score that is a number (scaled, in the log2 domain, 0.18 of fp32's range), so
// that scores of minus infinity weigh nothing and minus infinity is not subtracted from itself.
constexpr float DP_FLOOR = -1e38f;

// Self-tests: partials are published when they have been given up; no warp's first tile ever comes.
constexpr int DP_LATE = 1, DP_LOST = 2;

constexpr int dp_tile_rows(int D) { return DP_STAGE_BYTES / (4 * D); }

struct DecodePagedArgs {
  const __nv_bfloat16* q;
  const int32_t *table, *seq_lens;
  int pages_per_seq, page_size, B, Hq, g;
  int chunks;       // groups of up to DP_HEADS query heads per cache head
  int units;        // units per sequence: cache heads * chunks
  int grid;
  float c2;
  unsigned long long wait_ns;
  float *out, *lse;
  // workspace: [2 * grid] flags, then as many partials of DP_HEADS * (D + 2) floats: of the unit that
  // a block's shares begin inside, of the last one that they begin
  unsigned long long* flags;
  unsigned long long call;  // what marks a partial of this call as written; its complement: as given up
  int selftest;             // DP_LATE, DP_LOST or 0
  float* partials;
};

__device__ __forceinline__ int rows_of(const DecodePagedArgs& a, int b) {
  const long long most = static_cast<long long>(a.pages_per_seq) * a.page_size;
  const int n = __ldg(a.seq_lens + b);
  return n < 0 ? 0 : (n < most ? n : static_cast<int>(most));
}

__device__ __forceinline__ unsigned long long ld_flag(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long swap_flag(unsigned long long* p, unsigned long long v) {
  unsigned long long was;
  asm volatile("atom.acq_rel.gpu.global.exch.b64 %0, [%1], %2;" : "=l"(was) : "l"(p), "l"(v) : "memory");
  return was;
}

// (a 64-bit division takes several times as long as one of 32 bits)
__device__ __forceinline__ long long quotient64(long long n, long long d) {
  return ((n | d) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(n) / static_cast<uint32_t>(d)) : n / d;
}

// The cut: `total` pieces (a unit's DP_UNIT_COST, then its tiles) in S shares, the first `extra` of
// them one piece longer.
struct Cut {
  long long total, each, extra;
  int S;
  __device__ __forceinline__ Cut(long long total_, int most) : total(total_) {
    S = total < most ? static_cast<int>(total) : most;
    each = S > 0 ? quotient64(total, S) : 0;
    extra = total - each * S;
  }
  __device__ __forceinline__ long long begin(int s) const { return s * each + (s < extra ? s : extra); }
  __device__ __forceinline__ int owner(long long x) const {  // the share that holds piece x
    const long long longer = extra * (each + 1);
    return static_cast<int>(x < longer ? quotient64(x, each + 1) : extra + quotient64(x - longer, each));
  }
};

// A walk over the units of a share.
struct Walk {
  int b, n, tiles;       // sequence, its rows and tiles per unit
  int unit;              // of the sequence
  int t0, t1;            // the share's tiles of the unit (none where it has a part of the unit's cost alone)
  int p1;                // the share's end in pieces of the unit
  long long left;        // pieces of the share behind p1

  __device__ __forceinline__ void enter(int p0) {  // the unit from piece p0 on; `left` counts from there
    const int pieces = tiles + DP_UNIT_COST;
    p1 = left < pieces - p0 ? p0 + static_cast<int>(left) : pieces;
    left -= p1 - p0;
    t0 = p0 > DP_UNIT_COST ? p0 - DP_UNIT_COST : 0;
    t1 = p1 > DP_UNIT_COST ? p1 - DP_UNIT_COST : 0;
  }
};

// The next unit of the share; false at its end.
template <int D>
__device__ __forceinline__ bool walk_next(const DecodePagedArgs& a, Walk& w) {
  if (w.left <= 0) return false;
  if (++w.unit == a.units) {
    w.unit = 0;
    do {
      w.n = rows_of(a, ++w.b);
    } while (w.n == 0 && w.b + 1 < a.B);
    w.tiles = (w.n + dp_tile_rows(D) - 1) / dp_tile_rows(D);
  }
  w.enter(0);
  return true;
}

template <int D, int NH>
__global__ void __launch_bounds__(DP_THREADS, 1)
decode_paged_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const DecodePagedArgs a) {
  constexpr int ROWS = dp_tile_rows(D);   // cache rows per stage
  constexpr int HALVES = D / 64;          // 64-element (128-byte) column blocks of a row
  constexpr int KS = D / 16;              // k-steps of S, and pairs of 8-column tiles of the output
  constexpr int BOX = ROWS * 128;         // bytes of one column block of a tile
  constexpr int PART = DP_HEADS * (D + 2);  // floats of a partial: maxima, sums, outputs
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[DP_WARPS][DP_STAGES];
  __shared__ long long scan_s[DP_WARPS], run_s[DP_THREADS];
  // a warp's partials: of the unit that its share begins inside, of the last one that it begins
  struct Left {
    int b, unit;   // b < 0: none
    bool more;     // the unit goes on in the next share
  };
  __shared__ Left left_s[DP_WARPS][2];
  __shared__ Left ending_s;
  __shared__ int late_s, publish_s[2];
  __shared__ long long first_tile_s;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  float* parts = reinterpret_cast<float*>(smem + DP_WARPS * DP_STAGES * DP_STAGE_BYTES);  // [warp][2][PART]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int gid = lane >> 2, tig = lane & 3;   // mma fragment coordinates
  const uint32_t ring = smem_u32(smem) + warp * (DP_STAGES * DP_STAGE_BYTES);
  const uint32_t bar = smem_u32(&bars[warp][0]);
  if (lane == 0) {
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
    for (int s = 0; s < DP_STAGES; ++s) mbar_init(bar + 8u * s, 1);
    mbar_fence_init();
    fence_proxy_async();
    left_s[warp][0].b = left_s[warp][1].b = -1;
  }
  __syncwarp();
  pdl_wait();  // everything above touched this block's shared memory only

  // ---- the warps' shares.  Every thread adds up the pieces of its run of sequences.
  if (threadIdx.x == 0) {
    late_s = publish_s[0] = publish_s[1] = 0;
    ending_s.b = -1;
  }
  const int run = (a.B + DP_THREADS - 1) / DP_THREADS, b_lo = min(static_cast<int>(threadIdx.x) * run, a.B),
            b_hi = min(b_lo + run, a.B);
  auto pieces_of = [&](int b) {  // of one unit
    const int t = (rows_of(a, b) + ROWS - 1) / ROWS;
    return static_cast<long long>(t > 0 ? t + DP_UNIT_COST : 0);
  };
  long long mine = 0;
  for (int k = 0; k < run; ++k) {
    const int b = b_lo + k;
    const long long p = b < b_hi ? pieces_of(b) : 1;
    mine += b < b_hi ? p : 0;
    // sequences without rows: zeros, each by a warp of one block
    for (unsigned none = __ballot_sync(0xffffffffu, p == 0 && b % gridDim.x == blockIdx.x); none; none &= none - 1) {
      const size_t bh = static_cast<size_t>(__shfl_sync(0xffffffffu, b, __ffs(none) - 1)) * a.Hq;
      for (int e = lane; e < a.Hq * D; e += 32) a.out[bh * D + e] = 0.f;
      if (a.lse)
        for (int h = lane; h < a.Hq; h += 32) a.lse[bh + h] = -INFINITY;
    }
  }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  run_s[threadIdx.x] = upto - mine;
  if (lane == 31) scan_s[warp] = upto;
  __syncthreads();
  long long warp_before[DP_WARPS + 1];  // pieces in front of each warp's runs
  warp_before[0] = 0;
#pragma unroll
  for (int w = 0; w < DP_WARPS; ++w) warp_before[w + 1] = warp_before[w] + scan_s[w];
  const Cut cut(warp_before[DP_WARPS] * a.units, a.grid * DP_WARPS);
  const int share0 = static_cast<int>(blockIdx.x) * DP_WARPS;
  if (share0 >= cut.S) return;
  const int shares = min(DP_WARPS, cut.S - share0);  // of the block
  Walk cur = {};
  bool some = share0 + warp < cut.S;
  long long off = 0;  // of the warp's share in its first sequence, then in its first unit
  if (some) {
    // the run that holds the share's first piece: the last one that begins at or in front of it
    const long long lo = cut.begin(share0 + warp);
    int in = 0;
    long long from = 0;
#pragma unroll
    for (int w = 0; w < DP_WARPS; ++w) {
      const long long p = (warp_before[w] + run_s[w * 32 + lane]) * a.units;
      const unsigned reached = __ballot_sync(0xffffffffu, p <= lo);
      if (reached) {
        const int last = 31 - __clz(reached);
        in = w * 32 + last;
        from = __shfl_sync(0xffffffffu, p, last);
      }
    }
    cur.b = in * run;
    off = lo - from;
    for (;; ++cur.b) {  // its sequences
      cur.n = rows_of(a, cur.b);
      const long long size = pieces_of(cur.b) * a.units;
      if (off < size || cur.b + 1 >= a.B) break;
      off -= size;
    }
    cur.tiles = (cur.n + ROWS - 1) / ROWS;
    const int pieces = cur.tiles + DP_UNIT_COST;
    cur.unit = static_cast<int>(quotient64(off, pieces));
    off -= static_cast<long long>(cur.unit) * pieces;
    cur.left = cut.begin(share0 + warp + 1) - lo;
    cur.enter(static_cast<int>(off));
  }
  if (threadIdx.x == 0)  // the first tile of the unit that the block begins inside, among all pieces
    first_tile_s = cut.begin(share0) - off + DP_UNIT_COST;

  // ---- the warp's tiles.  `ahead` is at the next one to be requested; its page numbers are fetched
  // when the one before is requested.
  Walk ahead = cur;
  bool tiles_left = some;
  int at = cur.t0, page[ROWS / DP_BOX_ROWS];
  auto find_page = [&] {  // settles `ahead` on a tile (or behind the share) and fetches its page numbers
    while (tiles_left && at >= ahead.t1) {
      tiles_left = walk_next<D>(a, ahead);
      at = ahead.t0;
      // the unit's queries, on their way into L1
      const int head = ahead.unit / a.chunks, h0 = (ahead.unit - head * a.chunks) * DP_HEADS;
      const int bytes = min(DP_HEADS, a.g - h0) * D * 2;
      const char* q = reinterpret_cast<const char*>(a.q + (static_cast<size_t>(ahead.b) * a.Hq + head * a.g + h0) * D);
      for (int i = lane * 64; i < bytes; i += 32 * 64) asm volatile("prefetch.global.L1 [%0];" ::"l"(q + i));
    }
    if (tiles_left)
#pragma unroll
      for (int i = 0; i < ROWS / DP_BOX_ROWS; ++i) {
        const int r = at * ROWS + i * DP_BOX_ROWS;
        const int pg = r / a.page_size;
        page[i] = r < ahead.n ? __ldg(a.table + static_cast<long long>(ahead.b) * a.pages_per_seq + pg) : -1;
      }
  };
  int issued = 0;
  const int lost = a.selftest == DP_LOST ? 0 : -1;
  auto request = [&] {  // K and V of the tile at hand, then on to the next
    if (!tiles_left) return;
    if (lane == 0 && issued != lost) {
      const uint32_t dst = ring + (issued % DP_STAGES) * DP_STAGE_BYTES, bs = bar + 8u * (issued % DP_STAGES);
      const int head = ahead.unit / a.chunks;
      mbar_expect_tx(bs, DP_STAGE_BYTES);
#pragma unroll
      for (int i = 0; i < ROWS / DP_BOX_ROWS; ++i) {
        const int r = at * ROWS + i * DP_BOX_ROWS, row = r % a.page_size;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          tma_load_4d(dst + h * BOX + i * (DP_BOX_ROWS * 128), &tmK, bs, h * 64, row, head, page[i]);
          tma_load_4d(dst + (HALVES + h) * BOX + i * (DP_BOX_ROWS * 128), &tmV, bs, h * 64, row, head, page[i]);
        }
      }
    }
    __syncwarp();
    ++issued;
    ++at;
    find_page();
  };
  find_page();
  for (int s = 0; s < DP_STAGES; ++s) request();

  constexpr int NT = (3 * NH + 7) / 8;          // instructions with V per 16 keys and dimensions
  const int term0 = (2 * tig) / NH;             // this lane's columns carry terms term0, term0 + 8 / NH, ...
  const int lrow_k = lane & 15, lchunk_k = lane >> 4;
  const int lrow_v = (lane & 7) + ((lane >> 4) << 3), lchunk_v = (lane >> 3) & 1;
  int n = 0;
  bool failed = false;
  for (; some; some = walk_next<D>(a, cur)) {
    if (cur.t1 <= cur.t0) continue;
    const int head = cur.unit / a.chunks, h0 = (cur.unit - head * a.chunks) * DP_HEADS, gc = min(DP_HEADS, a.g - h0);
    // Q as the B operand: column gid is head h0 + gid % NH (zero beyond gc)
    uint32_t qb[KS][2];
    {
      const int h = gid % NH;
      const __nv_bfloat16* qh = a.q + (static_cast<size_t>(cur.b) * a.Hq + head * a.g + h0 + h) * D + 2 * tig;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          qb[k][i] = h < gc ? __ldg(reinterpret_cast<const uint32_t*>(qh + k * 16 + i * 8)) : 0u;
    }
    // Dimensions 16 j + gid (+ 8) of columns 2 tig, 2 tig + 1.  The matrix instructions cut what they add
    // instead of rounding it, which adds up to 2e-6 of a result over a hundred tiles: every FLUSH tiles
    // their sums go to others that are rounded (5e-7 then, at no cost that shows).
    constexpr int FLUSH = 8;
    float acc[KS][4], sums[KS][4];
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = sums[j][i] = 0.f;
    int flush = FLUSH;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // of columns 2 tig + {0, 1}; l: this lane's keys
    for (int t = cur.t0; t < cur.t1 && !failed; ++t) {
      const int s = n % DP_STAGES;
      if (!wait_copy(bar + 8u * s, (n / DP_STAGES) & 1, a.wait_ns)) {
        failed = true;
        // never leave with copies in flight
        for (int i = n + 1; i < issued; ++i) wait_copy(bar + 8u * (i % DP_STAGES), (i / DP_STAGES) & 1, a.wait_ns);
        break;
      }
      ++n;
      const uint32_t kb = ring + s * DP_STAGE_BYTES, vb = kb + HALVES * BOX;
#pragma unroll
      for (int sub = 0; sub < ROWS / 16; ++sub) {
        const int key0 = t * ROWS + sub * 16;
        const int rk = sub * 16 + lrow_k, rv = sub * 16 + lrow_v;
        float sc[2][4];  // two chains, even and odd k-steps
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[0][i] = sc[1][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t x[4];
          ldsm_x4(kb + (k >> 2) * BOX + rk * 128 + ((((k & 3) * 2 + lchunk_k) ^ (rk & 7)) << 4), x);
          mma_16816(sc[k & 1], x[0], x[1], x[2], x[3], qb[k][0], qb[k][1]);
        }
        const bool whole = key0 + 16 <= cur.n;
        float p[4];  // keys gid (0, 1) and gid + 8 (2, 3) of the lane's two columns
#pragma unroll
        for (int i = 0; i < 4; ++i)
          p[i] = whole || key0 + gid + (i >> 1) * 8 < cur.n ? (sc[0][i] + sc[1][i]) * a.c2 : -INFINITY;
        float mx[2] = {fmaxf(p[0], p[2]), fmaxf(p[1], p[3])};
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], o));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], o));
        }
        if (__any_sync(0xffffffffu, mx[0] > m[0] || mx[1] > m[1])) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float mn = fmaxf(m[c], mx[c]);
            const float corr = ex2_approx(m[c] - fmaxf(mn, DP_FLOOR));  // (nothing summed yet: 0)
            l[c] *= corr;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
              acc[j][c] *= corr;
              acc[j][c + 2] *= corr;
              sums[j][c] *= corr;
              sums[j][c + 2] *= corr;
            }
            m[c] = mn;
          }
        }
        // (no key yet, as in a subtile past the last row of a 32-row tile: p = 0, whatever the reference;
        // a NaN stays one)
        const float ref[2] = {fmaxf(m[0], DP_FLOOR), fmaxf(m[1], DP_FLOOR)};
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = ex2_approx(p[i] - ref[i & 1]);
        l[0] += p[0] + p[2];
        l[1] += p[1] + p[3];
        uint32_t lo3[3], hi3[3];  // terms of keys gid and gid + 8
        split_bf16<3>(p[0], p[1], lo3);
        split_bf16<3>(p[2], p[3], hi3);
        uint32_t bt[NT][2];      // P^T as the B operand: keys 2 tig, + 1 (and 8 further on) of column gid
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const int term = term0 + i * (8 / NH);
          bt[i][0] = transpose8(term == 0 ? lo3[0] : (term == 1 ? lo3[1] : (term == 2 ? lo3[2] : 0u)));
          bt[i][1] = transpose8(term == 0 ? hi3[0] : (term == 1 ? hi3[1] : (term == 2 ? hi3[2] : 0u)));
        }
        uint32_t keep[2] = {0xffffffffu, 0xffffffffu};  // keys 2 tig, + 1 and 8 further on: rows that exist
        if (!whole)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int key = key0 + 2 * tig + 8 * i;
            keep[i] = (key < cur.n ? 0xffffu : 0u) | (key + 1 < cur.n ? 0xffff0000u : 0u);
          }
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          uint32_t x[4];
          ldsm_x4_trans(vb + (j >> 2) * BOX + rv * 128 + ((((j & 3) * 2 + lchunk_v) ^ (rv & 7)) << 4), x);
#pragma unroll
          for (int i = 0; i < NT; ++i)
            mma_16816(acc[j], x[0] & keep[0], x[1] & keep[0], x[2] & keep[1], x[3] & keep[1], bt[i][0], bt[i][1]);
        }
      }
      __syncwarp();  // every lane has read the stage
      request();
      if (--flush == 0) {
        flush = FLUSH;
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sums[j][i] += acc[j][i];
            acc[j][i] = 0.f;
          }
      }
    }
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] += sums[j][i];
    if (failed) l[0] = l[1] = NAN;  // the outputs of this unit and of those behind it become NaN
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      l[0] += __shfl_xor_sync(0xffffffffu, l[0], o);
      l[1] += __shfl_xor_sync(0xffffffffu, l[1], o);
    }
    // the columns of one head (its terms) are NH apart: NH / 2 lanes
#pragma unroll
    for (int o = NH / 2; o < 4; o <<= 1)
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] += __shfl_xor_sync(0xffffffffu, acc[j][i], o);

    if (failed) m[0] = m[1] = 0.f;
    if (cur.t0 == 0 && cur.t1 == cur.tiles) {  // the whole unit
      if (tig < NH / 2)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int h = 2 * tig + c;
          if (h >= gc) continue;
          const size_t bh = static_cast<size_t>(cur.b) * a.Hq + head * a.g + h0 + h;
          const float inv = l[c] == 0.f ? 0.f : 1.f / l[c];
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            a.out[bh * D + 16 * j + gid] = acc[j][c] * inv;
            a.out[bh * D + 16 * j + gid + 8] = acc[j][c + 2] * inv;
          }
          if (a.lse && gid == 0) a.lse[bh] = (m[c] + log2f(l[c])) * 0.6931471805599453f;
        }
    } else {
      const int which = cur.t0 == 0;
      float* part = parts + (warp * 2 + which) * PART;
      if (tig < NH / 2)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int h = 2 * tig + c;
          if (gid == 0) {
            part[h] = m[c];
            part[DP_HEADS + h] = l[c];
          }
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            part[2 * DP_HEADS + h * D + 16 * j + gid] = acc[j][c];
            part[2 * DP_HEADS + h * D + 16 * j + gid + 8] = acc[j][c + 2];
          }
        }
      if (lane == 0) left_s[warp][which] = Left{cur.b, cur.unit, cur.t1 < cur.tiles};
    }
  }

  // ---- the block's partials in the order of its shares: entry 2 w + {0, 1} is what warp w left.  A
  // unit's are consecutive: where it begins (or the block does), then one per warp until it ends.
  // A warp folds a head of a unit.  From here on the code runs once, so it is bound by fetching
  // instructions: rolled loops (for one sequence of 777 rows the call takes 9.6 us, 13.2 with unrolled ones).
  __syncthreads();
  float* own = reinterpret_cast<float*>(smem);  // the rings are idle: this block's part of a unit that ends here
  constexpr int E = D / 32;  // elements of a head per lane
  uint32_t present, more;
  {
    const Left x = lane < 2 * DP_WARPS ? left_s[lane >> 1][lane & 1] : Left{-1, 0, false};
    present = __ballot_sync(0xffffffffu, x.b >= 0);
    more = __ballot_sync(0xffffffffu, x.b >= 0 && x.more);
  }
  constexpr uint32_t EVEN = 0x55555555u & ((1u << 2 * DP_WARPS) - 1);
  int item = 0;
  for (uint32_t begins = present & ~(EVEN & ~1u); begins; begins &= begins - 1) {
    const int i = __ffs(begins) - 1, w = i >> 1;
    const Left u = left_s[w][i & 1];
    int count = 1;
    bool on = more >> i & 1;  // the unit goes on: to the first later entry of a share that it does not fill, if there is one
    if (on) {
      const uint32_t ends = present & ~more & EVEN & ~((2u << i) - 1);
      on = ends == 0;
      count = (on ? shares : (__ffs(ends) + 1) / 2) - w;
    }
    const int head = u.unit / a.chunks, h0 = (u.unit - head * a.chunks) * DP_HEADS, gc = min(DP_HEADS, a.g - h0);
    const bool begun = i & 1, complete = begun && !on;
    float* to = begun || on ? a.partials + static_cast<size_t>(2 * blockIdx.x + begun) * PART : own;
#pragma unroll 1
    for (int h = 0; h < gc; ++h) {
      if (item++ % DP_WARPS != warp) continue;
      auto part = [&](int k) { return parts + (k == 0 ? i : 2 * (w + k)) * PART; };
      const int mine = lane & 7;
      const float mk = mine < count ? part(mine)[h] : -INFINITY;
      float M = fmaxf(mk, DP_FLOOR), L = 0.f, o[E] = {};
#pragma unroll
      for (int x = 1; x < 8; x <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
      const float f = ex2_approx(mk - M);
#pragma unroll 1
      for (int k = 0; k < count; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, k);
        const float* p = part(k);
        L = fmaf(p[DP_HEADS + h], fk, L);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(p[2 * DP_HEADS + h * D + E * lane + e], fk, o[e]);
      }
      if (complete) {
        const size_t bh = static_cast<size_t>(u.b) * a.Hq + head * a.g + h0 + h;
        const float inv = L == 0.f ? 0.f : __fdividef(1.f, L);
#pragma unroll
        for (int e = 0; e < E; ++e) a.out[bh * D + E * lane + e] = o[e] * inv;
        if (a.lse && lane == 0) a.lse[bh] = (M + __log2f(L)) * 0.6931471805599453f;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) to[2 * DP_HEADS + h * D + E * lane + e] = o[e];
        if (lane == 0) {
          to[h] = M;
          to[DP_HEADS + h] = L;
          if (h == 0 && on) publish_s[begun] = 1;  // the unit ends in a later block
          if (h == 0 && !on) ending_s = u;
        }
      }
    }
  }
  __syncthreads();
  if (const int i = DP_THREADS - 1 - static_cast<int>(threadIdx.x); i < 2 && publish_s[i]) {
    unsigned long long* flag = a.flags + 2 * blockIdx.x + i;
    if (a.selftest == DP_LATE) {
      const unsigned long long t0 = globaltimer_ns();
      while (ld_flag(flag) != ~a.call && globaltimer_ns() - t0 < 4 * a.wait_ns) {
      }
    }
    __threadfence();
    if (swap_flag(flag, a.call) == ~a.call) *flag = 0;  // nobody waits any more
  }
  const Left ending = ending_s;
  if (ending.b < 0) return;

  // ---- a unit that began in an earlier block ends here: join the partials of the blocks from there on
  const int first = cut.owner(first_tile_s) / DP_WARPS, count = static_cast<int>(blockIdx.x) - first;
  auto slot_of = [&](int k) { return 2 * (first + k) + (k == 0); };
  const int head = ending.unit / a.chunks, h0 = (ending.unit - head * a.chunks) * DP_HEADS, gc = min(DP_HEADS, a.g - h0);
  if (static_cast<int>(threadIdx.x) < count) {
    unsigned long long* flag = a.flags + slot_of(threadIdx.x);
    const unsigned long long t0 = globaltimer_ns();
    bool there;
    while (!(there = ld_flag(flag) == a.call) && globaltimer_ns() - t0 <= a.wait_ns) {
    }
    // read, or given up: unless it came in that moment, the publisher clears it
    if (there || swap_flag(flag, ~a.call) == a.call) *flag = 0;
    else late_s = 1;
  }
  __syncthreads();
  // DP_WARPS / 2^x warps per head, each with every so many-th partial; then theirs and the block's own
  const int heads_log2 = gc > 4 ? 3 : (gc > 2 ? 2 : (gc > 1 ? 1 : 0)), ways = DP_WARPS >> heads_log2;
  const int h = warp & ((1 << heads_log2) - 1), way = warp >> heads_log2;
  float* sums = own + PART + warp * (D + 2);  // [warp]: maximum, sum, output
  float M = DP_FLOOR, L = 0.f, o[E] = {};
  if (h < gc) {
#pragma unroll 4
    for (int k = way; k < count; k += ways) {
      const float* p = a.partials + static_cast<size_t>(slot_of(k)) * PART;
      const float mk = __ldcg(p + h), lk = __ldcg(p + DP_HEADS + h);
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = __ldcg(p + 2 * DP_HEADS + h * D + E * lane + e);
      const float Mn = fmaxf(M, mk), c = ex2_approx(M - Mn), f = ex2_approx(mk - Mn);
      M = Mn;
      L = fmaf(L, c, lk * f);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], c, x[e] * f);
    }
    if (lane == 0) {
      sums[0] = M;
      sums[1] = L;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[2 + E * lane + e] = o[e];
  }
  __syncthreads();
  if (way > 0 || h >= gc) return;
#pragma unroll 1
  for (int k = 1; k <= ways; ++k) {
    const bool last = k == ways;
    const float* p = last ? own : sums + (k << heads_log2) * (D + 2);
    const float mk = last ? own[h] : p[0], lk = last ? own[DP_HEADS + h] : p[1];
    const float* x = last ? own + 2 * DP_HEADS + h * D : p + 2;
    const float Mn = fmaxf(M, mk), c = ex2_approx(M - Mn), f = ex2_approx(mk - Mn);
    M = Mn;
    L = fmaf(L, c, lk * f);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], c, x[E * lane + e] * f);
  }
  if (late_s) L = NAN;
  const size_t bh = static_cast<size_t>(ending.b) * a.Hq + head * a.g + h0 + h;
  const float inv = L == 0.f ? 0.f : __fdividef(1.f, L);
#pragma unroll
  for (int e = 0; e < E; ++e) a.out[bh * D + E * lane + e] = o[e] * inv;
  if (a.lse && lane == 0) a.lse[bh] = (M + __log2f(L)) * 0.6931471805599453f;
}

// A number that no other call has: partials of an earlier call, of another process in the same memory
// or of whatever was there do not pass for this call's.  (The SplitMix64 generator of Steele, Lea and Flood, 2014: a
// counter with an odd step, mixed one to one.)
unsigned long long call_number() {
  static const unsigned long long seed =
      static_cast<unsigned long long>(std::chrono::system_clock::now().time_since_epoch().count()) ^
      (static_cast<unsigned long long>(getpid()) << 40);
  static std::atomic<unsigned long long> calls{0};
  for (;;) {
    unsigned long long x = seed + ++calls * 0x9e3779b97f4a7c15ull;  // (odd: a step through all 64-bit numbers)
    x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;                    // mixed one to one
    x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
    x ^= x >> 31;
    if (x != 0 && x != ~0ull) return x;  // (0 is a cleared flag, and must not be a complement either)
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

template <int D, int NH>
cudaError_t launch_decode_paged(const CUtensorMap& tmK, const CUtensorMap& tmV, const DecodePagedArgs& a, cudaStream_t stream) {
  constexpr int SMEM = DP_WARPS * DP_STAGES * DP_STAGE_BYTES + 2 * DP_WARPS * DP_HEADS * (D + 2) * 4 + 1024;
  auto kernel = decode_paged_kernel<D, NH>;
  static DeviceOnce ready;
  if (!ready.done()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    ready.set();
  }
  return launch_pdl(kernel, dim3(a.grid), dim3(DP_THREADS), SMEM, stream, tmK, tmV, a);
}

bool strides_ok(const int64_t* s, int d) {
  if (!s) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 1 || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return s[2] >= d;
}

bool pool_map(CUtensorMap* m, const void* pool, const int64_t* s, int d, int page_size, int heads, int num_pages) {
  using u64 = unsigned long long;
  const u64 dims[4] = {static_cast<u64>(d), static_cast<u64>(page_size), static_cast<u64>(heads), static_cast<u64>(num_pages)};
  const u64 strides[3] = {static_cast<u64>(s[2]) * 2, static_cast<u64>(s[1]) * 2, static_cast<u64>(s[0]) * 2};
  const unsigned box[4] = {64, DP_BOX_ROWS, 1, 1};
  return encode_tensor_map(m, pool, 4, dims, strides, box);
}

}  // namespace
}  // namespace snapkv

extern "C" size_t snapkv_decode_paged_workspace_size(int B, int Hq, int Hc, int d) {
  using namespace snapkv;
  if (B < 1 || Hq < 1 || Hc < 1 || Hq % Hc != 0 || (d != 64 && d != 128)) return 0;
  return align256(2 * DP_MAX_GRID * sizeof(unsigned long long)) +
         align256(static_cast<size_t>(2) * DP_MAX_GRID * DP_HEADS * (d + 2) * sizeof(float));
}

namespace snapkv {
namespace {

snapkv_status_t decode_paged(const void* q_cur, const void* k_pool, const void* v_pool, const int64_t* k_strides,
                             const int64_t* v_strides, const int32_t* page_table, int pages_per_seq, int page_size,
                             int num_pages, const int32_t* seq_lens, int B, int Hq, int Hc, int d, float* out,
                             float* out_lse, void* workspace, size_t workspace_bytes, void* stream, int selftest) {
  if (B < 1 || Hq < 1 || Hc < 1 || Hq % Hc != 0 || d < 1 || pages_per_seq < 1 || page_size < 1 || num_pages < 1 ||
      page_size % DP_BOX_ROWS != 0)
    return SNAPKV_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || static_cast<long long>(B) * Hq > 65535 ||
      static_cast<long long>(pages_per_seq) * page_size >= (1ll << 31) - 64)
    return SNAPKV_ERR_UNSUPPORTED;
  if (!q_cur || !k_pool || !v_pool || !page_table || !seq_lens || !out) return SNAPKV_ERR_INVALID_ARG;
  for (const void* p : {q_cur, k_pool, v_pool})
    if (reinterpret_cast<uintptr_t>(p) & 15) return SNAPKV_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(page_table), static_cast<const void*>(seq_lens),
                        static_cast<const void*>(out), static_cast<const void*>(out_lse)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return SNAPKV_ERR_INVALID_ARG;
  if (!strides_ok(k_strides, d) || !strides_ok(v_strides, d)) return SNAPKV_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
      workspace_bytes < snapkv_decode_paged_workspace_size(B, Hq, Hc, d))
    return SNAPKV_ERR_WORKSPACE;
  CUtensorMap tmK, tmV;
  if (!pool_map(&tmK, k_pool, k_strides, d, page_size, Hc, num_pages) ||
      !pool_map(&tmV, v_pool, v_strides, d, page_size, Hc, num_pages))
    return SNAPKV_ERR_CUDA;
  DecodePagedArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q_cur);
  a.table = page_table, a.seq_lens = seq_lens;
  a.pages_per_seq = pages_per_seq, a.page_size = page_size, a.B = B, a.Hq = Hq, a.g = Hq / Hc;
  a.chunks = (a.g + DP_HEADS - 1) / DP_HEADS;
  a.units = Hc * a.chunks;
  a.grid = sm_count() < DP_MAX_GRID ? sm_count() : DP_MAX_GRID;
  a.c2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(d)));
  a.wait_ns = wait_limit_setting();
  a.out = out, a.lse = out_lse;
  a.flags = static_cast<unsigned long long*>(workspace);
  a.call = call_number();
  a.selftest = selftest;
  a.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + align256(2 * DP_MAX_GRID * sizeof(unsigned long long)));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto f = d == 128 ? (a.g <= 2 ? launch_decode_paged<128, 2> : (a.g <= 4 ? launch_decode_paged<128, 4> : launch_decode_paged<128, 8>))
                    : (a.g <= 2 ? launch_decode_paged<64, 2> : (a.g <= 4 ? launch_decode_paged<64, 4> : launch_decode_paged<64, 8>));
  return f(tmK, tmV, a, s) == cudaSuccess ? SNAPKV_OK : SNAPKV_ERR_CUDA;
}

}  // namespace
}  // namespace snapkv

extern "C" snapkv_status_t snapkv_decode_paged(const void* q_cur, const void* k_pool, const void* v_pool,
                                               const int64_t* k_strides, const int64_t* v_strides,
                                               const int32_t* page_table, int pages_per_seq, int page_size,
                                               int num_pages, const int32_t* seq_lens, int B, int Hq, int Hc, int d,
                                               float* out, float* out_lse, void* workspace, size_t workspace_bytes,
                                               void* stream) {
  return snapkv::decode_paged(q_cur, k_pool, v_pool, k_strides, v_strides, page_table, pages_per_seq, page_size,
                              num_pages, seq_lens, B, Hq, Hc, d, out, out_lse, workspace, workspace_bytes, stream, 0);
}

extern "C" snapkv_status_t snapkv_selftest_late_partials(const void* q_cur, const void* k_pool, const void* v_pool,
                                                         const int64_t* k_strides, const int64_t* v_strides,
                                                         const int32_t* page_table, int pages_per_seq, int page_size,
                                                         int num_pages, const int32_t* seq_lens, int B, int Hq, int Hc,
                                                         int d, float* out, float* out_lse, void* workspace,
                                                         size_t workspace_bytes, void* stream) {
  return snapkv::decode_paged(q_cur, k_pool, v_pool, k_strides, v_strides, page_table, pages_per_seq, page_size,
                              num_pages, seq_lens, B, Hq, Hc, d, out, out_lse, workspace, workspace_bytes, stream,
                              snapkv::DP_LATE);
}

extern "C" snapkv_status_t snapkv_selftest_lost_rows(const void* q_cur, const void* k_pool, const void* v_pool,
                                                     const int64_t* k_strides, const int64_t* v_strides,
                                                     const int32_t* page_table, int pages_per_seq, int page_size,
                                                     int num_pages, const int32_t* seq_lens, int B, int Hq, int Hc, int d,
                                                     float* out, float* out_lse, void* workspace, size_t workspace_bytes,
                                                     void* stream) {
  return snapkv::decode_paged(q_cur, k_pool, v_pool, k_strides, v_strides, page_table, pages_per_seq, page_size,
                              num_pages, seq_lens, B, Hq, Hc, d, out, out_lse, workspace, workspace_bytes, stream,
                              snapkv::DP_LOST);
}
