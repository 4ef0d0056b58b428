// Appending to a paged cache with the position rotation on the way.  Pair r of a head turns by
// positions[t] * inv_freq[r]: (x, y) -> (x cos - y sin, x sin + y cos).
//
// Bound by HBM for prompts, by latency for a generation step.  A block takes a few tokens with all
// their heads.  First a warp per token finds the token's sequence, page and angles, once for all heads;
// then a thread moves items of 16 elements (two 16-byte vectors: the two halves of eight pairs) of one
// token and one place in the head, head after head, so that its sines and cosines stay in registers.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/snapkv.h"
#include "launch.cuh"
#include "snapkv_internal.h"

namespace snapkv {
namespace {

constexpr int AP_THREADS = 256;

struct AppendArgs {
  const uint16_t *k, *v, *q;
  long long k_st[3], v_st[3], q_st[3];
  const int32_t *cu, *cache_lens, *positions, *table;
  const float* inv_freq;
  int half;  // rot / 2, 0 without rotation
  int pages_per_seq, page_size, num_pages, B, T, Hq, Hkv, Hc;
  uint16_t *q_out, *k_pool, *v_pool;
  long long kp[3], vp[3];
};

// The last sequence that starts at or in front of token t, and its start: a warp probes 32 at a time.
__device__ __forceinline__ int sequence_of(const AppendArgs& a, int t, int lane, int* start) {
  int lo = 0, len = a.B;
  for (;;) {
    const int step = (len + 31) / 32;
    const int v = lane * step < len ? __ldg(a.cu + lo + lane * step) : 0x7fffffff;
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, v <= t) | 1u);
    lo += last * step;
    if (step == 1) {
      *start = __shfl_sync(0xffffffffu, v, last);
      return lo;
    }
    len = min(step, len - last * step);
  }
}

__device__ __forceinline__ float lo_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// TB tokens per block: 8 where there are many (a head's rows are then consecutive in memory for eight
// tokens in caches stored by heads), 1 for generation steps.
template <int D, bool INTERLEAVED, int TB>
__global__ void __launch_bounds__(AP_THREADS) append_kernel(const AppendArgs a) {
  constexpr int ITEMS = D / 16;                        // of a head
  constexpr int STEP = AP_THREADS / (ITEMS * TB);      // heads in flight
  __shared__ __align__(16) float cs[TB][D / 2], sn[TB][D / 2];  // (read as float4)
  __shared__ long long src_b[TB], src_i[TB], k_to[TB], v_to[TB];  // sequence and row of the source; targets or -1
  __shared__ int live[TB];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  if (warp < TB) {
    const int t = blockIdx.x * TB + warp;
    int b = 0, start = 0;
    bool in = t < a.T;
    if (in && a.cu) {
      in = t < __ldg(a.cu + a.B);
      b = sequence_of(a, t, lane, &start);
      in = in && t >= start;
    } else if (in) {
      const int n = a.T / a.B;
      b = t / n;
      start = b * n;
    }
    if (in) {
      const long long slot = static_cast<long long>(__ldg(a.cache_lens + b)) + (t - start);
      const long long pos = a.positions ? __ldg(a.positions + t) : slot;
      // Angles of far positions lose their fraction of a turn in 32 bits: 64 up to the reduction.
      for (int r = lane; r < a.half; r += 32) {
        const double turns = static_cast<double>(pos) * __ldg(a.inv_freq + r) * 0.15915494309189535;  // 1 / (2 pi)
        sincospif(2.f * static_cast<float>(turns - rint(turns)), &sn[warp][r], &cs[warp][r]);
      }
      if (lane == 0) {
        src_b[warp] = a.cu ? 0 : b;
        src_i[warp] = a.cu ? t : t - start;
        long long kd = -1, vd = -1;
        if (slot >= 0 && slot < static_cast<long long>(a.pages_per_seq) * a.page_size) {
          const int s = static_cast<int>(slot), pg = s / a.page_size, row = s - pg * a.page_size;
          const int page = __ldg(a.table + static_cast<long long>(b) * a.pages_per_seq + pg);
          if (page >= 0 && page < a.num_pages) {
            kd = page * a.kp[0] + row * a.kp[2];
            vd = page * a.vp[0] + row * a.vp[2];
          }
        }
        k_to[warp] = kd;
        v_to[warp] = vd;
      }
    }
    if (lane == 0) live[warp] = in;
  }
  __syncthreads();
  const int j = threadIdx.x % ITEMS, tok = threadIdx.x / ITEMS % TB, h0 = threadIdx.x / (ITEMS * TB);
  if (!live[tok]) return;
  // the item's two vectors, and whether it is turned
  const bool turn = 8 * j < a.half;
  const int v0 = turn && !INTERLEAVED ? j : 2 * j, v1 = turn && !INTERLEAVED ? j + a.half / 8 : 2 * j + 1;
  float c[8], s[8];
  if (turn)
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(&cs[tok][8 * j + e]), y = *reinterpret_cast<const float4*>(&sn[tok][8 * j + e]);
      c[e] = x.x, c[e + 1] = x.y, c[e + 2] = x.z, c[e + 3] = x.w;
      s[e] = y.x, s[e + 1] = y.y, s[e + 2] = y.z, s[e + 3] = y.w;
    }
  auto turned = [&](uint4& p, uint4& q) {
    uint32_t x[4] = {p.x, p.y, p.z, p.w}, y[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (INTERLEAVED) {  // pairs (lo, hi): of the first vector 0 .. 3, of the second 4 .. 7
        const float xl = lo_bf16(x[i]), xh = hi_bf16(x[i]), yl = lo_bf16(y[i]), yh = hi_bf16(y[i]);
        x[i] = pack_bf16(xl * c[i] - xh * s[i], xl * s[i] + xh * c[i]);
        y[i] = pack_bf16(yl * c[4 + i] - yh * s[4 + i], yl * s[4 + i] + yh * c[4 + i]);
      } else {
        const float xl = lo_bf16(x[i]), xh = hi_bf16(x[i]), yl = lo_bf16(y[i]), yh = hi_bf16(y[i]);
        x[i] = pack_bf16(xl * c[2 * i] - yl * s[2 * i], xh * c[2 * i + 1] - yh * s[2 * i + 1]);
        y[i] = pack_bf16(xl * s[2 * i] + yl * c[2 * i], xh * s[2 * i + 1] + yh * c[2 * i + 1]);
      }
    }
    p = make_uint4(x[0], x[1], x[2], x[3]);
    q = make_uint4(y[0], y[1], y[2], y[3]);
  };
  // heads h0, h0 + STEP, ... of a tensor, four at a time in flight
  auto move = [&](const uint16_t* from, long long from_head, int heads, bool rotate, uint16_t* to, long long to_head, int reps) {
    for (int h = h0; h < heads; h += 4 * STEP) {
      uint4 x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (h + i * STEP < heads) {
          const uint4* p = reinterpret_cast<const uint4*>(from + (h + i * STEP) * from_head);
          x[i] = p[v0];
          y[i] = p[v1];
        }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (h + i * STEP < heads) {
          if (rotate) turned(x[i], y[i]);
          uint16_t* base = to + (h + i * STEP) * reps * to_head;
          for (int m = 0; m < reps; ++m) {
            uint4* p = reinterpret_cast<uint4*>(base + m * to_head);
            p[v0] = x[i];
            p[v1] = y[i];
          }
        }
    }
  };
  const long long b = src_b[tok], i = src_i[tok], kd = k_to[tok], vd = v_to[tok];
  const int reps = a.Hc / a.Hkv;
  if (kd >= 0) {
    move(a.k + b * a.k_st[0] + i * a.k_st[1], a.k_st[2], a.Hkv, turn, a.k_pool + kd, a.kp[1], reps);
    move(a.v + b * a.v_st[0] + i * a.v_st[1], a.v_st[2], a.Hkv, false, a.v_pool + vd, a.vp[1], reps);
  }
  if (a.q)
    move(a.q + b * a.q_st[0] + i * a.q_st[1], a.q_st[2], a.Hq, turn,
         a.q_out + (static_cast<long long>(blockIdx.x) * TB + tok) * a.Hq * D, D, 1);
}

template <int D, bool INTERLEAVED>
cudaError_t launch_append(const AppendArgs& a, cudaStream_t stream) {
  // eight tokens per block once that leaves every SM a few blocks
  if (a.T >= 8 * 4 * sm_count())
    return launch_pdl(append_kernel<D, INTERLEAVED, 8>, dim3((a.T + 7) / 8), dim3(AP_THREADS), 0, stream, a);
  return launch_pdl(append_kernel<D, INTERLEAVED, 1>, dim3(a.T), dim3(AP_THREADS), 0, stream, a);
}

bool token_strides_ok(const int64_t* s, int d) {
  if (!s) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] < (i ? d : 1) || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return true;
}
bool pool_strides_ok(const int64_t* s, int d) {
  if (!s) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 1 || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return s[2] >= d;
}

}  // namespace
}  // namespace snapkv

extern "C" snapkv_status_t snapkv_append_paged(const void* k_new, const void* v_new, const int64_t* k_new_strides,
                                               const int64_t* v_new_strides, const int32_t* cu_tokens,
                                               const int32_t* cache_lens, const int32_t* positions,
                                               const float* inv_freq, int rot, int interleaved, const void* q,
                                               const int64_t* q_strides, void* q_out, void* k_pool, void* v_pool,
                                               const int64_t* k_strides, const int64_t* v_strides,
                                               const int32_t* page_table, int pages_per_seq, int page_size,
                                               int num_pages, int B, int T, int Hq, int Hkv, int Hc, int d,
                                               void* stream) {
  using namespace snapkv;
  if (B < 1 || T < 0 || Hkv < 1 || Hc < 1 || Hc % Hkv != 0 || d < 1 || pages_per_seq < 1 || page_size < 1 ||
      num_pages < 1 || (!cu_tokens && T % B != 0) || (q && Hq < 1))
    return SNAPKV_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || static_cast<long long>(pages_per_seq) * page_size >= (1ll << 31) - 64)
    return SNAPKV_ERR_UNSUPPORTED;
  if (!k_new || !v_new || !cache_lens || !k_pool || !v_pool || !page_table || (q && (!inv_freq || !q_out)))
    return SNAPKV_ERR_INVALID_ARG;
  if (inv_freq && (rot < 2 || rot > d || rot % 2 != 0)) return SNAPKV_ERR_INVALID_ARG;
  if (inv_freq && rot % 16 != 0) return SNAPKV_ERR_UNSUPPORTED;
  for (const void* p : {k_new, v_new, q, static_cast<const void*>(q_out), static_cast<const void*>(k_pool),
                        static_cast<const void*>(v_pool)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return SNAPKV_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(cu_tokens), static_cast<const void*>(cache_lens),
                        static_cast<const void*>(positions), static_cast<const void*>(inv_freq),
                        static_cast<const void*>(page_table)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return SNAPKV_ERR_INVALID_ARG;
  if (!token_strides_ok(k_new_strides, d) || !token_strides_ok(v_new_strides, d) ||
      (q && !token_strides_ok(q_strides, d)) || !pool_strides_ok(k_strides, d) || !pool_strides_ok(v_strides, d))
    return SNAPKV_ERR_INVALID_ARG;
  if (T == 0) return SNAPKV_OK;
  AppendArgs a = {};
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.q = static_cast<const uint16_t*>(q);
  for (int i = 0; i < 3; ++i) {
    a.k_st[i] = k_new_strides[i];
    a.v_st[i] = v_new_strides[i];
    a.q_st[i] = q ? q_strides[i] : 0;
    a.kp[i] = k_strides[i];
    a.vp[i] = v_strides[i];
  }
  a.cu = cu_tokens, a.cache_lens = cache_lens, a.positions = positions, a.table = page_table, a.inv_freq = inv_freq;
  a.half = inv_freq ? rot / 2 : 0;
  a.pages_per_seq = pages_per_seq, a.page_size = page_size, a.num_pages = num_pages;
  a.B = B, a.T = T, a.Hq = Hq, a.Hkv = Hkv, a.Hc = Hc;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_pool = static_cast<uint16_t*>(k_pool);
  a.v_pool = static_cast<uint16_t*>(v_pool);
  auto f = d == 128 ? (interleaved ? launch_append<128, true> : launch_append<128, false>)
                    : (interleaved ? launch_append<64, true> : launch_append<64, false>);
  return f(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? SNAPKV_OK : SNAPKV_ERR_CUDA;
}
