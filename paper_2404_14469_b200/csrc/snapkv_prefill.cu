// The prompt's own attention (the phase in front of the compression step): causal, grouped heads,
// sequences of different lengths.  Per query i of a sequence with Lq queries and Lk keys:
//   out_i = sum_j p_ij v_j / l_i,  p_ij = exp(s_ij - m_i),  s_ij = q_i.k_j / sqrt(d),  j <= Lk - Lq + i
// with m_i the running maximum and l_i the running sum; lse_i = m_i + ln l_i.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/snapkv.h"
#include "launch.cuh"
#include "snapkv_internal.h"

namespace snapkv {
namespace {

constexpr int PF_MAX_SEQS = 32;  // sequences that share a launch
constexpr int PF_WARPS = 8, PF_KEYS = 32;

struct PrefillSeq {
  int lq, lk;
  long long q0, k0;  // first token
};
struct PrefillSeqs {
  PrefillSeq s[PF_MAX_SEQS];
};
struct PrefillArgs {
  const __nv_bfloat16 *q, *k, *v;
  long long qt, qh, kt, kh, vt, vh;
  int Hq, g, W, b0;
  float c2;
  __nv_bfloat16* out;
  float *lse, *lse_obs;
};

// One warp per query, one lane per key of a tile.
template <int D>
__global__ void __launch_bounds__(PF_WARPS * 32) prefill_kernel(const PrefillArgs a, const PrefillSeqs seqs) {
  __shared__ float ks[PF_KEYS][D + 1], vs[PF_KEYS][D], qs[PF_WARPS][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y;
  const PrefillSeq s = seqs.s[blockIdx.z];
  const int i0 = blockIdx.x * PF_WARPS, i = i0 + warp;
  if (i0 >= s.lq) return;
  pdl_wait();
  const int last = s.lk - s.lq + min(i0 + PF_WARPS, s.lq) - 1;  // of the block's last query
  const int mine = i < s.lq ? s.lk - s.lq + i : -1;
  for (int c = lane; c < D; c += 32)
    qs[warp][c] = i < s.lq ? __bfloat162float(a.q[(s.q0 + i) * a.qt + h * a.qh + c]) : 0.f;
  float m = -INFINITY, l = 0.f, acc[D / 32] = {};
  for (int j0 = 0; j0 <= last; j0 += PF_KEYS) {
    __syncthreads();
    for (int e = threadIdx.x; e < PF_KEYS * D; e += PF_WARPS * 32) {
      const int r = e / D, c = e % D, j = j0 + r;
      const bool in = j <= last;
      ks[r][c] = in ? __bfloat162float(a.k[(s.k0 + j) * a.kt + (h / a.g) * a.kh + c]) : 0.f;
      vs[r][c] = in ? __bfloat162float(a.v[(s.k0 + j) * a.vt + (h / a.g) * a.vh + c]) : 0.f;
    }
    __syncthreads();
    float x = 0.f;
    for (int c = 0; c < D; ++c) x = fmaf(qs[warp][c], ks[lane][c], x);
    x = j0 + lane <= mine ? x * a.c2 : -INFINITY;
    float mn = x;
    for (int o = 16; o; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    mn = fmaxf(fmaxf(mn, m), -1e30f);
    const float corr = exp2f(m - mn), p = exp2f(x - mn);
    m = mn;
    l = l * corr + p;
    for (int t = 0; t < D / 32; ++t) acc[t] *= corr;
    for (int r = 0; r < PF_KEYS; ++r) {
      const float pr = __shfl_sync(0xffffffffu, p, r);
      if (pr != 0.f)
        for (int t = 0; t < D / 32; ++t) acc[t] = fmaf(pr, vs[r][lane + 32 * t], acc[t]);
    }
  }
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (i >= s.lq) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const long long row = (s.q0 + i) * a.Hq + h;
  for (int t = 0; t < D / 32; ++t) a.out[row * D + lane + 32 * t] = __float2bfloat16(acc[t] * inv);
  if (lane == 0) {
    const float e = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    if (a.lse) a.lse[row] = e;
    if (i >= s.lq - a.W)
      a.lse_obs[(static_cast<long long>(a.b0 + blockIdx.z) * a.Hq + h) * a.W + i - (s.lq - a.W)] = e;
  }
}

bool strides_ok(const int64_t* s, int d) {
  for (int i = 0; i < 2; ++i)
    if (s[i] < d || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return true;
}

}  // namespace
}  // namespace snapkv

extern "C" snapkv_status_t snapkv_prefill_attention(const void* q, const void* k, const void* v,
                                                    const int64_t* q_strides, const int64_t* k_strides,
                                                    const int64_t* v_strides, const int32_t* q_lens,
                                                    const int32_t* k_lens, const int64_t* q_starts,
                                                    const int64_t* k_starts, int B, int Hq, int Hkv, int d, int W,
                                                    void* out, float* out_lse, float* lse_obs, void* stream) {
  using namespace snapkv;
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || d < 1 || W < 0 || !q_lens) return SNAPKV_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || W > 128 || Hq > 65535) return SNAPKV_ERR_UNSUPPORTED;
  if (!q || !k || !v || !out || (W > 0) != (lse_obs != nullptr)) return SNAPKV_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, static_cast<const void*>(out)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return SNAPKV_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(out_lse) | reinterpret_cast<uintptr_t>(lse_obs)) & 3) return SNAPKV_ERR_INVALID_ARG;
  const int64_t dq[2] = {static_cast<int64_t>(Hq) * d, d}, dk[2] = {static_cast<int64_t>(Hkv) * d, d};
  const int64_t *qs = q_strides ? q_strides : dq, *ks = k_strides ? k_strides : dk, *vs = v_strides ? v_strides : dk;
  if (!strides_ok(qs, d) || !strides_ok(ks, d) || !strides_ok(vs, d)) return SNAPKV_ERR_INVALID_ARG;
  constexpr int64_t MAX_TOKENS = 1ll << 31;
  int64_t q_end = 0, k_end = 0;
  for (int b = 0; b < B; ++b) {
    const int lq = q_lens[b], lk = k_lens ? k_lens[b] : lq;
    if (lq < 0 || lk < 0 || lq < W) return SNAPKV_ERR_INVALID_ARG;
    const int64_t q0 = q_starts ? q_starts[b] : q_end, k0 = k_starts ? k_starts[b] : k_end;
    if (q0 < q_end || q0 > MAX_TOKENS || k0 < 0 || k0 > MAX_TOKENS) return SNAPKV_ERR_INVALID_ARG;
    q_end = q0 + lq;
    k_end = k0 + lk;
    if (q_end > MAX_TOKENS || k_end > MAX_TOKENS) return SNAPKV_ERR_INVALID_ARG;
  }
  PrefillArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.qt = qs[0], a.qh = qs[1], a.kt = ks[0], a.kh = ks[1], a.vt = vs[0], a.vh = vs[1];
  a.Hq = Hq, a.g = Hq / Hkv, a.W = W;
  a.c2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(d)));
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = out_lse, a.lse_obs = lse_obs;
  int64_t q_at = 0, k_at = 0;
  for (int b0 = 0; b0 < B; b0 += PF_MAX_SEQS) {
    PrefillSeqs seqs = {};
    const int n = B - b0 < PF_MAX_SEQS ? B - b0 : PF_MAX_SEQS;
    int most = 0;
    for (int i = 0; i < n; ++i) {
      PrefillSeq& s = seqs.s[i];
      s.lq = q_lens[b0 + i];
      s.lk = k_lens ? k_lens[b0 + i] : s.lq;
      s.q0 = q_starts ? q_starts[b0 + i] : q_at;
      s.k0 = k_starts ? k_starts[b0 + i] : k_at;
      q_at = s.q0 + s.lq;
      k_at = s.k0 + s.lk;
      if (s.lq > most) most = s.lq;
    }
    if (most == 0) continue;
    a.b0 = b0;
    const dim3 grid((most + PF_WARPS - 1) / PF_WARPS, Hq, n);
    const cudaError_t e = launch_pdl(d == 128 ? prefill_kernel<128> : prefill_kernel<64>, grid, dim3(PF_WARPS * 32), 0,
                                     static_cast<cudaStream_t>(stream), a, seqs);
    if (e != cudaSuccess) return SNAPKV_ERR_CUDA;
  }
  return SNAPKV_OK;
}
