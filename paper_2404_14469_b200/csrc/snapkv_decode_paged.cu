// One generation step's attention over a paged cache with a length per sequence:
// out = softmax(q . K^T / sqrt(d)) V over rows 0 .. seq_lens[b] - 1 of every sequence.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/snapkv.h"
#include "launch.cuh"
#include "snapkv_internal.h"

namespace snapkv {
namespace {

constexpr int DP_WARPS = 8;

struct DecodePagedArgs {
  const __nv_bfloat16 *q, *k, *v;
  long long kp[3], vp[3];
  const int32_t *table, *seq_lens;
  int pages_per_seq, page_size, num_pages, Hq, g;
  float c2;
  float *out, *lse;
};

// A block per query head; a warp takes every DP_WARPS-th row, its lanes the elements.
template <int D>
__global__ void __launch_bounds__(DP_WARPS * 32) decode_paged_kernel(const DecodePagedArgs a) {
  constexpr int E = D / 32;
  __shared__ float ms[DP_WARPS], ls[DP_WARPS], os[DP_WARPS][D];
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, c = h / a.g;
  const long long most = static_cast<long long>(a.pages_per_seq) * a.page_size;
  const long long want = a.seq_lens[b];
  const int n = static_cast<int>(want < 0 ? 0 : (want < most ? want : most));
  float q[E], acc[E] = {}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) q[e] = __bfloat162float(a.q[static_cast<long long>(blockIdx.x) * D + lane + 32 * e]);
  for (int r = warp; r < n; r += DP_WARPS) {
    const int pg = r / a.page_size, row = r - pg * a.page_size;
    const int page = a.table[static_cast<long long>(b) * a.pages_per_seq + pg];
    const bool in = page >= 0 && page < a.num_pages;
    const __nv_bfloat16 *kr = a.k + page * a.kp[0] + c * a.kp[1] + row * a.kp[2],
                        *vr = a.v + page * a.vp[0] + c * a.vp[1] + row * a.vp[2];
    float x = 0.f;
    for (int e = 0; e < E; ++e) x = fmaf(q[e], in ? __bfloat162float(kr[lane + 32 * e]) : 0.f, x);
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    x *= a.c2;
    const float mn = fmaxf(m, x), corr = exp2f(m - mn), p = exp2f(x - mn);
    m = mn;
    l = l * corr + p;
    for (int e = 0; e < E; ++e) acc[e] = fmaf(p, in ? __bfloat162float(vr[lane + 32 * e]) : 0.f, acc[e] * corr);
  }
  for (int e = 0; e < E; ++e) os[warp][lane + 32 * e] = acc[e];
  if (lane == 0) {
    ms[warp] = m;
    ls[warp] = l;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < DP_WARPS; ++w) M = fmaxf(M, ms[w]);
  for (int w = 0; w < DP_WARPS; ++w) L += ms[w] == -INFINITY ? 0.f : ls[w] * exp2f(ms[w] - M);
  for (int e = threadIdx.x; e < D; e += DP_WARPS * 32) {
    float o = 0.f;
    for (int w = 0; w < DP_WARPS; ++w) o += ms[w] == -INFINITY ? 0.f : os[w][e] * exp2f(ms[w] - M);
    a.out[static_cast<long long>(blockIdx.x) * D + e] = n > 0 ? o / L : 0.f;
  }
  if (a.lse && threadIdx.x == 0) a.lse[blockIdx.x] = n > 0 ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

bool strides_ok(const int64_t* s, int d) {
  if (!s) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 1 || (s[i] & 7) || s[i] >= (1ll << 39)) return false;
  return s[2] >= d;
}

}  // namespace
}  // namespace snapkv

extern "C" size_t snapkv_decode_paged_workspace_size(int B, int Hq, int Hc, int d) {
  if (B < 1 || Hq < 1 || Hc < 1 || Hq % Hc != 0 || (d != 64 && d != 128)) return 0;
  return 256;
}

extern "C" snapkv_status_t snapkv_decode_paged(const void* q_cur, const void* k_pool, const void* v_pool,
                                               const int64_t* k_strides, const int64_t* v_strides,
                                               const int32_t* page_table, int pages_per_seq, int page_size,
                                               int num_pages, const int32_t* seq_lens, int B, int Hq, int Hc, int d,
                                               float* out, float* out_lse, void* workspace, size_t workspace_bytes,
                                               void* stream) {
  using namespace snapkv;
  if (B < 1 || Hq < 1 || Hc < 1 || Hq % Hc != 0 || d < 1 || pages_per_seq < 1 || page_size < 1 || num_pages < 1 ||
      page_size % 16 != 0)
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
  DecodePagedArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q_cur);
  a.k = static_cast<const __nv_bfloat16*>(k_pool);
  a.v = static_cast<const __nv_bfloat16*>(v_pool);
  for (int i = 0; i < 3; ++i) {
    a.kp[i] = k_strides[i];
    a.vp[i] = v_strides[i];
  }
  a.table = page_table, a.seq_lens = seq_lens;
  a.pages_per_seq = pages_per_seq, a.page_size = page_size, a.num_pages = num_pages;
  a.Hq = Hq, a.g = Hq / Hc;
  a.c2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(d)));
  a.out = out, a.lse = out_lse;
  const cudaError_t e = launch_pdl(d == 128 ? decode_paged_kernel<128> : decode_paged_kernel<64>, dim3(B * Hq),
                                   dim3(DP_WARPS * 32), 0, static_cast<cudaStream_t>(stream), a);
  return e == cudaSuccess ? SNAPKV_OK : SNAPKV_ERR_CUDA;
}
