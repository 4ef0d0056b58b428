// Appending to a paged cache with the position rotation on the way.  Pair r of a head turns by
// positions[t] * inv_freq[r]: (x, y) -> (x cos - y sin, x sin + y cos).
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

// The sequence of token t, its place in it and whether there is one.
__device__ __forceinline__ bool locate(const AppendArgs& a, int t, int* b, int* i) {
  if (!a.cu) {
    const int n = a.T / a.B;
    *b = t / n;
    *i = t - *b * n;
    return true;
  }
  if (t >= a.cu[a.B] || t < a.cu[0]) return false;
  int lo = 0, hi = a.B - 1;  // the last sequence that starts at or in front of t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  *b = lo;
  *i = t - a.cu[lo];
  return true;
}

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(AP_THREADS) append_kernel(const AppendArgs a) {
  __shared__ float cs[D / 2], sn[D / 2];
  pdl_wait();
  const int t = blockIdx.x;
  int b, i;
  if (!locate(a, t, &b, &i)) return;
  const long long slot = static_cast<long long>(a.cache_lens[b]) + i;
  // Angles of far positions lose their fraction of a turn in 32 bits: 64 up to the reduction.
  for (int r = threadIdx.x; r < a.half; r += AP_THREADS) {
    const double angle = static_cast<double>(a.positions ? a.positions[t] : slot) * a.inv_freq[r];
    const double turns = angle * 0.15915494309189535;  // 1 / (2 pi)
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &sn[r], &cs[r]);
  }
  __syncthreads();
  uint16_t *kd = nullptr, *vd = nullptr;
  if (slot >= 0 && slot < static_cast<long long>(a.pages_per_seq) * a.page_size) {
    const int pg = static_cast<int>(slot / a.page_size), row = static_cast<int>(slot - static_cast<long long>(pg) * a.page_size);
    const int page = a.table[static_cast<long long>(b) * a.pages_per_seq + pg];
    if (page >= 0 && page < a.num_pages) {
      kd = a.k_pool + page * a.kp[0] + row * a.kp[2];
      vd = a.v_pool + page * a.vp[0] + row * a.vp[2];
    }
  }
  const long long at = a.cu ? t : i, seq = a.cu ? 0 : b;
  const uint16_t* ks = a.k + seq * a.k_st[0] + at * a.k_st[1];
  const uint16_t* vs = a.v + seq * a.v_st[0] + at * a.v_st[1];
  const uint16_t* qs = a.q ? a.q + seq * a.q_st[0] + at * a.q_st[1] : nullptr;
  auto turned = [&](const uint16_t* x, int c) {  // element c of a rotated head
    const float self = __uint_as_float(static_cast<uint32_t>(x[c]) << 16);
    if (c >= 2 * a.half) return x[c];
    const int r = INTERLEAVED ? c >> 1 : (c < a.half ? c : c - a.half);
    const bool first = INTERLEAVED ? !(c & 1) : c < a.half;
    const int oc = INTERLEAVED ? c ^ 1 : (first ? c + a.half : c - a.half);
    const float other = __uint_as_float(static_cast<uint32_t>(x[oc]) << 16);
    const __nv_bfloat16 y = __float2bfloat16(first ? self * cs[r] - other * sn[r] : other * sn[r] + self * cs[r]);
    return __bfloat16_as_ushort(y);
  };
  const int reps = a.Hc / a.Hkv;
  if (kd)
    for (int e = threadIdx.x; e < a.Hkv * D; e += AP_THREADS) {
      const int h = e / D, c = e % D;
      const uint16_t x = turned(ks + h * a.k_st[2], c), y = vs[h * a.v_st[2] + c];
      for (int m = 0; m < reps; ++m) {
        kd[(h * reps + m) * a.kp[1] + c] = x;
        vd[(h * reps + m) * a.vp[1] + c] = y;
      }
    }
  if (qs)
    for (int e = threadIdx.x; e < a.Hq * D; e += AP_THREADS)
      a.q_out[static_cast<long long>(t) * a.Hq * D + e] = turned(qs + e / D * a.q_st[2], e % D);
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
  if (d != 64 && d != 128) return SNAPKV_ERR_UNSUPPORTED;
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
  auto kernel = d == 128 ? (interleaved ? append_kernel<128, true> : append_kernel<128, false>)
                         : (interleaved ? append_kernel<64, true> : append_kernel<64, false>);
  const cudaError_t e = launch_pdl(kernel, dim3(T), dim3(AP_THREADS), 0, static_cast<cudaStream_t>(stream), a);
  return e == cudaSuccess ? SNAPKV_OK : SNAPKV_ERR_CUDA;
}
