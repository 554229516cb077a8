// Causal attention over a paged KV cache (kv_attend): a warp per row and head.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rs_internal.h"

namespace rs {

namespace {

template <class T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }

// One pass with the running maximum m, sum l and weighted values o of the
// softmax: a new score s moves m to m' = max(m, s) and scales l and o by
// exp(m - m').
template <class T, int D>
__global__ void __launch_bounds__(128) k_kv_attend_rows(KvAttendArgs a) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (w >= (int64_t)a.b.n_tokens * a.n_heads) return;
  const int r = (int)(w / a.n_heads), h = (int)(w - (int64_t)r * a.n_heads);
  const int kh = h / (a.n_heads / a.c.n_kv_heads);
  int req = -1, limit = 0;
  if (a.b.n_req > 0 && r < a.b.q_start[a.b.n_req]) {
    int lo = 0, hi = a.b.n_req;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.b.q_start[mid] <= r) lo = mid; else hi = mid;
    }
    req = lo;
    limit = min(a.b.kv_len[req] - (a.b.q_start[req + 1] - r) + 1, a.b.max_blocks * 16);
  }
  const T* q = static_cast<const T*>(a.q) + r * a.q_ts + h * a.q_hs;
  float qf[E], o[E];
#pragma unroll
  for (int e = 0; e < E; e++) { qf[e] = to_f(q[lane * E + e]) * a.scale; o[e] = 0.0f; }
  float m = -INFINITY, l = 0.0f;
  for (int j = 0; j < limit; j++) {
    const int id = a.b.table[(int64_t)req * a.b.table_stride + (j >> 4)];
    const bool in = id >= 0 && id < a.c.n_blocks;
    const int64_t off = id * a.c.stride_block + kh * a.c.stride_head + (j & 15) * a.c.stride_token + lane * E;
    float s = 0.0f;
    if (in)
#pragma unroll
      for (int e = 0; e < E; e++) s = fmaf(qf[e], to_f(static_cast<const T*>(a.c.k)[off + e]), s);
#pragma unroll
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(~0u, s, x);
    const float m2 = fmaxf(m, s), f = __expf(m - m2), p = __expf(s - m2);
    l = fmaf(l, f, p);
#pragma unroll
    for (int e = 0; e < E; e++) {
      const float v = in ? to_f(static_cast<const T*>(a.c.v)[off + e]) : 0.0f;
      o[e] = fmaf(o[e], f, p * v);
    }
    m = m2;
  }
  T* out = static_cast<T*>(a.out) + r * a.o_ts + h * a.o_hs;
#pragma unroll
  for (int e = 0; e < E; e++) out[lane * E + e] = from_f<T>(limit > 0 ? o[e] / l : 0.0f);
  if (a.lse && lane == 0) a.lse[w] = limit > 0 ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_kv_attend(const KvAttendArgs& a, cudaStream_t st) {
  const int64_t grid = ((int64_t)a.b.n_tokens * a.n_heads + 3) / 4;
  const bool h = a.c.dtype == RS_FP16;
  if (a.c.head_dim == 64) {
    if (h) k_kv_attend_rows<__half, 64><<<(unsigned)grid, 128, 0, st>>>(a);
    else k_kv_attend_rows<__nv_bfloat16, 64><<<(unsigned)grid, 128, 0, st>>>(a);
  } else {
    if (h) k_kv_attend_rows<__half, 128><<<(unsigned)grid, 128, 0, st>>>(a);
    else k_kv_attend_rows<__nv_bfloat16, 128><<<(unsigned)grid, 128, 0, st>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace rs
