// Attention of one new token per sequence over a paged cache (last_cache_attention).
//
// out = sum_p exp(z_p - m) v_p / sum_p exp(z_p - m), z_p = scale q.k_p, with the running
// maximum m of the keys seen so far: one pass over K and V.
#include <cuda_bf16.h>

#include "cache_internal.h"
#include "last_device.cuh"

namespace last {

namespace {

constexpr int kThreads = 128;
constexpr int kMaxDim = 256;

// One CTA per (sequence, q-head); each warp takes every fourth key, each lane eight
// coordinates, and the warps' sums are joined at the end.
template <typename T>
__global__ void __launch_bounds__(kThreads) attend_kernel(const __grid_constant__ AttendArgs p) {
  __shared__ float acc_s[kThreads / 32][kMaxDim], m_s[kThreads / 32], l_s[kThreads / 32];
  __shared__ unsigned flags;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.cache.dim;
  unsigned *status = reinterpret_cast<unsigned *>(p.ws);
  if (threadIdx.x == 0) flags = 0;
  const long long items = (long long)p.seq.batch * p.q_heads;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    __syncthreads();
    const int b = (int)(it / p.q_heads), h = (int)(it - (long long)b * p.q_heads);
    const int g = h / (p.q_heads / p.cache.heads);
    const long long room = (long long)p.seq.max_pages * p.cache.page_size;
    int end = p.seq.lens[b], begin = p.seq.begin ? p.seq.begin[b] : 0;
    if (end < 0 || begin < 0 || end > room) {
      if (threadIdx.x == 0) flags = kErrCacheIndex;
      end = end > room ? (int)room : end;
      begin = begin < 0 ? 0 : begin;
    }
    const T *q = reinterpret_cast<const T *>(p.q + b * p.q_stride) + (long long)h * D;
    float qv[kMaxDim / 32], o[kMaxDim / 32], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < kMaxDim / 32; ++e) {
      const int d = e * 32 + lane;
      qv[e] = d < D ? (float)q[d] : 0.0f;
      o[e] = 0.0f;
    }
    for (int i = begin + warp; i < end; i += kThreads / 32) {
      const int page = p.seq.table[b * p.seq.table_stride + i / p.cache.page_size];
      if (page < 0 || page >= p.cache.num_pages) {
        if (lane == 0) atomicOr(&flags, kErrCacheIndex);
        continue;
      }
      const long long at = page * p.cache.page_stride + g * p.cache.head_stride + (i % p.cache.page_size) * p.cache.token_stride;
      const T *k = reinterpret_cast<const T *>(p.cache.k + at), *v = reinterpret_cast<const T *>(p.cache.v + at);
      float z = 0.0f;
#pragma unroll
      for (int e = 0; e < kMaxDim / 32; ++e)
        if (e * 32 + lane < D) z = fmaf(qv[e], (float)k[e * 32 + lane], z);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(~0u, z, x);
      z *= p.scale;
      if (z == -INFINITY) continue;
      const float top = fmaxf(m, z), f = expf(m - top), w = expf(z - top);
      m = top;
      l = l * f + w;
#pragma unroll
      for (int e = 0; e < kMaxDim / 32; ++e)
        if (e * 32 + lane < D) o[e] = o[e] * f + w * (float)v[e * 32 + lane];
    }
    if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
    for (int e = 0; e < kMaxDim / 32; ++e) acc_s[warp][e * 32 + lane] = o[e];
    __syncthreads();
    float top = -INFINITY, total = 0.0f, f[kThreads / 32];
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, m_s[w]);
    for (int w = 0; w < kThreads / 32; ++w) {
      f[w] = m_s[w] == -INFINITY ? (l_s[w] == 0.0f ? 0.0f : l_s[w]) : expf(m_s[w] - top);
      total += l_s[w] * f[w];
    }
    T *out = reinterpret_cast<T *>(p.out + b * p.out_stride) + (long long)h * D;
    for (int d = threadIdx.x; d < D; d += kThreads) {
      float x = 0.0f;
      for (int w = 0; w < kThreads / 32; ++w) x += acc_s[w][d] * f[w];
      out[d] = (T)(total == 0.0f ? 0.0f : x / total);
    }
    if (p.lse != nullptr && threadIdx.x == 0) p.lse[(long long)b * p.q_heads + h] = logf(total) + (total == 0.0f ? 0.0f : top);
  }
  __syncthreads();
  if (threadIdx.x == 0) post_status(status, blockIdx.x, gridDim.x, flags);
}

}  // namespace

size_t attend_scratch_bytes(int, int, int, int) { return 0; }

cudaError_t launch_attend(const AttendArgs &a, cudaStream_t s) {
  const long long items = (long long)a.seq.batch * a.q_heads;
  const int grid = (int)(items < 1 ? 1 : items < kMaxStatus ? items : kMaxStatus);
  if (a.elem == 4) attend_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else attend_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace last
