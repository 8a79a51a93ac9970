// Rotary positions with several axes, on heads in memory (last_rope, last_rope_backward) and
// on the way into a paged cache (last_cache_append).
//
// Pair (a, b) of token t, frequency i, becomes (a cos phi - b sin phi, a sin phi + b cos phi)
// with phi = pos[axis(i)][t] * f_i.  The angle is formed in turns: pos * (f_i / 2 pi) as a
// 64-bit fixed-point product wraps modulo one turn exactly, so that no position, however
// long, loses bits of phi; one sine and cosine serve all heads of the token.
#include <cuda_bf16.h>

#include <cstring>

#include "cache_internal.h"
#include "last_device.cuh"

namespace last {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;        // loads a thread has in flight
constexpr int kMaxTokens = 16;   // per CTA

template <int BYTES> struct Pack;
template <> struct Pack<16> { using type = uint4; };
template <> struct Pack<8> { using type = uint2; };
template <> struct Pack<4> { using type = uint32_t; };
template <> struct Pack<2> { using type = uint16_t; };

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

// x / n for 0 <= x < 2^17, 1 <= n <= 2^14, with m = ceil(2^32 / n).
__device__ __forceinline__ int quotient(int x, int n, uint32_t m) {
  return n == 1 ? x : (int)__umulhi((uint32_t)x, m);
}

// Byte offset of new token t's slot in its cache layer; -1 (and a flag) if it has none.
__device__ long long slot_of(const RotaryArgs &p, int t, unsigned *bad) {
  int b = t, behind = 1;   // tokens from t to the end of its sequence
  if (p.cu_new != nullptr) {
    int lo = 0, hi = p.seq.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.cu_new[mid] <= t) lo = mid; else hi = mid - 1;
    }
    b = lo;
    const int first = p.cu_new[b], end = p.cu_new[b + 1];
    behind = end > t && first <= t ? end - t : 0;
  }
  const long long at = (long long)p.seq.lens[b] - behind;
  if (behind > 0 && at >= 0 && at < (long long)p.seq.max_pages * p.cache.page_size) {
    const int i = (int)(at / p.cache.page_size);
    const int page = p.seq.table[b * p.seq.table_stride + i];
    if (page >= 0 && page < p.cache.num_pages)
      return page * p.cache.page_stride + (at - (long long)i * p.cache.page_size) * p.cache.token_stride;
  }
  *bad = kErrCacheIndex;
  return -1;
}

// Heads of a few tokens per CTA: the angles' sines and cosines go to shared memory while
// the first loads are under way, then every thread turns VEC pairs of one row at a time.
template <typename T, int VEC, bool ADJACENT, bool APPEND>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryArgs p, int per_cta, uint32_t rows_m,
                                                          uint32_t kv_m, bool wide) {
  using V = typename Pack<VEC * (int)sizeof(T)>::type;
  __shared__ float2 turn[kMaxTokens * kMaxRotPairs];   // (cos, sin) [token][pair]
  __shared__ long long slot[kMaxTokens];
  __shared__ unsigned flags;
  const int tid = threadIdx.x, half = p.rot.half, heads = p.q.heads + p.k.heads;
  if (APPEND && tid == 0) flags = 0;
  const int chunks = half / VEC;   // of a row, side by side in a warp
  const int c = chunks > 0 ? tid % chunks : 0, pass = chunks > 0 ? kThreads / chunks : 1;
  const int first = chunks > 0 ? tid / chunks : 0;
  const int ia = (ADJACENT ? 2 * c : c) * VEC, ib = ADJACENT ? ia + VEC : half + ia;   // elements
  const int groups = (p.tokens + per_cta - 1) / per_cta;

  for (int g = blockIdx.x; g < groups; g += gridDim.x) {
    const int t0 = g * per_cta, nt = min(per_cta, p.tokens - t0);
    // rows: the rotated heads of the tokens, token-major
    const int rows = first < pass && chunks > 0 ? nt * heads : 0;
    auto row_in = [&](int t, int h) -> const char * {
      return h < p.q.heads ? p.q.in + (t0 + t) * p.q.in_token + h * p.q.in_head
                           : p.k.in + (t0 + t) * p.k.in_token + (h - p.q.heads) * p.k.in_head;
    };
    V a[kBatch], b[kBatch];
    auto load = [&](int at) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int r = at + u * pass;
        if (r < rows) {
          const int t = quotient(r, heads, rows_m);
          const char *x = row_in(t, r - t * heads);
          a[u] = *reinterpret_cast<const V *>(x + ia * sizeof(T));
          b[u] = *reinterpret_cast<const V *>(x + ib * sizeof(T));
        }
      }
    };
    load(first);

    __syncthreads();   // the previous tokens' angles and slots are read, flags is zero
    if (half > 0) {
      const int lanes = kThreads / half, i = tid % half;
      if (tid / half < lanes) {
        const unsigned long long f = p.rot.turn[i];
        const int32_t *pos = p.positions + p.rot.axis[i] * p.axis_stride + t0;
        for (int t = tid / half; t < nt; t += lanes) {
          const long long phase = (long long)((unsigned long long)(long long)pos[t] * f);
          float sn, cs;
          sincospif((float)phase * 0x1p-63f, &sn, &cs);   // phase: 2^-64 turns
          turn[t * half + i] = make_float2(cs, p.backward ? -sn : sn);
        }
      }
    }
    if (APPEND && tid < nt) {
      unsigned bad = 0;
      slot[tid] = slot_of(p, t0 + tid, &bad);
      if (bad) atomicOr(&flags, bad);
    }
    __syncthreads();

    auto row_out = [&](int t, int h) -> char * {
      if (h < p.q.heads) return p.q.out + (t0 + t) * p.q.out_token + h * p.q.out_head;
      if (!APPEND) return p.k.out + (t0 + t) * p.k.out_token + (h - p.q.heads) * p.k.out_head;
      return slot[t] < 0 ? nullptr : p.cache.k + slot[t] + (h - p.q.heads) * p.cache.head_stride;
    };
    for (int base = first; base < rows; base += pass * kBatch) {
      if (base != first) load(base);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int r = base + u * pass;
        if (r >= rows) break;
        const int t = quotient(r, heads, rows_m);
        char *y = row_out(t, r - t * heads);
        T ea[VEC], eb[VEC];
        memcpy(ea, &a[u], sizeof(V));
        memcpy(eb, &b[u], sizeof(V));
        const float2 *cs = turn + t * half + c * VEC;
        if (!ADJACENT || VEC == 1) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float x0 = to_f32(ea[e]), x1 = to_f32(eb[e]);
            ea[e] = from_f32<T>(x0 * cs[e].x - x1 * cs[e].y);
            eb[e] = from_f32<T>(x0 * cs[e].y + x1 * cs[e].x);
          }
        } else {
#pragma unroll
          for (int e = 0; e + 1 < VEC; e += 2) {
            const float2 w0 = cs[e / 2], w1 = cs[VEC / 2 + e / 2];
            const float x0 = to_f32(ea[e]), x1 = to_f32(ea[e + 1]), z0 = to_f32(eb[e]), z1 = to_f32(eb[e + 1]);
            ea[e] = from_f32<T>(x0 * w0.x - x1 * w0.y);
            ea[e + 1] = from_f32<T>(x0 * w0.y + x1 * w0.x);
            eb[e] = from_f32<T>(z0 * w1.x - z1 * w1.y);
            eb[e + 1] = from_f32<T>(z0 * w1.y + z1 * w1.x);
          }
        }
        if (y != nullptr) {
          V va, vb;
          memcpy(&va, ea, sizeof(V));
          memcpy(&vb, eb, sizeof(V));
          *reinterpret_cast<V *>(y + ia * sizeof(T)) = va;
          *reinterpret_cast<V *>(y + ib * sizeof(T)) = vb;
        }
      }
    }

    // elements past the rotated ones are copied
    const int tail = (p.dim - 2 * half) / VEC;
    for (int i = tid; i < nt * heads * tail; i += kThreads) {
      const int r = i / tail, e = 2 * half + (i - r * tail) * VEC;
      const int t = quotient(r, heads, rows_m), h = r - t * heads;
      char *y = row_out(t, h);
      if (y != nullptr)
        *reinterpret_cast<V *>(y + e * sizeof(T)) = *reinterpret_cast<const V *>(row_in(t, h) + e * sizeof(T));
    }
    if (APPEND) {   // V, in 16-byte pieces where its alignment allows
      auto copy_v = [&](auto piece) {
        using P = decltype(piece);
        const int n = p.dim * (int)sizeof(T) / (int)sizeof(P);
        for (int i = tid; i < nt * p.v.heads * n; i += kThreads) {
          const int r = i / n, t = quotient(r, p.v.heads, kv_m), h = r - t * p.v.heads;
          if (slot[t] >= 0)
            reinterpret_cast<P *>(p.cache.v + slot[t] + h * p.cache.head_stride)[i - r * n] =
                reinterpret_cast<const P *>(p.v.in + (t0 + t) * p.v.in_token + h * p.v.in_head)[i - r * n];
        }
      };
      if (wide) copy_v(uint4{});
      else copy_v(typename Pack<sizeof(T)>::type{});
    }
  }
  if (APPEND) {
    __syncthreads();
    if (tid == 0) post_status(p.status, blockIdx.x, gridDim.x, flags);
  }
}

bool rows_aligned(const HeadRows &h, int bytes, bool out) {
  auto ok = [&](long long v) { return v % bytes == 0; };
  return h.heads == 0 ||
         (ok((long long)reinterpret_cast<uintptr_t>(h.in)) && ok(h.in_token) && ok(h.in_head) &&
          (!out || (ok((long long)reinterpret_cast<uintptr_t>(h.out)) && ok(h.out_token) && ok(h.out_head))));
}

template <typename T, int VEC>
void launch(const RotaryArgs &a, int grid, int per_cta, bool wide, cudaStream_t s) {
  auto magic = [](int n) { return (uint32_t)(((1ull << 32) + (unsigned)n - 1) / (unsigned)(n > 0 ? n : 1)); };
  const uint32_t rm = magic(a.q.heads + a.k.heads), km = magic(a.v.heads);
  auto go = [&](auto kernel) { kernel<<<grid, kThreads, 0, s>>>(a, per_cta, rm, km, wide); };
  if (a.rot.adjacent)
    a.append ? go(rotary_kernel<T, VEC, true, true>) : go(rotary_kernel<T, VEC, true, false>);
  else
    a.append ? go(rotary_kernel<T, VEC, false, true>) : go(rotary_kernel<T, VEC, false, false>);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t s) {
  // the widest vector that every row's parts are whole numbers of, up to 16 bytes
  int vec = 16 / a.elem;
  while (vec > 1 && (a.rot.half % vec != 0 || a.dim % vec != 0 || !rows_aligned(a.q, vec * a.elem, true) ||
                     !rows_aligned(a.k, vec * a.elem, !a.append)))
    vec /= 2;
  const bool wide = a.append && rows_aligned(a.v, 16, false);
  // tokens per CTA: as many as its threads hold in one batch of loads, fewer where the GPU would not be full
  const int heads = a.q.heads + a.k.heads, chunks = a.rot.half / vec;
  int per = kThreads * kBatch / (heads * (chunks > 0 ? chunks : 1));
  per = per < 1 ? 1 : per > kMaxTokens ? kMaxTokens : per;
  const int sms = sm_count();
  while (per > 1 && (a.tokens + per - 1) / per < 2 * sms) --per;
  int grid = (a.tokens + per - 1) / per;
  if (a.append && grid > kMaxStatus) grid = kMaxStatus;   // a status word each
  if (grid < 1) grid = 1;
  if (a.elem == 4) {
    vec == 4 ? launch<float, 4>(a, grid, per, wide, s) : vec == 2 ? launch<float, 2>(a, grid, per, wide, s)
                                                                 : launch<float, 1>(a, grid, per, wide, s);
  } else {
    using B = __nv_bfloat16;
    vec == 8 ? launch<B, 8>(a, grid, per, wide, s) : vec == 4 ? launch<B, 4>(a, grid, per, wide, s)
    : vec == 2 ? launch<B, 2>(a, grid, per, wide, s) : launch<B, 1>(a, grid, per, wide, s);
  }
  return cudaGetLastError();
}

}  // namespace last
