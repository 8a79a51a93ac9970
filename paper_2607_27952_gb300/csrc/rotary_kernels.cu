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
constexpr int kBatch = 4;        // items of a lane in flight

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

// x / n for x n < 2^32, with m = ceil(2^32 / n).
__device__ __forceinline__ int quotient(int x, int n, uint32_t m) {
  return n == 1 ? x : (int)__umulhi((uint32_t)x, m);
}
uint32_t magic(int n) { return (uint32_t)(((1ull << 32) + (unsigned)n - 1) / (unsigned)(n > 0 ? n : 1)); }

struct Split {       // of a token's work
  int parts;         // warps per token
  int rounds;        // of 32 items (pairs of VEC-element pieces) per part
  int chunks, tail;  // items and single pieces behind them of a row
  uint32_t chunks_m, tail_m;
};

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

// A warp takes a token (or, of few tokens, a part of its rows) at a time.  Its lanes turn VEC pairs of a row
// in each round and load those of the fourth round from there, of the next token if need be, so that loads
// are always under way; the sines and cosines of a token lie in the warp's own shared memory, and warps do
// not wait for each other.  Rows are q's, k's and, for a cache, v's heads, which are copied.
template <typename T, int VEC, bool ADJACENT, bool APPEND>
__global__ void __launch_bounds__(kThreads, 3) rotary_kernel(const __grid_constant__ RotaryArgs p, const Split w) {
  using V = typename Pack<VEC * (int)sizeof(T)>::type;
  constexpr int kSets = kMaxRotPairs / 32;
  __shared__ float2 tables[kThreads / 32][kMaxRotPairs];   // (cos, sin) of pair c VEC + e at [e chunks + c]
  __shared__ unsigned flags;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = p.rot.half, warps = gridDim.x * (kThreads / 32);
  const int turned = p.q.heads + p.k.heads, rows = turned + (APPEND ? p.v.heads : 0), items = rows * w.chunks;
  float2 *turn = tables[warp];
  if (APPEND) {
    if (threadIdx.x == 0) flags = 0;
    __syncthreads();
  }
  auto share = [&](int n, int part, int &i0, int &i1) {
    i0 = w.parts == 1 ? 0 : (int)((long long)n * part / w.parts);
    i1 = w.parts == 1 ? n : (int)((long long)n * (part + 1) / w.parts);
  };
  auto row_in = [&](int t, int h) -> const char * {
    if (h < p.q.heads) return p.q.in + t * p.q.in_token + h * p.q.in_head;
    if (!APPEND || h < turned) return p.k.in + t * p.k.in_token + (h - p.q.heads) * p.k.in_head;
    return p.v.in + t * p.v.in_token + (h - turned) * p.v.in_head;
  };
  // a lane's frequencies, read once: lanes reading parameters at different places do so one by one
  unsigned long long freq[kSets];
  uint32_t axes = 0;
#pragma unroll
  for (int n = 0; n < kSets; ++n) {
    const int i = lane + 32 * n;
    freq[n] = i < half ? p.rot.turn[i] : 0;
    axes |= i < half ? (uint32_t)p.rot.axis[i] << (8 * n) : 0u;
  }

  const int units = p.tokens * w.parts;
  int load_unit = blockIdx.x * (kThreads / 32) + warp, load_round = 0;
  V a[kBatch], b[kBatch];
  auto load = [&](int n) {   // the next round's items
    if (load_unit >= units) return;
    const int t = w.parts == 1 ? load_unit : load_unit / w.parts;
    int i0, i1;
    share(items, load_unit - t * w.parts, i0, i1);
    const int i = i0 + load_round * 32 + lane;
    if (i < i1) {
      const int h = quotient(i, w.chunks, w.chunks_m), c = i - h * w.chunks;
      const T *x = reinterpret_cast<const T *>(row_in(t, h)) + (ADJACENT ? 2 * c : c) * VEC;
      a[n] = *reinterpret_cast<const V *>(x);
      b[n] = *reinterpret_cast<const V *>(x + (ADJACENT ? VEC : half));
    }
    if (++load_round == w.rounds) {
      load_round = 0;
      load_unit += warps;
    }
  };
#pragma unroll
  for (int n = 0; n < kBatch; ++n) load(n);

  int unit = blockIdx.x * (kThreads / 32) + warp, round = 0, t = 0, i0 = 0, i1 = 0;
  long long slot = 0;
  while (unit < units) {
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (unit >= units) break;
      if (round == 0) {   // a new token
        t = w.parts == 1 ? unit : unit / w.parts;
        share(items, unit - t * w.parts, i0, i1);
        __syncwarp();
#pragma unroll
        for (int m = 0; m < kSets; ++m) {
          const int i = lane + 32 * m;
          if (i >= half) break;
          const long long at = p.positions[(long long)(axes >> (8 * m) & 255) * p.axis_stride + t];
          const long long phase = (long long)((unsigned long long)at * freq[m]);
          float sn, cs;
          sincospif((float)phase * 0x1p-63f, &sn, &cs);   // phase: 2^-64 turns
          turn[(i % VEC) * w.chunks + i / VEC] = make_float2(cs, p.backward ? -sn : sn);
        }
        if (APPEND) {
          unsigned bad = 0;
          slot = slot_of(p, t, &bad);
          if (bad && lane == 0) atomicOr(&flags, bad);
        }
        __syncwarp();
      }
      auto row_out = [&](int h) -> char * {
        if (h < p.q.heads) return p.q.out + t * p.q.out_token + h * p.q.out_head;
        if (!APPEND) return p.k.out + t * p.k.out_token + (h - p.q.heads) * p.k.out_head;
        if (slot < 0) return nullptr;
        return h < turned ? p.cache.k + slot + (h - p.q.heads) * p.cache.head_stride
                          : p.cache.v + slot + (h - turned) * p.cache.head_stride;
      };
      const int i = i0 + round * 32 + lane;
      if (i < i1) {
        const int h = quotient(i, w.chunks, w.chunks_m), c = i - h * w.chunks;
        char *y = row_out(h);
        V va = a[n], vb = b[n];
        if (!APPEND || h < turned) {
          T ea[VEC], eb[VEC];
          memcpy(ea, &va, sizeof(V));
          memcpy(eb, &vb, sizeof(V));
          if (!ADJACENT || VEC == 1) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const float2 cs = turn[e * w.chunks + c];
              const float x0 = to_f32(ea[e]), x1 = to_f32(eb[e]);
              ea[e] = from_f32<T>(x0 * cs.x - x1 * cs.y);
              eb[e] = from_f32<T>(x0 * cs.y + x1 * cs.x);
            }
          } else {
#pragma unroll
            for (int e = 0; e + 1 < VEC; e += 2) {
              const float2 w0 = turn[e / 2 * w.chunks + c], w1 = turn[(VEC / 2 + e / 2) * w.chunks + c];
              const float x0 = to_f32(ea[e]), x1 = to_f32(ea[e + 1]), z0 = to_f32(eb[e]), z1 = to_f32(eb[e + 1]);
              ea[e] = from_f32<T>(x0 * w0.x - x1 * w0.y);
              ea[e + 1] = from_f32<T>(x0 * w0.y + x1 * w0.x);
              eb[e] = from_f32<T>(z0 * w1.x - z1 * w1.y);
              eb[e + 1] = from_f32<T>(z0 * w1.y + z1 * w1.x);
            }
          }
          memcpy(&va, ea, sizeof(V));
          memcpy(&vb, eb, sizeof(V));
        }
        if (!APPEND || y != nullptr) {
          T *to = reinterpret_cast<T *>(y) + (ADJACENT ? 2 * c : c) * VEC;
          *reinterpret_cast<V *>(to) = va;
          *reinterpret_cast<V *>(to + (ADJACENT ? VEC : half)) = vb;
        }
      }
      load(n);
      if (++round >= w.rounds) {
        if (w.tail > 0) {   // elements past the rotated ones are copied
          int j0, j1;
          share(rows * w.tail, unit - t * w.parts, j0, j1);
          for (int j = j0 + lane; j < j1; j += 32) {
            const int h = quotient(j, w.tail, w.tail_m), e = 2 * half + (j - h * w.tail) * VEC;
            char *y = row_out(h);
            if (y != nullptr)
              *reinterpret_cast<V *>(y + e * sizeof(T)) = *reinterpret_cast<const V *>(row_in(t, h) + e * sizeof(T));
          }
        }
        round = 0;
        unit += warps;
      }
    }
  }
  if (APPEND) {
    __syncthreads();
    if (threadIdx.x == 0) post_status(p.status, blockIdx.x, gridDim.x, flags);
  }
}

bool rows_aligned(const HeadRows &h, int bytes, bool out) {
  auto ok = [&](long long v) { return v % bytes == 0; };
  return h.heads == 0 ||
         (ok((long long)reinterpret_cast<uintptr_t>(h.in)) && ok(h.in_token) && ok(h.in_head) &&
          (!out || (ok((long long)reinterpret_cast<uintptr_t>(h.out)) && ok(h.out_token) && ok(h.out_head))));
}

template <typename T, int VEC>
void launch(const RotaryArgs &a, int grid, const Split &w, cudaStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, kThreads, 0, s>>>(a, w); };
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
                     !rows_aligned(a.k, vec * a.elem, !a.append) || !rows_aligned(a.v, vec * a.elem, false)))
    vec /= 2;
  Split w;
  w.chunks = a.rot.half / vec;
  w.tail = (a.dim - 2 * a.rot.half) / vec;
  w.chunks_m = magic(w.chunks);
  w.tail_m = magic(w.tail);
  // one warp a token, or as many as leave each one a round, where the SMs would not have eight each
  const int rows = a.q.heads + a.k.heads + a.v.heads, items = rows * (w.chunks > w.tail ? w.chunks : w.tail);
  const int sms = sm_count(), most = items > 32 ? items / 32 : 1;
  w.parts = a.tokens > 0 && a.tokens < sms * 8 ? sms * 8 / a.tokens : 1;
  if (w.parts > most) w.parts = most;
  w.rounds = ((rows * w.chunks + w.parts - 1) / w.parts + 31) / 32;
  const long long units = (long long)a.tokens * w.parts, per = kThreads / 32;
  long long grid = (units + per - 1) / per;
  if (grid > sms * 3) grid = sms * 3;
  if (a.append && grid > kMaxStatus) grid = kMaxStatus;   // a status word each
  if (grid < 1) grid = 1;
  const int g = (int)grid;
  if (a.elem == 4) {
    vec == 4 ? launch<float, 4>(a, g, w, s) : vec == 2 ? launch<float, 2>(a, g, w, s) : launch<float, 1>(a, g, w, s);
  } else {
    using B = __nv_bfloat16;
    vec == 8 ? launch<B, 8>(a, g, w, s) : vec == 4 ? launch<B, 4>(a, g, w, s)
    : vec == 2 ? launch<B, 2>(a, g, w, s) : launch<B, 1>(a, g, w, s);
  }
  return cudaGetLastError();
}

}  // namespace last
