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
constexpr int kCtas = 2;         // per SM, at up to 128 registers: 3 and 4 spill (215 and 405 us against 189 for
                                 // 94208 tokens of 24 heads)

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

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\t"
      "mov.b64 {%0, %1}, z;\n\t}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
template <typename T> __device__ __forceinline__ float2 get2(const T *x);
template <> __device__ __forceinline__ float2 get2(const float *x) { return make_float2(x[0], x[1]); }
template <> __device__ __forceinline__ float2 get2(const __nv_bfloat16 *x) {
  uint32_t v;
  memcpy(&v, x, 4);
  return make_float2(bf16lo(v), bf16hi(v));
}
template <typename T> __device__ __forceinline__ void set2(T *x, float2 v);
template <> __device__ __forceinline__ void set2(float *x, float2 v) { x[0] = v.x; x[1] = v.y; }
template <> __device__ __forceinline__ void set2(__nv_bfloat16 *x, float2 v) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v.y), "f"(v.x));
  memcpy(x, &r, 4);
}

// A row's items (pairs of VEC-element pieces, the first `turned` of them rotated, the others copied) lie side
// by side in a warp, `heads` rows at a time.
struct Split {
  int parts;            // warps per token
  int items, turned;    // of a row
  int columns;          // passes over rows of more than 32 items
  int heads;
  bool tail;            // one piece is left behind the items
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

// The cosines and sines of a lane's VEC pairs.
template <int VEC, bool ADJACENT> struct Turns {
  static constexpr bool kPacked = !ADJACENT && VEC > 1;
  float2 c[VEC > 1 ? VEC / 2 : 1], s[VEC > 1 ? VEC / 2 : 1];   // of two pairs; adjacent: pairs e < VEC / 2 and the rest
  __device__ __forceinline__ void load(const float *table, int items, int column) {
    if constexpr (kPacked) {
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const float4 x = reinterpret_cast<const float4 *>(table)[e * items + column];
        c[e] = make_float2(x.x, x.y);
        s[e] = make_float2(x.z, x.w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < (VEC > 1 ? VEC / 2 : 1); ++e) {
        const float2 x = reinterpret_cast<const float2 *>(table)[e * items + column];
        const float2 y = VEC > 1 ? reinterpret_cast<const float2 *>(table)[(VEC / 2 + e) * items + column] : x;
        c[e] = make_float2(x.x, y.x);
        s[e] = make_float2(x.y, y.y);
      }
    }
  }
  template <typename T> __device__ __forceinline__ void apply(T *a, T *b) const {
    if constexpr (kPacked) {
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const float2 x = get2(a + 2 * e), y = get2(b + 2 * e), ys = mul2(y, s[e]);
        set2(a + 2 * e, fma2(x, c[e], make_float2(-ys.x, -ys.y)));
        set2(b + 2 * e, fma2(x, s[e], mul2(y, c[e])));
      }
    } else if constexpr (VEC == 1) {
      const float x = to_f32(a[0]), y = to_f32(b[0]);
      a[0] = from_f32<T>(fmaf(x, c[0].x, -y * s[0].x));
      b[0] = from_f32<T>(fmaf(x, s[0].x, y * c[0].x));
    } else {
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const float2 x = get2(a + 2 * e), y = get2(b + 2 * e);
        set2(a + 2 * e, make_float2(fmaf(x.x, c[e].x, -x.y * s[e].x), fmaf(x.x, s[e].x, x.y * c[e].x)));
        set2(b + 2 * e, make_float2(fmaf(y.x, c[e].y, -y.y * s[e].y), fmaf(y.x, s[e].y, y.y * c[e].y)));
      }
    }
  }
};

// A warp takes a token, or, of few tokens, every `parts`-th group of its rows.  The first loads of all its
// tensors are under way while the token's sines and cosines go to the warp's own shared memory; from there
// each lane keeps those of its column for all heads.  Warps do not wait for each other.
// Bound by HBM: 16512 tokens of 20 heads by 128 in bf16 (169 MB) 29 us, 5.8 TB/s; appending 94208 tokens of 24 heads
// (1.16 GB) 186 us, 6.2 TB/s.  Sines and cosines read from shared memory for every head: 35 and 242 us.
template <typename T, int VEC, bool ADJACENT, bool APPEND>
__global__ void __launch_bounds__(kThreads, kCtas) rotary_kernel(const __grid_constant__ RotaryArgs p, const Split w) {
  using V = typename Pack<VEC * (int)sizeof(T)>::type;
  using R = Turns<VEC, ADJACENT>;
  // of pair c VEC + e: cosine and sine at [e turned + c], or, two pairs a time, both cosines and both sines at
  // [e / 2 turned + c]
  __shared__ alignas(16) float tables[kThreads / 32][2 * kMaxRotPairs];
  __shared__ unsigned long long freqs[kMaxRotPairs];
  __shared__ uint8_t axes[kMaxRotPairs];
  __shared__ unsigned flags;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = p.rot.half, warps = gridDim.x * (kThreads / 32);
  float *table = tables[warp];
  for (int i = threadIdx.x; i < half; i += kThreads) {
    // through memory addresses: a warp's lanes would read parameters at different places one by one
    const RotaryTable *rot = &p.rot;
    asm("mov.b64 %0, %0;" : "+l"(rot));
    freqs[i] = rot->turn[i];
    axes[i] = rot->axis[i];
  }
  if (APPEND && threadIdx.x == 0) flags = 0;
  __syncthreads();
  grid_begins();

  const bool across = w.columns > 1;
  const int width = max(w.items, 1), sub = across ? 0 : lane / width;   // row of the group
  const bool idle = sub >= w.heads;
  const int step = w.heads * w.parts, units = p.tokens * w.parts;
  for (int unit = blockIdx.x * (kThreads / 32) + warp; unit < units; unit += warps) {
    const int t = w.parts == 1 ? unit : unit / w.parts, first = sub + (unit - t * w.parts) * w.heads;
    long long slot = 0;
    for (int col = 0; col < w.columns; ++col) {
      const int c = across ? lane + 32 * col : lane - sub * width;
      const bool off = idle || c >= w.items, rotated = c < w.turned;
      // an item's first piece, and from there to its second
      const int at = (!rotated ? 2 * half + (c - w.turned) * 2 * VEC : ADJACENT ? 2 * c * VEC : c * VEC) * (int)sizeof(T);
      const int far = (rotated && !ADJACENT ? half : VEC) * (int)sizeof(T);
      const int nq = off || first >= p.q.heads ? 0 : (p.q.heads - first + step - 1) / step;
      const int nk = off || first >= p.k.heads ? 0 : (p.k.heads - first + step - 1) / step;
      const char *q = p.q.in + t * p.q.in_token + first * p.q.in_head + at, *k = p.k.in + t * p.k.in_token + first * p.k.in_head + at;
      const char *v = APPEND ? p.v.in + t * p.v.in_token + first * p.v.in_head + at : nullptr;
      const long long q_step = step * p.q.in_head, k_step = step * p.k.in_head, v_step = step * p.v.in_head;
      V a[kBatch], b[kBatch], ka, kb, va, vb;
      auto load_q = [&](int r) {
#pragma unroll
        for (int n = 0; n < kBatch; ++n)
          if (r + n < nq) {
            a[n] = *reinterpret_cast<const V *>(q + n * q_step);
            b[n] = *reinterpret_cast<const V *>(q + n * q_step + far);
          }
        q += kBatch * q_step;
      };
      load_q(0);
      if (nk > 0) {
        ka = *reinterpret_cast<const V *>(k);
        kb = *reinterpret_cast<const V *>(k + far);
        if (APPEND) {
          va = *reinterpret_cast<const V *>(v);
          vb = *reinterpret_cast<const V *>(v + far);
        }
      }
      if (col == 0) {   // the token's angles, and its slot
        __syncwarp();
        for (int i = lane; i < half; i += 32) {
          const long long phase = (long long)((unsigned long long)(long long)p.positions[axes[i] * p.axis_stride + t] * freqs[i]);
          float sn, cs;
          sincospif((float)phase * 0x1p-63f, &sn, &cs);   // phase: 2^-64 turns
          sn = p.backward ? -sn : sn;
          const int e = i % VEC, j = i / VEC;
          if (R::kPacked) {
            float *to = table + ((e / 2) * w.turned + j) * 4 + (e & 1);
            to[0] = cs;
            to[2] = sn;
          } else {
            *reinterpret_cast<float2 *>(table + (e * w.turned + j) * 2) = make_float2(cs, sn);
          }
        }
        if (APPEND) {
          unsigned bad = 0;
          slot = slot_of(p, t, &bad);
          if (bad && lane == 0) atomicOr(&flags, bad);
        }
        __syncwarp();
      }
      R turns;
      if (!off && rotated) turns.load(table, w.turned, c);
      auto turn = [&](V &x, V &y) {
        if (!rotated) return;
        T ex[VEC], ey[VEC];
        memcpy(ex, &x, sizeof(V));
        memcpy(ey, &y, sizeof(V));
        turns.apply(ex, ey);
        memcpy(&x, ex, sizeof(V));
        memcpy(&y, ey, sizeof(V));
      };
      char *qo = p.q.out + t * p.q.out_token + first * p.q.out_head + at;
      const long long qo_step = step * p.q.out_head;
      for (int r = 0; r < nq; r += kBatch) {
        if (r > 0) load_q(r);
#pragma unroll
        for (int n = 0; n < kBatch; ++n)
          if (r + n < nq) {
            turn(a[n], b[n]);
            *reinterpret_cast<V *>(qo + n * qo_step) = a[n];
            *reinterpret_cast<V *>(qo + n * qo_step + far) = b[n];
          }
        qo += kBatch * qo_step;
      }
      if (APPEND && slot < 0) continue;
      char *ko = APPEND ? p.cache.k + slot + first * p.cache.head_stride + at : p.k.out + t * p.k.out_token + first * p.k.out_head + at;
      char *vo = APPEND ? p.cache.v + slot + first * p.cache.head_stride + at : nullptr;
      const long long ko_step = step * (APPEND ? p.cache.head_stride : p.k.out_head);
      for (int r = 0; r < nk; ++r) {
        if (r > 0) {
          k += k_step;
          ka = *reinterpret_cast<const V *>(k);
          kb = *reinterpret_cast<const V *>(k + far);
          if (APPEND) {
            v += v_step;
            va = *reinterpret_cast<const V *>(v);
            vb = *reinterpret_cast<const V *>(v + far);
          }
        }
        turn(ka, kb);
        *reinterpret_cast<V *>(ko) = ka;
        *reinterpret_cast<V *>(ko + far) = kb;
        ko += ko_step;
        if (APPEND) {
          *reinterpret_cast<V *>(vo) = va;
          *reinterpret_cast<V *>(vo + far) = vb;
          vo += ko_step;
        }
      }
    }
    if (w.tail && unit - t * w.parts == 0) {   // the piece that no item holds
      const int e = (p.dim - VEC) * (int)sizeof(T);
      auto copy = [&](const char *in, long long in_head, char *out, long long out_head, int heads) {
        for (int h = lane; h < heads; h += 32)
          *reinterpret_cast<V *>(out + h * out_head + e) = *reinterpret_cast<const V *>(in + h * in_head + e);
      };
      copy(p.q.in + t * p.q.in_token, p.q.in_head, p.q.out + t * p.q.out_token, p.q.out_head, p.q.heads);
      if (!APPEND) copy(p.k.in + t * p.k.in_token, p.k.in_head, p.k.out + t * p.k.out_token, p.k.out_head, p.k.heads);
      if (APPEND && slot >= 0) {
        copy(p.k.in + t * p.k.in_token, p.k.in_head, p.cache.k + slot, p.cache.head_stride, p.k.heads);
        copy(p.v.in + t * p.v.in_token, p.v.in_head, p.cache.v + slot, p.cache.head_stride, p.v.heads);
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
cudaError_t launch(const RotaryArgs &a, int grid, const Split &w, cudaStream_t s) {
  auto go = [&](auto kernel) { return launch_early(kernel, dim3(grid), kThreads, 0, s, a, w); };
  if (a.rot.adjacent)
    return a.append ? go(rotary_kernel<T, VEC, true, true>) : go(rotary_kernel<T, VEC, true, false>);
  return a.append ? go(rotary_kernel<T, VEC, false, true>) : go(rotary_kernel<T, VEC, false, false>);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t s) {
  // the widest vector that every row's parts are whole numbers of, up to 16 bytes
  int vec = 16 / a.elem;
  while (vec > 1 && (a.rot.half % vec != 0 || a.dim % vec != 0 || !rows_aligned(a.q, vec * a.elem, true) ||
                     !rows_aligned(a.k, vec * a.elem, !a.append) || !rows_aligned(a.v, vec * a.elem, false)))
    vec /= 2;
  Split w;
  w.turned = a.rot.half / vec;
  w.items = w.turned + (a.dim - 2 * a.rot.half) / (2 * vec);
  w.tail = (a.dim - 2 * a.rot.half) / vec % 2 != 0;
  w.columns = w.items > 32 ? (w.items + 31) / 32 : 1;
  w.heads = w.columns > 1 ? 1 : w.items > 0 ? 32 / w.items : 32;
  // Parts of a token per warp: the fewest rounds on the busiest warp, its angles (and slot) taken for two
  const int sms = sm_count(), warps = sms * kCtas * (kThreads / 32);
  auto rounds = [&](int heads, int parts) { return (heads + w.heads * parts - 1) / (w.heads * parts); };
  const int most = rounds(a.q.heads > a.k.heads ? a.q.heads : a.k.heads, 1);
  w.parts = 1;
  long long best = -1;
  for (int parts = 1; parts <= most && parts <= 32; ++parts) {
    const int work = rounds(a.q.heads, parts) + rounds(a.k.heads, parts) + rounds(a.v.heads, parts);
    const long long cost = ((long long)a.tokens * parts + warps - 1) / warps * (w.columns * work + 2);
    if (best < 0 || cost < best) {
      best = cost;
      w.parts = parts;
    }
  }
  const long long units = (long long)a.tokens * w.parts, per = kThreads / 32;
  long long grid = (units + per - 1) / per;
  if (grid > sms * kCtas) grid = sms * kCtas;
  if (a.append && grid > kMaxStatus) grid = kMaxStatus;   // a status word each
  if (grid < 1) grid = 1;
  const int g = (int)grid;
  if (a.elem == 4)
    return vec == 4 ? launch<float, 4>(a, g, w, s) : vec == 2 ? launch<float, 2>(a, g, w, s) : launch<float, 1>(a, g, w, s);
  using B = __nv_bfloat16;
  return vec == 8 ? launch<B, 8>(a, g, w, s) : vec == 4 ? launch<B, 4>(a, g, w, s)
         : vec == 2 ? launch<B, 2>(a, g, w, s) : launch<B, 1>(a, g, w, s);
}

}  // namespace last
