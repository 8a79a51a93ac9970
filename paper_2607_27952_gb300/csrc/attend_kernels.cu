// Attention of one new token per sequence over a paged cache (last_cache_attention).
//
// With z_p = scale q.k_p in units of log 2 and the running maximum m of the keys seen so far,
//   l <- l 2^(m - m') + sum 2^(z_p - m'),  o <- o 2^(m - m') + sum 2^(z_p - m') v_p
// is one pass over K and V; sums over parts of the keys join by the same rule, so that the
// keys of all sequences and kv-heads are cut into equal shares, one per SM, wherever the
// cuts fall (join_kernel adds up what a cut has parted).  The work is reading K and V: each
// is read once for up to 16 query heads of its kv-head.
//
// A CTA: one warp keeps a ring of tiles filled with TMA boxes of the pages (128-byte swizzle),
// eight take quarters of every other tile, each with sums of its own, and add them up where
// the CTA's part of a (sequence, head) ends.
#include <cuda_bf16.h>

#include "cache_internal.h"
#include "last_device.cuh"
#include "last_internal.h"
#include "tensor_map.h"

namespace last {

namespace {

constexpr int kWarps = 8;                      // consumers
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kSlices = 4, kGroups = 2;        // quarters of a tile; warps by turns
constexpr int kRows = 16;                      // query heads of one pass over a kv-head
constexpr int kMaxWorkers = 256;
constexpr int kMaxStages = 12;
constexpr int kMergeRows = 8, kMergeCols = 128, kMergeLd = kMergeCols + 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct TileInfo {   // what the producer says of a tile
  int seq, head;    // head: pass over a kv-head
  int lo, hi;       // keys of the tile that count
  int flags;
};
// First and last tile of the CTA's part of a (sequence, head); the part is all of it; it is not the
// CTA's first one.
constexpr int kFirst = 1, kLast = 2, kWhole = 4, kLater = 8;
constexpr int kStatFloats = 2 * kRows;   // of a parted sum: maximum and denominator per head, then the rows

struct Shape {      // the same for every CTA
  AttendArgs a;
  int group, passes, heads;   // q-heads per kv-head, passes over a kv-head, passes in all
  int box, stages, chunks;    // rows of a TMA box; ring; 128-byte columns of a row
  int tile;                   // keys
  int rows;                   // heads of a pass at most
  float scale2;               // scale log2 e
  long long *first;           // [batch + 1] first tile of each sequence (in the workspace)
  float *parts;               // [workers][2] sums that a cut has parted
};

struct Shared {
  unsigned long long full[kMaxStages], empty[kMaxStages], sync, never;
  TileInfo info[kMaxStages];
  float top[kWarps][kRows], sum[kWarps][kRows], factor[kWarps][kRows], all[kRows], total[kRows];
  float merge[kWarps][kMergeRows][kMergeLd];
  long long warp_tiles[kWarps + 1], start_first;
  int start_seq;
  unsigned flags;
  volatile unsigned dead;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A whole warp waits, with a limit; the first to give up has every other wait of the CTA end too.
__device__ __forceinline__ bool wait(Shared &sm, unsigned long long *bar, uint32_t parity) {
  bool ok = false;
  for (uint32_t i = 0; i < kWaitLimit && !ok; ++i) {
    ok = mbar_try_wait(bar, parity);
    if ((i & 31) == 31 && sm.dead) break;
  }
  if (__all_sync(~0u, ok)) return true;
  sm.dead = 1;
  return false;
}

// The consumers' barrier (bounded, unlike a hardware one).
__device__ __forceinline__ bool consumers_sync(Shared &sm, uint32_t &parity) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(&sm.sync);
  parity ^= 1;
  return wait(sm, &sm.sync, parity ^ 1);
}

struct Keys {
  int begin, end;
};
__device__ __forceinline__ Keys keys_of(const AttendArgs &a, int b, unsigned *bad) {
  const long long room = (long long)a.seq.max_pages * a.cache.page_size;
  int end = a.seq.lens[b], begin = a.seq.begin ? a.seq.begin[b] : 0;
  if (end < 0 || end > room || begin < 0) *bad = kErrCacheIndex;
  end = end > room ? (int)room : end;
  begin = begin < 0 ? 0 : begin;
  return Keys{begin, end};
}
__device__ __forceinline__ int tiles_of(Keys k, int tile) {
  return k.begin < k.end ? (k.end - 1) / tile - k.begin / tile + 1 : 0;
}

// ---- consumers: bf16, on the tensor cores ----
// S = Q K^T with the heads as the 16 rows of an MMA, then O += P V.  With at most 8 heads rows 8..15
// are free and take what the cut of P to bf16 leaves out, so that P carries 16 bits for nothing;
// with more heads a second product adds it.
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two values rounded to bf16, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
// Two weights cut to bf16, and what the cut left: not negative, and not zero for a weight above zero, so
// that an infinite value comes out as the weight times it.
__device__ __forceinline__ uint32_t pack_down(float x, float y) {
  uint32_t r;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_rest(float x, float y, uint32_t down) {
  return pack_bf16(fmaxf(x - bf16lo(down), x * 0x1p-30f), fmaxf(y - bf16hi(down), y * 0x1p-30f));
}

template <int CHUNKS, bool FEW>   // 128-byte columns of a row; at most 8 heads
struct Bf16Part {
  static constexpr int kTile = 64;
  static constexpr int kHeadRows = FEW ? 8 : 16;
  uint32_t q[CHUNKS * 4][FEW ? 2 : 4];
  float o[CHUNKS * 8][4], m[2], l[2];

  __device__ bool start(const Shape &p, Shared &, char *, uint32_t &, int b, int h0, int n) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, D = p.a.cache.dim;
    const char *base = p.a.q + b * p.a.q_stride + (long long)h0 * D * 2;
    auto get = [&](int row, int d) {
      return row < n && d < D ? *reinterpret_cast<const uint32_t *>(base + ((long long)row * D + d) * 2) : 0u;
    };
#pragma unroll
    for (int s = 0; s < CHUNKS * 4; ++s) {
      q[s][0] = get(g, s * 16 + 2 * t);
      q[s][1] = get(g, s * 16 + 2 * t + 8);
      if (!FEW) {
        q[s][2] = get(g + 8, s * 16 + 2 * t);
        q[s][3] = get(g + 8, s * 16 + 2 * t + 8);
      }
    }
#pragma unroll
    for (int i = 0; i < CHUNKS * 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.0f;
    return true;
  }

  // 16 keys (quarter `slice`) of the tile at k, v; keys lo <= i < hi of the tile count.
  __device__ void tile(const Shape &p, char *, const char *k, const char *v, int slice, int lo, int hi) {
    const int lane = threadIdx.x & 31, t = lane & 3, D = p.a.cache.dim;
    const int row0 = slice * 16;
    if (row0 >= hi || row0 + 16 <= lo) return;
    float s[2][4] = {};
    {   // rows of K as the MMA's columns: matrices (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 7) + ((lane >> 4) << 3), sub = (lane >> 3) & 1;
      const uint32_t base = smem_addr(k) + row * 128;
#pragma unroll
      for (int i = 0; i < CHUNKS * 4; ++i) {
        if (i * 16 >= D) break;
        uint32_t f[4];
        ldsm4(f, base + (i >> 2) * (kTile * 128) + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4));
        mma16816(s[0], q[i][0], FEW ? 0u : q[i][2], q[i][1], FEW ? 0u : q[i][3], f[0], f[1]);
        mma16816(s[1], q[i][0], FEW ? 0u : q[i][2], q[i][1], FEW ? 0u : q[i][3], f[2], f[3]);
      }
    }
    const bool part = lo > row0 || hi < row0 + 16;
    uint32_t keep[2] = {~0u, ~0u};   // halves of V's fragments whose keys count
    if (part) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = row0 + j * 8 + 2 * t + e;
          if (key < lo || key >= hi) {
            s[j][e] = s[j][2 + e] = -INFINITY;
            keep[j] &= e ? 0x0000ffffu : 0xffff0000u;
          }
        }
    }
    constexpr int R = FEW ? 1 : 2;
    float alpha[2] = {1.0f, 1.0f};
    bool moved = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1])) * p.scale2;
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
      if (x > m[r]) {
        alpha[r] = exp2_fast(m[r] - x);
        m[r] = x;
        moved = true;
      }
      const float ref = m[r] == -INFINITY ? 0.0f : m[r];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) s[j][2 * r + e] = exp2_fast(fmaf(s[j][2 * r + e], p.scale2, -ref));
      l[r] = l[r] * alpha[r] + ((s[0][2 * r] + s[0][2 * r + 1]) + (s[1][2 * r] + s[1][2 * r + 1]));
    }
    if (FEW) alpha[1] = alpha[0];
    if (__any_sync(~0u, moved)) {
#pragma unroll
      for (int i = 0; i < CHUNKS * 8; ++i) {
        o[i][0] *= alpha[0];
        o[i][1] *= alpha[0];
        o[i][2] *= alpha[1];
        o[i][3] *= alpha[1];
      }
    }
    const uint32_t h0 = pack_down(s[0][0], s[0][1]), h2 = pack_down(s[1][0], s[1][1]);
    const uint32_t r0 = pack_rest(s[0][0], s[0][1], h0), r2 = pack_rest(s[1][0], s[1][1], h2);
    const uint32_t h1 = FEW ? r0 : pack_down(s[0][2], s[0][3]), h3 = FEW ? r2 : pack_down(s[1][2], s[1][3]);
    const uint32_t r1 = FEW ? 0u : pack_rest(s[0][2], s[0][3], h1), r3 = FEW ? 0u : pack_rest(s[1][2], s[1][3], h3);
    {   // V transposed on the way: matrices (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 15), sub = lane >> 4;
      const uint32_t base = smem_addr(v) + row * 128;
#pragma unroll
      for (int i = 0; i < CHUNKS * 4; ++i) {
        if (i * 16 >= D) break;
        uint32_t f[4];
        ldsm4t(f, base + (i >> 2) * (kTile * 128) + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4));
        if (part) {   // an infinity or NaN times a weight of zero would still show
          f[0] &= keep[0];
          f[1] &= keep[1];
          f[2] &= keep[0];
          f[3] &= keep[1];
        }
        mma16816(o[2 * i], h0, h1, h2, h3, f[0], f[1]);
        mma16816(o[2 * i + 1], h0, h1, h2, h3, f[2], f[3]);
        if (!FEW) {
          mma16816(o[2 * i], r0, r1, r2, r3, f[0], f[1]);
          mma16816(o[2 * i + 1], r0, r1, r2, r3, f[2], f[3]);
        }
      }
    }
  }

  __device__ void stats(float *top, float *sum) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < (FEW ? 1 : 2); ++r) {
      float x = l[r] + __shfl_xor_sync(~0u, l[r], 1);
      x += __shfl_xor_sync(~0u, x, 2);
      if ((lane & 3) == 0) {
        top[(lane >> 2) + 8 * r] = m[r];
        sum[(lane >> 2) + 8 * r] = x;
      }
    }
  }
  // Rows row0 .. row0 + 7 and columns col0 .. col0 + 127 of the sums times factor[row].
  __device__ void put(int row0, int col0, const float *factor, float (*to)[kMergeLd]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float f = factor[row0 + g];
#pragma unroll
    for (int i = 0; i < CHUNKS * 8; ++i) {
      const int c = i * 8 + 2 * t - col0;
      if (i * 8 < col0 || i * 8 >= col0 + kMergeCols) continue;
      float2 x;
      if (FEW) x = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
      else x = row0 == 0 ? make_float2(o[i][0], o[i][1]) : make_float2(o[i][2], o[i][3]);
      *reinterpret_cast<float2 *>(&to[g][c]) = make_float2(x.x * f, x.y * f);
    }
  }
};

// ---- consumers: fp32, on the CUDA cores ----
// Logits: 4 lanes a key, 8 keys a warp, the heads' q broadcast from shared memory.  O: the lanes
// across the row's columns (with short rows several keys at once), the weights broadcast.
template <int HEADS, int WIDE>   // heads held; 128-column blocks of a row
struct F32Part {
  static constexpr int kTile = 32;
  static constexpr int kHeadRows = HEADS;
  float o[HEADS][WIDE][4], m[HEADS], l[HEADS];

  static __device__ __forceinline__ int lanes_across(int D) {   // lanes that share a row of V
    const int n = D / 4;
    return n > 16 ? 32 : n > 8 ? 16 : n > 4 ? 8 : n > 2 ? 4 : n;
  }
  // q is kept in shared memory for all warps: the last part's sums are joined, so nobody reads the old one.
  __device__ bool start(const Shape &p, Shared &sm, char *scratch, uint32_t &parity, int b, int h0, int n) {
    const int D = p.a.cache.dim;
    const float *base = reinterpret_cast<const float *>(p.a.q + b * p.a.q_stride) + (long long)h0 * D;
    float4 *qs = reinterpret_cast<float4 *>(scratch);
    for (int i = threadIdx.x; i < HEADS * D / 4; i += kWarps * 32)
      qs[i] = i < n * D / 4 ? reinterpret_cast<const float4 *>(base)[i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!consumers_sync(sm, parity)) return false;
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      m[h] = -INFINITY;
      l[h] = 0.0f;
#pragma unroll
      for (int w = 0; w < WIDE; ++w) o[h][w][0] = o[h][w][1] = o[h][w][2] = o[h][w][3] = 0.0f;
    }
    return true;
  }
  __device__ void tile(const Shape &p, char *scratch, const char *k, const char *v, int slice, int lo, int hi) {
    const int lane = threadIdx.x & 31, D = p.a.cache.dim, cols = D / 4;
    const int row0 = slice * 8;
    if (row0 >= hi || row0 + 8 <= lo) return;
    const float4 *qs = reinterpret_cast<const float4 *>(scratch);
    float *ps = reinterpret_cast<float *>(scratch) + HEADS * (D + 8 * (threadIdx.x >> 5));   // this warp's [8 keys][HEADS]
    const int row = row0 + (lane & 7);
    float s[HEADS] = {};
    for (int c = lane >> 3; c < cols; c += 4) {
      const float4 x = *reinterpret_cast<const float4 *>(k + (c >> 3) * (kTile * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4));
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        const float4 y = qs[h * cols + c];
        s[h] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[h]))));
      }
    }
    const bool counts = row >= lo && row < hi;
    bool moved = false;
    float alpha[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      s[h] += __shfl_xor_sync(~0u, s[h], 8);
      s[h] += __shfl_xor_sync(~0u, s[h], 16);
      if (!counts) s[h] = -INFINITY;
      float x = s[h] * p.scale2;
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
      x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
      alpha[h] = 1.0f;
      if (x > m[h]) {
        alpha[h] = exp2_fast(m[h] - x);
        m[h] = x;
        moved = true;
      }
      s[h] = exp2_fast(fmaf(s[h], p.scale2, m[h] == -INFINITY ? 0.0f : -m[h]));
      l[h] = l[h] * alpha[h] + s[h];
    }
    if (moved) {   // the same in every lane
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int w = 0; w < WIDE; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[h][w][e] *= alpha[h];
    }
    __syncwarp();
    if (lane < 8) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h) ps[lane * HEADS + h] = s[h];
    }
    __syncwarp();
    const int across = lanes_across(D), c0 = lane & (across - 1);
    for (int i = lane / across; i < 8; i += 32 / across) {
      const int r = row0 + i;
      if (r < lo || r >= hi) continue;
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        const int c = c0 + 32 * w;
        if (c >= cols) break;
        const float4 x = *reinterpret_cast<const float4 *>(v + (c >> 3) * (kTile * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          const float y = ps[i * HEADS + h];
          o[h][w][0] = fmaf(y, x.x, o[h][w][0]);
          o[h][w][1] = fmaf(y, x.y, o[h][w][1]);
          o[h][w][2] = fmaf(y, x.z, o[h][w][2]);
          o[h][w][3] = fmaf(y, x.w, o[h][w][3]);
        }
      }
    }
  }
  __device__ void stats(float *top, float *sum) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      float x = l[h] + __shfl_xor_sync(~0u, l[h], 1);
      x += __shfl_xor_sync(~0u, x, 2);
      x += __shfl_xor_sync(~0u, x, 4);
      if (lane == 0) {
        top[h] = m[h];
        sum[h] = x;
      }
    }
  }
  __device__ void put(int row0, int col0, const float *factor, float (*to)[kMergeLd], int D) {
    const int lane = threadIdx.x & 31, across = lanes_across(D);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h < row0 || h >= row0 + kMergeRows) continue;
      const float f = factor[h];
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        if (w * 128 != col0) continue;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = o[h][w][e];
          for (int d = across; d < 32; d <<= 1) x[e] += __shfl_xor_sync(~0u, x[e], d);
        }
        if (lane < across) *reinterpret_cast<float4 *>(&to[h - row0][lane * 4]) = make_float4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
      }
    }
  }
};
template <int C, bool F> __device__ __forceinline__ void put(Bf16Part<C, F> &p, int r, int c, const float *f, float (*to)[kMergeLd], int) { p.put(r, c, f, to); }
template <int H, int W> __device__ __forceinline__ void put(F32Part<H, W> &p, int r, int c, const float *f, float (*to)[kMergeLd], int D) { p.put(r, c, f, to, D); }

__device__ __forceinline__ float join_factor(float top, float all) { return top == -INFINITY ? 1.0f : exp2_fast(top - all); }
__device__ __forceinline__ float lse_of(float top, float sum) { return sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2; }

// Adds up the warps' sums of the CTA's part of a (sequence, head): to the output where the part is
// all of it, else to the workspace.
template <typename Part, typename T>
__device__ bool finish(const Shape &p, Shared &sm, Part &part, const TileInfo &ti, uint32_t &parity) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = p.a.cache.dim;
  const int kv = ti.head / p.passes, pass = ti.head - kv * p.passes;
  const int h0 = kv * p.group + pass * kRows, n = min(kRows, p.group - pass * kRows);
  part.stats(sm.top[warp], sm.sum[warp]);
  if (!consumers_sync(sm, parity)) return false;
  if (lane < Part::kHeadRows) {
    float all = sm.top[0][lane], total = 0.0f;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all = fmaxf(all, sm.top[w][lane]);
    sm.factor[warp][lane] = join_factor(sm.top[warp][lane], all);
    if (warp == 0) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) total += sm.sum[w][lane] * join_factor(sm.top[w][lane], all);
      sm.all[lane] = all;
      sm.total[lane] = total;
    }
  }
  __syncwarp();
  float *slot = p.parts + ((long long)blockIdx.x * 2 + (ti.flags & kLater ? 1 : 0)) * (kStatFloats + p.rows * D);
  for (int row0 = 0; row0 < n; row0 += kMergeRows)
    for (int col0 = 0; col0 < D; col0 += kMergeCols) {
      put(part, row0, col0, sm.factor[warp], sm.merge[warp], D);
      if (!consumers_sync(sm, parity)) return false;
      for (int i = threadIdx.x; i < kMergeRows * kMergeCols / 2; i += kWarps * 32) {
        const int rr = i / (kMergeCols / 2), r = row0 + rr, cc = (i % (kMergeCols / 2)) * 2, c = col0 + cc;
        if (r >= n || c >= D) continue;
        float2 x = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 y = *reinterpret_cast<const float2 *>(&sm.merge[w][rr][cc]);
          x.x += y.x;
          x.y += y.y;
        }
        const float total = sm.total[r];
        if (ti.flags & kWhole) {
          const float f = total == 0.0f ? 0.0f : 1.0f / total;
          T *out = reinterpret_cast<T *>(p.a.out + ti.seq * p.a.out_stride) + (long long)(h0 + r) * D + c;
          if (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(out) = pack_bf16(x.x * f, x.y * f);
          else *reinterpret_cast<float2 *>(out) = make_float2(x.x * f, x.y * f);
          if (p.a.lse != nullptr && c == 0) p.a.lse[(long long)ti.seq * p.a.q_heads + h0 + r] = lse_of(sm.all[r], total);
        } else {
          *reinterpret_cast<float2 *>(slot + kStatFloats + r * D + c) = x;
          if (c == 0) *reinterpret_cast<float2 *>(slot + 2 * r) = make_float2(sm.all[r], total);
        }
      }
      if (!consumers_sync(sm, parity)) return false;
    }
  return true;
}

template <typename Part, typename T>
__device__ void consume(const Shape &p, Shared &sm, char *ring, char *scratch, int tiles) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = p.chunks * Part::kTile * 128;
  Part part;
  uint32_t parity = 0;
  int stage = 0, round = 0;
  for (int it = 0; it < tiles; ++it) {
    if (!wait(sm, &sm.full[stage], round & 1)) return;
    const TileInfo ti = sm.info[stage];
    if (ti.flags & kFirst) {
      const int kv = ti.head / p.passes, pass = ti.head - kv * p.passes;
      if (!part.start(p, sm, scratch, parity, ti.seq, kv * p.group + pass * kRows, min(kRows, p.group - pass * kRows))) return;
    }
    if ((it & (kGroups - 1)) == warp / kSlices) {
      const char *k = ring + (long long)stage * 2 * half;
      part.tile(p, scratch, k, k + half, warp % kSlices, ti.lo, ti.hi);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.empty[stage]);
    if ((ti.flags & kLast) && !finish<Part, T>(p, sm, part, ti, parity)) return;
    if (++stage == p.stages) {
      stage = 0;
      ++round;
    }
  }
}

struct Walk {   // tile `at` of the `tiles` of sequence seq, pass head
  int seq, head, at, tiles;
  Keys keys;
};
__device__ __forceinline__ void advance(const Shape &p, Walk &w) {
  unsigned bad = 0;
  if (++w.at < w.tiles) return;
  w.at = 0;
  if (++w.head < p.heads) return;
  w.head = 0;
  do {
    if (++w.seq >= p.a.seq.batch) return;
    w.keys = keys_of(p.a, w.seq, &bad);
    w.tiles = tiles_of(w.keys, p.tile);
  } while (w.tiles == 0);
}

// One warp fills the ring.  A tile's boxes (whole pages, or parts of them) are spread over the lanes, and the
// next tile's pages are looked up while this one waits for room.
template <int TILE, int ELEM>
__device__ void produce(const Shape &p, Shared &sm, char *ring, const CUtensorMap *kmap, const CUtensorMap *vmap, Walk w,
                        int tiles) {
  const int lane = threadIdx.x & 31, boxes = TILE / p.box, mine = lane & (boxes - 1);
  const int ops = boxes * p.chunks * 2, half = p.chunks * TILE * 128, size = p.a.cache.page_size;
  auto lookup = [&](const Walk &x, int &row) {   // page and first row of this lane's box; -1: no key in it counts
    const int key = (x.keys.begin / TILE + x.at) * TILE + mine * p.box;
    row = key % size;
    if (key >= x.keys.end || key + p.box <= x.keys.begin) return -1;
    const int page = p.a.seq.table[x.seq * p.a.seq.table_stride + key / size];
    if (page >= 0 && page < p.a.cache.num_pages) return page;
    atomicOr(&sm.flags, kErrCacheIndex);
    return 0;   // any page will do: the call is reported
  };
  int row, next_row = 0, page = lookup(w, row), next_page = -1, stage = 0, round = 0;
  bool fresh = true, later = false, begun = false;
  for (int it = 0; it < tiles; ++it) {
    Walk next = w;
    if (it + 1 < tiles) {
      advance(p, next);
      next_page = lookup(next, next_row);
    }
    if (it >= p.stages && !wait(sm, &sm.empty[stage], (round & 1) ^ 1)) return;
    const bool last = it + 1 == tiles || w.at + 1 == w.tiles;
    if (fresh) begun = w.at == 0;
    const int loaded = __popc(__ballot_sync(~0u, lane < boxes && page >= 0));
    if (lane == 0) {
      const int k0 = (w.keys.begin / TILE + w.at) * TILE;
      TileInfo ti;
      ti.seq = w.seq;
      ti.head = w.head;
      ti.lo = w.keys.begin - k0;
      ti.hi = w.keys.end - k0;
      ti.flags = (fresh ? kFirst : 0) | (last ? kLast : 0) | (begun && w.at + 1 == w.tiles ? kWhole : 0) | (later ? kLater : 0);
      sm.info[stage] = ti;
      mbar_expect_tx(&sm.full[stage], loaded * p.box * 128 * p.chunks * 2);
    }
    __syncwarp();
    if (page >= 0) {
      const int kv = w.head / p.passes;
      char *to = ring + (long long)stage * 2 * half + mine * p.box * 128;
      for (int o = lane; o < ops; o += 32) {
        const int c = (o / boxes) >> 1;
        if ((o / boxes) & 1) tma_load_4d(to + half + c * TILE * 128, vmap, c * (128 / ELEM), row, kv, page, &sm.full[stage]);
        else tma_load_4d(to + c * TILE * 128, kmap, c * (128 / ELEM), row, kv, page, &sm.full[stage]);
      }
    }
    fresh = last;
    later |= last;
    w = next;
    page = next_page;
    row = next_row;
    if (++stage == p.stages) {
      stage = 0;
      ++round;
    }
  }
}

template <typename Part, typename T>
__global__ void __launch_bounds__(kThreads, 1)
attend_kernel(const __grid_constant__ Shape p, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ char smem_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.a.seq.batch;
  char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  Shared &sm = *reinterpret_cast<Shared *>(ring + (long long)p.stages * 2 * p.chunks * Part::kTile * 128);
  char *scratch = reinterpret_cast<char *>(&sm + 1);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], kWarps);
    }
    mbar_init(&sm.sync, kWarps);
    mbar_init(&sm.never, 1);
    fence_mbar_init();
    sm.flags = 0;
    sm.dead = 0;
    sm.start_seq = -1;
  }

  // this CTA's share of all tiles: each thread counts some sequences' tiles
  unsigned bad = 0;
  const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += (long long)tiles_of(keys_of(p.a, b, &bad), p.tile) * p.heads;
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long x = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sm.warp_tiles[warp] = upto;
  __syncthreads();
  if (bad) atomicOr(&sm.flags, bad);
  long long total = 0;
  for (int w = 0; w <= kWarps; ++w) {
    if (w < warp) upto += sm.warp_tiles[w];
    total += sm.warp_tiles[w];
  }
  // no share is empty: with fewer tiles than CTAs the last CTAs have none
  const long long shares = total < gridDim.x ? total : gridDim.x;
  const long long t0 = blockIdx.x < shares ? total * blockIdx.x / shares : total;
  const long long t1 = blockIdx.x < shares ? total * (blockIdx.x + 1) / shares : total;
  const bool here = t0 < t1 && t0 >= upto - mine && t0 < upto;
  if (here || blockIdx.x == 0) {
    long long at = upto - mine;
    for (int b = b0; b < b1; ++b) {
      const long long n = (long long)tiles_of(keys_of(p.a, b, &bad), p.tile) * p.heads;
      if (blockIdx.x == 0) p.first[b] = at;
      if (here && t0 >= at && t0 < at + n) {
        sm.start_seq = b;
        sm.start_first = at;
      }
      at += n;
    }
  }
  if (blockIdx.x == 0 && tid == 0) p.first[B] = total;
  __syncthreads();

  const int tiles = (int)(t1 - t0);
  if (tiles > 0) {
    if (warp == kWarps) {
      Walk w;
      w.seq = sm.start_seq;
      w.keys = keys_of(p.a, w.seq, &bad);
      w.tiles = tiles_of(w.keys, p.tile);
      const long long at = t0 - sm.start_first;
      w.head = (int)(at / w.tiles);
      w.at = (int)(at - (long long)w.head * w.tiles);
      produce<Part::kTile, (int)sizeof(T)>(p, sm, ring, &kmap, &vmap, w, tiles);
    } else {
      consume<Part, T>(p, sm, ring, scratch, tiles);
    }
  }
  __syncthreads();
  if (sm.dead && tid < 32) wait_out(&sm.never);   // copies that nobody waited for
  if (tid == 0) post_status(reinterpret_cast<unsigned *>(p.a.ws), blockIdx.x, gridDim.x, sm.flags | (sm.dead ? kErrTimeout : 0u));
}

// What the cuts between the CTAs' shares have parted, one query head per CTA; and the outputs of sequences
// without a key.
constexpr int kJoinThreads = 256;
static_assert(kJoinThreads >= kMaxWorkers, "a thread per part");

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Shape p, int workers) {
  __shared__ float factor[kJoinThreads], red[kJoinThreads / 32];
  __shared__ float4 rows[kJoinThreads / 32][64];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, D = p.a.cache.dim;
  const int b = blockIdx.x / p.a.q_heads, h = blockIdx.x - b * p.a.q_heads;
  const int kv = h / p.group, pass = (h - kv * p.group) / kRows, r = h - kv * p.group - pass * kRows;
  const long long total = p.first[p.a.seq.batch], tiles = (p.first[b + 1] - p.first[b]) / p.heads;
  const long long begin = p.first[b] + (kv * p.passes + pass) * tiles;
  T *out = reinterpret_cast<T *>(p.a.out + b * p.a.out_stride) + (long long)h * D;
  float *lse = p.a.lse == nullptr ? nullptr : p.a.lse + (long long)b * p.a.q_heads + h;
  if (tiles == 0) {
    for (int d = tid; d < D; d += kJoinThreads) out[d] = (T)0.0f;
    if (lse != nullptr && tid == 0) *lse = -INFINITY;
    return;
  }
  // share w: the tiles total w / workers up to total (w + 1) / workers
  if (workers > total) workers = (int)total;
  const int w0 = (int)(((begin + 1) * workers - 1) / total), w1 = (int)(((begin + tiles) * workers - 1) / total);
  if (w0 == w1) return;   // one CTA wrote the output
  const long long stride = kStatFloats + p.rows * D;
  auto part = [&](int w) {   // a CTA's first part unless its share begins before the (sequence, head)
    return p.parts + (2LL * w + (total * w / workers < begin ? 1 : 0)) * stride;
  };
  float top = -INFINITY, sum = 0.0f;
  if (w0 + tid <= w1) {
    const float2 x = *reinterpret_cast<const float2 *>(part(w0 + tid) + 2 * r);
    top = x.x;
    sum = x.y;
  }
  float all = top;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) all = fmaxf(all, __shfl_xor_sync(~0u, all, x));
  if (lane == 0) red[warp] = all;
  __syncthreads();
  all = red[0];
#pragma unroll
  for (int w = 1; w < kJoinThreads / 32; ++w) all = fmaxf(all, red[w]);
  const float f = join_factor(top, all);
  factor[tid] = f;
  sum *= f;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(~0u, sum, x);
  __syncthreads();
  if (lane == 0) red[warp] = sum;
  float4 acc[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
#pragma unroll 4
  for (int w = w0 + warp; w <= w1; w += kJoinThreads / 32) {
    const float4 *x = reinterpret_cast<const float4 *>(part(w) + kStatFloats + r * D);
    const float g = factor[w - w0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (lane + 32 * i < D / 4) {
        const float4 y = x[lane + 32 * i];
        acc[i].x = fmaf(y.x, g, acc[i].x);
        acc[i].y = fmaf(y.y, g, acc[i].y);
        acc[i].z = fmaf(y.z, g, acc[i].z);
        acc[i].w = fmaf(y.w, g, acc[i].w);
      }
  }
  rows[warp][lane] = acc[0];
  rows[warp][lane + 32] = acc[1];
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) sum += red[w];
  for (int d = tid; d < D; d += kJoinThreads) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 32; ++w) x += reinterpret_cast<const float *>(rows[w])[d];
    out[d] = (T)(sum == 0.0f ? 0.0f : x / sum);
  }
  if (lse != nullptr && tid == 0) *lse = lse_of(all, sum);
}

constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }

template <typename Part, typename T>
cudaError_t launch(Shape p, cudaStream_t s) {
  const AttendArgs &a = p.a;
  const CacheLayer &c = a.cache;
  p.tile = Part::kTile;
  p.box = Part::kTile;
  while (c.page_size % p.box != 0) p.box /= 2;
  const size_t scratch = sizeof(T) == 4 ? (size_t)Part::kHeadRows * (c.dim + 8 * kWarps) * 4 : 0;
  const size_t stage = (size_t)2 * p.chunks * Part::kTile * 128, fixed = 1024 + sizeof(Shared) + scratch;
  p.stages = (int)((kSmemOptinSm100 - fixed) / stage);
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  const size_t smem = fixed + p.stages * stage;
  CUtensorMap maps[2];
  const uint64_t row = (uint64_t)c.dim * sizeof(T);
  const uint64_t dims[4] = {(uint64_t)c.dim, (uint64_t)c.page_size, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint64_t strides[3] = {(uint64_t)c.token_stride, c.heads > 1 ? (uint64_t)c.head_stride : row,
                               c.num_pages > 1 ? (uint64_t)c.page_stride : row};
  const uint32_t box[4] = {128 / (uint32_t)sizeof(T), (uint32_t)p.box, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (!encode_rows_map(&maps[i], i ? c.v : c.k, sizeof(T) == 4, 4, dims, strides, box)) return cudaErrorInvalidValue;
  const void *fn = reinterpret_cast<const void *>(&attend_kernel<Part, T>);
  cudaError_t e = allow_smem(fn, smem);
  if (e != cudaSuccess) return e;
  int workers = sm_count();
  workers = workers < kMaxWorkers ? workers : kMaxWorkers;
  attend_kernel<Part, T><<<workers, kThreads, smem, s>>>(p, maps[0], maps[1]);
  if ((e = cudaGetLastError()) != cudaSuccess || a.seq.batch == 0) return e;
  cudaLaunchConfig_t q = {};
  q.gridDim = dim3((unsigned)(a.seq.batch * (long long)a.q_heads));
  q.blockDim = dim3(kJoinThreads);
  q.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // its launch overlaps the kernel it waits for
  at[0].val.programmaticStreamSerializationAllowed = 1;
  q.attrs = at;
  q.numAttrs = 1;
  return cudaLaunchKernelEx(&q, join_kernel<T>, p, workers);
}

template <int CHUNKS>
cudaError_t launch_bf16(const Shape &p, cudaStream_t s) {
  return p.rows <= 8 ? launch<Bf16Part<CHUNKS, true>, __nv_bfloat16>(p, s) : launch<Bf16Part<CHUNKS, false>, __nv_bfloat16>(p, s);
}
template <int WIDE>
cudaError_t launch_f32(const Shape &p, cudaStream_t s) {
  if (p.rows <= 1) return launch<F32Part<1, WIDE>, float>(p, s);
  if (p.rows <= 2) return launch<F32Part<2, WIDE>, float>(p, s);
  if (p.rows <= 4) return launch<F32Part<4, WIDE>, float>(p, s);
  if (p.rows <= 8) return launch<F32Part<8, WIDE>, float>(p, s);
  return launch<F32Part<16, WIDE>, float>(p, s);
}

}  // namespace

size_t attend_scratch_bytes(int batch, int q_heads, int kv_heads, int dim) {
  const int group = q_heads / kv_heads, rows = group < kRows ? group : kRows;
  return align256(sizeof(long long) * ((size_t)batch + 1)) + align256(sizeof(float) * kMaxWorkers * 2 * (kStatFloats + (size_t)rows * dim));
}

cudaError_t launch_attend(const AttendArgs &a, cudaStream_t s) {
  Shape p{};
  p.a = a;
  p.group = a.q_heads / a.cache.heads;
  p.passes = (p.group + kRows - 1) / kRows;
  p.heads = p.passes * a.cache.heads;
  p.rows = p.group < kRows ? p.group : kRows;
  p.chunks = (a.cache.dim * a.elem + 127) / 128;
  p.scale2 = a.scale * kLog2e;
  p.first = reinterpret_cast<long long *>(a.ws + kStatusBytes);
  p.parts = reinterpret_cast<float *>(a.ws + kStatusBytes + align256(sizeof(long long) * ((size_t)a.seq.batch + 1)));
  if ((long long)a.seq.batch * a.q_heads > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (a.elem == 4) return p.chunks <= 4 ? launch_f32<1>(p, s) : launch_f32<2>(p, s);
  switch (p.chunks) {
    case 1: return launch_bf16<1>(p, s);
    case 2: return launch_bf16<2>(p, s);
    case 3: return launch_bf16<3>(p, s);
    default: return launch_bf16<4>(p, s);
  }
}

}  // namespace last
