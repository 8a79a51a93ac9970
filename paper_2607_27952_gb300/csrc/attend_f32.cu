// Cache attention over fp32 keys and values: the products on the CUDA cores.
#include "attend_impl.cuh"

namespace last {

namespace {

// ---- consumers: fp32, on the CUDA cores ----
// Bound by HBM with one head a kv-head and rows of whole 128-byte columns (16 kv-heads of 74010 keys by 128, 1.21 GB:
// 180 us, 6.7 TB/s); rows of 320 bytes are fetched as 384 (the same by 80, 758 MB: 155 us, 4.9 TB/s).  With many heads
// bound by this layout's reads of q and of the weights from shared memory (4 x 17970 keys by 64, 12 heads on 2: 35 us
// against 11 of HBM).  16 heads spill 64 bytes up to 128 elements (4 x 20000 keys by 128: 48 us) and 660 past
// them (by 256: 184 us; 8 heads 48).
// Logits: 4 lanes a key, 8 keys a warp, the heads' q broadcast from shared memory.  O: the lanes
// across the row's columns (with short rows several keys at once), the weights broadcast.
template <int HEADS, int WIDE>   // heads held; 128-column blocks of a row
struct F32Part {
  static constexpr int kTile = 32, kWarpKeys = 8, kCtas = HEADS <= 4 && WIDE == 1 ? 3 : 2;
  static constexpr int kHeadRows = HEADS;
  float o[HEADS][WIDE][4], m[HEADS], l[HEADS];

  static __device__ __forceinline__ int lanes_across(int D) {   // lanes that share a row of V
    const int n = D / 4;
    return n > 16 ? 32 : n > 8 ? 16 : n > 4 ? 8 : n > 2 ? 4 : n;
  }
  // Heads past the pass's n start from +inf: their logits, of whatever the slot holds, then never move the maxima.
  __device__ void start(const Shape &, const char *, int n) {
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      m[h] = h < n ? -INFINITY : INFINITY;
      l[h] = 0.0f;
#pragma unroll
      for (int w = 0; w < WIDE; ++w) o[h][w][0] = o[h][w][1] = o[h][w][2] = o[h][w][3] = 0.0f;
    }
  }
  // A box holds 8 keys and more: the warp's are all in one.
  static __device__ __forceinline__ bool skips(const Shape &p, unsigned skip, int row0) { return skip >> (row0 >> p.box_log) & 1; }

  // Weights of the tile's 8 keys from row0 on, kept in this warp's ps [8 keys][HEADS]; keys lo <= i < hi of
  // the tile count.  q: the heads' rows (past the pass's heads anything: neither their sums nor their logits are used).
  __device__ void logits(const Shape &p, const char *q, float *ps, const char *k, int row0, int lo, int hi, unsigned) {
    const int lane = threadIdx.x & 31, D = p.a.cache.dim, cols = D / 4, column = 128 << p.box_log;
    const float4 *qs = reinterpret_cast<const float4 *>(q);
    const int row = row0 + (lane & 7);
    const char *kr = k + row_at(p, row);
    float s[HEADS] = {};
#pragma unroll 2
    for (int c = lane >> 3; c < cols; c += 4) {
      const float4 x = *reinterpret_cast<const float4 *>(kr + (c >> 3) * column + (((c & 7) ^ (row & 7)) << 4));
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        const float4 y = qs[h * cols + c];
        s[h] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[h]))));
      }
    }
    const bool counts = row >= lo && row < hi;
    bool above = false;
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      s[h] += __shfl_xor_sync(~0u, s[h], 8);
      s[h] += __shfl_xor_sync(~0u, s[h], 16);
      s[h] = counts ? s[h] : -INFINITY;
      above |= s[h] * p.scale2 > m[h] + 8.0f;   // as for bf16: the maximum follows from a weight of 256 on
    }
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        float x = s[h] * p.scale2;
        x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
        x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
        x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
        const float alpha = x > m[h] ? exp2_fast(m[h] - x) : 1.0f;
        m[h] = fmaxf(m[h], x);
        l[h] *= alpha;
#pragma unroll
        for (int w = 0; w < WIDE; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[h][w][e] *= alpha;
      }
    }
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      s[h] = exp2_fast(fmaf(s[h], p.scale2, m[h] == -INFINITY ? 0.0f : -m[h]));
      l[h] += s[h];
    }
    __syncwarp();
    if (lane < 8) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h) ps[lane * HEADS + h] = s[h];
    }
    __syncwarp();
  }
  __device__ void values(const Shape &p, const float *ps, const char *v, int row0, int lo, int hi) {
    const int lane = threadIdx.x & 31, D = p.a.cache.dim, cols = D / 4, column = 128 << p.box_log;
    const int across = lanes_across(D), c0 = lane & (across - 1);
#pragma unroll 2
    for (int i = lane / across; i < 8; i += 32 / across) {
      const int r = row0 + i;
      const bool counts = r >= lo && r < hi;   // an infinity or NaN times a weight of zero would still show
      const char *vr = v + row_at(p, r);
      float y[HEADS];
      if constexpr (HEADS % 4 == 0) {
#pragma unroll
        for (int h = 0; h < HEADS; h += 4) *reinterpret_cast<float4 *>(y + h) = *reinterpret_cast<const float4 *>(ps + i * HEADS + h);
      } else {
#pragma unroll
        for (int h = 0; h < HEADS; ++h) y[h] = ps[i * HEADS + h];
      }
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        const int c = c0 + 32 * w;
        if (c >= cols) break;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (counts) x = *reinterpret_cast<const float4 *>(vr + (c >> 3) * column + (((c & 7) ^ (r & 7)) << 4));
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          o[h][w][0] = fmaf(y[h], x.x, o[h][w][0]);
          o[h][w][1] = fmaf(y[h], x.y, o[h][w][1]);
          o[h][w][2] = fmaf(y[h], x.z, o[h][w][2]);
          o[h][w][3] = fmaf(y[h], x.w, o[h][w][3]);
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
  // Rows row0 .. row0 + rows - 1 and columns col0 .. col0 + cols - 1 of the sums.
  __device__ void put(int row0, int rows, int col0, int cols, int ld, float *to, int D) {
    const int lane = threadIdx.x & 31, across = lanes_across(D);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h < row0 || h >= row0 + rows) continue;
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = o[h][w][e];
          for (int d = across; d < 32; d <<= 1) x[e] += __shfl_xor_sync(~0u, x[e], d);
        }
        const int c = w * 128 + lane * 4 - col0;
        if (lane < across && c >= 0 && c < cols) *reinterpret_cast<float4 *>(to + (h - row0) * ld + c) = make_float4(x[0], x[1], x[2], x[3]);
      }
    }
  }
};

template <int WIDE>
cudaError_t launch_heads(const Shape &p, cudaStream_t s) {
  if (p.rows <= 1) return launch<F32Part<1, WIDE>, float>(p, s);
  if (p.rows <= 4) return launch<F32Part<4, WIDE>, float>(p, s);
  if (p.rows <= 8) return launch<F32Part<8, WIDE>, float>(p, s);
  return launch<F32Part<16, WIDE>, float>(p, s);
}

}  // namespace

cudaError_t launch_attend_f32(const Shape &p, cudaStream_t s) {
  return p.chunks <= 4 ? launch_heads<1>(p, s) : launch_heads<2>(p, s);
}

}  // namespace last
