// Cache attention over bf16 keys and values: the products on the tensor cores.
#include "attend_impl.cuh"

namespace last {

namespace {

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
  static constexpr int kTile = 64, kWarpKeys = 16;
  static constexpr int kHeadRows = FEW ? 8 : 16;
  uint32_t q[CHUNKS * 4][FEW ? 2 : 4];
  float o[CHUNKS * 8][4], m[2], l[2];
  static constexpr int kR1 = FEW ? 0 : 1, kR2 = FEW ? 0 : 2, kR3 = FEW ? 0 : 3;
  uint32_t w[4], rest[FEW ? 1 : 4], keep[2];   // the tile's weights; masks of its values
  bool part;

  // q: the n heads' rows in shared memory.
  __device__ void start(const Shape &p, const char *qs, int n) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, D = p.a.cache.dim;
    auto get = [&](int row, int d) {
      return row < n && d < D ? *reinterpret_cast<const uint32_t *>(qs + (row * D + d) * 2) : 0u;
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
  }

  // Weights of the tile's 16 keys from row0 on; keys lo <= i < hi of the tile count.
  __device__ void logits(const Shape &p, const char *, float *, const char *k, int row0, int lo, int hi) {
    const int lane = threadIdx.x & 31, t = lane & 3, D = p.a.cache.dim, column = 128 << p.box_log;
    float s[2][4] = {};
    {   // rows of K as the MMA's columns: matrices (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 7) + ((lane >> 4) << 3), sub = (lane >> 3) & 1;
      const uint32_t base = smem_addr(k) + row_at(p, row);
#pragma unroll
      for (int i = 0; i < CHUNKS * 4; ++i) {
        if (i * 16 >= D) break;
        uint32_t f[4];
        ldsm4(f, base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4));
        mma16816(s[0], q[i][0], FEW ? 0u : q[i][2], q[i][1], FEW ? 0u : q[i][3], f[0], f[1]);
        mma16816(s[1], q[i][0], FEW ? 0u : q[i][2], q[i][1], FEW ? 0u : q[i][3], f[2], f[3]);
      }
    }
    part = lo > row0 || hi < row0 + 16;
    keep[0] = keep[1] = ~0u;   // halves of V's fragments whose keys count
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
    w[0] = pack_down(s[0][0], s[0][1]);
    w[2] = pack_down(s[1][0], s[1][1]);
    const uint32_t r0 = pack_rest(s[0][0], s[0][1], w[0]), r2 = pack_rest(s[1][0], s[1][1], w[2]);
    if (FEW) {
      w[1] = r0;
      w[3] = r2;
    } else {
      w[1] = pack_down(s[0][2], s[0][3]);
      w[3] = pack_down(s[1][2], s[1][3]);
      rest[0] = r0;
      rest[kR1] = pack_rest(s[0][2], s[0][3], w[1]);
      rest[kR2] = r2;
      rest[kR3] = pack_rest(s[1][2], s[1][3], w[3]);
    }
  }

  __device__ void values(const Shape &p, const float *, const char *v, int row0, int, int) {
    const int lane = threadIdx.x & 31, D = p.a.cache.dim, column = 128 << p.box_log;
    {   // V transposed on the way: matrices (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 15), sub = lane >> 4;
      const uint32_t base = smem_addr(v) + row_at(p, row);
#pragma unroll
      for (int i = 0; i < CHUNKS * 4; ++i) {
        if (i * 16 >= D) break;
        uint32_t f[4];
        ldsm4t(f, base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4));
        if (part) {   // an infinity or NaN times a weight of zero would still show
          f[0] &= keep[0];
          f[1] &= keep[1];
          f[2] &= keep[0];
          f[3] &= keep[1];
        }
        mma16816(o[2 * i], w[0], w[1], w[2], w[3], f[0], f[1]);
        mma16816(o[2 * i + 1], w[0], w[1], w[2], w[3], f[2], f[3]);
        if (!FEW) {
          mma16816(o[2 * i], rest[0], rest[kR1], rest[kR2], rest[kR3], f[0], f[1]);
          mma16816(o[2 * i + 1], rest[0], rest[kR1], rest[kR2], rest[kR3], f[2], f[3]);
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
  // Rows row0 .. row0 + rows - 1 and columns col0 .. col0 + cols - 1 of the sums.
  __device__ void put(int row0, int rows, int col0, int cols, int ld, float *to, int) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int r = 0; r < (FEW ? 1 : 2); ++r) {
      const int row = g + 8 * r - row0;
      if (row < 0 || row >= rows) continue;
#pragma unroll
      for (int i = 0; i < CHUNKS * 8; ++i) {
        if (i * 8 < col0 || i * 8 >= col0 + cols) continue;
        const float2 x = FEW ? make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]) : make_float2(o[i][2 * r], o[i][2 * r + 1]);
        *reinterpret_cast<float2 *>(to + row * ld + i * 8 + 2 * t - col0) = x;
      }
    }
  }
};

template <int CHUNKS>
cudaError_t launch_chunks(const Shape &p, cudaStream_t s) {
  return p.rows <= 8 ? launch<Bf16Part<CHUNKS, true>, __nv_bfloat16>(p, s) : launch<Bf16Part<CHUNKS, false>, __nv_bfloat16>(p, s);
}

}  // namespace

cudaError_t launch_attend_bf16(const Shape &p, cudaStream_t s) {
  switch (p.chunks) {
    case 1: return launch_chunks<1>(p, s);
    case 2: return launch_chunks<2>(p, s);
    case 3: return launch_chunks<3>(p, s);
    default: return launch_chunks<4>(p, s);
  }
}

}  // namespace last
