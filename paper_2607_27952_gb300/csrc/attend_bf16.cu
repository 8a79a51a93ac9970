// Cache attention over bf16 keys and values: the products on the tensor cores.
#include "attend_impl.cuh"

namespace last {

namespace {

// ---- consumers: bf16, on the tensor cores ----
// S^T = K Q^T with 16 keys as the rows of an MMA and 8 heads as its columns, then O^T += V^T P^T: K and V come
// from shared memory as they lie, and eight heads fill the MMA.  P is cut to bf16 in two parts, so that it
// carries 16 bits.  The maximum that the weights are taken against follows the logits only once one
// exceeds it by 8 (a weight of 256): most tiles then need neither the exchange nor the rescaling.
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// Per tile of 64 keys by 128 a warp's logits take 700 cycles and its values 500 (with heads as rows, twice the
// products at 8 heads, 1080 and 850).
template <int CHUNKS, int EIGHTS>   // 128-byte columns of a row; groups of 8 heads
struct Bf16Part {
  static constexpr int kTile = 64, kWarpKeys = 16, kHeadRows = 8 * EIGHTS, kCtas = CHUNKS * EIGHTS == 1 ? 3 : 2;
  static constexpr int kSteps = CHUNKS * 4;                           // 16-wide along a row
  // Fragments in flight: four, or two where the sums take most of a thread's 168 registers.  <4, 2> (rows wider than
  // 192, 9 to 16 heads) spills all the same, 1.8 KB: 4 x 20000 keys by 256 take 75 us with 16 heads, 30 with 8.
  static constexpr int kAhead = CHUNKS * EIGHTS > 4 ? 2 : 4;
  static constexpr bool kKeepQ = CHUNKS * EIGHTS < 6;                 // else its fragments are read for every tile
  uint32_t q[kKeepQ ? kSteps : 1][2 * EIGHTS];
  int heads;
  float o[kSteps][EIGHTS][4];                             // (d g, head 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1)
  float m[EIGHTS][2], l[EIGHTS][2];                       // heads 2t, 2t + 1; l over this lane's keys
  uint32_t w[EIGHTS][4], keep[2];                         // the tile's weights, cut and rest; masks of its values
  bool part;

  // Step s of q, whose heads' rows lie in shared memory.
  __device__ __forceinline__ void get_q(uint32_t (&x)[2 * EIGHTS], const char *qs, int s, int D) const {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int e = 0; e < 2 * EIGHTS; ++e) {
      const int row = g + 8 * (e >> 1), d = s * 16 + 2 * t + 8 * (e & 1);
      x[e] = row < heads && d < D ? *reinterpret_cast<const uint32_t *>(qs + (row * D + d) * 2) : 0u;
    }
  }
  __device__ void start(const Shape &p, const char *qs, int n) {
    heads = n;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (kKeepQ) get_q(q[kKeepQ ? s : 0], qs, s, p.a.cache.dim);
#pragma unroll
    for (int e = 0; e < EIGHTS; ++e) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) o[i][e][0] = o[i][e][1] = o[i][e][2] = o[i][e][3] = 0.0f;
      m[e][0] = m[e][1] = -INFINITY;
      l[e][0] = l[e][1] = 0.0f;
    }
  }

  // The warp's keys may lie in two boxes: logits() looks at each.
  static __device__ __forceinline__ bool skips(const Shape &, unsigned, int) { return false; }

  // Weights of the tile's 16 keys from row0 on; keys lo <= i < hi of the tile count, but for those of the boxes in skip.
  __device__ void logits(const Shape &p, const char *qs, float *, const char *k, int row0, int lo, int hi, unsigned skip) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, D = p.a.cache.dim, column = 128 << p.box_log;
    float s[2][EIGHTS][4] = {};   // even and odd steps
    {   // 8 x 8 blocks (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 15), sub = lane >> 4;
      const uint32_t base = smem_addr(k) + row_at(p, row);
      auto at = [&](int i) { return base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4); };
      uint32_t f[kAhead][4];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i * 16 < D) ldsm4(f[i], at(i));
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (i * 16 >= D) break;
        uint32_t (&x)[2 * EIGHTS] = q[kKeepQ ? i : 0];
        if (!kKeepQ) get_q(x, qs, i, D);
#pragma unroll
        for (int e = 0; e < EIGHTS; ++e) mma16816(s[i & 1][e], f[i % kAhead], x[2 * e], x[2 * e + 1]);
        if (i + kAhead < kSteps && (i + kAhead) * 16 < D) ldsm4(f[i % kAhead], at(i + kAhead));
      }
    }
    part = lo > row0 || hi < row0 + 16 || skip != 0;
    auto counts = [&](int key) { return key >= lo && key < hi && (skip >> (key >> p.box_log) & 1) == 0; };
    keep[0] = keep[1] = ~0u;   // halves of V's fragments whose keys count
    if (part) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (!counts(row0 + j * 8 + 2 * t + e)) keep[j] &= e ? 0x0000ffffu : 0xffff0000u;
        }
        if (!counts(row0 + j * 8 + g))
#pragma unroll
          for (int e = 0; e < EIGHTS; ++e) s[0][e][2 * j] = s[0][e][2 * j + 1] = s[1][e][2 * j] = s[1][e][2 * j + 1] = -INFINITY;
      }
    }
    float top[EIGHTS][2];
    bool above = false;
#pragma unroll
    for (int e = 0; e < EIGHTS; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[0][e][h] += s[1][e][h];
        s[0][e][2 + h] += s[1][e][2 + h];
        top[e][h] = fmaxf(s[0][e][h], s[0][e][2 + h]) * p.scale2;
        above |= top[e][h] > m[e][h] + 8.0f;
      }
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int e = 0; e < EIGHTS; ++e) {
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = top[e][h];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
          alpha[h] = x > m[e][h] ? exp2_fast(m[e][h] - x) : 1.0f;
          m[e][h] = fmaxf(m[e][h], x);
          l[e][h] *= alpha[h];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          o[i][e][0] *= alpha[0];
          o[i][e][1] *= alpha[1];
          o[i][e][2] *= alpha[0];
          o[i][e][3] *= alpha[1];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < EIGHTS; ++e) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = exp2_fast(fmaf(s[0][e][i], p.scale2, m[e][i & 1] == -INFINITY ? 0.0f : -m[e][i & 1]));
      l[e][0] += x[0] + x[2];
      l[e][1] += x[1] + x[3];
#pragma unroll
      for (int j = 0; j < 2; ++j) {   // keys j * 8 + g, to keys j * 8 + 2t and 2t + 1 of head g
        const uint32_t down = pack_down(x[2 * j], x[2 * j + 1]);
        w[e][j] = transpose8(down);
        w[e][2 + j] = transpose8(pack_rest(x[2 * j], x[2 * j + 1], down));
      }
    }
  }

  __device__ void values(const Shape &p, const float *, const char *v, int row0, int, int) {
    const int lane = threadIdx.x & 31, D = p.a.cache.dim, column = 128 << p.box_log;
    // 8 x 8 blocks, transposed on the way: (keys 0-7 | 8-15) x (16-byte column even | odd)
    const int row = row0 + (lane & 7) + (lane >> 4) * 8, sub = lane >> 3 & 1;
    const uint32_t base = smem_addr(v) + row_at(p, row);
    auto at = [&](int i) { return base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4); };
    uint32_t f[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i * 16 < D) ldsm4t(f[i], at(i));
#pragma unroll
    for (int i = 0; i < kSteps; i += 2) {   // two steps together: the products of one wait for each other
      if (i * 16 >= D) break;
      const bool both = (i + 1) * 16 < D;
      uint32_t (&x)[4] = f[i % kAhead], (&y)[4] = f[(i + 1) % kAhead];
      if (part) {   // an infinity or NaN times a weight of zero would still show
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] &= keep[j >> 1];
          y[j] &= keep[j >> 1];
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < EIGHTS; ++e) {
          mma16816(o[i][e], x, w[e][2 * r], w[e][2 * r + 1]);
          if (both) mma16816(o[i + 1][e], y, w[e][2 * r], w[e][2 * r + 1]);
        }
#pragma unroll
      for (int j = i + kAhead; j < i + kAhead + 2; ++j)
        if (j < kSteps && j * 16 < D) ldsm4t(f[j % kAhead], at(j));
    }
  }

  __device__ void stats(float *top, float *sum) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < EIGHTS; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = l[e][h];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(~0u, x, d);
        if (lane < 4) {
          top[8 * e + 2 * lane + h] = m[e][h];
          sum[8 * e + 2 * lane + h] = x;
        }
      }
  }
  // Rows row0 .. row0 + rows - 1 and columns col0 .. col0 + cols - 1 of the sums.
  __device__ void put(int row0, int rows, int col0, int cols, int ld, float *to, int) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int e = 0; e < EIGHTS; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 8 * e + 2 * t + h - row0;
        if (row < 0 || row >= rows) continue;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          if (i * 16 < col0 || i * 16 >= col0 + cols) continue;
          float *x = to + row * ld + i * 16 + g - col0;
          x[0] = o[i][e][h];
          x[8] = o[i][e][2 + h];
        }
      }
  }
};

template <int CHUNKS>
cudaError_t launch_chunks(const Shape &p, cudaStream_t s) {
  return p.rows <= 8 ? launch<Bf16Part<CHUNKS, 1>, __nv_bfloat16>(p, s) : launch<Bf16Part<CHUNKS, 2>, __nv_bfloat16>(p, s);
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
