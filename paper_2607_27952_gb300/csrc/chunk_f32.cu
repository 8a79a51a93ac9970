// Chunk and differential attention over fp32 keys and values: the products on the CUDA cores.
//
// A CTA holds a block of 64 rows and passes its keys in tiles of 64: S = Q K^T with 4 x 4 results a thread, a running maximum
// and sum per row (kept by the 16 threads that share it), O = O + P V with 4 rows x 4 columns a thread and
// 64 columns of V.  diff passes the keys twice, a map at a time, and keeps the first map's O in shared memory.
#include "chunk_impl.cuh"

namespace last {

namespace {

constexpr int kSimtThreads = 256, kSimtRows = 64, kSimtKeys = 64, kPad = 4;

struct alignas(16) SimtShared {
  ChunkShare share;
  unsigned long long sums[kSimtThreads / 32];
  long long at[kSimtKeys];   // where a key of the tile lies in its head's pages; -1: no row of the block sees it, or its page is out of range
  unsigned flags;
};

// CTAs of an SM, by registers.  All shares run at once: a second wave of them would begin when the first has ended.
template <int NC>
constexpr int kSimtCtas = NC <= 2 ? 2 : 1;

// NC: 64-column blocks of a value.
template <int NC>
__global__ void __launch_bounds__(kSimtThreads, kSimtCtas<NC>) chunk_f32_kernel(const __grid_constant__ ChunkShape p) {
  extern __shared__ float4 smem4[];
  const ChunkArgs &a = p.a;
  const int D = a.cache.dim, ld = D + kPad, ldv = p.dv + kPad, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  SimtShared &sm = *reinterpret_cast<SimtShared *>(smem4);
  float *qs = reinterpret_cast<float *>(&sm + 1), *ks = qs + kSimtRows * ld, *vs = ks + kSimtKeys * ld, *ps = vs + kSimtKeys * ldv;
  float *os = ps + kSimtRows * (kSimtKeys + kPad);   // diff: the first map's
  if (tid == 0) sm.flags = 0;
  grid_begins();
  __syncthreads();
  chunk_share<kSimtThreads>(p, blockIdx.x, sm.sums, &sm.share, &sm.flags);
  const CacheLayer &c = a.cache;
  ChunkWalk walk(sm.share);
  ChunkItem it;
  const int fours = D / 4;
  while (walk.next(p, &it)) {
    float o[4][NC][4], m[4], l[4];
    for (int map = 0; map < p.maps; ++map) {
      __syncthreads();
      for (int i = tid; i < kSimtRows * fours; i += kSimtThreads) {
        const int r = i / fours, d = (i - r * fours) * 4;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (r < it.rows) {
          const int t = (it.r0 + r) / p.group, h = it.unit * p.group + (it.r0 + r) - t * p.group;
          x = *reinterpret_cast<const float4 *>(a.q + (long long)(it.s.first + t) * a.q_stride + ((long long)(p.maps == 2 ? 2 * h + map : h) * D + d) * 4);
        }
        *reinterpret_cast<float4 *>(qs + r * ld + d) = x;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.0f;
      }
      int lo[4], hi[4];   // keys that this thread's rows see
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = ty * 4 + i, t = (it.r0 + r) / p.group;
        lo[i] = r < it.rows ? chunk_lo(a, it.s, t) : 0;   // rows of no token see everything, their q is zero
        hi[i] = r < it.rows ? chunk_hi(a, it.s, t) : 0x7fffffff;
      }
      const bool works = (tid >> 5) * 8 < it.rows;        // the warp has a row
      if (it.t.count > 0)
        for (int k = it.k0; k < it.k1; ++k) {
          const int key0 = (it.t.first + k) * kSimtKeys;
          __syncthreads();
          if (tid < kSimtKeys) {
            const int key = key0 + tid;
            long long at = -1;
            if (key >= it.t.lo && key < it.t.hi) {
              const int page = a.seq.table[it.seq * a.seq.table_stride + key / c.page_size];
              if ((unsigned)page < (unsigned)c.num_pages) at = page * c.page_stride + key % c.page_size * c.token_stride;
              else atomicOr(&sm.flags, kErrCacheIndex);
            }
            sm.at[tid] = at;
          }
          __syncthreads();
          // a warp every eighth row, its lanes the pieces of K and V; rows that are not there are zeros
          for (int d4 = tid & 31; d4 < fours + p.dv / 4; d4 += 32) {
            const bool is_v = d4 >= fours;
            const int d = (is_v ? d4 - fours : d4) * 4, head = it.unit * p.maps + (is_v ? d / D : map);
            const char *from = (is_v ? c.v : c.k) + head * c.head_stride + (is_v ? d % D : d) * 4;
            float *to = is_v ? vs + d : ks + d;
            const int pitch = is_v ? ldv : ld;
            float4 x[kSimtKeys / 8];
#pragma unroll
            for (int i = 0; i < kSimtKeys / 8; ++i) {
              const long long at = sm.at[i * 8 + (tid >> 5)];
              x[i] = at >= 0 ? *reinterpret_cast<const float4 *>(from + at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int i = 0; i < kSimtKeys / 8; ++i) *reinterpret_cast<float4 *>(to + (i * 8 + (tid >> 5)) * pitch) = x[i];
          }
          bool there[4];   // of keys tx + 16 j
#pragma unroll
          for (int j = 0; j < 4; ++j) there[j] = sm.at[tx + 16 * j] >= 0;
          __syncthreads();
          float s[4][4] = {};
#pragma unroll 4
          for (int d = 0; works && d < D; d += 4) {
            float4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[i] = *reinterpret_cast<const float4 *>(qs + (ty * 4 + i) * ld + d);
              y[i] = *reinterpret_cast<const float4 *>(ks + (tx + 16 * i) * ld + d);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                s[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j]))));
          }
          bool hidden = false;   // some row does not see some key that is there
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int key = key0 + tx + 16 * j;
              const bool sees = there[j] && key >= lo[i] && key < hi[i];
              hidden |= there[j] && !sees;
              s[i][j] = sees ? s[i][j] * p.scale2 : -INFINITY;
              top = fmaxf(top, s[i][j]);
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
            top = fmaxf(top, m[i]);
            const float alpha = m[i] == top ? 1.0f : chunk_exp2(m[i] - top), off = top == -INFINITY ? 0.0f : top;
            m[i] = top;
            l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][j][e] *= alpha;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              s[i][j] = chunk_exp2(s[i][j] - off);
              l[i] += s[i][j];
              ps[(ty * 4 + i) * (kSimtKeys + kPad) + tx + 16 * j] = s[i][j];
            }
          }
          hidden = __syncthreads_or(hidden);
          for (int k4 = 0; works && k4 < kSimtKeys; k4 += 4) {
            float4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4 *>(ps + (ty * 4 + i) * (kSimtKeys + kPad) + k4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < NC; ++j) {
                if (tx * 4 + 64 * j >= p.dv) break;
                const float4 y = *reinterpret_cast<const float4 *>(vs + (k4 + e) * ldv + tx * 4 + 64 * j);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float x = e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w;
                  if (hidden && x == 0.0f) continue;   // an infinity or NaN that the row does not see would show
                  o[i][j][0] = fmaf(x, y.x, o[i][j][0]);
                  o[i][j][1] = fmaf(x, y.y, o[i][j][1]);
                  o[i][j][2] = fmaf(x, y.z, o[i][j][2]);
                  o[i][j][3] = fmaf(x, y.w, o[i][j][3]);
                }
              }
          }
        }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(~0u, l[i], x);
      if (!it.whole) {
        float *slot = chunk_slot(p, blockIdx.x, map, it.second);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = ty * 4 + i;
          if (r >= it.rows) continue;
          if (tx == 0) {
            slot[r] = m[i];
            slot[p.pitch + r] = l[i];
          }
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            const int d = tx * 4 + 64 * j;
            if (d < p.dv)
              reinterpret_cast<float4 *>(slot + 2 * p.pitch)[(long long)(d / 4) * p.pitch + r] = make_float4(o[i][j][0], o[i][j][1], o[i][j][2], o[i][j][3]);
          }
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float g = l[i] == 0.0f ? 0.0f : 1.0f / l[i];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][j][e] = l[i] == 0.0f ? 0.0f : o[i][j][e] * g;
        const int r = ty * 4 + i;
        if (p.maps == 1 || map == 1 || r >= it.rows) continue;
#pragma unroll
        for (int j = 0; j < NC; ++j)   // read back by the same thread
          if (tx * 4 + 64 * j < p.dv)
            *reinterpret_cast<float4 *>(os + r * ldv + tx * 4 + 64 * j) = make_float4(o[i][j][0], o[i][j][1], o[i][j][2], o[i][j][3]);
      }
    }
    if (!it.whole) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = ty * 4 + i;
      const int t = (it.r0 + r) / p.group, h = it.unit * p.group + (it.r0 + r) - t * p.group;
      const bool live = r < it.rows;
      if (p.maps == 2) {
        const float lam = live ? a.lambda[h] : 0.0f;
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const int d = tx * 4 + 64 * j;
          if (d >= p.dv || !live) continue;
          const float4 y = *reinterpret_cast<const float4 *>(os + r * ldv + d);
          o[i][j][0] = y.x - lam * o[i][j][0];
          o[i][j][1] = y.y - lam * o[i][j][1];
          o[i][j][2] = y.z - lam * o[i][j][2];
          o[i][j][3] = y.w - lam * o[i][j][3];
#pragma unroll
          for (int e = 0; e < 4; ++e) sq = fmaf(o[i][j][e], o[i][j][e], sq);
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) sq += __shfl_xor_sync(~0u, sq, x);
        const float f = chunk_norm(a, sq, p.dv);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int d = tx * 4 + 64 * j + e;
            if (d < p.dv) o[i][j][e] *= f * (a.norm_weight ? a.norm_weight[d] : 1.0f);
          }
      }
      if (!live) continue;
      if (p.maps == 1 && a.lse != nullptr && tx == 0) a.lse[(long long)(it.s.first + t) * a.q_heads + h] = chunk_lse(m[i], l[i]);
      float *out = reinterpret_cast<float *>(a.out + (long long)(it.s.first + t) * a.out_stride) + (long long)h * p.dv;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        if (tx * 4 + 64 * j < p.dv) *reinterpret_cast<float4 *>(out + tx * 4 + 64 * j) = make_float4(o[i][j][0], o[i][j][1], o[i][j][2], o[i][j][3]);
    }
  }
  __syncthreads();
  if (tid == 0) {
    p.cuts[blockIdx.x] = chunk_cut(p, sm.share.end);
    post_status(reinterpret_cast<unsigned *>(a.ws), blockIdx.x, gridDim.x, sm.flags);
  }
}

template <int NC>
cudaError_t launch_f32(ChunkShape p, cudaStream_t s) {
  const int D = p.a.cache.dim;
  const size_t smem = sizeof(SimtShared) + sizeof(float) * ((kSimtRows + kSimtKeys) * (D + kPad) + kSimtKeys * (p.dv + kPad) +
                                                             kSimtRows * (kSimtKeys + kPad) + (p.maps == 2 ? kSimtRows * (p.dv + kPad) : 0));
  p.block = p.pitch = kSimtRows;
  p.tile = kSimtKeys;
  const int ctas = (int)((227 << 10) / (smem + 1024));
  int shares = sm_count() * (ctas < kSimtCtas<NC> ? ctas : kSimtCtas<NC>);
  p.shares = shares < kMaxShares ? shares : kMaxShares;
  cudaError_t e = allow_smem(reinterpret_cast<const void *>(&chunk_f32_kernel<NC>), smem);
  if (e != cudaSuccess) return e;
  e = launch_early(chunk_f32_kernel<NC>, dim3(p.shares), kSimtThreads, smem, s, p);
  return e == cudaSuccess ? launch_chunk_join(p, s) : e;
}

}  // namespace

cudaError_t launch_chunk_f32(ChunkShape p, cudaStream_t s) {
  switch ((p.dv + 63) / 64) {
    case 1: return launch_f32<1>(p, s);
    case 2: return launch_f32<2>(p, s);
    case 3: return launch_f32<3>(p, s);
    default: return launch_f32<4>(p, s);
  }
}

}  // namespace last
