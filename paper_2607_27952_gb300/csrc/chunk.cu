// Chunk and differential attention: the workspace, the choice of the kernel, and the sums that cuts have parted.
#include "chunk_impl.cuh"

namespace last {

namespace {

constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <int N>
struct Count {
  static constexpr int value = N;
};

template <typename T>
__device__ __forceinline__ void join_store(T *to, const float (&v)[8], int n) {   // 4 or 8 of v
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
    if (n > 4) *reinterpret_cast<float4 *>(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    __nv_bfloat162 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<uint4 *>(x);
  }
}

// CTA (w, y) belongs to the item that share w ends within, if any.  The CTAs of all its cuts divide its rows, 32 at a
// time (8, 16 where blocks have no more): a lane has a row, a warp's 32 / rows lanes of a row and the warps the groups of 8 columns by turns.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) chunk_join_kernel(const __grid_constant__ ChunkShape p) {
  __shared__ int first_cut, last_cut, share_of[kMaxShares + 1], parts;
  __shared__ float squares[kJoinWarps][32];
  grid_begins();
  const ChunkArgs &a = p.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, w = blockIdx.x;
  const int4 x = p.cuts[w];
  if (x.w == 0) return;
  if (tid == 0) {
    first_cut = w;
    last_cut = w;
  }
  __syncthreads();
  auto tile_at = [&](int i) {   // of the cut behind share i, if it is in this item
    const int4 c = p.cuts[i];
    return c.x == x.x && c.y == x.y && c.z == x.z ? c.w : 0;
  };
  for (int i = tid; i < p.shares; i += kJoinThreads)
    if (tile_at(i) > 0) {
      atomicMin(&first_cut, i);
      atomicMax(&last_cut, i);
    }
  __syncthreads();
  const int end = min(last_cut + 1, p.shares - 1);   // the last share with a part
  if (warp == 0) {   // the shares with a part: the first, and those that end at another tile than the one before
    int n = 0;
    for (int i0 = first_cut; i0 <= end; i0 += 32) {   // the cuts in between are in the item too
      const int i = i0 + lane;
      const bool some = i <= end && (i == first_cut || i > last_cut || tile_at(i) != tile_at(i - 1));
      const unsigned all = __ballot_sync(~0u, some);
      if (some) share_of[n + __popc(all & ((1u << lane) - 1))] = i;
      n += __popc(all);
    }
    if (lane == 0) parts = n;
  }
  __syncthreads();
  const int per = p.block <= 8 ? 8 : p.block <= 16 ? 16 : 32, groups = kJoinWarps * (32 / per);
  const int in_row = lane & (per - 1), group = warp * (32 / per) + lane / per;
  const int me = (w - first_cut) * gridDim.y + blockIdx.y, ctas = (last_cut - first_cut + 1) * gridDim.y;
  unsigned bad = 0;
  const ChunkSeq s = chunk_seq(a, x.x, &bad);
  const int r0 = x.z * p.block, rows = (int)min((long long)p.block, (long long)s.n * p.group - r0);
  for (int row0 = me * per; row0 < rows; row0 += ctas * per) {
    const int r = row0 + in_row;
    const bool live = r < rows;
    const int t = (r0 + (live ? r : 0)) / p.group, h = x.y * p.group + (r0 + (live ? r : 0)) - t * p.group;
    float acc[4][8], sq = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[j][e] = 0.0f;
    for (int map = 0; map < p.maps; ++map) {
      auto slot = [&](int i) { return chunk_slot(p, share_of[i], map, i == 0); };   // an item begins in its first share
      float all = -INFINITY, sum = 0.0f;
      if (live) {
#pragma unroll 8
        for (int i = 0; i < parts; ++i) all = fmaxf(all, slot(i)[r]);
#pragma unroll 8
        for (int i = 0; i < parts; ++i) sum = fmaf(chunk_factor(slot(i)[r], all), slot(i)[p.pitch + r], sum);
      }
      const float weight = map == 0 ? 1.0f : live ? -a.lambda[h] : 0.0f;
      if (live && p.maps == 1 && a.lse != nullptr && group == 0) a.lse[(long long)(s.first + t) * a.q_heads + h] = chunk_lse(all, sum);
      if (!live || sum == 0.0f) continue;
      const float g = weight / sum;
      auto add = [&](int i, auto last) {   // the groups of 8 columns of the thread: four, or one
        const float *from = slot(i);
        const float f = chunk_factor(from[r], all) * g;
#pragma unroll
        for (int j = 0; j < decltype(last)::value; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int four = (group + groups * j) * 2 + e;
            if (four * 4 >= p.dv) continue;
            const float4 y = reinterpret_cast<const float4 *>(from + 2 * p.pitch)[(long long)four * p.pitch + r];
            acc[j][4 * e] = fmaf(y.x, f, acc[j][4 * e]);
            acc[j][4 * e + 1] = fmaf(y.y, f, acc[j][4 * e + 1]);
            acc[j][4 * e + 2] = fmaf(y.z, f, acc[j][4 * e + 2]);
            acc[j][4 * e + 3] = fmaf(y.w, f, acc[j][4 * e + 3]);
          }
      };
      if (groups * 8 >= p.dv) {   // parts' loads side by side
#pragma unroll 8
        for (int i = 0; i < parts; ++i) add(i, Count<1>{});
      } else {
        for (int i = 0; i < parts; ++i) add(i, Count<4>{});
      }
    }
    if (p.maps == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(acc[j][e], acc[j][e], sq);
      __syncthreads();
      squares[warp][lane] = sq;
      __syncthreads();
      sq = 0.0f;
      for (int i = 0; i < kJoinWarps; ++i)
        for (int j = in_row; j < 32; j += per) sq += squares[i][j];
      const float f = chunk_norm(a, sq, p.dv);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = (group + groups * j) * 8 + e;
          if (d < p.dv) acc[j][e] *= f * (a.norm_weight ? a.norm_weight[d] : 1.0f);
        }
    }
    if (!live) continue;
    T *out = reinterpret_cast<T *>(a.out + (long long)(s.first + t) * a.out_stride) + (long long)h * p.dv;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = (group + groups * j) * 8;
      if (d < p.dv) join_store(out + d, acc[j], p.dv - d);
    }
  }
}

}  // namespace

// Parts: a block's rows and one value more each for maximum and sum, in two slots of every share and map.
static size_t parts_bytes(int dim, int elem) {
  auto all = [&](int maps) -> size_t {
    const int dv = dim * maps, columns = (dim + 15) / 16 * 16 * maps;
    if (maps == 2 && dim > 128) return 0;
    const size_t slots = 2 * (elem == 4 ? kMaxShares * maps : kMaxTensorCtas);
    return align256(sizeof(float) * slots * chunk_slot_floats(elem == 4 ? 64 : columns <= 128 ? 256 : 128, dv));
  };
  return all(1) > all(2) ? all(1) : all(2);
}
// diff, bf16: half of a block's rows and 16 columns at a time, per CTA.
static size_t exchange_bytes(int dim, int elem) {
  const int columns = (dim + 15) / 16 * 16 * 2;
  return elem == 4 || dim > 128 ? 0 : align256(sizeof(float) * kMaxTensorCtas * 64 * (columns <= 128 ? 2 : 1) * columns);
}

size_t chunk_scratch_bytes(int dim, int elem) {
  return align256(sizeof(int4) * kMaxShares) + parts_bytes(dim, elem) + exchange_bytes(dim, elem);
}

cudaError_t launch_chunk_join(const ChunkShape &p, cudaStream_t s) {
  const dim3 grid(p.shares, (p.block + 31) / 32);   // a CTA for 32 rows of an item with one cut
  return p.a.elem == 4 ? launch_early(chunk_join_kernel<float>, grid, kJoinThreads, 0, s, p)
                       : launch_early(chunk_join_kernel<__nv_bfloat16>, grid, kJoinThreads, 0, s, p);
}

cudaError_t launch_chunk(const ChunkArgs &a, cudaStream_t s) {
  ChunkShape p{};
  p.a = a;
  p.maps = a.diff ? 2 : 1;
  p.units = a.cache.heads / p.maps;
  p.group = a.q_heads / a.cache.heads;
  p.dv = a.cache.dim * p.maps;
  p.scale2 = a.scale * kChunkLog2e;
  // measured, 128 / 384 / 448 / 512 / 1024 / 1536 keys: prompts of 24 x 264 - 4352 tokens 624 / 520 / 523 / 526 / 579 / 629 us, differential prefill of
  // 4 x 2944 tokens 634 / 523 / 500 / 488 / 422 / 441 us (its items are 128 rows, and the CTAs of a cluster wait for each other at their ends)
  p.item_keys = a.elem == 4 ? 128 : a.diff ? 1024 : 448;
  p.cuts = reinterpret_cast<int4 *>(a.ws + kStatusBytes);
  p.parts = reinterpret_cast<float *>(a.ws + kStatusBytes + align256(sizeof(int4) * kMaxShares));
  float *exchange = reinterpret_cast<float *>(reinterpret_cast<char *>(p.parts) + parts_bytes(a.cache.dim, a.elem));
  if (a.elem == 4) return launch_chunk_f32(p, s);
  // few rows per sequence, on average: no tile of 128 rows is worth its products.  Measured with 4 query heads a kv-head, 64 sequences of 650 keys and 8
  // of 20000, few rows' kernel against tiles, us: width 128, 16 rows 37 / 47 and 75 / 92, 20 rows 50 / 48 and 122 / 95; 64, 16 rows 29 / 43 and 56 / 77, 20
  // rows 38 / 44 and 90 / 79; 80, 8 rows 30 / 46 and 63 / 86, 12 rows 42 / 46 and 105 / 88.  Differences, 128, 8 rows 45 / 71 and 87 / 121, 12 rows 61 / 72
  // and 140 / 126; 64, 8 rows 34 / 59 and 62 / 104, 12 rows 43 / 59 and 96 / 108; 80, 8 rows 53 / 63 and 111 / 116, 12 rows 79 / 63 and 184 / 121.
  const long long rows = a.seq.batch > 0 ? ((long long)a.tokens * p.group + a.seq.batch - 1) / a.seq.batch : 0;
  const int d = a.cache.dim;
  const bool whole = d == 64 || d == 128;
  if (rows <= (a.diff || !whole ? 8 : 16)) {
    // their items end sooner: differential tokens over 127 x 64 and once 131072 keys 146 / 122 / 129 / 141 us with 128 / 256 / 448 / 1024, over 32
    // sequences of 64 - 20000 keys 418 / 415 / 417 / 424; chunks 87 / 84 / 86 / 91 and 393 / 392 / 389 / 394
    p.item_keys = 256;
    if (a.diff) return whole ? launch_diff_few(p, s) : launch_diff_few_any(p, s);
    if (!whole) return launch_chunk_few_any(p, s);
    return d == 64 ? launch_chunk_few_64(p, rows > 8, s) : launch_chunk_few_128(p, rows > 8, s);
  }
  return launch_chunk_bf16(p, exchange, s);
}

}  // namespace last
