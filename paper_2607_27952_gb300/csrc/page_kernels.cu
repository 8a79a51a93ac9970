// Pages of a cache copied (last_cache_copy) and caches cut to the kept tokens
// (last_cache_compact): copies of head rows, every layer, K and V.
#include "cache_internal.h"
#include "last_device.cuh"

namespace last {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;   // 16-byte pieces of a thread in flight
constexpr int kMaxRows = 4096, kCompactCtas = 3;   // per SM

// x / n; m = ceil(2^32 / n) where x n < 2^32 for every x, else 0.
__device__ __forceinline__ int quotient(int x, int n, uint32_t m) {
  return n == 1 ? x : m != 0 ? (int)__umulhi((uint32_t)x, m) : x / n;
}

// A warp takes BATCH pieces a lane of one page of one layer of K or V at a time.  Bound by HBM: 2048 pages of
// 4 layers (537 MB) 82 us, 6.6 TB/s.
template <int BATCH>
__global__ void __launch_bounds__(kThreads) copy_kernel(const __grid_constant__ PagesArgs p, int n, const int32_t *src,
                                                        const int32_t *dst, int blocks) {
  grid_begins();
  unsigned flags = 0;
  const int lane = threadIdx.x & 31, vec = p.row_bytes / 16, per_page = p.heads * p.page_size * vec;
  const long long items = (long long)n * p.layers * 2 * blocks, step = (long long)gridDim.x * (kThreads / 32);
  for (long long it = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); it < items; it += step) {
    const long long page = blocks == 1 ? it : it / blocks;
    const int block = (int)(it - page * blocks), i = (int)(page / (2 * p.layers)), lk = (int)(page - (long long)i * 2 * p.layers);
    const int from = src[i], to = dst[i];
    if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) {
      flags = kErrCacheIndex;
      continue;
    }
    if (from == to) continue;
    char *base = (lk & 1 ? p.v : p.k) + (lk >> 1) * p.layer_stride;
    const char *x = base + from * p.page_stride;
    char *y = base + to * p.page_stride;
    auto at = [&](int e) {
      if (p.packed) return e * 16LL;
      const int r = e / vec, h = r / p.page_size;
      return h * p.head_stride + (r - h * p.page_size) * p.token_stride + (e - r * vec) * 16;
    };
    const int e = block * 32 * BATCH + lane;
    uint4 v[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (e + u * 32 < per_page) v[u] = *reinterpret_cast<const uint4 *>(x + at(e + u * 32));
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (e + u * 32 < per_page) *reinterpret_cast<uint4 *>(y + at(e + u * 32)) = v[u];
  }
  flags = __syncthreads_or((int)flags);
  if (threadIdx.x == 0) post_status(p.status, blockIdx.x, gridDim.x, flags ? kErrCacheIndex : 0u);
}

// A warp takes a token of a shortened sequence (or, of few tokens, a part of its rows): its place and its
// source are looked up once for all layers and heads, whose rows' addresses each CTA keeps (TABLE:
// where there are no more than kMaxRows).  The tokens of 32 sequences at a time are counted by
// the lanes, every warp alike, and dealt out in turn.  Bound by HBM: 17449 tokens of 4 layers by 4 heads
// (286 MB in rows of 256 bytes) 48 us, 5.9 TB/s; with addresses formed anew for every piece 50 us, with
// two more CTAs per SM and spilled registers 55 us.
template <bool TABLE>
__global__ void __launch_bounds__(kThreads, kCompactCtas) compact_kernel(const __grid_constant__ CompactArgs a, int rows,
                                                                         uint32_t vec_m, uint32_t heads_m) {
  extern __shared__ char *row_at[];   // K or V, layer, head
  const PagesArgs &p = a.p;
  auto row_of = [&](int r) {
    const int lk = quotient(r, p.heads, heads_m);
    return (lk & 1 ? p.v : p.k) + (lk >> 1) * p.layer_stride + (r - lk * p.heads) * p.head_stride;
  };
  if (TABLE) {
    for (int r = threadIdx.x; r < rows; r += kThreads) row_at[r] = row_of(r);
    __syncthreads();
  }
  grid_begins();
  const int lane = threadIdx.x & 31, ps = p.page_size, vec = p.row_bytes / 16, items = rows * vec;
  const int warps = gridDim.x * (kThreads / 32), me = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  unsigned flags = 0;
  long long dealt = 0;   // units of the sequences before
  for (int b0 = 0; b0 < a.seq.batch; b0 += 32) {
    const int mine = b0 + lane;
    int len = 0, first = 0, span = 0, kept = 0, k0 = 0, total = 0;
    if (mine < a.seq.batch) {
      len = a.seq.lens[mine];
      k0 = a.cu_keep[mine];
      const int k1 = a.cu_keep[mine + 1];
      first = a.span_begin ? a.span_begin[mine] : 0;
      span = a.span_len ? a.span_len[mine] : len;
      const bool ok = len >= 0 && first >= 0 && span >= 0 && first <= len && span <= len - first && k0 >= 0 && k0 <= k1 &&
                      k1 <= a.num_idx && len <= (long long)a.seq.max_pages * ps &&
                      (long long)len - span + (k1 - k0) <= (long long)a.dst_max_pages * ps;
      kept = k1 - k0;
      total = ok ? len - span + kept : 0;
      if (!ok) flags = kErrCacheIndex;
      else if (me == 0) a.lens_out[mine] = total;
    }
    long long upto = total;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long x = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += x;
    }
    const long long tokens = __shfl_sync(~0u, upto, 31);
    if (tokens == 0) continue;
    // of few tokens, parts of no less than 4 pieces a lane
    const int most = items / (32 * kBatch);
    int parts = tokens < warps ? (int)(warps / tokens) : 1;
    parts = parts > most ? (most > 1 ? most : 1) : parts;
    const long long units = tokens * parts;
    for (long long u = ((long long)me - dealt % warps + warps) % warps; u < units; u += warps) {
      const long long tok = parts == 1 ? u : u / parts;
      const int part = (int)(u - tok * parts);
      const int own = __popc(__ballot_sync(~0u, upto <= tok));   // the sequence whose tokens hold it
      const int b = b0 + own, j = (int)(tok - (__shfl_sync(~0u, upto, own) - __shfl_sync(~0u, total, own)));
      const int f = __shfl_sync(~0u, first, own), sp = __shfl_sync(~0u, span, own), kp = __shfl_sync(~0u, kept, own);
      int from = j;
      if (j >= f + kp) from = j + sp - kp;
      else if (j >= f) {
        const int i = a.idx[__shfl_sync(~0u, k0, own) + j - f];
        from = i >= 0 && i < sp ? f + i : -1;
      }
      const int to_page = a.dst_table[b * a.dst_stride + j / ps];
      const int page = from >= 0 ? a.seq.table[b * a.seq.table_stride + from / ps] : -1;
      if (page < 0 || page >= p.num_pages || to_page < 0 || to_page >= p.num_pages) {
        flags = kErrCacheIndex;
        continue;
      }
      const long long x = page * p.page_stride + (from % ps) * p.token_stride;
      const long long y = to_page * p.page_stride + (j % ps) * p.token_stride;
      if (x == y) continue;
      const int i0 = parts == 1 ? 0 : (int)((long long)items * part / parts);
      const int i1 = parts == 1 ? items : (int)((long long)items * (part + 1) / parts);
      for (int i = i0 + lane; i < i1; i += 32 * kBatch) {
        uint4 v[kBatch];
        char *at[kBatch];   // piece of the token
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
          const int r = quotient(min(i + n * 32, items - 1), vec, vec_m);
          at[n] = (TABLE ? row_at[r] : row_of(r)) + (i + n * 32 - r * vec) * 16;
          if (i + n * 32 < i1) v[n] = *reinterpret_cast<const uint4 *>(at[n] + x);
        }
#pragma unroll
        for (int n = 0; n < kBatch; ++n)
          if (i + n * 32 < i1) *reinterpret_cast<uint4 *>(at[n] + y) = v[n];
      }
    }
    dealt += units;
  }
  flags = __syncthreads_or((int)flags);
  if (threadIdx.x == 0) post_status(p.status, blockIdx.x, gridDim.x, flags ? kErrCacheIndex : 0u);
}

int grid_of(long long items) {
  const long long most = sm_count() * 8LL < kMaxStatus ? sm_count() * 8LL : kMaxStatus;
  return (int)(items < 1 ? 1 : items < most ? items : most);
}

}  // namespace

cudaError_t launch_page_copy(const PagesArgs &args, int n, const int32_t *src, const int32_t *dst, cudaStream_t s) {
  PagesArgs p = args;
  // a page's rows one after the other, in either order
  const long long row = p.row_bytes, ps = p.page_size;
  p.packed = (p.token_stride == row && (p.heads == 1 || p.head_stride == row * ps)) ||
             (p.token_stride == row * p.heads && (p.heads == 1 || p.head_stride == row));
  const long long pieces = (long long)p.heads * p.page_size * (p.row_bytes / 16), pages = (long long)n * p.layers * 2;
  auto go = [&](auto kernel, int batch) {
    const int blocks = (int)((pieces + 32 * batch - 1) / (32 * batch));
    const long long items = pages * blocks;
    return launch_early(kernel, dim3(grid_of((items + kThreads / 32 - 1) / (kThreads / 32))), kThreads, 0, s, p, n, src, dst, blocks);
  };
  // eight pieces a lane where that leaves every SM its warps several times over: 2048 pages of 4 layers
  // 86.0 us with four, 81.5 with eight; 64 pages 3.3 and 3.8
  return pages * pieces >= 32LL * 8 * 256 * sm_count() ? go(copy_kernel<8>, 8) : go(copy_kernel<4>, 4);
}

cudaError_t launch_compact(const CompactArgs &a, cudaStream_t s) {
  const int rows = a.p.layers * 2 * a.p.heads, vec = a.p.row_bytes / 16;
  auto magic = [](long long most, int n) {
    return most * n < 1LL << 32 ? (uint32_t)(((1ull << 32) + (unsigned)n - 1) / (unsigned)n) : 0u;
  };
  const long long most = (long long)a.seq.batch * a.dst_max_pages * a.p.page_size * rows * vec / (32 * kBatch);   // units
  const long long ctas = (long long)sm_count() * kCompactCtas, need = most / (kThreads / 32) + 1;
  const int grid = (int)(need < ctas ? need : ctas < kMaxStatus ? ctas : kMaxStatus);
  const uint32_t vm = magic((long long)rows * vec, vec), hm = magic(rows, a.p.heads);
  if (rows <= kMaxRows)
    return launch_early(compact_kernel<true>, dim3(grid), kThreads, rows * sizeof(char *), s, a, rows, vm, hm);
  return launch_early(compact_kernel<false>, dim3(grid), kThreads, 0, s, a, rows, vm, hm);
}

}  // namespace last
