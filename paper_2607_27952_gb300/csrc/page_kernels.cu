// Pages of a cache copied (last_cache_copy) and caches cut to the kept tokens
// (last_cache_compact): copies of head rows, every layer, K and V.
#include "cache_internal.h"
#include "last_device.cuh"

namespace last {

namespace {

constexpr int kThreads = 256;

// One page of one layer of K or V per step.
__global__ void __launch_bounds__(kThreads) copy_kernel(const __grid_constant__ PagesArgs p, int n, const int32_t *src,
                                                        const int32_t *dst) {
  unsigned flags = 0;
  const int vec = p.row_bytes / 16, per_page = p.heads * p.page_size * vec;
  const long long items = (long long)n * p.layers * 2;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int i = (int)(it / (2 * p.layers)), lk = (int)(it - (long long)i * 2 * p.layers);
    const int from = src[i], to = dst[i];
    if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) {
      flags = kErrCacheIndex;
      continue;
    }
    if (from == to) continue;
    char *base = (lk & 1 ? p.v : p.k) + (lk >> 1) * p.layer_stride;
    const char *x = base + from * p.page_stride;
    char *y = base + to * p.page_stride;
    for (int e = threadIdx.x; e < per_page; e += kThreads) {
      const int r = e / vec, h = r / p.page_size;
      const long long at = h * p.head_stride + (r - h * p.page_size) * p.token_stride + (e - r * vec) * 16;
      *reinterpret_cast<uint4 *>(y + at) = *reinterpret_cast<const uint4 *>(x + at);
    }
  }
  if (threadIdx.x == 0) post_status(p.status, blockIdx.x, gridDim.x, flags);
}

// One destination page of one layer of K or V per step.
__global__ void __launch_bounds__(kThreads) compact_kernel(const __grid_constant__ CompactArgs a) {
  const PagesArgs &p = a.p;
  unsigned flags = 0;
  const int vec = p.row_bytes / 16, ps = p.page_size;
  const long long items = (long long)a.seq.batch * a.dst_max_pages * p.layers * 2;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int lk = (int)(it % (2 * p.layers));
    const long long bp = it / (2 * p.layers);
    const int b = (int)(bp / a.dst_max_pages), page = (int)(bp - (long long)b * a.dst_max_pages);
    const int len = a.seq.lens[b], k0 = a.cu_keep[b], k1 = a.cu_keep[b + 1];
    const int first = a.span_begin ? a.span_begin[b] : 0, span = a.span_len ? a.span_len[b] : len;
    const bool ok = len >= 0 && first >= 0 && span >= 0 && first <= len && span <= len - first && k0 >= 0 && k0 <= k1 &&
                    k1 <= a.num_idx && len <= (long long)a.seq.max_pages * ps &&
                    (long long)len - span + (k1 - k0) <= (long long)a.dst_max_pages * ps;
    if (!ok) {
      flags |= kErrCacheIndex;
      continue;
    }
    const int kept = k1 - k0, total = len - span + kept;
    if (page == 0 && lk == 0 && threadIdx.x == 0) a.lens_out[b] = total;
    const int rows = min(ps, total - page * ps);
    if (rows <= 0) continue;
    const int to = a.dst_table[b * a.dst_stride + page];
    if (to < 0 || to >= p.num_pages) {
      flags |= kErrCacheIndex;
      continue;
    }
    char *base = (lk & 1 ? p.v : p.k) + (lk >> 1) * p.layer_stride;
    for (int e = threadIdx.x; e < rows * p.heads * vec; e += kThreads) {
      const int r = e / vec, h = r / rows, j = page * ps + (r - h * rows);
      int from = j;
      if (j >= first + kept) from = j + span - kept;
      else if (j >= first) {
        const int i = a.idx[k0 + j - first];
        from = i >= 0 && i < span ? first + i : -1;
      }
      const int sp = from >= 0 ? a.seq.table[b * a.seq.table_stride + from / ps] : -1;
      if (sp < 0 || sp >= p.num_pages) {
        flags |= kErrCacheIndex;
        continue;
      }
      const long long x = sp * p.page_stride + (from % ps) * p.token_stride, y = to * p.page_stride + (j % ps) * p.token_stride;
      if (x == y) continue;
      const long long in = h * p.head_stride + (e - r * vec) * 16;
      *reinterpret_cast<uint4 *>(base + y + in) = *reinterpret_cast<const uint4 *>(base + x + in);
    }
  }
  flags = __syncthreads_or((int)flags);
  if (threadIdx.x == 0) post_status(p.status, blockIdx.x, gridDim.x, flags ? kErrCacheIndex : 0u);
}

int grid_of(long long items) {
  const long long most = sm_count() * 8LL < kMaxStatus ? sm_count() * 8LL : kMaxStatus;
  return (int)(items < 1 ? 1 : items < most ? items : most);
}

}  // namespace

cudaError_t launch_page_copy(const PagesArgs &p, int n, const int32_t *src, const int32_t *dst, cudaStream_t s) {
  copy_kernel<<<grid_of((long long)n * p.layers * 2), kThreads, 0, s>>>(p, n, src, dst);
  return cudaGetLastError();
}

cudaError_t launch_compact(const CompactArgs &a, cudaStream_t s) {
  compact_kernel<<<grid_of((long long)a.seq.batch * a.dst_max_pages * a.p.layers * 2), kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace last
