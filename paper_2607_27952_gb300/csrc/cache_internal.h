// What the key-value cache's entry points hand to their kernels.
#pragma once

#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>

#include "last.h"

namespace last {

// Device status of the cache calls.  They copy nothing into the workspace beforehand, so a
// flag word would start undefined: every CTA writes its own word instead, and the first
// one writes word 0 = kErrList | number of words, for last_poll to gather.
constexpr unsigned kErrList = 1u << 31;
constexpr unsigned kErrCacheIndex = 8u;   // a page, an index or a length was out of range
constexpr int kStatusBegin = 64;          // first CTA's word
constexpr int kMaxStatus = 4032;          // CTAs of one launch at most
constexpr size_t kStatusBytes = 4 * (kStatusBegin + kMaxStatus);

constexpr int kMaxRotPairs = 128;
constexpr int kMaxAxes = 4;

// One layer of a cache (strides in bytes).
struct CacheLayer {
  char *k, *v;
  long long page_stride, head_stride, token_stride;
  int num_pages, page_size, heads, dim;
};

struct SequenceView {
  const int32_t *table, *lens, *begin;
  long long table_stride;
  int batch, max_pages;
};

// Angles in units of 2^-64 turns per position: position * turn wraps modulo one turn.
struct RotaryTable {
  unsigned long long turn[kMaxRotPairs];
  uint8_t axis[kMaxRotPairs];
  int half;       // pairs
  int adjacent;   // pairs of neighbours
};

struct HeadRows {   // strides in bytes
  const char *in;
  char *out;
  long long in_token, in_head, out_token, out_head;
  int heads;
};

struct RotaryArgs {
  RotaryTable rot;
  HeadRows q, k, v;   // last_rope: q, k; append: k and v go to the cache
  const int32_t *positions;
  long long axis_stride;
  int tokens, dim, elem;
  bool backward, append;
  CacheLayer cache;
  SequenceView seq;
  const int32_t *cu_new;
  unsigned *status;
};

struct AttendArgs {
  CacheLayer cache;
  SequenceView seq;
  int q_heads, elem;
  float scale;
  const char *q;
  char *out;
  long long q_stride, out_stride;   // bytes
  float *lse;
  char *ws;
};

struct ChunkArgs {   // attention of several new tokens per sequence; diff: the difference of two maps
  CacheLayer cache;
  SequenceView seq;
  const int32_t *cu_new;
  int tokens, q_heads, elem;
  float scale;
  bool causal, diff;
  int window;                       // 0: none
  const char *q;
  char *out;
  long long q_stride, out_stride;   // bytes
  float *lse;
  const float *lambda, *norm_weight;
  float norm_eps, out_scale;
  char *ws;
};

struct PagesArgs {   // copy and compact: every layer
  char *k, *v;
  long long layer_stride, page_stride, head_stride, token_stride;   // bytes
  int layers, num_pages, page_size, heads, row_bytes;
  bool packed;   // copy: a page's rows follow each other without a gap
  unsigned *status;
};

struct CompactArgs {
  PagesArgs p;
  SequenceView seq;
  const int32_t *dst_table;
  long long dst_stride;
  int dst_max_pages;
  const int32_t *span_begin, *span_len, *cu_keep, *idx;
  int num_idx;
  int32_t *lens_out;
};

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t s);
cudaError_t launch_attend(const AttendArgs &a, cudaStream_t s);
cudaError_t launch_chunk(const ChunkArgs &a, cudaStream_t s);
cudaError_t launch_page_copy(const PagesArgs &a, int n, const int32_t *src, const int32_t *dst, cudaStream_t s);
cudaError_t launch_compact(const CompactArgs &a, cudaStream_t s);
// Workspace of the attention behind the status words.
size_t attend_scratch_bytes(int q_heads, int kv_heads, int dim);
size_t chunk_scratch_bytes(int dim, int elem);

// SMs of the current device.
int sm_count();

#ifdef __CUDACC__
// Kernels of the cache are launched as soon as the one before them in the stream has all its CTAs running, and
// wait here, before they touch memory, for it to end: the launch itself costs nothing then.
__device__ __forceinline__ void grid_begins() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, const A &...args) {
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  c.attrs = at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, P(args)...);
}
__device__ __forceinline__ void post_status(unsigned *status, unsigned cta, unsigned ctas, unsigned flags) {
  status[kStatusBegin + cta] = flags;
  if (cta == 0) status[0] = kErrList | ctas;
}
#endif

}  // namespace last
