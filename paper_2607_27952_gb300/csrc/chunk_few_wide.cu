// Few rows per sequence, chunk attention over heads of 136 to 256 elements.
#include "chunk_few_impl.cuh"

namespace last {

cudaError_t launch_chunk_few_wide(const ChunkShape &p, cudaStream_t s) {
  const Few f = few_of(p);
  return p.a.cache.dim <= 192 ? launch_kind<Kind<3, 1, 1>>(f, s) : launch_kind<Kind<4, 1, 1>>(f, s);
}

}  // namespace last
