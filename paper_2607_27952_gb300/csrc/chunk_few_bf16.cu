// Few rows per sequence, chunk attention over heads of up to 128 elements.
#include "chunk_few_impl.cuh"

namespace last {

cudaError_t launch_chunk_few(const ChunkShape &p, int rows, cudaStream_t s) {
  const Few f = few_of(p);
  if (p.a.cache.dim > 128) return launch_chunk_few_wide(p, s);
  if (p.a.cache.dim <= 64) return rows > 8 ? launch_kind<Kind<1, 2, 1>>(f, s) : launch_kind<Kind<1, 1, 1>>(f, s);
  return rows > 8 ? launch_kind<Kind<2, 2, 1>>(f, s) : launch_kind<Kind<2, 1, 1>>(f, s);
}

}  // namespace last
