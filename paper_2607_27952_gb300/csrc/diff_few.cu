// Few rows per sequence, differential attention: heads of 64 and 128 elements.
#include "chunk_few_impl.cuh"

namespace last {

cudaError_t launch_diff_few(const ChunkShape &p, cudaStream_t s) {
  const Few f = few_of(p);
  return p.a.cache.dim == 64 ? launch_kind<Kind<1, 1, 2, true>>(f, s) : launch_kind<Kind<2, 1, 2, true>>(f, s);
}

}  // namespace last
