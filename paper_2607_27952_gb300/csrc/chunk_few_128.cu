// Few rows per sequence, chunk attention: heads of 128 elements.
#include "chunk_few_impl.cuh"

namespace last {

cudaError_t launch_chunk_few_128(const ChunkShape &p, bool sixteen, cudaStream_t s) {
  const Few f = few_of(p);
  return sixteen ? launch_kind<Kind<2, 2, 1, true>>(f, s) : launch_kind<Kind<2, 1, 1, true>>(f, s);
}

}  // namespace last
