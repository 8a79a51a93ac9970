// Few rows per sequence, chunk attention: heads of any other number of elements.
#include "chunk_few_impl.cuh"

namespace last {

cudaError_t launch_chunk_few_any(const ChunkShape &p, cudaStream_t s) {
  const Few f = few_of(p);
  switch ((p.a.cache.dim + 63) / 64) {
    case 1: return launch_kind<Kind<1, 1, 1, false>>(f, s);
    case 2: return launch_kind<Kind<2, 1, 1, false>>(f, s);
    case 3: return launch_kind<Kind<3, 1, 1, false>>(f, s);
    default: return launch_kind<Kind<4, 1, 1, false>>(f, s);
  }
}

}  // namespace last
