// Cache attention: the workspace and the choice of the kernel.
#include "attend_impl.cuh"

namespace last {

namespace {

constexpr size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t attend_scratch_bytes(int q_heads, int kv_heads, int dim) {
  const int group = q_heads / kv_heads, rows = group < kRows ? group : kRows;
  return align256(sizeof(int4) * kMaxWorkers) + align256(sizeof(float) * kMaxWorkers * 2 * (kStatFloats + (size_t)rows * dim));
}

cudaError_t launch_attend(const AttendArgs &a, cudaStream_t s) {
  Shape p{};
  p.a = a;
  p.group = a.q_heads / a.cache.heads;
  p.passes = (p.group + kRows - 1) / kRows;
  p.heads = p.passes * a.cache.heads;
  p.rows = p.group < kRows ? p.group : kRows;
  p.chunks = (a.cache.dim * a.elem + 127) / 128;
  p.scale2 = a.scale * kLog2e;
  p.jobs = reinterpret_cast<int4 *>(a.ws + kStatusBytes);
  p.parts = reinterpret_cast<float *>(a.ws + kStatusBytes + align256(sizeof(int4) * kMaxWorkers));
  return a.elem == 4 ? launch_attend_f32(p, s) : launch_attend_bf16(p, s);
}

}  // namespace last
