// Attention of chunks of new tokens over a paged cache (last_cache_chunk_attention, last_cache_diff_attention):
// what the kernels for bf16 and fp32 share.
//
// The new tokens of a sequence and the query heads of one kv-head are rows of one matrix, token by token
// (row r: token r / group, head r % group), cut into blocks.  An item is a block and a kv-head; its keys are
// tiles.  All items' tiles, one after the other, are cut into equal shares, one per CTA, wherever the cuts fall;
// sums that a cut has parted go to the workspace and join_kernel adds them up:
//   o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i,  m = max_i m_i.
// A share is found from the lengths alone: the cost of a sequence's first x blocks is a closed form
// (below), so that a CTA needs a sum over the sequences and a search over x, and a cut lies at the same
// tile for the CTAs on both of its sides.
//
// diff: maps 0 and 1 of a pair of query heads; a unit is a pair of kv-heads, and the value of a key is the pair's two
// rows of V side by side.
#pragma once

#include <cuda_bf16.h>

#include "cache_internal.h"
#include "last_device.cuh"
#include "last_internal.h"
#include "mma16816.cuh"

namespace last {

struct ChunkShape {   // the same for every CTA
  ChunkArgs a;
  int units, group;   // kv-heads (diff: pairs of them); query heads (pairs) per unit
  int block, tile;    // rows of an item, keys of a tile
  int pitch;          // rows of a part: the block's, up to a multiple of 4
  int dv, maps;       // width of a value; 2 for diff
  int shares;
  int item_keys;      // what an item costs beside its keys, in keys
  float scale2;       // times log2(e)
  int4 *cuts;         // [shares] where a share ends: sequence, unit, block, tile (0: between two items)
  float *parts;       // [shares][maps][2] parted sums: second one where an item begins in the share
};

// bf16 tiles: a CTA per SM.  fp32 and few rows: up to two, with smaller parts.
constexpr int kMaxTensorCtas = 160, kMaxShares = 2 * kMaxTensorCtas;
constexpr int kMaxKeys = 0x7fffff00;   // of a sequence: the last key's tile ends before 2^31
constexpr float kChunkLog2e = 1.4426950408889634f, kChunkLn2 = 0.6931471805599453f;

cudaError_t launch_chunk_f32(ChunkShape p, cudaStream_t s);
cudaError_t launch_chunk_bf16(ChunkShape p, float *exchange, cudaStream_t s);
// bf16, few rows; sixteen: in blocks of 16 instead of 8.
cudaError_t launch_chunk_few_64(const ChunkShape &p, bool sixteen, cudaStream_t s);
cudaError_t launch_chunk_few_128(const ChunkShape &p, bool sixteen, cudaStream_t s);
cudaError_t launch_chunk_few_any(const ChunkShape &p, cudaStream_t s);
cudaError_t launch_diff_few(const ChunkShape &p, cudaStream_t s);
cudaError_t launch_diff_few_any(const ChunkShape &p, cudaStream_t s);
// Adds up what the cuts have parted.
cudaError_t launch_chunk_join(const ChunkShape &p, cudaStream_t s);

// A part: its rows' maxima and sums, then four columns of all rows at a time.
__host__ __device__ inline size_t chunk_slot_floats(int pitch, int dv) { return (size_t)pitch * (dv + 2); }

#ifdef __CUDACC__
__device__ __forceinline__ float *chunk_slot(const ChunkShape &p, int share, int map, int second) {
  return p.parts + (((size_t)share * p.maps + map) * 2 + second) * chunk_slot_floats(p.pitch, p.dv);
}

__device__ __forceinline__ float chunk_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Waits end after two seconds by the clock.
constexpr unsigned long long kWaitNanoseconds = 2000000000ull;
struct ChunkLimit {
  unsigned long long begin = 0;
  uint32_t tries = 0;
  template <typename S>
  __device__ __forceinline__ bool over(const S &sm) {
    if ((tries++ & 63) != 0) return false;
    unsigned long long now;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
    if (begin == 0) begin = now;
    return sm.dead != 0 || now - begin > kWaitNanoseconds;
  }
};
// A whole warp waits, with a limit; the first to give up has every other wait of the CTA end too.  Warps that meet
// in barriers go on after a wait that gave up, with whatever is there, to the end of their item, so that no barrier waits for one
// that has left; the others leave.
template <typename S>
__device__ __forceinline__ bool wait(S &sm, unsigned long long *bar, uint32_t parity) {
  bool ok = mbar_try_wait(bar, parity);
  if (!ok)
    for (ChunkLimit limit; !ok && !limit.over(sm);) ok = mbar_try_wait(bar, parity);
  if (__all_sync(~0u, ok)) return true;
  sm.dead = 1;
  return false;
}

struct ChunkSeq {   // n new tokens from token `first` on, behind `base` cached ones; keys begin .. lens - 1
  int first, n, base, begin, lens;
};
// New tokens out of range: none are there.  A length or first key out of range: there is no key.
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs &a, int b, unsigned *bad) {
  ChunkSeq s{0, 0, 0, 0, 0};
  const int first = a.cu_new ? a.cu_new[b] : b, next = a.cu_new ? a.cu_new[b + 1] : b + 1;
  const int lens = a.seq.lens[b], begin = a.seq.begin ? a.seq.begin[b] : 0;
  if (first < 0 || next < first || next > a.tokens) {
    *bad = kErrCacheIndex;
    return s;
  }
  s.first = first;
  s.n = next - first;
  if (s.n == 0) return s;
  if (lens < s.n || lens > kMaxKeys || lens > (long long)a.seq.max_pages * a.cache.page_size || begin < 0) {
    *bad = kErrCacheIndex;
    return s;
  }
  s.base = lens - s.n;
  s.begin = begin;
  s.lens = lens;
  return s;
}
// Keys lo .. hi - 1 that new token i sees.
__device__ __forceinline__ int chunk_lo(const ChunkArgs &a, const ChunkSeq &s, int i) {
  return a.window > 0 ? max(s.begin, s.base + i - (a.window - 1)) : s.begin;
}
__device__ __forceinline__ int chunk_hi(const ChunkArgs &a, const ChunkSeq &s, int i) {
  return a.causal ? min(s.base + i + 1, s.lens) : s.lens;
}

struct ChunkTiles {   // of rows r0 .. r1 - 1: visible keys of any of them, and their tiles
  int lo, hi, first, count;
};
__device__ __forceinline__ ChunkTiles chunk_tiles(const ChunkShape &p, const ChunkSeq &s, int r0, int r1) {
  ChunkTiles t;
  t.lo = chunk_lo(p.a, s, r0 / p.group);
  t.hi = chunk_hi(p.a, s, (r1 - 1) / p.group);
  t.first = t.lo / p.tile;
  t.count = t.lo < t.hi ? (t.hi - 1) / p.tile - t.first + 1 : 0;
  return t;
}
__device__ __forceinline__ int chunk_blocks(const ChunkShape &p, const ChunkSeq &s) {
  return (int)(((long long)s.n * p.group + p.block - 1) / p.block);
}

// Cost of a unit's first x blocks, in keys times group: block y sees, of its last row, base - begin + (y + 1) block /
// group keys, none below zero and no more than the window (with the block's own tokens) or the sequence has.  The host refuses calls whose
// sums could reach 2^62.
struct ChunkCost {
  long long a, most, item;
  int block;
  bool flat;
  __device__ ChunkCost(const ChunkShape &p, const ChunkSeq &s) {
    const long long g = p.group, all = g * max(0, s.lens - s.begin);
    block = p.block;
    item = g * p.item_keys;
    flat = !p.a.causal;
    a = g * ((long long)s.base - s.begin);
    most = p.a.window > 0 ? min(all, g * p.a.window + p.block) : all;
  }
  __device__ long long upto(long long x) const {
    if (flat) return x * (most + item);
    const long long none = a < 0 ? -a / block : 0, grow = most > a ? (most - a) / block : 0;
    const long long x0 = min(x, none), x1 = min(x, max(none, grow));
    return (x1 - x0) * a + block * (x1 * (x1 + 1) - x0 * (x0 + 1)) / 2 + (x - x1) * most + x * item;
  }
};

struct ChunkPos {   // the tiles of item (seq, unit, block) before `tile` are behind it
  int seq, unit, block, tile;
};
__device__ __forceinline__ bool same_item(const ChunkPos &x, const ChunkPos &y) {
  return x.seq == y.seq && x.unit == y.unit && x.block == y.block;
}

__device__ inline ChunkPos chunk_locate(const ChunkShape &p, const ChunkSeq &s, int b, unsigned long long at) {
  const ChunkCost cost(p, s);
  const int blocks = chunk_blocks(p, s);
  const unsigned long long per = cost.upto(blocks);
  ChunkPos pos;
  pos.seq = b;
  pos.unit = (int)(at / per);
  const long long rest = (long long)(at - per * pos.unit);
  int x = 0, end = blocks;   // the last x whose blocks before cost no more than `rest`
  while (end - x > 1) {
    const int mid = x + (end - x) / 2;
    if (cost.upto(mid) <= rest) x = mid;
    else end = mid;
  }
  pos.block = x;
  const long long before = cost.upto(x);
  const int rows = (int)min((long long)p.block, (long long)s.n * p.group - (long long)x * p.block);
  const int tiles = max(1, chunk_tiles(p, s, x * p.block, x * p.block + rows).count);
  pos.tile = (int)((double)(rest - before) / (double)(cost.upto(x + 1) - before) * tiles + 0.5);
  return pos;
}

// Where this CTA's share begins and ends, by all threads (`sums`: one per warp).  A position behind the
// last item has seq = batch.
struct ChunkShare {
  ChunkPos begin, end;
};
template <int THREADS>
__device__ void chunk_share(const ChunkShape &p, int share, unsigned long long *sums, ChunkShare *out, unsigned *flags) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.a.seq.batch;
  constexpr int kShareWarps = THREADS / 32;
  unsigned bad = 0;
  unsigned long long mine = 0;
  const int per = (B + THREADS - 1) / THREADS, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  for (int b = b0; b < b1; ++b) {
    const ChunkSeq s = chunk_seq(p.a, b, &bad);
    if (s.n > 0) mine += ChunkCost(p, s).upto(chunk_blocks(p, s)) * p.units;
  }
  unsigned long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long x = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sums[warp] = upto;
  if (tid == 0) out->begin = out->end = ChunkPos{B, 0, 0, 0};
  __syncthreads();
  if (bad) atomicOr(flags, bad);
  unsigned long long total = 0;
  for (int w = 0; w < kShareWarps; ++w) {
    if (w < warp) upto += sums[w];
    total += sums[w];
  }
  const unsigned long long whole = total / p.shares, rest = total - whole * p.shares;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned long long w = share + i, at = whole * w + rest * w / p.shares;
    if (at < upto - mine || at >= upto) continue;
    unsigned long long from = at - (upto - mine);
    for (int b = b0; b < b1; ++b) {
      const ChunkSeq s = chunk_seq(p.a, b, &bad);
      const unsigned long long cost = s.n > 0 ? ChunkCost(p, s).upto(chunk_blocks(p, s)) * p.units : 0;
      if (from < cost) {
        (i ? out->end : out->begin) = chunk_locate(p, s, b, from);
        break;
      }
      from -= cost;
    }
  }
  __syncthreads();
}

// The items of a share one after the other.
struct ChunkItem {
  ChunkSeq s;
  int seq, unit, block;
  int r0, rows;         // of the sequence's rows
  ChunkTiles t;         // of all rows
  int k0, k1;           // this share's of the item's tiles
  bool whole;
  int second;           // slot of a part
};
struct ChunkWalk {
  ChunkPos at, end;
  ChunkSeq s;
  int blocks, loaded;   // loaded: the sequence that s is of
  __device__ explicit ChunkWalk(const ChunkShare &sh) : at(sh.begin), end(sh.end), blocks(0), loaded(-1) {}
  __device__ bool next(const ChunkShape &p, ChunkItem *o) {
    unsigned bad = 0;
    while (at.seq < p.a.seq.batch) {
      if (loaded != at.seq) {
        s = chunk_seq(p.a, at.seq, &bad);
        blocks = chunk_blocks(p, s);
        loaded = at.seq;
      }
      const bool last = same_item(at, end);
      if (at.seq > end.seq) return false;
      if (at.block < blocks) {
        o->s = s;
        o->seq = at.seq;
        o->unit = at.unit;
        o->block = at.block;
        o->r0 = at.block * p.block;
        o->rows = (int)min((long long)p.block, (long long)s.n * p.group - o->r0);
        o->t = chunk_tiles(p, s, o->r0, o->r0 + o->rows);
        const int tiles = max(1, o->t.count);
        o->k0 = at.tile;
        o->k1 = last ? min(end.tile, tiles) : tiles;
        o->whole = o->k0 == 0 && o->k1 == tiles;
        o->second = o->k0 == 0;
      } else {
        o->k0 = o->k1 = 0;
      }
      // on to the next item
      if (last) at = ChunkPos{p.a.seq.batch, 0, 0, 0};
      else {
        at.tile = 0;
        if (++at.block >= blocks) {
          at.block = 0;
          if (++at.unit >= p.units || blocks == 0) {
            at.unit = 0;
            ++at.seq;
          }
        }
      }
      if (o->k0 < o->k1) return true;
    }
    return false;
  }
};
// A cut inside an item, else tile 0.
__device__ __forceinline__ int4 chunk_cut(const ChunkShape &p, const ChunkPos &e) {
  int tile = 0;
  if (e.seq < p.a.seq.batch) {
    unsigned bad = 0;
    const ChunkSeq s = chunk_seq(p.a, e.seq, &bad);
    const int r0 = e.block * p.block, rows = (int)min((long long)p.block, (long long)s.n * p.group - r0);
    if (e.tile < max(1, chunk_tiles(p, s, r0, r0 + rows).count)) tile = e.tile;
  }
  return make_int4(e.seq, e.unit, e.block, tile);
}

__device__ __forceinline__ float chunk_factor(float top, float all) { return top == -INFINITY ? 1.0f : chunk_exp2(top - all); }
__device__ __forceinline__ float chunk_lse(float top, float sum) {
  return sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kChunkLn2;
}
// What a row of diff is multiplied by besides the weights, from the sum of its squares.
__device__ __forceinline__ float chunk_norm(const ChunkArgs &a, float squares, int dv) {
  if (a.norm_weight == nullptr) return a.out_scale;
  const float mean = squares / (float)dv + a.norm_eps;
  return mean == 0.0f ? 0.0f : a.out_scale / sqrtf(mean);
}
#endif

}  // namespace last
