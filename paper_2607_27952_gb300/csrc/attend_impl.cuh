// Attention of one new token per sequence over a paged cache (last_cache_attention).
//
// With z_p = scale q.k_p in units of log 2 and the running maximum m of the keys seen so far,
//   l <- l 2^(m - m') + sum 2^(z_p - m'),  o <- o 2^(m - m') + sum 2^(z_p - m') v_p
// is one pass over K and V; sums over parts of the keys join by the same rule, so that the
// keys of all sequences and kv-heads are cut into equal shares, one per CTA, wherever the
// cuts fall (join_kernel adds up what a cut has parted).  The work is reading K and V: each
// is read once for up to 16 query heads of its kv-head.
//
// A CTA: one warp keeps a ring of tiles filled with TMA boxes of the pages (128-byte swizzle),
// four take a quarter of every tile each, with sums of their own, and one adds them up where
// the CTA's part of a (sequence, head) ends.  Two CTAs per SM keep some 160 KB of K and V under way.
//
// Bound by HBM: 1.42 GB of K and V (6 sequences of about 115 thousand keys) take 211 us, 6.7 TB/s; 340 MB (64 of
// about 650 keys, 16 kv-heads) 59.5 us, of which 8 are the start (lengths, page table, first tile: three reads
// that wait for each other) and the join: 6.6 TB/s in between.  A tile of 64 keys by 128 arrives every 2600 cycles and its
// products take 1450; one CTA of eight such warps and one loader per SM took 87 and 294 us.
#pragma once

#include <cuda_bf16.h>

#include "cache_internal.h"
#include "last_device.cuh"
#include "last_internal.h"
#include "mma16816.cuh"
#include "tensor_map.h"

namespace last {

struct Shape {      // the same for every CTA
  AttendArgs a;
  int group, passes, heads;   // q-heads per kv-head, passes over a kv-head, passes in all
  int box_log, chunks;        // rows of a TMA box; 128-byte columns of a row
  int stages, slots;          // ring; parts whose q is kept
  bool joined;                // a box holds all of them
  int page_log;               // of the page size, -1 if it is no power of two
  int tile;                   // keys
  int rows;                   // heads of a pass at most
  float scale2;               // scale log2 e
  int4 *jobs;                 // [CTAs] of the (sequence, head) that a CTA's share ends within: these, the share it
                              // begins in, and 2 x shares it spans (0: none) + whether it is the first one's second part
  float *parts;               // [CTAs][2] sums that a cut has parted
};

cudaError_t launch_attend_bf16(const Shape &p, cudaStream_t s);
cudaError_t launch_attend_f32(const Shape &p, cudaStream_t s);

namespace {

constexpr int kWarps = 4;                      // consumers: a quarter of every tile each
constexpr int kThreads = 32 * (kWarps + 2);    // and one to load, one to add up
constexpr int kRows = 16;                      // query heads of one pass over a kv-head
constexpr int kMaxWorkers = 480;               // CTAs
constexpr int kMaxStages = 12;                 // of the ring: K or V of a tile each
constexpr int kMergeFloats = 512;              // of a warp's sums laid down at a time: 8 x 64, 4 x 128 or 2 x 256
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct TileInfo {   // what the producer says of a tile
  int seq, head;    // head: pass over a kv-head
  int lo, hi;       // keys of the tile that count
  int flags, slot;  // slot: of the part's q
};
// First and last tile of the CTA's part of a (sequence, head); the part is all of it; it is not the
// CTA's first one.
constexpr int kFirst = 1, kLast = 2, kWhole = 4, kLater = 8, kEnd = 16;   // kEnd: the CTA's last tile
constexpr int kSkip = 8;   // flags from this bit on: boxes of the tile whose page is out of range, left out
constexpr int kStatFloats = 2 * kRows;   // of a parted sum: maximum and denominator per head, then the rows

struct Keys {
  int begin, end;
};
struct Walk {   // tile `at` of the `tiles` of sequence seq, pass head
  int seq, head, at, tiles;
  Keys keys;
};

struct alignas(16) Merge {
  float rows[kWarps][kMergeFloats + 8 * 8];   // 8 floats apart
  float top[kWarps][kRows], sum[kWarps][kRows];
  unsigned long long laid, read;
  TileInfo info;
};

struct alignas(16) Shared {
  unsigned long long full[kMaxStages], empty[kMaxStages], never;
  TileInfo info[kMaxStages];
  Merge merge[2];
  float scale[kWarps][8];   // of the pass being added up
  bool none[8];
  int4 job;
  Walk start;
  unsigned warp_tiles[kWarps + 2];
  unsigned flags;
  volatile unsigned dead;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A whole warp waits, with a limit; the first to give up has every other wait of the CTA end too.
__device__ __forceinline__ bool wait(Shared &sm, unsigned long long *bar, uint32_t parity) {
  bool ok = false;
  for (uint32_t i = 0; i < kWaitLimit && !ok; ++i) {
    ok = mbar_try_wait(bar, parity);
    if ((i & 31) == 31 && sm.dead) break;
  }
  if (__all_sync(~0u, ok)) return true;
  sm.dead = 1;
  return false;
}

// A sequence whose length or first key is out of range has none.
__device__ __forceinline__ Keys keys_of(const AttendArgs &a, int b, unsigned *bad) {
  const long long room = (long long)a.seq.max_pages * a.cache.page_size;
  const int end = a.seq.lens[b], begin = a.seq.begin ? a.seq.begin[b] : 0;
  if (end >= 0 && end <= room && begin >= 0) return Keys{begin, end};
  *bad = kErrCacheIndex;
  return Keys{0, 0};
}
__device__ __forceinline__ int tiles_of(Keys k, int tile) {
  return k.begin < k.end ? (k.end - 1) / tile - k.begin / tile + 1 : 0;
}

// Where a row of a tile lies: boxes of 2^box_log rows, in each the 128-byte columns one after the other.
__device__ __forceinline__ uint32_t row_at(const Shape &p, int row) {
  return ((row >> p.box_log) * p.chunks << (p.box_log + 7)) + (row & ((1 << p.box_log) - 1)) * 128;
}

__device__ __forceinline__ float join_factor(float top, float all) { return top == -INFINITY ? 1.0f : exp2_fast(top - all); }
__device__ __forceinline__ float lse_of(float top, float sum) { return sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2; }

// The warps' sums of the CTA's part of a (sequence, head) are added up by a warp of its own, as many rows
// and columns at a time as a buffer holds, while the others go on with the next part.  Two buffers by turns.
struct Pass {   // the same sequence of passes on both sides
  int row_log, cols, ld;   // rows and columns at a time
  __device__ Pass(int n) : row_log(n > 4 ? 3 : n > 2 ? 2 : 1), cols(kMergeFloats >> row_log), ld(cols + 8) {}
};

template <typename Part>
__device__ bool lay_down(const Shape &p, Shared &sm, Part &part, const TileInfo &ti, int &passes) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = p.a.cache.dim;
  const int n = min(kRows, p.group - ti.head % p.passes * kRows);
  const Pass s(n);
  for (int row0 = 0; row0 < n; row0 += 1 << s.row_log)
    for (int col0 = 0; col0 < D; col0 += s.cols, ++passes) {
      Merge &m = sm.merge[passes & 1];
      if (passes > 1 && !wait(sm, &m.read, (passes >> 1 & 1) ^ 1)) return false;
      part.stats(m.top[warp], m.sum[warp]);
      part.put(row0, 1 << s.row_log, col0, s.cols, s.ld, m.rows[warp], D);
      if (threadIdx.x == 0) m.info = ti;
      __syncwarp();
      if (lane == 0) mbar_arrive(&m.laid);
    }
  return true;
}

// The outputs of sequences without a key, a CTA after the other.
template <typename T>
__device__ void write_empty(const Shape &p) {
  const int lane = threadIdx.x & 31;
  unsigned bad = 0;
  for (int b = blockIdx.x; b < p.a.seq.batch; b += gridDim.x) {
    if (tiles_of(keys_of(p.a, b, &bad), p.tile) > 0) continue;
    uint4 *out = reinterpret_cast<uint4 *>(p.a.out + b * p.a.out_stride);
    for (int i = lane; i < p.a.q_heads * p.a.cache.dim * (int)sizeof(T) / 16; i += 32) out[i] = make_uint4(0, 0, 0, 0);
    if (p.a.lse != nullptr)
      for (int i = lane; i < p.a.q_heads; i += 32) p.a.lse[(long long)b * p.a.q_heads + i] = -INFINITY;
  }
}

// To the output where the part is all of its (sequence, head), else to the workspace.
template <typename T>
__device__ void add_up(const Shape &p, Shared &sm) {
  const int lane = threadIdx.x & 31, D = p.a.cache.dim;
  for (int passes = 0, flags = 0; !(flags & kEnd);) {
    if (!wait(sm, &sm.merge[passes & 1].laid, passes >> 1 & 1)) return;
    const TileInfo ti = sm.merge[passes & 1].info;
    flags = ti.flags;
    const int kv = ti.head / p.passes, pass = ti.head - kv * p.passes;
    const int h0 = kv * p.group + pass * kRows, n = min(kRows, p.group - pass * kRows);
    const Pass s(n);
    float *slot = p.parts + ((long long)blockIdx.x * 2 + (flags & kLater ? 1 : 0)) * (kStatFloats + p.rows * D);
    T *out = reinterpret_cast<T *>(p.a.out + ti.seq * p.a.out_stride) + (long long)h0 * D;
    for (int row0 = 0; row0 < n; row0 += 1 << s.row_log)
      for (int col0 = 0; col0 < D; col0 += s.cols, ++passes) {
        Merge &m = sm.merge[passes & 1];
        if (row0 + col0 > 0 && !wait(sm, &m.laid, passes >> 1 & 1)) return;
        // lane: warp lane / 8, row lane % 8
        const int w = lane >> 3, r = row0 + (lane & 7);
        const bool live = r < n && (lane & 7) < 1 << s.row_log;
        const float top = live ? m.top[w][r] : -INFINITY;
        float all = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
        all = fmaxf(all, __shfl_xor_sync(~0u, all, 16));
        const float f = join_factor(top, all);
        float total = live ? m.sum[w][r] * f : 0.0f;
        total += __shfl_xor_sync(~0u, total, 8);
        total += __shfl_xor_sync(~0u, total, 16);
        const float g = flags & kWhole ? 1.0f / total : 1.0f;
        if (w == 0 && live && col0 == 0) {
          if (!(flags & kWhole)) *reinterpret_cast<float2 *>(slot + 2 * r) = make_float2(all, total);
          else if (p.a.lse != nullptr) p.a.lse[(long long)ti.seq * p.a.q_heads + h0 + r] = lse_of(all, total);
        }
        sm.scale[w][lane & 7] = f * g;
        if (w == 0) sm.none[lane & 7] = (flags & kWhole) && total == 0.0f;   // no key has a weight
        __syncwarp();
        const int fours_log = 31 - __clz(s.cols) - 2;   // of a row
#pragma unroll
        for (int i = lane; i < kMergeFloats / 4; i += 32) {
          const int rr = i >> fours_log, c = (i & ((1 << fours_log) - 1)) * 4;
          if (row0 + rr >= n || col0 + c >= D) continue;
          float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int v = 0; v < kWarps; ++v) {
            const float4 y = *reinterpret_cast<const float4 *>(&m.rows[v][rr * s.ld + c]);
            const float k = sm.scale[v][rr];
            x.x = fmaf(y.x, k, x.x);
            x.y = fmaf(y.y, k, x.y);
            x.z = fmaf(y.z, k, x.z);
            x.w = fmaf(y.w, k, x.w);
          }
          if (sm.none[rr]) x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          const int at = (row0 + rr) * D + col0 + c;
          if (!(flags & kWhole)) *reinterpret_cast<float4 *>(slot + kStatFloats + at) = x;
          else if (sizeof(T) == 4) *reinterpret_cast<float4 *>(out + at) = x;
          else *reinterpret_cast<uint2 *>(out + at) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&m.read);
      }
  }
}

// Rows of a slot for q: the fp32 consumers read as many heads as they hold.
template <typename Part, typename T>
__host__ __device__ __forceinline__ int slot_rows(const Shape &p) { return sizeof(T) == 4 ? Part::kHeadRows : p.rows; }

template <typename Part, typename T>
__device__ void consume(const Shape &p, Shared &sm, char *ring, char *qs, float *weights, int tiles) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = p.chunks * Part::kTile * 128;
  const int q_bytes = slot_rows<Part, T>(p) * p.a.cache.dim * (int)sizeof(T);
  Part part;
  int stage = 0, round = 0, passes = 0;
  auto give_back = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.empty[stage]);
    if (++stage == p.stages) {
      stage = 0;
      ++round;
    }
  };
  weights += warp * 8 * Part::kHeadRows;
  for (int it = 0; it < tiles; ++it) {
    if (!wait(sm, &sm.full[stage], round & 1)) return;
    const TileInfo ti = sm.info[stage];
    const char *q = qs + ti.slot * q_bytes;
    if (ti.flags & kFirst) part.start(p, q, min(kRows, p.group - ti.head % p.passes * kRows));
    const unsigned skip = (unsigned)ti.flags >> kSkip;
    const bool mine = warp * Part::kWarpKeys < ti.hi && (warp + 1) * Part::kWarpKeys > ti.lo && !Part::skips(p, skip, warp * Part::kWarpKeys);
    if (mine) part.logits(p, q, weights, ring + (long long)stage * half, warp * Part::kWarpKeys, ti.lo, ti.hi, skip);
    give_back();
    if (!wait(sm, &sm.full[stage], round & 1)) return;
    if (mine) part.values(p, weights, ring + (long long)stage * half, warp * Part::kWarpKeys, ti.lo, ti.hi);
    give_back();
    if ((ti.flags & kLast) && !lay_down(p, sm, part, ti, passes)) return;
  }
}

// The whole warp goes on to the next tile; sequences without one are passed over 32 at a time.
__device__ __forceinline__ void advance(const Shape &p, Walk &w) {
  unsigned bad = 0;
  if (++w.at < w.tiles) return;
  w.at = 0;
  if (++w.head < p.heads) return;
  w.head = 0;
  for (int b0 = w.seq + 1; b0 < p.a.seq.batch; b0 += 32) {
    const int b = b0 + (threadIdx.x & 31);
    Keys k{0, 0};
    if (b < p.a.seq.batch) k = keys_of(p.a, b, &bad);
    const int n = tiles_of(k, p.tile);
    const unsigned some = __ballot_sync(~0u, n > 0);
    if (some == 0) continue;
    const int lane = __ffs(some) - 1;
    w.seq = b0 + lane;
    w.keys.begin = __shfl_sync(~0u, k.begin, lane);
    w.keys.end = __shfl_sync(~0u, k.end, lane);
    w.tiles = __shfl_sync(~0u, n, lane);
    return;
  }
}

// One warp fills the ring, K and V of a tile by turns.  A tile's boxes (whole pages, or parts of them) are spread
// over the lanes, and the next tile's pages are looked up while this one waits for room.  The heads' rows of q
// come with the K of a part's first tile.  They have a slot for every K the ring can hold: when a slot's turn
// comes again, as many tiles lie between and the last K of its part has been given back.
template <typename Part, typename T>
__device__ void produce(const Shape &p, Shared &sm, char *ring, char *qs, const CUtensorMap *kmap, const CUtensorMap *vmap,
                        Walk w, int tiles, unsigned upto, unsigned total, unsigned shares) {
  constexpr int kTile = Part::kTile;
  const int lane = threadIdx.x & 31, box = 1 << p.box_log, boxes = kTile >> p.box_log, mine = lane & (boxes - 1);
  const int ops = boxes * (p.joined ? 1 : p.chunks), half = p.chunks * kTile * 128;
  const int size = p.a.cache.page_size, row_bytes = p.a.cache.dim * (int)sizeof(T);
  auto box_key = [&](const Walk &x) { return (x.keys.begin / kTile + x.at) * kTile + mine * box; };
  // begin - box, not key + box: that passes 2^31 behind the last key that a length can say
  auto counts = [&](const Walk &x) { return box_key(x) < x.keys.end && box_key(x) > x.keys.begin - box; };
  auto lookup = [&](const Walk &x) {   // page of this lane's box, as the table has it
    const int key = box_key(x);
    return counts(x) ? p.a.seq.table[x.seq * p.a.seq.table_stride + (p.page_log >= 0 ? key >> p.page_log : key / size)] : 0;
  };
  int page = lookup(w), next_page = 0, stage = 0, round = 0, slot = 0;
  bool fresh = true, later = false, begun = false;
  for (int it = 0; it < tiles; ++it) {
    Walk next = w;
    if (it + 1 < tiles) {
      advance(p, next);
      next_page = lookup(next);   // not looked at before its own turn
    }
    const bool last = it + 1 == tiles || w.at + 1 == w.tiles;
    bool here = counts(w);
    int bytes = 0;
    if (fresh) begun = w.at == 0;
    const int kv = p.passes == 1 ? w.head : w.head / p.passes;
    const int row = p.page_log >= 0 ? box_key(w) & (size - 1) : box_key(w) % size;
#pragma unroll
    for (int is_v = 0; is_v < 2; ++is_v) {
      if (round > 0 && !wait(sm, &sm.empty[stage], (round & 1) ^ 1)) return;
      unsigned skip = 0;
      if (is_v == 0) {
        const bool bad = here && (unsigned)page >= (unsigned)p.a.cache.num_pages;
        if (bad) atomicOr(&sm.flags, kErrCacheIndex);
        here &= !bad;
        skip = __ballot_sync(~0u, lane < boxes && bad);
        bytes = __popc(__ballot_sync(~0u, lane < boxes && here)) * p.chunks * box * 128;
      }
      if (lane == 0) {
        if (is_v == 0) {
          const int k0 = (w.keys.begin / kTile + w.at) * kTile, pass = w.head - kv * p.passes;
          TileInfo ti;
          ti.seq = w.seq;
          ti.head = w.head;
          ti.lo = w.keys.begin - k0;
          ti.hi = w.keys.end - k0;
          ti.flags = (fresh ? kFirst : 0) | (last ? kLast : 0) | (begun && w.at + 1 == w.tiles ? kWhole : 0) | (later ? kLater : 0) |
                     (it + 1 == tiles ? kEnd : 0) | (int)(skip << kSkip);
          ti.slot = slot;
          sm.info[stage] = ti;
          const int q_bytes = fresh ? min(kRows, p.group - pass * kRows) * row_bytes : 0;
          mbar_expect_tx(&sm.full[stage], bytes + q_bytes);
          if (fresh)
            bulk_g2s(qs + slot * slot_rows<Part, T>(p) * row_bytes,
                     p.a.q + w.seq * p.a.q_stride + (long long)(kv * p.group + pass * kRows) * row_bytes, q_bytes, &sm.full[stage]);
        } else {
          mbar_expect_tx(&sm.full[stage], bytes);
        }
      }
      __syncwarp();
      if (here) {
        const CUtensorMap *map = is_v ? vmap : kmap;
        char *to = ring + (long long)stage * half + (mine * p.chunks << (p.box_log + 7));
        if (p.joined) {
          if (lane < boxes) tma_load_5d(to, map, 0, row, 0, kv, page, &sm.full[stage]);
        } else {
          for (int o = lane; o < ops; o += 32) {
            const int c = o / boxes;
            tma_load_4d(to + (c << (p.box_log + 7)), map, c * (128 / (int)sizeof(T)), row, kv, page, &sm.full[stage]);
          }
        }
      }
      if (++stage == p.stages) {
        stage = 0;
        ++round;
      }
    }
    if (it + 1 == tiles && w.at + 1 < w.tiles && lane == 0) {   // goes on in the next shares
      const unsigned long long first = upto - 1 - w.at, end = (unsigned long long)upto + (unsigned)(w.tiles - 1 - w.at);
      const int from = begun ? (int)blockIdx.x : (int)(((first + 1) * shares - 1) / total), to = (int)((end * shares - 1) / total);
      const bool second = begun ? later : (unsigned long long)total * from / shares < first;
      sm.job = make_int4(w.seq, w.head, from, 2 * (to - from + 1) + second);
    }
    fresh = last;
    later |= last;
    if (last && ++slot == p.slots) slot = 0;
    w = next;
    page = next_page;
  }
}

template <typename Part, typename T>
__global__ void __launch_bounds__(kThreads, Part::kCtas)
attend_kernel(const __grid_constant__ Shape p, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ char smem_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.a.seq.batch;
  char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  Shared &sm = *reinterpret_cast<Shared *>(ring + (long long)p.stages * p.chunks * Part::kTile * 128);
  char *qs = reinterpret_cast<char *>(&sm + 1);
  float *weights = reinterpret_cast<float *>(qs + p.slots * slot_rows<Part, T>(p) * p.a.cache.dim * (int)sizeof(T));
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" :: "l"(&vmap) : "memory");
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], kWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.merge[i].laid, kWarps);
      mbar_init(&sm.merge[i].read, 1);
    }
    mbar_init(&sm.never, 1);
    fence_mbar_init();
    sm.flags = 0;
    sm.dead = 0;
    sm.job = make_int4(0, 0, 0, 0);
  }
  grid_begins();

  // this CTA's share of all tiles: each thread counts some sequences' tiles
  unsigned bad = 0, mine = 0;
  const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  for (int b = b0; b < b1; ++b) mine += (unsigned)tiles_of(keys_of(p.a, b, &bad), p.tile) * p.heads;
  unsigned upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned x = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sm.warp_tiles[warp] = upto;
  __syncthreads();
  if (bad) atomicOr(&sm.flags, bad);
  unsigned total = 0;
  for (int w = 0; w < kWarps + 2; ++w) {
    if (w < warp) upto += sm.warp_tiles[w];
    total += sm.warp_tiles[w];
  }
  // share w: the tiles total w / shares up to total (w + 1) / shares.  None is empty: with fewer tiles than
  // CTAs the last CTAs have none
  const unsigned shares = min(total, gridDim.x), whole = shares > 0 ? total / shares : 0, rest = total - whole * shares;
  const bool some = blockIdx.x < shares;
  const unsigned t0 = some ? whole * blockIdx.x + rest * blockIdx.x / shares : total;
  const unsigned t1 = some ? whole * (blockIdx.x + 1) + rest * (blockIdx.x + 1) / shares : total;
  if (some && t0 >= upto - mine && t0 < upto) {
    unsigned at = t0 - (upto - mine);
    for (int b = b0; b < b1; ++b) {
      Walk w;
      w.keys = keys_of(p.a, b, &bad);
      w.tiles = tiles_of(w.keys, p.tile);
      if (at < (unsigned)w.tiles * p.heads) {
        w.seq = b;
        w.head = (int)(at / (unsigned)w.tiles);
        w.at = (int)(at - (unsigned)w.head * w.tiles);
        sm.start = w;
        break;
      }
      at -= (unsigned)w.tiles * p.heads;
    }
  }
  __syncthreads();

  const int tiles = (int)(t1 - t0);
  if (warp > kWarps) write_empty<T>(p);
  if (tiles > 0) {
    if (warp == kWarps) produce<Part, T>(p, sm, ring, qs, &kmap, &vmap, sm.start, tiles, t1, total, shares);
    else if (warp > kWarps) add_up<T>(p, sm);
    else consume<Part, T>(p, sm, ring, qs, weights, tiles);
  }
  __syncthreads();
  if (sm.dead && tid < 32) wait_out(&sm.never);   // copies that nobody waited for
  if (tid == 0) p.jobs[blockIdx.x] = sm.job;
  if (tid == 0) post_status(reinterpret_cast<unsigned *>(p.a.ws), blockIdx.x, gridDim.x, sm.flags | (sm.dead ? kErrTimeout : 0u));
}

// What the cuts between the CTAs' shares have parted.  CTA w belongs to the (sequence, head) that share w ends
// within, if any, and joins some of its heads: with few parts a warp takes a head, with many the whole CTA.
constexpr int kJoinThreads = 128, kJoinWarps = kJoinThreads / 32, kJoinBatch = 4;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Shape p) {
  __shared__ float factor[kMaxWorkers], red[2][kJoinWarps], sums[kJoinWarps][256];
  grid_begins();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, D = p.a.cache.dim;
  const int4 job = p.jobs[blockIdx.x];
  const int parts = job.w >> 1, first = job.z, kv = job.y / p.passes, pass = job.y - kv * p.passes;
  if (parts == 0) return;
  const int h0 = kv * p.group + pass * kRows, n = min(kRows, p.group - pass * kRows);
  const int me = (int)blockIdx.x - first, ctas = parts - 1;   // the last share's CTA belongs elsewhere
  const long long stride = kStatFloats + p.rows * D;
  auto part = [&](int i) { return p.parts + (2LL * (first + i) + (i == 0 ? job.w & 1 : 0)) * stride; };
  float4 x[kJoinBatch][2], acc[2];
  auto load = [&](int r, int i0, int step) {
#pragma unroll
    for (int m = 0; m < kJoinBatch; ++m)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (i0 + m * step < parts && lane + 32 * c < D / 4)
          x[m][c] = reinterpret_cast<const float4 *>(part(i0 + m * step) + kStatFloats + r * D)[lane + 32 * c];
  };
  auto add = [&](int m, float f) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (lane + 32 * c < D / 4) {
        acc[c].x = fmaf(x[m][c].x, f, acc[c].x);
        acc[c].y = fmaf(x[m][c].y, f, acc[c].y);
        acc[c].z = fmaf(x[m][c].z, f, acc[c].z);
        acc[c].w = fmaf(x[m][c].w, f, acc[c].w);
      }
  };
  auto write = [&](int r, int c, float4 v, float sum) {
    const float g = 1.0f / sum;
    if (sum == 0.0f) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    else v = make_float4(v.x * g, v.y * g, v.z * g, v.w * g);
    T *out = reinterpret_cast<T *>(p.a.out + job.x * p.a.out_stride) + (long long)(h0 + r) * D + 4 * c;
    if (sizeof(T) == 4) *reinterpret_cast<float4 *>(out) = v;
    else *reinterpret_cast<uint2 *>(out) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  };
  auto write_lse = [&](int r, float all, float sum) {
    if (p.a.lse != nullptr) p.a.lse[(long long)job.x * p.a.q_heads + h0 + r] = lse_of(all, sum);
  };

  if (parts <= 2 * kJoinBatch) {
    for (int r = me * kJoinWarps + warp; r < n; r += ctas * kJoinWarps) {
      load(r, 0, 1);
      const float2 s = lane < parts ? *reinterpret_cast<const float2 *>(part(lane) + 2 * r) : make_float2(-INFINITY, 0.0f);
      float all = s.x;
#pragma unroll
      for (int d = kJoinBatch; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor_sync(~0u, all, d));
      all = __shfl_sync(~0u, all, 0);
      const float f = join_factor(s.x, all);
      float sum = s.y * f;
#pragma unroll
      for (int d = kJoinBatch; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      sum = __shfl_sync(~0u, sum, 0);
      acc[0] = acc[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int i = 0; i < parts; i += kJoinBatch) {
        if (i > 0) load(r, i, 1);
#pragma unroll
        for (int m = 0; m < kJoinBatch; ++m) {
          const float g = __shfl_sync(~0u, f, i + m);
          if (i + m < parts) add(m, g);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (lane + 32 * c < D / 4) write(r, lane + 32 * c, acc[c], sum);
      if (lane == 0) write_lse(r, all, sum);
    }
    return;
  }
  for (int r = me; r < n; r += ctas) {
    load(r, warp, kJoinWarps);
    float all = -INFINITY, sum = 0.0f;
    for (int i = tid; i < parts; i += kJoinThreads) all = fmaxf(all, part(i)[2 * r]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor_sync(~0u, all, d));
    if (lane == 0) red[0][warp] = all;
    __syncthreads();
    all = red[0][0];
#pragma unroll
    for (int w = 1; w < kJoinWarps; ++w) all = fmaxf(all, red[0][w]);
    for (int i = tid; i < parts; i += kJoinThreads) {
      const float2 s = *reinterpret_cast<const float2 *>(part(i) + 2 * r);
      factor[i] = join_factor(s.x, all);
      sum += s.y * factor[i];
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if (lane == 0) red[1][warp] = sum;
    __syncthreads();
    acc[0] = acc[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = warp; i < parts; i += kJoinWarps * kJoinBatch) {
      if (i != warp) load(r, i, kJoinWarps);
#pragma unroll
      for (int m = 0; m < kJoinBatch; ++m)
        if (i + m * kJoinWarps < parts) add(m, factor[i + m * kJoinWarps]);
    }
    reinterpret_cast<float4 *>(sums[warp])[lane] = acc[0];
    reinterpret_cast<float4 *>(sums[warp])[lane + 32] = acc[1];
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += red[1][w];
    for (int c = tid; c < D / 4; c += kJoinThreads) {
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kJoinWarps; ++w) {
        const float4 y = reinterpret_cast<const float4 *>(sums[w])[c];
        v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
      }
      write(r, c, v, sum);
    }
    if (tid == 0) write_lse(r, all, sum);
    __syncthreads();
  }
}

template <typename Part, typename T>
cudaError_t launch(Shape p, cudaStream_t s) {
  const AttendArgs &a = p.a;
  const CacheLayer &c = a.cache;
  p.tile = Part::kTile;
  p.box_log = 0;
  while ((2 << p.box_log) <= Part::kTile && c.page_size % (2 << p.box_log) == 0) ++p.box_log;
  p.joined = c.dim * (int)sizeof(T) % 128 == 0;
  p.page_log = (c.page_size & (c.page_size - 1)) == 0 ? __builtin_ctz((unsigned)c.page_size) : -1;
  // CTAs of an SM share its 228 KB: 1 KB each is the system's, 6 KB are room for join_kernel
  constexpr size_t kShare = (size_t)(228 - 6) * 1024 / Part::kCtas / 1024 * 1024 - 2048;
  const size_t half = (size_t)p.chunks * Part::kTile * 128, q_slot = (size_t)slot_rows<Part, T>(p) * c.dim * sizeof(T);
  const size_t fixed = 1024 + sizeof(Shared) + (sizeof(T) == 4 ? kWarps * 8 * Part::kHeadRows * sizeof(float) : 0);
  auto smem_of = [&](int stages) { return fixed + stages * half + (stages + 1) / 2 * q_slot; };
  p.stages = kMaxStages;
  while (p.stages > 2 && smem_of(p.stages) > kShare) --p.stages;
  p.slots = (p.stages + 1) / 2;
  const size_t smem = smem_of(p.stages);
  // before the maps are encoded: a host thread's first runtime call gives it its context
  cudaError_t e = allow_smem(reinterpret_cast<const void *>(&attend_kernel<Part, T>), smem);
  if (e != cudaSuccess) return e;
  CUtensorMap maps[2];
  const uint64_t row = (uint64_t)c.dim * sizeof(T), head = c.heads > 1 ? (uint64_t)c.head_stride : row,
                 page = c.num_pages > 1 ? (uint64_t)c.page_stride : row, token = (uint64_t)c.token_stride;
  const uint64_t inner = 128 / sizeof(T);
  const uint64_t dims[4] = {(uint64_t)c.dim, (uint64_t)c.page_size, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint64_t dims5[5] = {inner, (uint64_t)c.page_size, (uint64_t)p.chunks, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint64_t strides[3] = {token, head, page}, strides5[4] = {token, 128, head, page};
  const uint32_t rows = 1u << p.box_log, box[4] = {(uint32_t)inner, rows, 1, 1}, box5[5] = {(uint32_t)inner, rows, (uint32_t)p.chunks, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (!encode_rows_map(&maps[i], i ? c.v : c.k, sizeof(T) == 4, p.joined ? 5 : 4, p.joined ? dims5 : dims,
                         p.joined ? strides5 : strides, p.joined ? box5 : box))
      return cudaErrorInvalidValue;
  // no more CTAs than the page tables have room for tiles
  const long long most = (long long)a.seq.batch * p.heads * ((long long)a.seq.max_pages * c.page_size / p.tile + 2);
  int workers = sm_count() * Part::kCtas;
  workers = workers < kMaxWorkers ? workers : kMaxWorkers;
  if (workers > most) workers = most > 0 ? (int)most : 1;
  e = launch_early(attend_kernel<Part, T>, dim3(workers), kThreads, smem, s, p, maps[0], maps[1]);
  if (e != cudaSuccess || a.seq.batch == 0) return e;
  return launch_early(join_kernel<T>, dim3(workers), kJoinThreads, 0, s, p);
}

}  // namespace
}  // namespace last
