// Chunk and differential attention over bf16 keys and values, few rows per sequence (single tokens, drafted tokens).
//
// Such a call reads K and V and computes little: tiles of 128 rows on tcgen05 would be empty for the most part.  S^T = K Q^T has 16
// keys as the rows of an MMA and 8 of a block's rows as its columns, O^T += V^T P^T follows from registers.  Four warps (diff: four
// per map) take a quarter of every tile of 64 keys each, with sums of their own; they add them up where the share's part of
// an item ends, while the ring goes on being filled.  One warp per map keeps K and V of its head on their way in TMA boxes and
// fetches the items' rows of q; the first one walks the items for all.
//
// Bound by HBM where rows of K are long runs and by the consumers' instructions for two maps: 64 x 5 new tokens over 592 - 704 keys, 16 kv-heads
// by 128, 72 us (4.8 TB/s; tiles of 128 rows on tcgen05 123), 64 differential single tokens 94 (234), 6 over 115 thousand keys 256 (5.6 TB/s; 322).
#pragma once

#include <cstddef>

#include "chunk_impl.cuh"
#include "tensor_map.h"

namespace last {

namespace {

constexpr int kTile = 64, kRingMax = 16, kItems = 4, kTileInfo = 16, kMergePad = 4;

struct Few {           // the same for every CTA
  ChunkShape p;
  int slots;           // panels of the ring: 64 keys or values of one head
  int box_log, page_log;
  bool joined;         // a box holds all 128-byte columns of its rows
};

struct Item {
  int seq, unit, first, r0, rows;
  int base, begin, lens;
  int ka, kb;               // key tiles of the share
  int lo, hi, all_lo, all_hi;   // keys that some row sees; that all rows see
  int whole, second;
};

template <int EIGHTS, int MAPS>
struct alignas(16) Shared {
  unsigned long long full[kRingMax], empty[kRingMax], item_full[kItems], item_empty[kItems], never;
  Item items[kItems];
  ChunkShare share;
  unsigned long long sums[16];
  alignas(16) float rows[4 * MAPS][8][64 + kMergePad];   // of a warp: 8 rows and 64 columns of its sums, read four at a time
  float top[4 * MAPS][8 * EIGHTS], sum[4 * MAPS][8 * EIGHTS];
  unsigned skip[MAPS][kTileInfo];            // boxes of the tiles on their way whose page is out of range
  unsigned flags;
  volatile unsigned dead;
};

// CHUNKS: 128-byte columns of a head's row; EIGHTS: groups of 8 rows of a block; FULL: the columns are, so that the steps along a
// row are known and their loads and products go between each other.
template <int CHUNKS, int EIGHTS, int MAPS, bool FULL>
struct Kind {
  static constexpr bool kFull = FULL;
  static __device__ __forceinline__ int dim(const ChunkShape &p) { return FULL ? CHUNKS * 64 : p.a.cache.dim; }
  static constexpr int kChunks = CHUNKS, kEights = EIGHTS, kMaps = MAPS, kRows = 8 * EIGHTS;
  static constexpr int kConsumers = 4 * MAPS, kThreads = 32 * (kConsumers + MAPS), kCtas = MAPS == 2 || CHUNKS > 2 ? 1 : 2;
  static constexpr int kSteps = CHUNKS * 4;   // 16-wide along a row
  static constexpr size_t kPanel = (size_t)CHUNKS * kTile * 128;
  using Sm = Shared<EIGHTS, MAPS>;
};

template <typename K>
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" :: "n"(32 * K::kConsumers) : "memory"); }
template <typename K>
__device__ __forceinline__ bool consumers_any(bool x) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
               "bar.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)x), "n"(32 * K::kConsumers) : "memory");
  return r != 0;
}

struct Place {
  int slot;
  uint32_t round;
  __device__ __forceinline__ void next(int slots) {
    if (++slot == slots) {
      slot = 0;
      round ^= 1;
    }
  }
};

// ---- one warp per map: items (the first), rows of q, K and V ----
template <typename K>
__device__ __forceinline__ void produce(const Few &f, typename K::Sm &sm, char *ring, char *qs, const CUtensorMap *kmap, const CUtensorMap *vmap, int map) {
  const ChunkShape &p = f.p;
  const CacheLayer &c = p.a.cache;
  const int lane = threadIdx.x & 31, box = 1 << f.box_log, boxes = kTile >> f.box_log, mine = lane & (boxes - 1);
  const bool joined = K::kFull || f.joined;
  const int ops = boxes * (joined ? 1 : K::kChunks), size = c.page_size, row_bytes = c.dim * 2;
  ChunkWalk walk(sm.share);
  ChunkItem it;
  Place at{0, 0};
  bool again = false;
  uint32_t tile = 0;
  auto step = [&](int n) {   // n <= slots
    for (int i = 0; i < n; ++i) {
      at.next(f.slots);
      again |= at.slot == 0;
    }
  };
  step(map);
  for (uint32_t n = 0;; ++n) {
    const int e = n % kItems;
    Item &o = sm.items[e];
    if (map == 0) {
      const bool more = walk.next(p, &it);
      if (n >= kItems && !wait(sm, &sm.item_empty[e], (n / kItems & 1) ^ 1)) return;
      if (lane == 0) {
        const bool some = more && it.t.count > 0;
        o.seq = more ? it.seq : -1;
        o.unit = it.unit;
        o.first = it.s.first;
        o.r0 = it.r0;
        o.rows = it.rows;
        o.base = it.s.base;
        o.begin = it.s.begin;
        o.lens = it.s.lens;
        o.ka = some ? it.t.first + it.k0 : 0;
        o.kb = some ? it.t.first + it.k1 : 0;
        o.lo = it.t.lo;
        o.hi = it.t.hi;
        o.all_lo = more ? chunk_lo(p.a, it.s, (it.r0 + it.rows - 1) / p.group) : 0;
        o.all_hi = more ? chunk_hi(p.a, it.s, it.r0 / p.group) : 0;
        o.whole = it.whole;
        o.second = it.second;
        mbar_arrive(&sm.item_full[e]);
      }
      __syncwarp();
      if (!more) return;
    } else if (!wait(sm, &sm.item_full[e], n / kItems & 1)) {
      return;
    }
    const int seq = o.seq, unit = o.unit, ka = o.ka, kb = o.kb, lo = o.lo, hi = o.hi, rows = o.rows, r0 = o.r0, first = o.first;
    __syncwarp();
    if (map > 0 && lane == 0) mbar_arrive(&sm.item_empty[e]);
    if (seq < 0) return;
    const int32_t *table = p.a.seq.table + seq * p.a.seq.table_stride;
    auto counts = [&](int j) { return j < kb && j * kTile + mine * box < hi && j * kTile + mine * box > lo - box; };
    auto lookup = [&](int j) {
      const int key = j * kTile + mine * box;
      return counts(j) ? table[f.page_log >= 0 ? key >> f.page_log : key / size] : -1;
    };
    int page = ka < kb ? lookup(ka) : -1;
    for (int j = ka; j < kb; ++j, ++tile) {
      const int next_page = lookup(j + 1);
      const bool wanted = counts(j), here = wanted && (unsigned)page < (unsigned)c.num_pages;
      const unsigned skip = __ballot_sync(~0u, lane < boxes && wanted && !here);
      const uint32_t bytes = __popc(__ballot_sync(~0u, lane < boxes && here)) * K::kChunks * box * 128;
      const int key = j * kTile + mine * box, row = f.page_log >= 0 ? key & (size - 1) : key % size;
      const int head = unit * K::kMaps + map;
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v) {
        if (again && !wait(sm, &sm.empty[at.slot], at.round ^ 1)) return;
        unsigned long long *bar = &sm.full[at.slot];
        const bool fresh = j == ka && !is_v;
        if (lane == 0) {
          if (!is_v) sm.skip[map][tile % kTileInfo] = skip;
          if (skip != 0) atomicOr(&sm.flags, kErrCacheIndex);
          mbar_expect_tx(bar, bytes + (fresh ? rows * row_bytes : 0));
        }
        __syncwarp();
        if (here) {
          const CUtensorMap *m = is_v ? vmap : kmap;
          char *to = ring + at.slot * K::kPanel + (mine * K::kChunks << (f.box_log + 7));
          if (joined) {
            if (lane < boxes) tma_load_5d(to, m, 0, row, 0, head, page, bar);
          } else {
            for (int i = lane; i < ops; i += 32) {
              const int x = i / boxes;
              tma_load_4d(to + (x << (f.box_log + 7)), m, x * 64, row, head, page, bar);
            }
          }
        }
        if (fresh && lane < rows) {
          const int tok = (r0 + lane) / p.group, h = unit * p.group + (r0 + lane) - tok * p.group;
          bulk_g2s(qs + ((e * K::kMaps + map) * K::kRows + lane) * row_bytes,
                   p.a.q + (long long)(first + tok) * p.a.q_stride + (long long)(K::kMaps * h + map) * row_bytes, row_bytes, bar);
        }
        step(K::kMaps);
      }
      page = next_page;
    }
  }
}

// ---- consumers ----
template <typename K>
struct Part {
  static constexpr int kSteps = K::kSteps, kEights = K::kEights, kValues = K::kMaps;
  static constexpr int kAhead = 4;
  uint32_t q[kSteps][2 * kEights];
  float o[kValues][kSteps][kEights][4];   // (d g, row 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1)
  float m[kEights][2], l[kEights][2];     // rows 2t, 2t + 1; l over this lane's keys
  uint32_t w[kEights][4], keep[2];        // the tile's weights, cut and rest; masks of its values
  int rlo[kEights][2], rhi[kEights][2];   // keys that rows 2t and 2t + 1 see
  bool part, mixed;                       // some of the warp's keys do not count; some count for some rows alone

  __device__ __forceinline__ void start(const ChunkShape &p, const Item &it) {
    const int t = threadIdx.x & 3;
    const ChunkSeq s{it.first, 0, it.base, it.begin, it.lens};
#pragma unroll
    for (int e = 0; e < kEights; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = 8 * e + 2 * t + h, tok = (it.r0 + r) / p.group;
        rlo[e][h] = r < it.rows ? chunk_lo(p.a, s, tok) : 0;   // rows of no token see everything: their q is zero
        rhi[e][h] = r < it.rows ? chunk_hi(p.a, s, tok) : 0x7fffffff;
        m[e][h] = -INFINITY;
        l[e][h] = 0.0f;
      }
#pragma unroll
    for (int v = 0; v < kValues; ++v)
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int e = 0; e < kEights; ++e) o[v][i][e][0] = o[v][i][e][1] = o[v][i][e][2] = o[v][i][e][3] = 0.0f;
  }
  __device__ __forceinline__ void get_q(const char *qs, int rows, int D) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int e = 0; e < 2 * kEights; ++e) {
        const int row = g + 8 * (e >> 1), d = s * 16 + 2 * t + 8 * (e & 1);
        q[s][e] = row < rows && d < D ? *reinterpret_cast<const uint32_t *>(qs + (row * D + d) * 2) : 0u;
      }
  }

  // Weights of the warp's 16 keys, row0 .. of the tile and key0 .. of the sequence.
  __device__ __forceinline__ void logits(const Few &f, const Item &it, uint32_t k, int row0, int key0, unsigned skip) {
    const int lane = threadIdx.x & 31, g = lane >> 2, D = K::dim(f.p), column = 128 << f.box_log;
    const float scale2 = f.p.scale2;
    float s[2][kEights][4] = {};   // even and odd steps
    {   // 8 x 8 blocks (keys 0-7 | 8-15) x (16-byte column even | odd)
      const int row = row0 + (lane & 15), sub = lane >> 4;
      const uint32_t base = k + row_at(f, row);
      auto at = [&](int i) { return base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4); };
      uint32_t x[kAhead][4];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i * 16 < D) ldsm4(x[i], at(i));
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (i * 16 >= D) break;
#pragma unroll
        for (int e = 0; e < kEights; ++e) mma16816(s[i & 1][e], x[i % kAhead], q[i][2 * e], q[i][2 * e + 1]);
        if (i + kAhead < kSteps && (i + kAhead) * 16 < D) ldsm4(x[i % kAhead], at(i + kAhead));
      }
    }
    part = it.all_lo > key0 || it.all_hi < key0 + 16 || skip != 0;
    mixed = part && (it.all_lo > key0 && it.all_lo > it.lo || it.all_hi < key0 + 16 && it.all_hi < it.hi);
    keep[0] = keep[1] = ~0u;   // halves of V's fragments whose keys count for some row
    if (part) {
      auto counts = [&](int i) { return key0 + i >= it.lo && key0 + i < it.hi && (skip >> ((row0 + i) >> f.box_log) & 1) == 0; };
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!counts(j * 8 + 2 * (lane & 3))) keep[j] &= 0xffff0000u;
        if (!counts(j * 8 + 2 * (lane & 3) + 1)) keep[j] &= 0x0000ffffu;
        const bool here = counts(j * 8 + g);
        const int key = key0 + j * 8 + g;
#pragma unroll
        for (int e = 0; e < kEights; ++e)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (!here || key < rlo[e][h] || key >= rhi[e][h]) s[0][e][2 * j + h] = s[1][e][2 * j + h] = -INFINITY;
      }
    }
    float top[kEights][2];
    bool above = false;
#pragma unroll
    for (int e = 0; e < kEights; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[0][e][h] += s[1][e][h];
        s[0][e][2 + h] += s[1][e][2 + h];
        top[e][h] = fmaxf(s[0][e][h], s[0][e][2 + h]) * scale2;
        above |= top[e][h] > m[e][h] + 8.0f;
      }
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int e = 0; e < kEights; ++e) {
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = top[e][h];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
          alpha[h] = x > m[e][h] ? chunk_exp2(m[e][h] - x) : 1.0f;
          m[e][h] = fmaxf(m[e][h], x);
          l[e][h] *= alpha[h];
        }
#pragma unroll
        for (int v = 0; v < kValues; ++v)
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            o[v][i][e][0] *= alpha[0];
            o[v][i][e][1] *= alpha[1];
            o[v][i][e][2] *= alpha[0];
            o[v][i][e][3] *= alpha[1];
          }
      }
    }
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = chunk_exp2(fmaf(s[0][e][i], scale2, m[e][i & 1] == -INFINITY ? 0.0f : -m[e][i & 1]));
      l[e][0] += x[0] + x[2];
      l[e][1] += x[1] + x[3];
#pragma unroll
      for (int j = 0; j < 2; ++j) {   // keys j * 8 + g, to keys j * 8 + 2t and 2t + 1 of row g
        const uint32_t down = pack_down(x[2 * j], x[2 * j + 1]);
        w[e][j] = transpose8(down);
        w[e][2 + j] = transpose8(pack_rest(x[2 * j], x[2 * j + 1], down));
      }
    }
  }

  static __device__ __forceinline__ uint32_t row_at(const Few &f, int row) {
    return ((row >> f.box_log) * K::kChunks << (f.box_log + 7)) + (row & ((1 << f.box_log) - 1)) * 128;
  }

  // o[v] += weights x V.
  template <int V>
  __device__ __forceinline__ void values(const Few &f, uint32_t panel, int row0, int key0) {
    const int lane = threadIdx.x & 31, D = K::dim(f.p), column = 128 << f.box_log;
    // 8 x 8 blocks, transposed on the way: (keys 0-7 | 8-15) x (16-byte column even | odd)
    const int row = row0 + (lane & 7) + (lane >> 4) * 8, sub = lane >> 3 & 1;
    const uint32_t base = panel + row_at(f, row);
    auto at = [&](int i) { return base + (i >> 2) * column + ((((i & 3) * 2 + sub) ^ (row & 7)) << 4); };
    if (mixed) {   // an infinity or NaN that some row does not see would show as its weight of zero times it
      bool odd = false;
#pragma unroll 1
      for (int i = 0; i * 16 < D; ++i) {
        uint32_t x[4];
        ldsm4t(x, at(i));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t y = x[j] & keep[j >> 1];
          odd |= (y & 0x7f80u) == 0x7f80u || (y & 0x7f800000u) == 0x7f800000u;
        }
      }
      if (__any_sync(~0u, odd)) {
        one_by_one<V>(f, panel, row0, key0);
        return;
      }
    }
    uint32_t x[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i * 16 < D) ldsm4t(x[i], at(i));
#pragma unroll
    for (int i = 0; i < kSteps; i += 2) {   // two steps together: the products of one wait for each other
      if (i * 16 >= D) break;
      const bool both = (i + 1) * 16 < D;
      uint32_t (&y)[4] = x[i % kAhead], (&z)[4] = x[(i + 1) % kAhead];
      if (part) {   // keys that no row sees
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] &= keep[j >> 1];
          z[j] &= keep[j >> 1];
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < kEights; ++e) {
          mma16816(o[V][i][e], y, w[e][2 * r], w[e][2 * r + 1]);
          if (both) mma16816(o[V][i + 1][e], z, w[e][2 * r], w[e][2 * r + 1]);
        }
#pragma unroll
      for (int j = i + kAhead; j < i + kAhead + 2; ++j)
        if (j < kSteps && j * 16 < D) ldsm4t(x[j % kAhead], at(j));
    }
  }

  // The same on the CUDA cores, each row with the keys that it sees alone.
  template <int V>
  __device__ __forceinline__ void one_by_one(const Few &f, uint32_t panel, int row0, int key0) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, D = K::dim(f.p), column = 128 << f.box_log;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
      const uint32_t base = panel + row_at(f, row0 + i);
      float k[kEights][2];   // weights of key i
      bool sees[kEights][2];
      // keep, of the lane that has the key as its 2t or 2t + 1
      const uint32_t kept = __shfl_sync(~0u, i < 8 ? keep[0] : keep[1], (i & 7) >> 1);
      const bool here = (kept >> (i & 1) * 16 & 1) != 0;
#pragma unroll
      for (int e = 0; e < kEights; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // row r = 2t + h has its weights in the lanes 4r .. 4r + 3: keys 2t', 2t' + 1
          const int from = (2 * t + h) * 4 + ((i & 7) >> 1);
          const uint32_t a = __shfl_sync(~0u, i < 8 ? w[e][0] : w[e][1], from), b = __shfl_sync(~0u, i < 8 ? w[e][2] : w[e][3], from);
          k[e][h] = (i & 1) ? bf16hi(a) + bf16hi(b) : bf16lo(a) + bf16lo(b);
          sees[e][h] = here && key0 + i >= rlo[e][h] && key0 + i < rhi[e][h];
        }
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (s * 16 >= D) break;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t at = base + (s >> 2) * column + ((((s & 3) * 2 + half) ^ ((row0 + i) & 7)) << 4) + g * 2;
          uint16_t bits;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(at) : "memory");
          const float v = __uint_as_float((uint32_t)bits << 16);
#pragma unroll
          for (int e = 0; e < kEights; ++e)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (sees[e][h]) o[V][s][e][2 * half + h] = fmaf(k[e][h], v, o[V][s][e][2 * half + h]);
        }
      }
    }
  }
};

// The warps' sums of an item, added up: to the output where the share has the whole item, else to the workspace.
template <typename K>
__device__ __forceinline__ void add_up(const Few &f, typename K::Sm &sm, Part<K> &part, const Item &it) {
  constexpr int kMaps = K::kMaps, kEights = K::kEights, kPasses = K::kMaps * K::kChunks;
  const ChunkShape &p = f.p;
  const ChunkArgs &a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3, D = K::dim(p);
#pragma unroll
  for (int e = 0; e < kEights; ++e)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x = part.l[e][h];
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(~0u, x, d);
      if (lane < 4) {
        sm.top[warp][8 * e + 2 * lane + h] = part.m[e][h];
        sm.sum[warp][8 * e + 2 * lane + h] = x;
      }
    }
  const int row = tid >> 4 & 7, col = (tid & 15) * 4;   // of a pass, by the first four warps
#pragma unroll
  for (int e = 0; e < kEights; ++e) {
    const int r = 8 * e + row;
    const bool live = r < it.rows && tid < 128;
    const int tok = (it.r0 + (live ? r : 0)) / p.group, h = it.unit * p.group + it.r0 + (live ? r : 0) - tok * p.group;
    float scale[kMaps][4], lam = 0.0f, x[kPasses][4];
    bool none[kMaps];
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      const int v = pass / K::kChunks, c = pass % K::kChunks;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float *to = &sm.rows[warp][2 * t][i * 16 + g];
        to[0] = part.o[v][4 * c + i][e][0];
        to[64 + kMergePad] = part.o[v][4 * c + i][e][1];
        to[8] = part.o[v][4 * c + i][e][2];
        to[64 + kMergePad + 8] = part.o[v][4 * c + i][e][3];
      }
      consumers_sync<K>();
      if (tid < 128) {
        if (pass == 0) {
#pragma unroll
          for (int map = 0; map < kMaps; ++map) {
            float all = -INFINITY, total = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) all = fmaxf(all, sm.top[4 * map + w][r]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              scale[map][w] = chunk_factor(sm.top[4 * map + w][r], all);
              total = fmaf(sm.sum[4 * map + w][r], scale[map][w], total);
            }
            none[map] = it.whole && total == 0.0f;
            if (it.whole) {
              const float inv = 1.0f / total;
#pragma unroll
              for (int w = 0; w < 4; ++w) scale[map][w] *= inv;
            }
            if (live && col == 0) {
              if (!it.whole) {
                float *slot = chunk_slot(p, blockIdx.x, map, it.second);
                slot[r] = all;
                slot[p.pitch + r] = total;
              } else if (kMaps == 1 && a.lse != nullptr) {
                a.lse[(long long)(it.first + tok) * a.q_heads + h] = chunk_lse(all, total);
              }
            }
          }
          if (kMaps == 2 && live) lam = a.lambda[h];
        }
        const bool in = c * 64 + col < D;
        float y[kMaps][4];
#pragma unroll
        for (int map = 0; map < kMaps; ++map) {
          float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float4 s = *reinterpret_cast<const float4 *>(&sm.rows[4 * map + w][row][col]);
            z.x = fmaf(s.x, scale[map][w], z.x);
            z.y = fmaf(s.y, scale[map][w], z.y);
            z.z = fmaf(s.z, scale[map][w], z.z);
            z.w = fmaf(s.w, scale[map][w], z.w);
          }
          if (none[map]) z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          y[map][0] = z.x;
          y[map][1] = z.y;
          y[map][2] = z.z;
          y[map][3] = z.w;
          if (!it.whole && live && in) {
            float *slot = chunk_slot(p, blockIdx.x, map, it.second);
            reinterpret_cast<float4 *>(slot + 2 * p.pitch)[(v * D + c * 64 + col) / 4 * p.pitch + r] = z;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[pass][i] = kMaps == 2 ? fmaf(-lam, y[kMaps - 1][i], y[0][i]) : y[0][i];
          if (!in) x[pass][i] = 0.0f;
        }
      }
      consumers_sync<K>();
    }
    if (!it.whole || tid >= 128) continue;
    float factor = 1.0f;
    if (kMaps == 2) {
      float squares = 0.0f;
#pragma unroll
      for (int pass = 0; pass < kPasses; ++pass)
#pragma unroll
        for (int i = 0; i < 4; ++i) squares = fmaf(x[pass][i], x[pass][i], squares);
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) squares += __shfl_xor_sync(~0u, squares, d);
      factor = chunk_norm(a, squares, p.dv);
    }
    if (!live) continue;
    char *out = a.out + (long long)(it.first + tok) * a.out_stride + (long long)h * p.dv * 2;
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      const int d = pass % K::kChunks * 64 + col, at = pass / K::kChunks * D + d;
      if (d >= D) continue;
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = x[pass][i];
        if (kMaps == 2) y[i] *= factor * (a.norm_weight != nullptr ? a.norm_weight[at + i] : 1.0f);
      }
      *reinterpret_cast<uint2 *>(out + at * 2) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
    }
  }
}

template <typename K>
__device__ __forceinline__ void consume(const Few &f, typename K::Sm &sm, char *ring, char *qs) {
  const ChunkShape &p = f.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, map = warp >> 2, row0 = (warp & 3) * 16, D = K::dim(p);
  const uint32_t ring_at = smem_addr(ring);
  Part<K> part;
  Place at{0, 0};
  uint32_t tile = 0;
  auto give_back = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.empty[at.slot]);
    at.next(f.slots);
  };
  auto panel = [&]() { return ring_at + (uint32_t)(at.slot * K::kPanel); };
  for (uint32_t n = 0;; ++n) {
    const int e = n % kItems;
    const bool here = wait(sm, &sm.item_full[e], n / kItems & 1);
    if (consumers_any<K>(!here)) return;
    const Item it = sm.items[e];
    if (it.seq < 0) return;
    part.start(p, it);
    bool taken = false;
    for (int j = it.ka; j < it.kb; ++j, ++tile) {
      const int key0 = j * kTile + row0;
      const bool mine = key0 < it.hi && key0 + 16 > it.lo;
#pragma unroll
      for (int x = 0; x < K::kMaps; ++x) {
        wait(sm, &sm.full[at.slot], at.round);
        if (x == map) {
          if (!taken) {
            part.get_q(qs + (e * K::kMaps + map) * K::kRows * D * 2, it.rows, D);
            taken = true;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_empty[e]);
          }
          if (mine) part.logits(f, it, panel(), row0, key0, sm.skip[map][tile % kTileInfo]);
        }
        give_back();
      }
      wait(sm, &sm.full[at.slot], at.round);
      if (mine) part.template values<0>(f, panel(), row0, key0);
      give_back();
      if (K::kMaps == 2) {
        wait(sm, &sm.full[at.slot], at.round);
        if (mine) part.template values<K::kMaps - 1>(f, panel(), row0, key0);
        give_back();
      }
    }
    if (!taken) {   // no key: all that it says is in registers
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.item_empty[e]);
    }
    add_up<K>(f, sm, part, it);
  }
}

template <typename K>
__global__ void __launch_bounds__(K::kThreads, K::kCtas)
chunk_few_kernel(const __grid_constant__ Few f, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ char smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5;
  char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  typename K::Sm &sm = *reinterpret_cast<typename K::Sm *>(ring + f.slots * K::kPanel);
  char *qs = reinterpret_cast<char *>(&sm + 1);
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" :: "l"(&vmap) : "memory");
    for (int i = 0; i < f.slots; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], K::kConsumers);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&sm.item_full[i], 1);
      mbar_init(&sm.item_empty[i], K::kConsumers + K::kMaps - 1);
    }
    mbar_init(&sm.never, 1);
    fence_mbar_init();
    sm.flags = 0;
    sm.dead = 0;
  }
  grid_begins();
  __syncthreads();
  chunk_share<K::kThreads>(f.p, blockIdx.x, sm.sums, &sm.share, &sm.flags);
  if (warp < K::kConsumers) consume<K>(f, sm, ring, qs);
  else produce<K>(f, sm, ring, qs, &kmap, &vmap, warp - K::kConsumers);
  __syncthreads();
  if (sm.dead && warp == 0) wait_out(&sm.never);   // copies that nobody waited for
  if (tid == 0) {
    f.p.cuts[blockIdx.x] = chunk_cut(f.p, sm.share.end);
    post_status(reinterpret_cast<unsigned *>(f.p.a.ws), blockIdx.x, gridDim.x, sm.flags | (sm.dead ? kErrTimeout : 0u));
  }
}

template <typename K>
cudaError_t launch_kind(Few f, cudaStream_t s) {
  ChunkShape &p = f.p;
  const CacheLayer &c = p.a.cache;
  p.block = p.pitch = K::kRows;
  p.tile = kTile;
  f.joined = c.dim * 2 % 128 == 0;
  // CTAs of an SM share its 228 KB: 1 KB each is the system's, 6 KB are room for the join
  constexpr size_t kMost = (size_t)(228 - 6) * 1024 / K::kCtas / 1024 * 1024 - 2048;
  static_assert(offsetof(typename K::Sm, rows) % 16 == 0, "read four floats at a time");
  static_assert(2 * K::kRows <= 128, "twice the tiles' shares, whose parts have 128 rows and more: room for two of these each");
  const size_t fixed = 1024 + sizeof(typename K::Sm) + (size_t)kItems * K::kMaps * K::kRows * c.dim * 2;
  f.slots = (int)((kMost - fixed) / K::kPanel);   // three at least: K and V of 64 keys, 32 KB each at most
  if (f.slots > kRingMax) f.slots = kRingMax;
  const size_t smem = fixed + f.slots * K::kPanel;
  // before the maps are encoded: a host thread's first runtime call gives it its context
  cudaError_t e = allow_smem(reinterpret_cast<const void *>(&chunk_few_kernel<K>), smem);
  if (e != cudaSuccess) return e;
  CUtensorMap maps[2];
  const uint64_t row = (uint64_t)c.dim * 2, head = c.heads > 1 ? (uint64_t)c.head_stride : row,
                 page = c.num_pages > 1 ? (uint64_t)c.page_stride : row, token = (uint64_t)c.token_stride;
  const uint64_t dims[4] = {(uint64_t)c.dim, (uint64_t)c.page_size, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint64_t dims5[5] = {64, (uint64_t)c.page_size, (uint64_t)K::kChunks, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint64_t strides[3] = {token, head, page}, strides5[4] = {token, 128, head, page};
  const uint32_t rows = 1u << f.box_log, box[4] = {64, rows, 1, 1}, box5[5] = {64, rows, (uint32_t)K::kChunks, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (!encode_rows_map(&maps[i], i ? c.v : c.k, false, f.joined ? 5 : 4, f.joined ? dims5 : dims, f.joined ? strides5 : strides,
                         f.joined ? box5 : box))
      return cudaErrorInvalidValue;
  p.shares = sm_count() * K::kCtas;
  if (p.shares > kMaxShares / K::kMaps) p.shares = kMaxShares / K::kMaps;
  e = launch_early(chunk_few_kernel<K>, dim3(p.shares), K::kThreads, smem, s, f, maps[0], maps[1]);
  return e == cudaSuccess ? launch_chunk_join(p, s) : e;
}

inline Few few_of(const ChunkShape &p) {
  Few f{};
  f.p = p;
  const int size = p.a.cache.page_size;
  while ((2 << f.box_log) <= kTile && size % (2 << f.box_log) == 0) ++f.box_log;
  f.page_log = (size & (size - 1)) == 0 ? __builtin_ctz((unsigned)size) : -1;
  return f;
}

}  // namespace
}  // namespace last
