// Chunk and differential attention over bf16 keys and values: both products on the tensor cores (tcgen05).
//
// A CTA holds 256 rows (two tiles of 128) where values are at most 128 wide, else 128.  Steps go key tile by key
// tile and, within, row tile by row tile:
//   S = Q K^T into one of two accumulators in TMEM; 8 warps turn it into weights P = 2^(scale2 S - m), rounded to
//   bf16 (diff: in two parts), a warp and its lanes' rows having 64 of the 128 keys, and put them back over S; O = O + P V in TMEM, P being
//   read from there.
// The next step's S is formed before this one's O, so that the tensor cores work while the weights are formed.
// The maximum m follows a row's logits only past a factor of 2^8 (weights are then at most 2^8, and O is rescaled by those warps,
// rarely); l sums the weights before they are rounded.
//
// Warps: 0-7 softmax and epilogue, 8 and 11 issue the products, 9 fills a ring of K and V panels (128 keys by up to 128 columns) with TMA
// boxes of the pages, 10 walks the share's items and fetches rows of Q.
// A weight of zero times an infinity or NaN would show.  V rows that no row sees are zeroed in shared memory before the product reads
// them.  Where some rows of a row tile see a key and others do not (at the mask's edges: one to four key tiles of a row tile), warp 9 looks at
// its row of V; is something not finite there, the product leaves those groups of 16 keys out and the softmax warps add them up row by row.
// diff: a cluster of two CTAs, one map each; each finishes half of the rows, with the other's half of O through L2.
//
// Bound by the way from S to P: 256 rows by 128 keys by 128 columns take 4600 cycles, of which the products are 2048 (16 x 2944 tokens,
// 16 heads on 4: 575 us, 0.99 PFLOP/s).  TMEM loads, the exchange of the maxima and the exponentials of a step follow each other;
// 16 softmax warps (687 us) or four buffers of 64 keys (618 us) made no step shorter.
#include "chunk_impl.cuh"
#include "tensor_map.h"

namespace last {

namespace {

constexpr int kThreads = 384, kSoftWarps = 8, kKeys = 128, kRingMax = 12, kItems = 4, kTileInfo = 16;
constexpr int kMmaWarp = 8, kLoadWarp = 9;   // 8 and 11 issue products, 10 walks the items
constexpr uint32_t kChunkBytes = kKeys * 128;   // 128 rows of 64 elements
constexpr int kOutColumn = 256;                 // of TMEM; S takes columns 0 - 127 and 128 - 255

struct Geometry {      // the same for every CTA
  ChunkShape p;
  int chunks;          // 64-column chunks of a head's row
  int panel_chunks;    // of the first panel: a panel is two chunks or one
  int columns;         // a head's row, up to a multiple of 16
  int slots;           // panels of the ring
  int box_log, page_log;
  int rows;            // of a row tile: whole tokens where a token's heads fit one
  bool q_boxes;        // a row tile of Q is one TMA box per chunk
  float *exchange;     // diff: [CTAs][row tiles][columns / 4][64 rows][4]
};

struct Item {
  int seq, unit, first, r0, rows;
  int base, begin, lens;
  int ka, kb;             // key tiles of the share
  int lo, hi;             // keys that some row sees
  int ta[2], tb[2];       // key tiles by row tile
  int tlo[2], thi[2];     // keys by row tile
  int ca[2], cb[2];       // key tiles by row tile whose keys all rows see (those of no row of the item aside)
  int qa, qb;             // key tiles for which that holds of all row tiles
  int alo[2], ahi[2];     // keys that all rows of a row tile see
  int whole, second;
};

constexpr size_t kHead = 3 << 10;   // shared memory before the panels, of which seven of 32 KB stand beside it

struct alignas(16) Shared {
  unsigned long long full[kRingMax], empty[kRingMax], q_full[2], q_empty[2], s_full[2], p_full[2][2], pv_done[2];
  unsigned long long item_full[kItems], item_empty[kItems], looked[kTileInfo], x_full, x_empty, never;   // looked: all of `skip` is there
  Item items[kItems];
  float row[2][128];      // a row's value of one half of the columns for the other
  ChunkShare share;
  unsigned long long sums[kThreads / 32];
  alignas(16) int2 boxes[16];   // of the key tile being fetched: first token, page
  // of the key tiles on their way: groups of 8 keys whose page is out of range; from bits 16 and 24 on, by row tile, groups of 16 that the product leaves out
  volatile unsigned skip[kTileInfo];
  uint32_t tmem;
  unsigned flags;
  volatile unsigned dead;
};
static_assert(sizeof(Shared) <= kHead, "the panels begin behind it");

// The same for one thread.
__device__ __forceinline__ bool wait_alone(Shared &sm, unsigned long long *bar, uint32_t parity) {
  bool ok = mbar_try_wait(bar, parity);
  if (!ok)
    for (ChunkLimit limit; !ok && !limit.over(sm);) ok = mbar_try_wait(bar, parity);
  if (!ok) sm.dead = 1;
  return ok;
}
// For what the other CTA of the cluster has written.
__device__ __forceinline__ bool wait_cluster(Shared &sm, unsigned long long *bar, uint32_t parity) {
  uint32_t ok = 0;
  for (ChunkLimit limit; !ok && !limit.over(sm);)
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  if (__all_sync(~0u, ok != 0)) return true;
  sm.dead = 1;
  return false;
}
// 32 columns of the warp's 32 TMEM lanes.
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      :: "r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
         "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D[tmem] (+)= A[tmem] * B[smem], issued by one thread.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               :: "r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Rows of 128 bytes with the 128-byte swizzle whose inner dimension is N: chunks of 64 columns kChunkBytes apart, 8 keys 1024.
__device__ __forceinline__ uint64_t desc_n_major(uint32_t saddr) {
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(kChunkBytes >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kNMajor = 1u << 16;   // of B, in the instruction descriptor

__device__ __forceinline__ uint64_t pack2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
// One lane of a converged warp, always the same.
__device__ __forceinline__ bool elected() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ void tma_box(uint32_t dst, const void *map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

// The two warps that share 32 rows.
__device__ __forceinline__ void pair_sync(int pair) { asm volatile("bar.sync %0, 64;" :: "r"(pair + 1) : "memory"); }
__device__ __forceinline__ bool pair_any(int pair, bool x) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
               "bar.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)x), "r"(pair + 1) : "memory");
  return r != 0;
}

// Steps go key tile by key tile, in each row tile by row tile (those with keys ta .. tb - 1), and are counted over all items.

// A place in the ring and whether its panel is of an even or odd round.
struct Place {
  int slot;
  uint32_t round;
  __device__ __forceinline__ void skip(const Geometry &g, int n) {   // n <= slots
    slot += n;
    if (slot >= g.slots) {
      slot -= g.slots;
      round ^= 1;
    }
  }
};

// TILES row tiles of a block, PANELS of a head's row, MAPS: 2 for diff.
template <int TILES, int PANELS, int MAPS>
struct Kind {
  static constexpr int kTiles = TILES, kPanels = PANELS, kMaps = MAPS, kValues = PANELS * MAPS;
  // Weights in two parts (the second what rounding has left) where a difference would magnify the rounding: its terms are
  // alike and cancel.  Else one rounding of the weights, as large as the output's own, because two parts take 28% longer (16 x 2944 tokens 742 us
  // and not 577): the error against 64 bits, in the norm, is 2.0e-3 for prompts and 2.3e-3 over long caches, of which the output's own is 1.6e-3 and 1.7e-3.
  static constexpr int kParts = MAPS;
};

// Query head of map `rank` of pair h, or h.
template <typename K>
struct MapHead {
  static __device__ __forceinline__ int of(int h, int rank) { return K::kMaps == 2 ? 2 * h + rank : h; }
};

// ---- warp 10: items and rows of Q ----
template <typename K>
__device__ __forceinline__ void query_role(const Geometry &g, Shared &sm, char *qs, const CUtensorMap *qmap, int rank) {
  const ChunkShape &p = g.p;
  const int lane = threadIdx.x & 31, D = p.a.cache.dim;
  ChunkWalk walk(sm.share);
  ChunkItem it;
  uint32_t n = 0, tile = 0;
  const int eights = g.chunks * 8;   // 16-byte pieces of a row, zeros past D
  const int four_tokens = 4 / p.group, four_rest = 4 % p.group;
  for (bool more = true; more; ++n) {
    more = walk.next(p, &it);
    const int e = n % kItems;
    if (n >= kItems && !wait(sm, &sm.item_empty[e], (n / kItems & 1) ^ 1)) return;
    Item &o = sm.items[e];
    const bool writes = lane == 0, some = more && it.t.count > 0;
    const int ka = some ? it.t.first + it.k0 : 0, kb = some ? it.t.first + it.k1 : 0;
    unsigned used = 0;   // row tiles with a step
    int qa = 0, qb = 0x7fffffff;
    if (writes) {
      o.seq = more ? it.seq : -1;
      o.unit = it.unit;
      o.first = it.s.first;
      o.r0 = it.r0;
      o.rows = it.rows;
      o.base = it.s.base;
      o.begin = it.s.begin;
      o.lens = it.s.lens;
      o.ka = ka;
      o.kb = kb;
      o.lo = it.t.lo;
      o.hi = it.t.hi;
      o.whole = it.whole;
      o.second = it.second;
    }
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      ChunkTiles x{0, 0, 0, 0};
      int ta = 0, tb = 0, alo = 0, ahi = 0;
      if (some && t * g.rows < it.rows) {
        const int r0 = it.r0 + t * g.rows, r1 = it.r0 + min(it.rows, t * g.rows + g.rows);
        x = chunk_tiles(p, it.s, r0, r1);
        alo = chunk_lo(p.a, it.s, (r1 - 1) / p.group);
        ahi = chunk_hi(p.a, it.s, r0 / p.group);
        ta = max(ka, x.first);
        tb = min(kb, x.first + x.count);
      }
      used |= (unsigned)(ta < tb) << t;
      if (writes) {
        o.ta[t] = ta;
        o.tb[t] = tb;
        o.tlo[t] = x.lo;
        o.thi[t] = x.hi;
        const int ca = alo <= it.t.lo ? 0 : (alo + kKeys - 1) / kKeys, cb = ahi >= it.t.hi ? 0x7fffffff : ahi / kKeys;
        if (ta < tb) {
          qa = max(qa, ca);
          qb = min(qb, cb);
        }
        o.ca[t] = ca;
        o.cb[t] = cb;
        o.alo[t] = alo;
        o.ahi[t] = ahi;
      }
    }
    if (writes) {
      o.qa = qa;
      o.qb = qb;
      mbar_arrive(&sm.item_full[e]);
    }
    __syncwarp();
    if (!more) return;
#pragma unroll 1
    for (int t = 0; t < K::kTiles; ++t) {
      if (!(used >> t & 1)) continue;
      const int slot = tile % K::kTiles;
      if (tile >= (uint32_t)K::kTiles && !wait(sm, &sm.q_empty[slot], (tile / K::kTiles & 1) ^ 1)) return;
      const uint32_t to = smem_addr(qs) + slot * g.chunks * kChunkBytes;
      if (g.q_boxes) {   // rows of other sequences behind the last one are nobody's
        if (elected()) {
          mbar_expect_tx(&sm.q_full[slot], g.chunks * g.rows * 128);
          const int tok = it.s.first + (it.r0 + t * g.rows) / p.group;
          for (int c = 0; c < g.chunks; ++c)
            tma_box(to + c * kChunkBytes, qmap, c * 64, it.unit * p.group, rank, tok, smem_addr(&sm.q_full[slot]));
        }
        __syncwarp();
        ++tile;
        continue;
      }
      // 32 / 8 rows at a time, 8 lanes to a row's 128 bytes
      int row = t * g.rows + (lane >> 3);
      int at = it.r0 + row, tok = at / p.group, h = at - tok * p.group;
#pragma unroll 2
      for (int r = lane >> 3; r < 128; r += 4, row += 4) {
        const bool live = r < g.rows && row < it.rows;
        const char *from = p.a.q + (live ? (long long)(it.s.first + tok) * p.a.q_stride + (long long)MapHead<K>::of(it.unit * p.group + h, rank) * D * 2 : 0);
        for (int c = lane & 7; c < eights; c += 8) {
          const uint32_t dst = to + (c >> 3) * kChunkBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4);
          const bool in = live && c * 8 < D;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(in ? from + c * 16 : p.a.q), "r"(in ? 16 : 0) : "memory");
        }
        h += four_rest;   // four rows on
        tok += four_tokens;
        if (h >= p.group) {
          h -= p.group;
          ++tok;
        }
      }
      cp_async_commit();
      cp_async_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[slot]);
      ++tile;
    }
  }
}

// ---- warp 9: K and V ----
// Groups of 16 of a step's 128 keys that the product has to leave out: those with a key that some rows of the row tile
// do not see (below all_lo or from all_hi on), where V's rows of such keys hold an infinity or NaN.  k0 .. k1 - 1: keys that the product reads and
// warps 8 and 11 do not zero.  v: V's first panel.  This warp has the time, for the ring is full: 16 x 2944 tokens take 577 us, 567 without a look, and
// 633 where the softmax warps look, which the tensor cores wait for and whose code fills the instruction cache.
template <typename K>
__device__ __noinline__ unsigned hidden_values(const Geometry &g, Shared &sm, uint32_t ring, Place v, int k0, int k1, int all_lo, int all_hi, unsigned skip) {
  const int h0 = min(k1, max(k0, all_lo)), h1 = min(k1, max(h0, all_hi)), n = (h0 - k0 + k1 - h1) * 8;   // pieces of 16 bytes of 64 columns
  if (n == 0) return 0;
  __nv_bfloat162 sum = __floats2bfloat162_rn(0.0f, 0.0f);   // of zeros times them: NaN once there was something
  const __nv_bfloat162 zero = sum;
#pragma unroll 1
  for (int i = 0; i < K::kValues; ++i) {
    if (!wait(sm, &sm.full[v.slot], v.round)) return 0;
    const int chunks = K::kPanels == 1 ? g.chunks : min(2, g.chunks - 2 * (i % K::kPanels));
    uint32_t chunk = ring + v.slot * g.panel_chunks * kChunkBytes + k0 * 128;
#pragma unroll 1
    for (int c = 0; c < chunks; ++c, chunk += kChunkBytes)
#pragma unroll 4
      for (int r = threadIdx.x & 31; r < n; r += 32) {
        __nv_bfloat162 x[4];
        uint32_t (&u)[4] = reinterpret_cast<uint32_t (&)[4]>(x);
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(chunk + (r + (r < (h0 - k0) * 8 ? 0 : (h1 - h0) * 8)) * 16) : "memory");
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = __hfma2(x[e], zero, sum);
      }
    v.skip(g, 1);
  }
  // rows of pages that are out of range are nobody's, and are zeroed meanwhile
  if (!__any_sync(~0u, skip != 0 || __low2float(sum) != 0.0f || __high2float(sum) != 0.0f)) return 0;
  auto groups = [](int from, int to) { return from < to ? (1u << ((to + 15) >> 4)) - (1u << (from >> 4)) : 0u; };
  return groups(k0, h0) | groups(h1, k1);
}

// The lanes look the boxes' pages up, a tile ahead; one lane issues all boxes (25 cycles each; a lane per box took 75).
template <typename K>
__device__ __forceinline__ void load_role(const Geometry &g, Shared &sm, char *ring, const CUtensorMap *kmap, const CUtensorMap *vmap, int rank) {
  const ChunkShape &p = g.p;
  const int lane = threadIdx.x & 31, box = 1 << g.box_log, boxes = kKeys >> g.box_log;
  const int size = p.a.cache.page_size;
  const uint32_t ring_at = smem_addr(ring);
  uint32_t tile = 0;
  Place at{0, 0};
  bool again = false;   // the ring has been filled once
  for (uint32_t n = 0;; ++n) {
    const int e = n % kItems;
    if (!wait(sm, &sm.item_full[e], n / kItems & 1)) return;
    const Item &it = sm.items[e];
    const int seq = it.seq, unit = it.unit, ka = it.ka, kb = it.kb, lo = it.lo, hi = it.hi, qa = it.qa, qb = it.qb;
    if (seq < 0) return;
    const int32_t *table = p.a.seq.table + seq * p.a.seq.table_stride;
    auto counts = [&](int j) { return lane < boxes && j < kb && j * kKeys + lane * box < hi && j * kKeys + lane * box > lo - box; };
    auto lookup = [&](int j) {
      const int key = j * kKeys + lane * box;
      return counts(j) ? table[g.page_log >= 0 ? key >> g.page_log : key / size] : -1;
    };
    int page = ka < kb ? lookup(ka) : -1;
    for (int j = ka; j < kb; ++j, ++tile) {
      const int next_page = lookup(j + 1);
      const bool wanted = counts(j), here = wanted && (unsigned)page < (unsigned)p.a.cache.num_pages;
      unsigned skip = __ballot_sync(~0u, wanted && !here);
      const unsigned there = __ballot_sync(~0u, here);
      if (skip) {
        if (lane == 0) atomicOr(&sm.flags, kErrCacheIndex);
        unsigned eights = 0;   // boxes to groups of 8 keys
        for (int i = 0; i < 16; ++i) eights |= (skip >> (i * 8 >> g.box_log) & 1) << i;
        skip = eights;
      }
      if (lane == 0) sm.skip[tile % kTileInfo] = skip;
      const int row = g.page_log >= 0 ? (j * kKeys + lane * box) & (size - 1) : (j * kKeys + lane * box) % size;
      if (lane < boxes) sm.boxes[lane] = make_int2(row, page);
      __syncwarp();
      const Place first = at;
#pragma unroll 1
      for (int i = 0; i < K::kPanels + K::kValues; ++i) {
        const int pi = i % K::kPanels, value = i / K::kPanels - 1;   // -1: K
        const int chunks = K::kPanels == 1 ? g.chunks : min(2, g.chunks - 2 * pi);
        if (again && !wait(sm, &sm.empty[at.slot], at.round ^ 1)) return;
        const uint32_t bar = smem_addr(&sm.full[at.slot]), panel = ring_at + at.slot * g.panel_chunks * kChunkBytes;
        const int head = unit * K::kMaps + (value < 0 ? rank : value);
        const CUtensorMap *map = value < 0 ? kmap : vmap;
        if (elected()) {
          mbar_expect_tx(&sm.full[at.slot], __popc(there) * chunks * box * 128);
          auto load = [&](int b, int first, int its_page) {
            const uint32_t to = panel + (b << (g.box_log + 7));
            tma_box(to, map, pi * 128, first, head, its_page, bar);
            if (chunks == 2) tma_box(to + kChunkBytes, map, pi * 128 + 64, first, head, its_page, bar);
          };
          if (there == (1u << boxes) - 1 && boxes >= 4) {
#pragma unroll 1
            for (int b = 0; b < boxes; b += 4) {
              const int4 f0 = reinterpret_cast<const int4 *>(sm.boxes)[b / 2], f1 = reinterpret_cast<const int4 *>(sm.boxes)[b / 2 + 1];
              load(b, f0.x, f0.y);
              load(b + 1, f0.z, f0.w);
              load(b + 2, f1.x, f1.y);
              load(b + 3, f1.z, f1.w);
            }
          } else {
#pragma unroll 1
            for (unsigned left = there; left != 0; left &= left - 1) {
              const int b = __ffs(left) - 1;
              const int2 from = sm.boxes[b];
              load(b, from.x, from.y);
            }
          }
        }
        __syncwarp();
        const int before = at.slot;
        at.skip(g, 1);
        again |= at.slot < before;
      }
      unsigned hand = 0;
#pragma unroll 1
      for (int t = 0; t < K::kTiles; ++t) {
        if (j >= qa && j < qb) break;
        if (j < it.ta[t] || j >= it.tb[t] || (j >= it.ca[t] && j < it.cb[t])) continue;
        const int key0 = j * kKeys, kmin = max(0, it.tlo[t] - key0), kmax = min(kKeys, it.thi[t] - key0);
        Place values = first;
        values.skip(g, K::kPanels);
        hand |= hidden_values<K>(g, sm, ring_at, values, max(kmin & ~15, lo - key0), min((kmax + 15) & ~15, min(kKeys, hi - key0)),
                                 it.alo[t] - key0, it.ahi[t] - key0, skip) << (16 + 8 * t);
      }
      if (lane == 0 && hand != 0) sm.skip[tile % kTileInfo] = skip | hand;
      if (lane == 0) mbar_arrive(&sm.looked[tile % kTileInfo]);
      page = next_page;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.item_empty[e]);
  }
}

// ---- warps 8 and 11: the products, all by one thread: votes and reconvergence took a third of the warps' time ----
// Each has one of the two accumulators of S: its steps are those of a row tile, or, of an item with one row tile, every other
// one.  A step's S goes to the tensor cores right behind O of the step before, whose weights lay where it goes: products
// of one thread run in the order they are issued.  What a warp works out and waits for in between hides behind the other's
// products.  A panel's room is free once both say so: a warp that has no use for a panel gives it back as it comes, so that neither
// mistakes a round of the ring for another.
struct Tiles {   // of an item, in registers
  int ka, kb, ta[2], tb[2], ca[2], cb[2], tlo[2], thi[2], lo, hi;
  __device__ __forceinline__ explicit Tiles(const Item &it) : ka(it.ka), kb(it.kb), lo(it.lo), hi(it.hi) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ta[t] = it.ta[t];
      tb[t] = it.tb[t];
      ca[t] = it.ca[t];
      cb[t] = it.cb[t];
      tlo[t] = it.tlo[t];
      thi[t] = it.thi[t];
    }
  }
  __device__ __forceinline__ bool on(int j, int t) const { return t == 0 ? j >= ta[0] && j < tb[0] : j >= ta[1] && j < tb[1]; }
  __device__ __forceinline__ bool two() const { return ta[0] < tb[0] && ta[1] < tb[1]; }
};

__device__ __forceinline__ void zero_rows(uint32_t panel, int chunks, int from, int to) {
#pragma unroll 1
  for (int c = 0; c < chunks; ++c)
#pragma unroll 8
    for (int i = from * 8; i < to * 8; ++i)
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" :: "r"(panel + c * kChunkBytes + i * 16), "r"(0) : "memory");
}

template <typename K>
__device__ __forceinline__ void product_role(const Geometry &g, Shared &sm, char *qs_, char *ring_, uint32_t tmem, int w) {
  const int D = g.p.a.cache.dim;
  const uint32_t ring = smem_addr(ring_), panel = (uint32_t)g.panel_chunks * kChunkBytes, rows = (uint32_t)g.chunks * (kChunkBytes >> 4);
  const uint64_t q_desc = umma_desc_sw128(smem_addr(qs_)), k_desc = umma_desc_sw128(ring), v_desc = desc_n_major(ring);
  const uint32_t st = tmem + w * 128;
  uint32_t s = 0, others = 0, tile = 0, q_tile = 0;   // own steps and the other warp's; key tiles; row tiles
  Place at{0, 0};
  for (uint32_t n = 0;; ++n) {
    const int e = n % kItems;
    if (!wait_alone(sm, &sm.item_full[e], n / kItems & 1)) return;
    const bool end = sm.items[e].seq < 0;
    const Tiles it(sm.items[e]);
    mbar_arrive(&sm.item_empty[e]);
    if (end) return;
    const bool two = it.two();
    const int t = two ? w : it.ta[0] < it.tb[0] ? 0 : 1, ta = t == 0 ? it.ta[0] : it.ta[1], tb = t == 0 ? it.tb[0] : it.tb[1];
    const int tlo = t == 0 ? it.tlo[0] : it.tlo[1], thi = t == 0 ? it.thi[0] : it.thi[1], ca = t == 0 ? it.ca[0] : it.ca[1], cb = t == 0 ? it.cb[0] : it.cb[1];
    const uint32_t turn = q_tile + (two ? w : 0), q = turn % K::kTiles, o = tmem + kOutColumn + t * 128;
    bool begun = false, waited = false;   // waited: for K of tile j
#pragma unroll 1
    for (int j = it.ka; j < it.kb; ++j, ++tile) {
      const bool own = two ? j >= ta && j < tb : ((j - it.ka) & 1) == w;
      const int key0 = j * kKeys, kmin = max(0, tlo - key0), kmax = min(kKeys, thi - key0);
      const int k0 = kmin >> 4, k1 = (kmax + 15) >> 4;
      if (own && !begun && !wait_alone(sm, &sm.q_full[q], turn / K::kTiles & 1)) return;
      // before S is there: who sees it sees all of sm.skip
      if (own && (j < ca || j >= cb) && !wait_alone(sm, &sm.looked[tile % kTileInfo], tile / kTileInfo & 1)) return;
#pragma unroll
      for (int pi = 0; pi < K::kPanels; ++pi) {
        if (!waited && !wait_alone(sm, &sm.full[at.slot], at.round)) return;
        if (own) {
          const uint64_t k_rows = k_desc + at.slot * (panel >> 4), q_rows = q_desc + q * rows + pi * 2 * (kChunkBytes >> 4);
          const uint32_t idesc = umma_idesc_bf16(128, k1 * 16);
          const int steps = (D - pi * 128 + 15) / 16;
          auto product = [&](int k) {
            const int off = ((k >> 2) * (int)kChunkBytes + (k & 3) * 32) >> 4;
            umma_bf16(st, q_rows + off, k_rows + off, idesc, (pi | k) != 0 ? 1u : 0u);
          };
          if (steps >= 8) {
#pragma unroll
            for (int k = 0; k < 8; ++k) product(k);
          } else {
#pragma unroll 1
            for (int k = 0; k < steps; ++k) product(k);
          }
          if (pi == K::kPanels - 1) umma_commit(&sm.s_full[w]);
          umma_commit(&sm.empty[at.slot]);
          if (pi == K::kPanels - 1 && j + (two ? 1 : 2) >= (two ? tb : it.kb)) {   // the row tile's last
            umma_commit(&sm.q_empty[q]);
            if (two) umma_commit(&sm.q_empty[q]);
          }
        } else {
          mbar_arrive(&sm.empty[at.slot]);
        }
        at.skip(g, 1);
      }
      const Place v0 = at;
      const unsigned info = sm.skip[tile % kTileInfo], skip = info & 0xffff;   // of pages: written before K's panels were asked for
      const unsigned hand = own ? info >> (16 + 8 * t) & 0xff : 0;   // if any, the softmax warps begin O
      const int from = max(0, it.lo - key0), to = min(kKeys, it.hi - key0);
#pragma unroll
      for (int i = 0; i < K::kValues; ++i) {
        if (!wait_alone(sm, &sm.full[at.slot], at.round)) return;
        if (!own) {
          mbar_arrive(&sm.empty[at.slot]);
        } else if (((from | to) & 15) != 0 || skip != 0) {   // what no row sees is zeroed (by both warps alike)
          const int chunks = K::kPanels == 1 ? g.chunks : min(2, g.chunks - 2 * (i % K::kPanels));
          zero_rows(ring + at.slot * panel, chunks, from & ~15, from);
          zero_rows(ring + at.slot * panel, chunks, to, (to + 15) & ~15);
#pragma unroll 1
          for (unsigned left = skip; left != 0; left &= left - 1)
            zero_rows(ring + at.slot * panel, chunks, (__ffs(left) - 1) * 8, __ffs(left) * 8);
          fence_proxy_async_smem();
        }
        at.skip(g, 1);
      }
      waited = false;
      if (own) {
        const bool full = k1 - k0 == 8 && hand == 0;
        // with two row tiles the next step is the next tile's: its K comes before these weights (and wants no room of this V)
        if (two && j + 1 < it.kb) {
          Place next = at;
#pragma unroll
          for (int pi = 0; pi < K::kPanels; ++pi) {
            if (!wait_alone(sm, &sm.full[next.slot], next.round)) return;
            next.skip(g, 1);
          }
          waited = true;
        }
        // one row tile: the other warp's O of the step before goes first
        if (!two && j > it.ka && !wait_alone(sm, &sm.pv_done[w ^ 1], (others - 1) & 1)) return;
        // the first and second 32 keys of either half
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (!wait_alone(sm, &sm.p_full[w][part], s & 1)) return;
          tc_fence_after();
          Place v = v0;
#pragma unroll
          for (int i = 0; i < K::kValues; ++i) {
            const int pi = i % K::kPanels, head = i / K::kPanels;
            const int width = K::kPanels == 1 ? g.columns : min(128, g.columns - pi * 128);
            const uint32_t idesc = umma_idesc_bf16(128, width) | kNMajor, d = o + head * g.columns + pi * 128;
            const uint64_t vd = v_desc + v.slot * (panel >> 4);
            if (full) {
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                  const int k = 4 * h + 2 * part + k2;
#pragma unroll
                  for (int x = 0; x < K::kParts; ++x)
                    umma_bf16_ts(d, st + 64 * h + 16 * part + 8 * k2 + 32 * x, vd + k * (2048 >> 4), idesc, part == 0 && h + k2 + x == 0 && j == ta ? 0u : 1u);
                }
            } else if (part == 1) {
#pragma unroll 1
              for (int k = k0; k < k1; ++k) {
                if (hand >> k & 1) continue;
#pragma unroll
                for (int x = 0; x < K::kParts; ++x)
                  umma_bf16_ts(d, st + 32 * x + (k >> 2) * 64 + (k & 3) * 8, vd + k * (2048 >> 4), idesc,
                               j == ta && k == k0 && x == 0 && hand == 0 ? 0u : 1u);
              }
            }
            if (part == 1) {
              if (i == K::kValues - 1) umma_commit(&sm.pv_done[w]);
              umma_commit(&sm.empty[v.slot]);
            }
            v.skip(g, 1);
          }
        }
        begun = true;
        ++s;
      }
      others += two ? it.on(j, w ^ 1) : !own;
    }
    // an item's only step was the other warp's: it has done with the row tile when both say so
    if (!two && !begun && it.ka < it.kb) {
      if (!wait_alone(sm, &sm.q_full[q], turn / K::kTiles & 1)) return;
      mbar_arrive(&sm.q_empty[q]);
    }
    q_tile += (it.ta[0] < it.tb[0]) + (it.ta[1] < it.tb[1]);
  }
}

// ---- warps 0 to 7 ----
struct Rows {      // what a thread keeps of a row tile
  float m, l;      // l: of this warp's keys
  int lo, hi;      // keys that its row sees
  bool started;
};

// O of the warp's 32 rows and its half of the columns, plus their weights times V of `groups`, each row with the keys that it sees
// (columns from .. to - 1 of the step) alone.  p: TMEM of the step's weights, out: of O; zero: O has not begun.
template <typename K>
__device__ __forceinline__ void add_by_hand(const Geometry &g, uint32_t ring, Place v, uint32_t p, uint32_t out, bool zero, int chunk0, int chunk1, unsigned groups,
                                            int from, int to, unsigned skip) {
  const int per = g.columns / 16;
#pragma unroll 1
  for (int c = chunk0; c < chunk1; ++c) {
    const int head = K::kMaps == 2 && c >= per, col = (c - head * per) * 16;
    Place at = v;
    at.skip(g, head * K::kPanels + (col >> 7));
    const uint32_t from_v = ring + at.slot * g.panel_chunks * kChunkBytes + (col >> 6 & 1) * kChunkBytes;
    uint32_t o[16];
    if (zero) {
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = 0;
    } else {
      tmem_ld16(out + c * 16, o);
    }
#pragma unroll 1
    for (unsigned left = groups; left != 0; left &= left - 1) {
      const int k = __ffs(left) - 1;
#pragma unroll 1
      for (int i = 0; i < 16; i += 2) {
        uint32_t two, rest = 0;
        const uint32_t w_at = p + (k >> 2) * 64 + (k & 3) * 8 + i / 2;
        tmem_ld1(w_at, &two);
        if (K::kParts == 2) tmem_ld1(w_at + 32, &rest);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = k * 16 + i + e;
          const float w = e ? bf16hi(two) + bf16hi(rest) : bf16lo(two) + bf16lo(rest);
          const bool sees = key >= from && key < to && !(skip >> (key >> 3) & 1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from_v + key * 128 + ((((col & 63) >> 3) + h) ^ (key & 7)) * 16) : "memory");
#pragma unroll
            for (int d = 0; d < 8; ++d) {
              uint32_t &y = o[h * 8 + d];
              if (sees) y = __float_as_uint(fmaf(w, d & 1 ? bf16hi(x[d / 2]) : bf16lo(x[d / 2]), __uint_as_float(y)));
            }
          }
        }
      }
    }
    tmem_st16(out + c * 16, o);
  }
  tmem_wait_st();
}

// Weights of the warp's 32 rows and 64 of the step's keys.  from, to: columns of these that the row sees.  There is one
// copy of this code for all row tiles and masks: with four of them the instruction cache missed all the time.
template <typename K>
__device__ __forceinline__ void weights(const Geometry &g, Shared &sm, Rows &r, uint32_t tmem, int t, int chunk0, int chunk1,
                                        int from, int to, unsigned skip, int b, bool two, uint32_t others, bool by_hand) {
  const bool masked = __any_sync(~0u, from > 0 || to < 64) || skip != 0;
  const int pair = (threadIdx.x >> 5) & 3, half = (threadIdx.x >> 5) >> 2, row = pair * 32 + (threadIdx.x & 31);
  const uint32_t lanes = (uint32_t)(pair * 32) << 16, st = tmem + lanes + b * 128 + half * 64;
  uint32_t v[64];
  tmem_ld32(st, v);
  tmem_ld32(st + 32, v + 32);
  tmem_wait_ld();
  if (masked) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int a = min(32, max(0, from - 32 * q)), b = min(32, max(0, to - 32 * q));
      unsigned sees = (b == 32 ? ~0u : (1u << b) - 1) & (a == 32 ? 0u : ~0u << a);
      if (skip != 0)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (skip >> (half * 8 + q * 4 + i) & 1) sees &= ~(0xffu << (8 * i));
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!(sees & (1u << i))) v[32 * q + i] = __float_as_uint(-INFINITY);
    }
  }
  float top[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    top[e] = fmaxf(__uint_as_float(v[e]), __uint_as_float(v[4 + e]));
#pragma unroll
    for (int i = 8; i < 64; i += 8) top[e] = fmaxf(fmaxf(top[e], __uint_as_float(v[i + e])), __uint_as_float(v[i + 4 + e]));
  }
  float mine = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * g.p.scale2;
  if (pair_any(pair, mine > r.m + 8.0f)) {
    sm.row[half][row] = mine;
    pair_sync(pair);
    mine = fmaxf(r.m, fmaxf(mine, sm.row[half ^ 1][row]));
    const float alpha = mine > r.m ? chunk_exp2(r.m - mine) : 1.0f;
    r.m = mine;
    r.l *= alpha;
    if (r.started) {
      if (!two) wait(sm, &sm.pv_done[b ^ 1], (others - 1) & 1);   // S of one row tile comes behind its own O
      tc_fence_after();
      for (int c = chunk0; c < chunk1; ++c) {
        uint32_t o[16];
        const uint32_t at = tmem + lanes + kOutColumn + t * 128 + c * 16;
        tmem_ld16(at, o);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
        tmem_st16(at, o);
      }
      tmem_wait_st();
    }
    pair_sync(pair);   // before the next maximum overwrites sm.row
  }
  const float off = r.m == -INFINITY ? 0.0f : -r.m;
  const uint64_t scale = pack2(g.p.scale2, g.p.scale2), shift = pack2(off, off);
  uint64_t sum[2] = {0, 0};
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t w[16], rest[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = 32 * q + 2 * i;
      const float2 x = unpack2(fma2(pack2(__uint_as_float(v[at]), __uint_as_float(v[at + 1])), scale, shift));
      const float e0 = chunk_exp2(x.x), e1 = chunk_exp2(x.y);
      w[i] = pack_bf16(e0, e1);
      sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
      if (K::kParts == 2) rest[i] = pack_bf16(e0 - bf16lo(w[i]), e1 - bf16hi(w[i]));
    }
    tmem_st16(st + 16 * q, w);
    if (K::kParts == 2) tmem_st16(st + 32 + 16 * q, rest);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && (q == 0 || !by_hand)) mbar_arrive(&sm.p_full[b][q]);   // of the half's first, then second 32 keys
  }
  const float2 total = unpack2(add2(sum[0], sum[1]));
  r.l += total.x + total.y;
}

// A row of a row tile at the end of its item.
struct RowEnd {
  float m, sum;    // of both warps' keys
  int tok, head;
  bool live, started;
};

// O of a warp's rows and its half of the columns: 16-column chunks chunk0 .. chunk1 - 1, for diff one of the value's two heads.
// Blocks of 32 columns are loaded, groups of 64 stored.
template <typename K>
struct Out {
  const Geometry &g;
  const Item &it;
  const RowEnd &r;
  int rank, t, half, chunk0, chunk1, skipped;   // skipped: chunks of the value's heads before
  uint32_t tmem;
  __device__ __forceinline__ Out(const Geometry &g, const Item &it, const RowEnd &r, int rank, int t, uint32_t tmem)
      : g(g), it(it), r(r), rank(rank), t(t), half(threadIdx.x >> 7), tmem(tmem) {
    const int per = g.columns / 16, all = per * K::kMaps;
    chunk0 = half ? (all + 1) / 2 : 0;
    chunk1 = half ? all : (all + 1) / 2;
    skipped = K::kMaps == 2 && half ? per : 0;
  }
  __device__ __forceinline__ int head() const { return K::kMaps == 2 ? half : 0; }
  __device__ __forceinline__ int col(int c) const { return (c - skipped) * 16; }                 // of its head
  __device__ __forceinline__ int column(int c) const { return head() * g.p.a.cache.dim + col(c); }   // of the value
  __device__ __forceinline__ bool two(int c) const { return c + 1 < chunk1; }
  __device__ __forceinline__ int width(int c) const { return min(two(c) ? 32 : 16, g.p.a.cache.dim - col(c)); }
  __device__ __forceinline__ void load(int c, float (&x)[32]) const {
    const uint32_t at = tmem + ((threadIdx.x >> 5 & 3) << 21) + kOutColumn + t * 128 + c * 16;
    uint32_t o[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = 0;
    if (r.started) {
      if (two(c)) {
        tmem_ld32(at, o);
        tmem_wait_ld();
      } else {
        tmem_ld16(at, o);
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(o[i]);
  }
  // 32 columns, from chunk c on, of every lane's row.  Pieces of 16 bytes change places among 4 lanes, so that these write 64 bytes
  // of one row: a lane per row would touch 32 lines with every store.
  __device__ __forceinline__ void store(int c, const float (&x)[32]) const {
    const int lane = threadIdx.x & 31;
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int b = 2; b > 0; b >>= 1) {
      const bool up = lane & b;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q & b) continue;   // pieces q and q + b: the one that is not this lane's goes
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t &low = w[4 * q + i], &high = w[4 * (q + b) + i];
          const uint32_t got = __shfl_xor_sync(~0u, up ? low : high, b);
          if (up) low = got;
          else high = got;
        }
      }
    }
    // piece q is now piece lane % 4 of the row of lane (lane & 28) + q
    const int mine = (lane & 3) * 8;
    const bool in = mine < width(c);
    const long long at = r.live ? (long long)(it.first + r.tok) * g.p.a.out_stride + (long long)r.head * g.p.dv * 2 : -1;
    char *out = g.p.a.out + (column(c) + mine) * 2;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const long long to = (long long)shfl_u64((unsigned long long)at, (lane & 28) + q);
      if (to >= 0 && in) *reinterpret_cast<uint4 *>(out + to) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
    }
  }
};

// To the output where the share has the whole item (diff: rows that the other CTA finishes to it), else to the workspace.
template <typename K>
__device__ __forceinline__ void finish(const Geometry &g, const Item &it, const RowEnd &r, int rank, int t, uint32_t tmem, bool sends, float *own) {
  const ChunkShape &p = g.p;
  const Out<K> o(g, it, r, rank, t, tmem);
  const int row = threadIdx.x & 127, all = g.columns / 16 * K::kMaps;
  const bool none = it.whole && r.sum == 0.0f;
  const float f = it.whole && !none ? 1.0f / r.sum : 1.0f;
  if (it.whole && K::kMaps == 2 && !sends) return;
  // a quarter of a part's or half's columns' rows lie side by side
  float4 *to = reinterpret_cast<float4 *>(own) + (long long)t * all * 256 + (row & 63);
  int stride = 64;
  if (!it.whole) {
    float *slot = chunk_slot(p, blockIdx.x / K::kMaps, rank, it.second);
    const int br = t * g.rows + row;
    if (r.live && o.half == 0) {
      slot[br] = r.m;
      slot[p.pitch + br] = r.sum;
    }
    to = reinterpret_cast<float4 *>(slot + 2 * p.pitch) + br;
    stride = p.pitch;
  } else if (K::kMaps == 1 && r.live && o.half == 0 && p.a.lse != nullptr) {
    p.a.lse[(long long)(it.first + r.tok) * p.a.q_heads + r.head] = chunk_lse(r.m, r.sum);
  }
#pragma unroll 1
  for (int c = o.chunk0; c < o.chunk1; c += 2) {
    float x[32];
    o.load(c, x);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = none ? 0.0f : x[i] * f;
    if (K::kMaps == 1 && it.whole) {
      o.store(c, x);
      continue;
    }
    float4 *at = to + (long long)(it.whole ? c * 4 : o.column(c) / 4) * stride;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r.live && i * 4 < o.width(c)) at[(long long)i * stride] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
}

// diff: the rows that this CTA finishes, with the other's half of the difference.
template <typename K>
__device__ __forceinline__ void finish_difference(const Geometry &g, Shared &sm, const Item &it, const RowEnd &r, int rank, int t, uint32_t tmem, const float4 *theirs) {
  const ChunkShape &p = g.p;
  const Out<K> o(g, it, r, rank, t, tmem);
  const int row = threadIdx.x & 127, pair = row >> 5, all = g.columns / 16 * K::kMaps;
  const float inv = r.sum == 0.0f ? 0.0f : 1.0f / r.sum, lam = p.a.lambda[r.head];
  const float f0 = rank == 0 ? inv : -lam * inv, f1 = rank == 0 ? -lam : 1.0f;
  const bool norm = p.a.norm_weight != nullptr;
  float sq = 0.0f, f = p.a.out_scale;
#pragma unroll 1
  for (int pass = norm ? 0 : 1; pass < 2; ++pass) {   // the squares, then the output
#pragma unroll 1
    for (int c = o.chunk0; c < o.chunk1; c += 2) {
      float x[32];
      o.load(c, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (r.live && i * 4 < o.width(c)) y = __ldcg(theirs + (long long)((t * all + c) * 4 + i) * 64 + (row & 63));
        const float z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * i + k] = (r.sum == 0.0f ? 0.0f : x[4 * i + k] * f0) + z[k] * f1;
      }
      if (pass == 0) {   // columns past D are zeros
#pragma unroll
        for (int i = 0; i < 32; ++i) sq = fmaf(x[i], x[i], sq);
        continue;
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] *= norm && i < o.width(c) ? f * p.a.norm_weight[o.column(c) + i] : f;
      o.store(c, x);
    }
    if (pass == 1) break;
    sm.row[o.half][row] = sq;
    pair_sync(pair);
    sq += sm.row[o.half ^ 1][row];
    pair_sync(pair);
    f = chunk_norm(p.a, sq, p.dv);
  }
}

template <typename K>
__device__ __forceinline__ void soft_role(const Geometry &g, Shared &sm, char *ring, uint32_t tmem, int rank) {
  const ChunkShape &p = g.p;
  const ChunkArgs &a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = warp & 3, half = warp >> 2, row = pair * 32 + lane;
  const int all = g.columns / 16 * K::kMaps, chunk0 = half ? (all + 1) / 2 : 0, chunk1 = half ? all : (all + 1) / 2;
  uint32_t steps[2] = {0, 0}, tile = 0, crossed = 0;   // of the two accumulators
  for (uint32_t n = 0;; ++n) {
    const int e = n % kItems;
    const bool here = wait(sm, &sm.item_full[e], n / kItems & 1);
    if (pair_any(pair, !here)) return;
    const Item it = sm.items[e];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.item_empty[e]);
    if (it.seq < 0) return;
    const ChunkSeq seq{it.first, 0, it.base, it.begin, it.lens};
    Rows r[2];
#pragma unroll
    for (int t = 0; t < K::kTiles; ++t) {
      const bool live = row < g.rows && t * g.rows + row < it.rows;
      const int tok = (it.r0 + t * g.rows + row) / p.group;
      r[t].m = live ? -INFINITY : INFINITY;                      // rows of no token, whatever they hold, never move the others' maxima,
      r[t].l = 0.0f;
      r[t].lo = live ? chunk_lo(a, seq, tok) : 0;                // and ask for no mask
      r[t].hi = live ? chunk_hi(a, seq, tok) : 0x7fffffff;
      r[t].started = false;
    }
    if (K::kTiles == 1) r[1] = r[0];
    const bool two = it.ta[0] < it.tb[0] && it.ta[1] < it.tb[1];
#pragma unroll 1
    for (int j = it.ka; j < it.kb; ++j, ++tile) {
#pragma unroll 1
      for (int t = 0; t < K::kTiles; ++t) {
        if (t == 0 ? j < it.ta[0] || j >= it.tb[0] : j < it.ta[1] || j >= it.tb[1]) continue;
        Rows x = t == 0 ? r[0] : r[1];
        const int b = two ? t : (j - it.ka) & 1;
        const uint32_t s = b == 0 ? steps[0] : steps[1], others = b == 0 ? steps[1] : steps[0];
        wait(sm, &sm.s_full[b], s & 1);
        tc_fence_after();
        if (t * g.rows + pair * 32 < it.rows) {   // else nobody's rows, whatever becomes of them
          const int key0 = j * kKeys, kmax = min(kKeys, (t == 0 ? it.thi[0] : it.thi[1]) - key0);
          const unsigned info = sm.skip[tile % kTileInfo], skip = info & 0xffff, hand = info >> (16 + 8 * t) & 0xff;
          // columns past kmax have not been computed
          const int from = max(0, min(kKeys, x.lo - key0)) - half * 64, to = max(0, min(kmax, x.hi - key0)) - half * 64;
          weights<K>(g, sm, x, tmem, t, chunk0, chunk1, from, to, skip, b, two, others, hand != 0);
          if (hand != 0) {   // the product waits for all weights then
            const uint32_t lanes = (uint32_t)(pair * 32) << 16;
            pair_sync(pair);   // the other half's are there
            if (!two && x.started) wait(sm, &sm.pv_done[b ^ 1], (others - 1) & 1);
            tc_fence_after();
            const uint32_t panel = tile * (K::kPanels + K::kValues) + K::kPanels;
            add_by_hand<K>(g, smem_addr(ring), Place{(int)(panel % g.slots), 0}, tmem + lanes + b * 128, tmem + lanes + kOutColumn + t * 128, !x.started, chunk0, chunk1, hand, from + half * 64,
                           to + half * 64, skip);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.p_full[b][1]);
          }
        } else if (lane == 0) {
          mbar_arrive(&sm.p_full[b][0]);
          mbar_arrive(&sm.p_full[b][1]);
        }
        x.started = true;
        (t == 0 ? r[0] : r[1]) = x;
        ++(b == 0 ? steps[0] : steps[1]);
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if (steps[b] > 0) wait(sm, &sm.pv_done[b], (steps[b] - 1) & 1);
    tc_fence_after();
    const bool sends = (pair >> 1) != rank;   // diff: the other CTA finishes these rows
    if (K::kMaps == 2 && it.whole && sends && crossed > 0) wait_cluster(sm, &sm.x_empty, (crossed - 1) & 1);
    const size_t stride = (size_t)64 * all * 16 * K::kTiles;
    auto end_of = [&](int t) {
      const Rows x = t == 0 ? r[0] : r[1];
      RowEnd end;
      sm.row[half][row] = x.l;
      pair_sync(pair);
      end.sum = x.l + sm.row[half ^ 1][row];
      pair_sync(pair);
      end.live = row < g.rows && t * g.rows + row < it.rows;
      const int at = it.r0 + (end.live ? t * g.rows + row : 0);
      end.tok = at / p.group;
      end.head = it.unit * p.group + at - end.tok * p.group;
      end.m = x.m;
      end.started = x.started;
      return end;
    };
#pragma unroll 1
    for (int t = 0; t < K::kTiles; ++t) {
      if (t * g.rows + pair * 32 >= it.rows) break;
      const RowEnd end = end_of(t);
      finish<K>(g, it, end, rank, t, tmem, sends, g.exchange + blockIdx.x * stride);
    }
    if (K::kMaps == 1 || !it.whole) continue;
    // ---- diff: the halves of the rows change places ----
    const uint32_t other = rank ^ 1;
    if (sends) {
      __threadfence();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_shared(&sm.x_full, other));
    } else {
      wait_cluster(sm, &sm.x_full, crossed & 1);
#pragma unroll 1
      for (int t = 0; t < K::kTiles; ++t) {
        if (t * g.rows + pair * 32 >= it.rows) break;
        const RowEnd end = end_of(t);
        finish_difference<K>(g, sm, it, end, rank, t, tmem, reinterpret_cast<const float4 *>(g.exchange + (blockIdx.x ^ 1) * stride));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_shared(&sm.x_empty, other));
    }
    ++crossed;
  }
}

template <typename K>
__global__ void __launch_bounds__(kThreads, 1)
chunk_bf16_kernel(const __grid_constant__ Geometry g, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                  const __grid_constant__ CUtensorMap qmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  Shared &sm = *reinterpret_cast<Shared *>(smem_raw);
  char *qs = smem_raw + kHead;
  char *ring = qs + (size_t)K::kTiles * g.chunks * kChunkBytes;
  const int tid = threadIdx.x, warp = tid >> 5;
  const int rank = K::kMaps == 2 ? (int)cluster_ctarank() : 0, share = blockIdx.x / K::kMaps;
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" :: "l"(&vmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" :: "l"(&qmap) : "memory");
    for (int i = 0; i < g.slots; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.q_full[i], 1);
      mbar_init(&sm.q_empty[i], 2);
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.p_full[i][0], kSoftWarps);
      mbar_init(&sm.p_full[i][1], kSoftWarps);
      mbar_init(&sm.pv_done[i], 1);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&sm.item_full[i], 1);
      mbar_init(&sm.item_empty[i], kSoftWarps + 3);
    }
    for (int i = 0; i < kTileInfo; ++i) mbar_init(&sm.looked[i], 1);
    mbar_init(&sm.x_full, kSoftWarps / 2);
    mbar_init(&sm.x_empty, kSoftWarps / 2);
    mbar_init(&sm.never, 1);
    fence_mbar_init();
    sm.flags = 0;
    sm.dead = 0;
  }
  if ((smem_addr(smem_raw) & 1023) != 0) {   // swizzled panels want it; the declaration asks for it
    grid_begins();
    if (tid == 0) {
      if (rank == 0) g.p.cuts[share] = make_int4(0, 0, 0, 0);
      post_status(reinterpret_cast<unsigned *>(g.p.a.ws), blockIdx.x, gridDim.x, kErrConfig);
    }
    return;
  }
  if (warp == kMmaWarp) tmem_alloc(&sm.tmem, 512);
  tc_fence_before();
  grid_begins();
  __syncthreads();
  tc_fence_after();
  chunk_share<kThreads>(g.p, share, sm.sums, &sm.share, &sm.flags);
  if (K::kMaps == 2) cluster_sync();   // the other CTA's barriers are there
  const uint32_t tmem = sm.tmem;
  // 384 x 168 registers at launch = 256 x 200 + 128 x 104
  if (warp < kSoftWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    soft_role<K>(g, sm, ring, tmem, rank);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == kMmaWarp || warp == kMmaWarp + 3) {
      if (elected()) product_role<K>(g, sm, qs, ring, tmem, warp != kMmaWarp);
    } else if (warp == kLoadWarp) load_role<K>(g, sm, ring, &kmap, &vmap, rank);
    else query_role<K>(g, sm, qs, &qmap, rank);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (sm.dead && warp == 0) wait_out(&sm.never);   // copies and products that nobody waited for
  if (tid == 0) {
    if (rank == 0) g.p.cuts[share] = chunk_cut(g.p, sm.share.end);
    post_status(reinterpret_cast<unsigned *>(g.p.a.ws), blockIdx.x, gridDim.x, sm.flags | (sm.dead ? kErrTimeout : 0u));
  }
  __syncwarp();
  if (K::kMaps == 2) cluster_sync();   // until the other one has done with this one's barriers
  else __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <typename K>
cudaError_t launch_kind(Geometry g, cudaStream_t s) {
  ChunkShape &p = g.p;
  const CacheLayer &c = p.a.cache;
  const int tokens = p.group <= 128 ? 128 / p.group : 0;   // of a row tile
  g.rows = tokens > 0 ? tokens * p.group : 128;
  p.block = g.rows * K::kTiles;
  p.pitch = (p.block + 3) & ~3;
  constexpr size_t kMost = 227 << 10;
  const size_t fixed = kHead + (size_t)K::kTiles * g.chunks * kChunkBytes, slot = (size_t)g.panel_chunks * kChunkBytes;
  g.slots = (int)((kMost - fixed) / slot);
  if (g.slots > kRingMax) g.slots = kRingMax;
  const size_t smem = fixed + g.slots * slot;
  // before the maps are encoded: a host thread's first runtime call gives it its context
  cudaError_t e = allow_smem(reinterpret_cast<const void *>(&chunk_bf16_kernel<K>), smem);
  if (e != cudaSuccess) return e;
  CUtensorMap maps[3];
  const uint64_t row = (uint64_t)c.dim * 2, strides[3] = {(uint64_t)c.token_stride, c.heads > 1 ? (uint64_t)c.head_stride : row,
                                                          c.num_pages > 1 ? (uint64_t)c.page_stride : row};
  const uint64_t dims[4] = {(uint64_t)c.dim, (uint64_t)c.page_size, (uint64_t)c.heads, (uint64_t)c.num_pages};
  const uint32_t box[4] = {64, 1u << g.box_log, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (!encode_rows_map(&maps[i], i ? c.v : c.k, false, 4, dims, strides, box)) return cudaErrorInvalidValue;
  // q by element, head of its map, map, token; what no map can say (tokens 0 or 2^40 bytes apart) goes by rows
  const uint64_t q_dims[4] = {(uint64_t)c.dim, (uint64_t)p.a.q_heads / K::kMaps, (uint64_t)K::kMaps, (uint64_t)(p.a.tokens > 0 ? p.a.tokens : 1)};
  const uint64_t q_strides[3] = {row * K::kMaps, row, p.a.tokens > 1 ? (uint64_t)p.a.q_stride : row * p.a.q_heads};
  const uint32_t q_box[4] = {64, (uint32_t)p.group, 1, (uint32_t)tokens};
  g.q_boxes = tokens > 0 && p.a.q != nullptr && q_strides[2] > 0 && encode_rows_map(&maps[2], p.a.q, false, 4, q_dims, q_strides, q_box);
  if (!g.q_boxes) maps[2] = maps[0];
  int ctas = sm_count();
  if (ctas > kMaxTensorCtas) ctas = kMaxTensorCtas;
  p.shares = ctas / K::kMaps;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.shares * K::kMaps);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim = {2, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = K::kMaps;
  e = cudaLaunchKernelEx(&cfg, chunk_bf16_kernel<K>, g, maps[0], maps[1], maps[2]);
  return e == cudaSuccess ? launch_chunk_join(p, s) : e;
}

}  // namespace

cudaError_t launch_chunk_bf16(ChunkShape p, float *exchange, cudaStream_t s) {
  const CacheLayer &c = p.a.cache;
  Geometry g{};
  p.tile = kKeys;
  g.columns = (c.dim + 15) / 16 * 16;
  g.chunks = (c.dim + 63) / 64;
  g.panel_chunks = g.chunks < 2 ? g.chunks : 2;
  g.exchange = exchange;
  g.box_log = 0;
  while ((2 << g.box_log) <= kKeys && c.page_size % (2 << g.box_log) == 0) ++g.box_log;
  g.page_log = (c.page_size & (c.page_size - 1)) == 0 ? __builtin_ctz((unsigned)c.page_size) : -1;
  g.p = p;
  if (p.maps == 2) return g.columns <= 64 ? launch_kind<Kind<2, 1, 2>>(g, s) : launch_kind<Kind<1, 1, 2>>(g, s);
  return g.columns <= 128 ? launch_kind<Kind<2, 1, 1>>(g, s) : launch_kind<Kind<1, 2, 1>>(g, s);
}

}  // namespace last
