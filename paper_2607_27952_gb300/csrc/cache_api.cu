// C-ABI entry points of the rotary positions and the key-value cache: argument checks and
// launches.  Nothing is copied from host memory: what the kernels need travels in their
// parameters.
#include "cache_internal.h"
#include "last_internal.h"

#include <cmath>
#include <cstring>
#include <exception>

namespace last {

int sm_count() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms > 0 ? sms : 1;
}

namespace {

last_status fail(last_status st, const std::string &msg) {
  set_error(msg);
  return st;
}
last_status invalid(const std::string &msg) { return fail(LAST_ERR_INVALID_ARG, msg); }

// No exception leaves a C entry.
template <typename F>
last_status guarded(F f) {
  try {
    return f();
  } catch (const std::exception &) {
    try {
      set_error("out of host memory");
    } catch (...) {
    }
    return LAST_ERR_CUDA;
  }
}

last_status launched(cudaError_t e, const char *what) {
  if (e == cudaSuccess) return LAST_OK;
  cudaGetLastError();   // reported here, and not by whoever asks the runtime next
  return fail(LAST_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

bool multiple16(long long bytes) { return (bytes & 15) == 0; }
bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
int elem_bytes(int32_t dtype) { return dtype == LAST_DTYPE_F32 ? 4 : 2; }

last_status check_dtype(int32_t dtype) {
  return dtype == LAST_DTYPE_F32 || dtype == LAST_DTYPE_BF16
             ? LAST_OK : invalid("dtype must be LAST_DTYPE_F32 or LAST_DTYPE_BF16");
}

// f / (2 pi) modulo 1 in units of 2^-64: the 24-bit significand times 1/(2 pi) to 128 bits
// after the point, in integers (the same on every host).
unsigned long long turn_of(float f) {
  uint32_t u;
  std::memcpy(&u, &f, sizeof u);
  const int biased = (int)(u >> 23 & 255), e = biased == 0 ? -149 : biased - 150;   // f = m 2^e
  const unsigned long long m = (u & 0x7fffffu) | (biased == 0 ? 0u : 0x800000u);
  constexpr unsigned long long kHi = 0x28be60db9391054aull, kLo = 0x7f09d5f47d4d3770ull;
  const unsigned __int128 lo = (unsigned __int128)m * kLo;
  const unsigned __int128 hi = (unsigned __int128)m * kHi + (unsigned long long)(lo >> 64);
  const unsigned long long w[3] = {(unsigned long long)lo, (unsigned long long)hi, (unsigned long long)(hi >> 64)};
  const int shift = 64 - e - 1;                       // one bit more, to round
  if (shift >= 192) return 0;
  auto bits = [&](int at) -> unsigned long long {     // 64 bits of the product from bit `at` on
    const int word = at / 64, off = at % 64;
    if (word >= 3) return 0;
    const unsigned long long above = word + 1 < 3 ? w[word + 1] : 0;
    return off == 0 ? w[word] : w[word] >> off | above << (64 - off);
  };
  return bits(shift + 1) + (bits(shift) & 1);
}

last_status make_rotary(const last_rotary *r, int head_dim, RotaryTable *t) {
  if (r->rot_dim < 2 || r->rot_dim % 2 != 0 || r->rot_dim > head_dim)
    return invalid("rot_dim must be even, 2 .. head_dim");
  if (r->num_axes < 1 || r->num_axes > kMaxAxes) return invalid("num_axes must be 1 .. 4");
  if (r->pairs != LAST_ROPE_HALF && r->pairs != LAST_ROPE_ADJACENT)
    return invalid("pairs must be LAST_ROPE_HALF or LAST_ROPE_ADJACENT");
  if (r->inv_freq == nullptr) return invalid("inv_freq is required");
  t->half = r->rot_dim / 2;
  t->adjacent = r->pairs == LAST_ROPE_ADJACENT;
  for (int i = 0; i < t->half; ++i) {
    const float f = r->inv_freq[i];
    const int a = r->axis == nullptr ? 0 : r->axis[i];
    if (!(f >= 0.0f && f <= 65536.0f)) return invalid("inv_freq must lie in 0 .. 65536");
    if (a < 0 || a >= r->num_axes) return invalid("axis must lie in 0 .. num_axes - 1");
    t->turn[i] = turn_of(f);
    t->axis[i] = (uint8_t)a;
  }
  return LAST_OK;
}

// Whether the pieces of `width` at i s0 + j s1, i < n0, j < n1, lie apart (all in the same unit).
bool apart(long long n0, long long s0, long long n1, long long s1, long long width) {
  using Wide = __int128;
  if (n0 < n1) return apart(n1, s1, n0, s0, width);
  if (n1 < 1) return true;
  const Wide a = s0 < 0 ? -(Wide)s0 : s0, b = s1 < 0 ? -(Wide)s1 : s1;
  if (n0 < 2 || n1 < 2) return (n0 < 2 || a >= width) && (n1 < 2 || b >= width);
  if (a < width || b < width) return false;
  if (a >= (n1 - 1) * b + width || b >= (n0 - 1) * a + width) return true;   // one inside the other
  for (Wide j = 1; j < n1 && j * b < (n0 - 1) * a + width; ++j) {   // the multiples of a on either side of j b
    const Wide i = j * b / a < n0 - 1 ? j * b / a : n0 - 1;
    if (j * b - i * a < width || (i + 1 < n0 && (i + 1) * a - j * b < width)) return false;
  }
  return true;
}

// `name`: of the argument, for the message.  need_out: q and k of last_rope.
last_status make_rows(const last_heads *h, int elem, int tokens, int dim, bool need_out, const char *name, HeadRows *o) {
  const std::string n(name);
  if (h->heads < 1 || h->heads > 8192) return invalid(n + ": heads must be 1 .. 8192");
  if (tokens > 0 && (h->in == nullptr || (need_out && h->out == nullptr)))
    return invalid(n + ": in" + (need_out ? " and out are" : " is") + " required");
  if (!aligned(h->in, elem) || (need_out && !aligned(h->out, elem))) return invalid(n + ": misaligned");
  if (need_out && !apart(tokens, h->out_token, h->heads, h->out_head, dim))
    return invalid(n + ": heads of out overlap each other");
  o->in = static_cast<const char *>(h->in);
  o->in_token = h->in_token * elem;
  o->in_head = h->in_head * elem;
  o->heads = h->heads;
  if (need_out) {
    o->out = static_cast<char *>(h->out);
    o->out_token = h->out_token * elem;
    o->out_head = h->out_head * elem;
  }
  return LAST_OK;
}

last_status check_tokens(int32_t n) {
  if (n < 0) return invalid("num_tokens < 0");
  return n <= 1 << 30 ? LAST_OK : fail(LAST_ERR_UNSUPPORTED, "num_tokens must be at most 2^30");
}

last_status check_positions(const int32_t *positions, int64_t axis_stride, int num_axes, int tokens) {
  if (tokens > 0 && positions == nullptr) return invalid("positions are required");
  if (num_axes > 1 && axis_stride < tokens) return invalid("axis_stride must be at least num_tokens");
  return LAST_OK;
}

last_status check_cache(const last_cache *c) {
  if (c == nullptr) return invalid("cache is NULL");
  last_status st = check_dtype(c->dtype);
  if (st != LAST_OK) return st;
  if (c->num_layers < 1 || c->num_pages < 1 || c->num_kv_heads < 1)
    return invalid("num_layers, num_pages and num_kv_heads must be positive");
  if (c->page_size < 8 || c->page_size % 8 != 0) return invalid("page_size must be a positive multiple of 8");
  if (c->head_dim < 1) return invalid("head_dim must be positive");
  const int e = elem_bytes(c->dtype);
  if (c->head_dim * (long long)e % 16 != 0 || c->head_dim > 256)
    return fail(LAST_ERR_UNSUPPORTED, "head_dim * elem_bytes must be a multiple of 16 and head_dim <= 256");
  if (c->page_size > (1 << 20) || c->num_kv_heads > 4096 || c->num_layers > 4096)
    return fail(LAST_ERR_UNSUPPORTED, "page_size must be at most 2^20, num_kv_heads and num_layers at most 4096");
  if ((long long)c->page_size * c->num_kv_heads * c->head_dim * e >= 1LL << 31)
    return fail(LAST_ERR_UNSUPPORTED, "a page of one layer must stay below 2^31 bytes");
  if ((long long)c->num_layers * c->num_kv_heads * c->head_dim * e >= 1LL << 31)
    return fail(LAST_ERR_UNSUPPORTED, "a token's K of all layers must stay below 2^31 bytes");
  if (c->k == nullptr || c->v == nullptr) return invalid("k and v are required");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return invalid("k and v must be 16-byte aligned");
  const int64_t strides[4] = {c->layer_stride, c->page_stride, c->head_stride, c->token_stride};
  for (int64_t s : strides) {
    if (s < 0 || s >= (int64_t)1 << 37) return invalid("cache strides must not be negative (nor reach 2^37)");
    if (!multiple16(s * e)) return invalid("cache strides must be multiples of 16 bytes");
  }
  if (c->token_stride < c->head_dim || (c->num_kv_heads > 1 && c->head_stride < c->head_dim) ||
      (c->num_pages > 1 && c->page_stride < c->head_dim))
    return invalid("cache strides must not be below head_dim");
  return LAST_OK;
}

// Of a cache that a call writes, no two of whose pages, heads and tokens (and layers, where it writes all) may share
// an element.  Layers that are one and the same get the same bytes.
last_status check_written(const last_cache *c, bool all_layers) {
  const long long n[4] = {c->num_pages, c->num_kv_heads, c->page_size, all_layers && c->layer_stride > 0 ? c->num_layers : 1};
  const long long s[4] = {c->page_stride, c->head_stride, c->token_stride, c->layer_stride};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (!apart(n[i], s[i], n[j], s[j], c->head_dim))
        return invalid("a cache that is written may not overlap itself: its strides are too small");
  return LAST_OK;
}

last_status check_sequences(const last_sequences *s) {
  if (s == nullptr) return invalid("sequences are NULL");
  if (s->batch < 0) return invalid("batch < 0");
  if (s->batch > 0 && (s->page_table == nullptr || s->lens == nullptr))
    return invalid("page_table and lens are required");
  if (s->max_pages < 0 || (s->batch > 1 && s->table_stride < s->max_pages))
    return invalid("table_stride must be at least max_pages, which must not be negative");
  return LAST_OK;
}

last_status check_layer(const last_cache *c, int32_t layer) {
  return layer >= 0 && layer < c->num_layers ? LAST_OK : invalid("layer must lie in 0 .. num_layers - 1");
}

last_status check_cache_ws(const void *ws, size_t ws_bytes, size_t need) {
  if (ws == nullptr) return invalid("workspace is NULL");
  if (!aligned(ws, 256)) return invalid("workspace must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(LAST_ERR_WORKSPACE_TOO_SMALL, "workspace needs " + std::to_string(need) + " bytes");
  return LAST_OK;
}

// Whether the `bytes` from `out` on hold any of `rows` rows of `width` int32 each, `stride` of them apart.
bool overlaps(const void *out, long long bytes, const int32_t *in, long long rows, long long stride, long long width) {
  if (in == nullptr || bytes <= 0 || rows <= 0 || width <= 0) return false;
  const auto begin = static_cast<__int128>(reinterpret_cast<uintptr_t>(out)) - static_cast<__int128>(reinterpret_cast<uintptr_t>(in));
  const __int128 end = begin + bytes, w = (__int128)width * 4, step = (__int128)stride * 4;
  if (rows == 1) return begin < w && end > 0;
  // row i takes i step .. i step + w: the first that ends behind `begin` and whether it starts before `end`
  __int128 i = begin < w ? 0 : (begin - w) / step + 1;
  return i < rows && i * step < end;
}

CacheLayer layer_of(const last_cache *c, int layer) {
  const int e = elem_bytes(c->dtype);
  CacheLayer l;
  l.k = static_cast<char *>(c->k) + (long long)layer * c->layer_stride * e;
  l.v = static_cast<char *>(c->v) + (long long)layer * c->layer_stride * e;
  l.page_stride = c->page_stride * e;
  l.head_stride = c->head_stride * e;
  l.token_stride = c->token_stride * e;
  l.num_pages = c->num_pages;
  l.page_size = c->page_size;
  l.heads = c->num_kv_heads;
  l.dim = c->head_dim;
  return l;
}

SequenceView view_of(const last_sequences *s) {
  return SequenceView{s->page_table, s->lens, s->key_begin, s->table_stride, s->batch, s->max_pages};
}

PagesArgs pages_of(const last_cache *c, void *ws) {
  const int e = elem_bytes(c->dtype);
  PagesArgs a;
  a.k = static_cast<char *>(c->k);
  a.v = static_cast<char *>(c->v);
  a.layer_stride = c->layer_stride * e;
  a.page_stride = c->page_stride * e;
  a.head_stride = c->head_stride * e;
  a.token_stride = c->token_stride * e;
  a.layers = c->num_layers;
  a.num_pages = c->num_pages;
  a.page_size = c->page_size;
  a.heads = c->num_kv_heads;
  a.row_bytes = c->head_dim * e;
  a.status = static_cast<unsigned *>(ws);
  return a;
}

last_status rope(const last_rotary *r, int32_t dtype, int32_t num_tokens, int32_t head_dim,
                 const int32_t *positions, int64_t axis_stride, const last_heads *q, const last_heads *k,
                 bool backward, void *stream) {
  last_status st = check_dtype(dtype);
  if (st != LAST_OK) return st;
  if (r == nullptr || q == nullptr) return invalid("r and q are required");
  if ((st = check_tokens(num_tokens)) != LAST_OK) return st;
  if (head_dim < 2) return invalid("head_dim must be at least 2");
  if (head_dim > 256) return fail(LAST_ERR_UNSUPPORTED, "head_dim must be at most 256");
  RotaryArgs a{};
  if ((st = make_rotary(r, head_dim, &a.rot)) != LAST_OK) return st;
  const int e = elem_bytes(dtype);
  if ((st = make_rows(q, e, num_tokens, head_dim, true, "q", &a.q)) != LAST_OK) return st;
  if (k != nullptr && (st = make_rows(k, e, num_tokens, head_dim, true, "k", &a.k)) != LAST_OK) return st;
  if ((st = check_positions(positions, axis_stride, r->num_axes, num_tokens)) != LAST_OK) return st;
  a.positions = positions;
  a.axis_stride = axis_stride;
  a.tokens = num_tokens;
  a.dim = head_dim;
  a.elem = e;
  a.backward = backward;
  if (num_tokens == 0) return LAST_OK;
  return launched(launch_rotary(a, static_cast<cudaStream_t>(stream)), "rotary launch");
}

}  // namespace
}  // namespace last

using namespace last;

extern "C" {

last_status last_rope(const last_rotary *r, int32_t dtype, int32_t num_tokens, int32_t head_dim,
                      const int32_t *positions, int64_t axis_stride, const last_heads *q,
                      const last_heads *k, void *stream) {
  return guarded([&] { return rope(r, dtype, num_tokens, head_dim, positions, axis_stride, q, k, false, stream); });
}

last_status last_rope_backward(const last_rotary *r, int32_t dtype, int32_t num_tokens, int32_t head_dim,
                               const int32_t *positions, int64_t axis_stride, const last_heads *q,
                               const last_heads *k, void *stream) {
  return guarded([&] { return rope(r, dtype, num_tokens, head_dim, positions, axis_stride, q, k, true, stream); });
}

last_status last_cache_workspace_size(const last_cache *c, int32_t batch, int32_t num_q_heads, size_t *bytes) {
  return guarded([&]() -> last_status {
    if (bytes == nullptr) return invalid("bytes is NULL");
    last_status st = check_cache(c);
    if (st != LAST_OK) return st;
    if (batch < 0) return invalid("batch < 0");
    if (num_q_heads < 1 || num_q_heads % c->num_kv_heads != 0)
      return invalid("num_q_heads must be a positive multiple of num_kv_heads");
    *bytes = kStatusBytes + attend_scratch_bytes(num_q_heads, c->num_kv_heads, c->head_dim);
    return LAST_OK;
  });
}

last_status last_cache_append(const last_cache *c, int32_t layer, const last_sequences *s, int32_t num_tokens,
                              const int32_t *cu_new, const last_rotary *r, const int32_t *positions,
                              int64_t axis_stride, const last_heads *q, const last_heads *k,
                              const last_heads *v, void *ws, size_t ws_bytes, void *stream) {
  return guarded([&]() -> last_status {
    last_status st = check_cache(c);
    if (st != LAST_OK || (st = check_layer(c, layer)) != LAST_OK || (st = check_sequences(s)) != LAST_OK) return st;
    if ((st = check_written(c, false)) != LAST_OK) return st;
    if ((st = check_tokens(num_tokens)) != LAST_OK) return st;
    if (cu_new == nullptr && num_tokens != s->batch)
      return invalid("without cu_new there is one token per sequence: num_tokens must be batch");
    if (num_tokens > 0 && s->batch == 0) return invalid("tokens without a sequence");
    if (k == nullptr || v == nullptr) return invalid("k and v are required");
    if (r == nullptr && q != nullptr) return invalid("q without a rotation");
    const int e = elem_bytes(c->dtype);
    RotaryArgs a{};
    if (r != nullptr) {
      if ((st = make_rotary(r, c->head_dim, &a.rot)) != LAST_OK) return st;
      if ((st = check_positions(positions, axis_stride, r->num_axes, num_tokens)) != LAST_OK) return st;
    }
    if (q != nullptr && (st = make_rows(q, e, num_tokens, c->head_dim, true, "q", &a.q)) != LAST_OK) return st;
    if ((st = make_rows(k, e, num_tokens, c->head_dim, false, "k", &a.k)) != LAST_OK) return st;
    if ((st = make_rows(v, e, num_tokens, c->head_dim, false, "v", &a.v)) != LAST_OK) return st;
    if (k->heads != c->num_kv_heads || v->heads != c->num_kv_heads)
      return invalid("k and v must have the cache's num_kv_heads heads");
    if ((st = check_cache_ws(ws, ws_bytes, kStatusBytes)) != LAST_OK) return st;
    a.positions = positions;
    a.axis_stride = axis_stride;
    a.tokens = num_tokens;
    a.dim = c->head_dim;
    a.elem = e;
    a.append = true;
    a.cache = layer_of(c, layer);
    a.seq = view_of(s);
    a.cu_new = cu_new;
    a.status = static_cast<unsigned *>(ws);
    return launched(launch_rotary(a, static_cast<cudaStream_t>(stream)), "append launch");
  });
}

last_status last_cache_attention(const last_cache *c, int32_t layer, const last_sequences *s,
                                 int32_t num_q_heads, float scale, const void *q, int64_t q_stride, void *out,
                                 int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
  return guarded([&]() -> last_status {
    last_status st = check_cache(c);
    if (st != LAST_OK || (st = check_layer(c, layer)) != LAST_OK || (st = check_sequences(s)) != LAST_OK) return st;
    if (num_q_heads < 1 || num_q_heads % c->num_kv_heads != 0)
      return invalid("num_q_heads must be a positive multiple of num_kv_heads");
    if (num_q_heads > 8192) return fail(LAST_ERR_UNSUPPORTED, "num_q_heads must be at most 8192");
    const int e = elem_bytes(c->dtype);
    // tiles of 32 keys and more are counted in 32 bits
    const double tiles = ((double)s->max_pages * c->page_size / 32 + 1) * s->batch * num_q_heads;
    if (tiles >= 2147483648.0)
      return fail(LAST_ERR_UNSUPPORTED, "batch * num_q_heads * (max_pages * page_size / 32 + 1) must stay below 2^31");
    if (s->batch > 0 && (q == nullptr || out == nullptr)) return invalid("q and out are required");
    if (!aligned(q, 16) || !aligned(out, 16)) return invalid("q and out must be 16-byte aligned");
    if (!multiple16(q_stride * e) || !multiple16(out_stride * e))
      return invalid("q_stride and out_stride must be multiples of 16 bytes");
    if (s->batch > 1 && out_stride < (int64_t)num_q_heads * c->head_dim)
      return invalid("out_stride must be at least num_q_heads * head_dim");
    if (!aligned(lse, 4)) return invalid("lse is misaligned");
    const size_t need = kStatusBytes + attend_scratch_bytes(num_q_heads, c->num_kv_heads, c->head_dim);
    if ((st = check_cache_ws(ws, ws_bytes, need)) != LAST_OK) return st;
    AttendArgs a{};
    a.cache = layer_of(c, layer);
    a.seq = view_of(s);
    a.q_heads = num_q_heads;
    a.elem = e;
    a.scale = scale > 0.0f ? scale : 1.0f / std::sqrt((float)c->head_dim);
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    a.q_stride = q_stride * e;
    a.out_stride = out_stride * e;
    a.lse = lse;
    a.ws = static_cast<char *>(ws);
    return launched(launch_attend(a, static_cast<cudaStream_t>(stream)), "attention launch");
  });
}

last_status last_cache_copy(const last_cache *c, int32_t num_copies, const int32_t *src, const int32_t *dst,
                            void *ws, size_t ws_bytes, void *stream) {
  return guarded([&]() -> last_status {
    last_status st = check_cache(c);
    if (st != LAST_OK) return st;
    if ((st = check_written(c, true)) != LAST_OK) return st;
    if (num_copies < 0) return invalid("num_copies < 0");
    if (num_copies > 0 && (src == nullptr || dst == nullptr)) return invalid("src and dst are required");
    if ((st = check_cache_ws(ws, ws_bytes, kStatusBytes)) != LAST_OK) return st;
    return launched(launch_page_copy(pages_of(c, ws), num_copies, src, dst, static_cast<cudaStream_t>(stream)),
                    "page copy launch");
  });
}

last_status last_cache_compact(const last_cache *c, const last_sequences *s, const int32_t *dst_table,
                               int32_t dst_max_pages, int64_t dst_stride, const int32_t *span_begin,
                               const int32_t *span_len, const int32_t *cu_keep, const int32_t *idx,
                               int32_t num_idx, int32_t *lens_out, void *ws, size_t ws_bytes, void *stream) {
  return guarded([&]() -> last_status {
    last_status st = check_cache(c);
    if (st != LAST_OK || (st = check_sequences(s)) != LAST_OK || (st = check_written(c, true)) != LAST_OK) return st;
    if (s->batch > 0 && (dst_table == nullptr || cu_keep == nullptr || lens_out == nullptr))
      return invalid("dst_table, cu_keep and lens_out are required");
    if ((span_begin == nullptr) != (span_len == nullptr)) return invalid("span_begin and span_len go together");
    if (dst_max_pages < (s->batch > 0 ? 1 : 0) || (s->batch > 1 && dst_stride < dst_max_pages))
      return invalid("dst_stride must be at least dst_max_pages, which must be positive");
    if (num_idx < 0 || (num_idx > 0 && idx == nullptr)) return invalid("idx must hold num_idx >= 0 entries");
    // other CTAs still read these while lens_out is written
    const long long b = s->batch, bytes = b * 4;
    if (overlaps(lens_out, bytes, s->lens, 1, 0, b) || overlaps(lens_out, bytes, span_begin, 1, 0, b) ||
        overlaps(lens_out, bytes, span_len, 1, 0, b) || overlaps(lens_out, bytes, cu_keep, 1, 0, b + 1) ||
        overlaps(lens_out, bytes, idx, 1, 0, num_idx) ||
        overlaps(lens_out, bytes, s->page_table, b, s->table_stride, s->max_pages) ||
        overlaps(lens_out, bytes, dst_table, b, dst_stride, dst_max_pages))
      return invalid("lens_out may not overlap lens, span_begin, span_len, cu_keep, idx or a page table");
    if ((st = check_cache_ws(ws, ws_bytes, kStatusBytes)) != LAST_OK) return st;
    CompactArgs a{};
    a.p = pages_of(c, ws);
    a.seq = view_of(s);
    a.dst_table = dst_table;
    a.dst_stride = dst_stride;
    a.dst_max_pages = dst_max_pages;
    a.span_begin = span_begin;
    a.span_len = span_len;
    a.cu_keep = cu_keep;
    a.idx = idx;
    a.num_idx = num_idx;
    a.lens_out = lens_out;
    return launched(launch_compact(a, static_cast<cudaStream_t>(stream)), "compaction launch");
  });
}

// ---- who holds which page (host) ----

static last_status check_pool(const last_page_pool *p) {
  if (p == nullptr) return invalid("pool is NULL");
  if (p->num_pages < 0 || (p->num_pages > 0 && (p->holders == nullptr || p->free_pages == nullptr)))
    return invalid("holders and free_pages are required");
  return LAST_OK;
}

static last_status check_pages(const last_page_pool *p, int32_t n, const int32_t *pages) {
  last_status st = check_pool(p);
  if (st != LAST_OK) return st;
  if (n < 0 || (n > 0 && pages == nullptr)) return invalid("pages must hold n >= 0 entries");
  if (p->num_free < 0 || p->num_free > p->num_pages) return invalid("num_free must lie in 0 .. num_pages");
  return LAST_OK;
}

last_status last_pages_init(last_page_pool *p) {
  return guarded([&]() -> last_status {
    last_status st = check_pool(p);
    if (st != LAST_OK) return st;
    for (int32_t i = 0; i < p->num_pages; ++i) {
      p->holders[i] = 0;
      p->free_pages[i] = p->num_pages - 1 - i;   // page 0 is handed out first
    }
    p->num_free = p->num_pages;
    return LAST_OK;
  });
}

last_status last_pages_take(last_page_pool *p, int32_t n, int32_t *pages) {
  return guarded([&]() -> last_status {
    last_status st = check_pages(p, n, pages);
    if (st != LAST_OK) return st;
    if (n > p->num_free)
      return fail(LAST_ERR_NO_PAGES, std::to_string(n) + " pages asked for, " + std::to_string(p->num_free) + " free");
    for (int32_t i = 0; i < n; ++i) {
      const int32_t g = p->free_pages[p->num_free - 1 - i];
      if (g < 0 || g >= p->num_pages || p->holders[g] != 0) return invalid("free_pages is not last_pages_init's");
    }
    for (int32_t i = 0; i < n; ++i) {
      pages[i] = p->free_pages[--p->num_free];
      p->holders[pages[i]] = 1;
    }
    return LAST_OK;
  });
}

last_status last_pages_share(last_page_pool *p, int32_t n, const int32_t *pages) {
  return guarded([&]() -> last_status {
    last_status st = check_pages(p, n, pages);
    if (st != LAST_OK) return st;
    for (int32_t i = 0; i < n; ++i)
      if (pages[i] < 0 || pages[i] >= p->num_pages || p->holders[pages[i]] <= 0)
        return invalid("page " + std::to_string(pages[i]) + " is out of range or free");
    for (int32_t i = 0; i < n; ++i) ++p->holders[pages[i]];
    return LAST_OK;
  });
}

last_status last_pages_release(last_page_pool *p, int32_t n, const int32_t *pages) {
  return guarded([&]() -> last_status {
    last_status st = check_pages(p, n, pages);
    if (st != LAST_OK) return st;
    for (int32_t i = 0; i < n; ++i) {
      const bool held = pages[i] >= 0 && pages[i] < p->num_pages && p->holders[pages[i]] > 0;
      if (held) {
        --p->holders[pages[i]];
        continue;
      }
      for (int32_t j = 0; j < i; ++j) ++p->holders[pages[j]];   // a page listed too often, too
      return invalid("page " + std::to_string(pages[i]) + " is out of range or free");
    }
    for (int32_t i = 0; i < n; ++i)
      if (p->holders[pages[i]] == 0) {
        p->holders[pages[i]] = -1;   // listed again: already on the stack
        p->free_pages[p->num_free++] = pages[i];
      }
    for (int32_t i = 0; i < n; ++i)
      if (p->holders[pages[i]] == -1) p->holders[pages[i]] = 0;
    return LAST_OK;
  });
}

}  // extern "C"
