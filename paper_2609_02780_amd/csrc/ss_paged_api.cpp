// C ABI of rotary positions and of the paged cache: argument validation and the
// attention's plan.  Every check runs before any HIP call.
#include "../../include/shallowstream.h"
#include "ss_paged.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

struct ss_cache {
  ss_cache_desc desc;
  char* arena;
};

namespace {

ss_status fail(ss_status st, const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return ss_fail_text(st, text);
}

// No C++ exception crosses the C ABI.
template <class F>
ss_status guarded(F&& body) noexcept {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(SS_ERR_INTERNAL, "out of host memory");
  } catch (...) {
    return fail(SS_ERR_INTERNAL, "unexpected C++ exception");
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr size_t kLeastWorkspace = 256;
constexpr int kMaxGroup = 16;

ss_status check_desc(const ss_cache_desc* d) {
  if (!d) return fail(SS_ERR_INVALID_ARGUMENT, "desc is NULL");
  if (d->n_layers < 1 || d->n_layers > 1024)
    return fail(SS_ERR_UNSUPPORTED, "n_layers %d outside 1..1024", d->n_layers);
  if (d->n_q_heads < 1 || d->n_kv_heads < 1) return fail(SS_ERR_INVALID_ARGUMENT, "head counts must be >= 1");
  if (d->n_q_heads % d->n_kv_heads != 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "n_q_heads %d is not a multiple of n_kv_heads %d", d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads / d->n_kv_heads > kMaxGroup)
    return fail(SS_ERR_UNSUPPORTED, "query heads per KV head %d > %d", d->n_q_heads / d->n_kv_heads, kMaxGroup);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(SS_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", d->head_dim);
  if ((int64_t)d->n_kv_heads * d->head_dim > 1024)
    return fail(SS_ERR_UNSUPPORTED, "n_kv_heads * head_dim %lld > 1024", (long long)d->n_kv_heads * d->head_dim);
  if (d->n_pages < 1 || d->n_pages > 0x7FFFFFFF)
    return fail(SS_ERR_INVALID_ARGUMENT, "n_pages %lld outside 1..2^31-1", (long long)d->n_pages);
  if (d->n_slots < 1 || d->n_slots > 1 << 20)
    return fail(SS_ERR_INVALID_ARGUMENT, "n_slots %d outside 1..2^20", d->n_slots);
  return SS_OK;
}

struct Layout {
  size_t k8, v8, ks, vs, ok, ov, total;
};
Layout layout(const ss_cache_desc& d) {
  const size_t L = (size_t)d.n_layers, pages = L * (size_t)d.n_pages * d.n_kv_heads;
  const size_t open = L * (size_t)d.n_slots * 2 * d.n_kv_heads, block = (size_t)ss::kBlockTokens * d.head_dim;
  Layout o{};
  size_t at = 0;
  auto part = [&](size_t& where, size_t bytes) {
    where = at;
    at = align256(at + bytes);
  };
  part(o.k8, pages * block);
  part(o.v8, pages * block);
  part(o.ks, pages * 4);
  part(o.vs, pages * 4);
  part(o.ok, open * block * 2);
  part(o.ov, open * block * 2);
  o.total = at;
  return o;
}

// One layer of the cache with the call's streams.
ss::PagedDev view(const ss_cache* c, const ss_cache_streams* s, int layer) {
  const ss_cache_desc& d = c->desc;
  const Layout o = layout(d);
  const size_t pages = (size_t)layer * d.n_pages * d.n_kv_heads, open = (size_t)layer * d.n_slots * 2 * d.n_kv_heads;
  const size_t block = (size_t)ss::kBlockTokens * d.head_dim;
  ss::PagedDev v;
  v.k8 = reinterpret_cast<uint8_t*>(c->arena + o.k8) + pages * block;
  v.v8 = reinterpret_cast<uint8_t*>(c->arena + o.v8) + pages * block;
  v.ks = reinterpret_cast<float*>(c->arena + o.ks) + pages;
  v.vs = reinterpret_cast<float*>(c->arena + o.vs) + pages;
  v.ok = reinterpret_cast<uint16_t*>(c->arena + o.ok) + open * block;
  v.ov = reinterpret_cast<uint16_t*>(c->arena + o.ov) + open * block;
  v.tables = s->tables;
  v.lengths = s->lengths;
  v.slots = s->slots;
  v.width = s->width;
  v.n_slots = d.n_slots;
  v.n_pages = (int)d.n_pages;
  v.Hk = d.n_kv_heads;
  return v;
}

ss_status check_tokens(int32_t n_tokens) {
  if (n_tokens < 1) return fail(SS_ERR_INVALID_ARGUMENT, "n_tokens %d < 1", n_tokens);
  if (n_tokens > ss::kPagedTokens) return fail(SS_ERR_UNSUPPORTED, "n_tokens %d > %d", n_tokens, ss::kPagedTokens);
  return SS_OK;
}

ss_status check_streams(const ss_cache* c, const ss_cache_streams* s, int32_t n_tokens, const int32_t* n, const char* what) {
  if (!c) return fail(SS_ERR_INVALID_ARGUMENT, "cache is NULL");
  if (!s) return fail(SS_ERR_INVALID_ARGUMENT, "streams is NULL");
  if (s->n_streams < 1 || s->n_streams > ss::kPagedStreams)
    return fail(SS_ERR_UNSUPPORTED, "n_streams %d outside 1..%d", s->n_streams, ss::kPagedStreams);
  if (s->width < 1 || s->width > ss::kPagedWidth)
    return fail(SS_ERR_UNSUPPORTED, "width %d outside 1..%d", s->width, ss::kPagedWidth);
  if (!s->tables || !s->lengths || !s->slots || !aligned(s->tables, 4) || !aligned(s->lengths, 4) || !aligned(s->slots, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "tables, lengths or slots NULL or misaligned");
  const ss_status st = check_tokens(n_tokens);
  if (st) return st;
  if (!n) {
    if (n_tokens % s->n_streams)
      return fail(SS_ERR_INVALID_ARGUMENT, "%d tokens are not the same number for each of %d streams", n_tokens, s->n_streams);
    return SS_OK;
  }
  int64_t sum = 0;
  for (int i = 0; i < s->n_streams; ++i) {
    if (n[i] < 0) return fail(SS_ERR_INVALID_ARGUMENT, "%s[%d] = %d is negative", what, i, n[i]);
    sum += n[i];
  }
  if (sum != n_tokens)
    return fail(SS_ERR_INVALID_ARGUMENT, "%s adds up to %lld, n_tokens is %d", what, (long long)sum, n_tokens);
  return SS_OK;
}

ss_status check_layer(const ss_cache* c, int32_t layer) {
  if (layer < 0 || layer >= c->desc.n_layers)
    return fail(SS_ERR_INVALID_ARGUMENT, "layer %d outside 0..%d", layer, c->desc.n_layers - 1);
  return SS_OK;
}

ss_status check_rows(const ss_rows* r, const char* what) {
  if (!r || !r->data || !aligned(r->data, 16))
    return fail(SS_ERR_INVALID_ARGUMENT, "%s NULL or not 16-byte aligned", what);
  if (r->head_stride < 0 || r->token_stride < 0 || r->head_stride % 8 || r->token_stride % 8)
    return fail(SS_ERR_INVALID_ARGUMENT, "strides of %s must be multiples of 8 elements and not negative", what);
  return SS_OK;
}

// Rows that are written: every head's every token has a place of its own.
ss_status check_written(const ss_rows* r, int64_t heads, int64_t tokens, int64_t d, const char* what) {
  const ss_status st = check_rows(r, what);
  if (st) return st;
  const int64_t hs = r->head_stride, ts = r->token_stride;
  const bool apart = (heads == 1 || tokens == 1) ? (heads == 1 || hs >= d) && (tokens == 1 || ts >= d)
                                                 : (ts >= d && hs >= (tokens - 1) * ts + d) ||
                                                       (hs >= d && ts >= (heads - 1) * hs + d);
  if (!apart) return fail(SS_ERR_INVALID_ARGUMENT, "rows of %s overlap", what);
  return SS_OK;
}

ss_status check_rotary(const ss_rotary* r, int32_t d) {
  if (!r->freqs || !aligned(r->freqs, 8)) return fail(SS_ERR_INVALID_ARGUMENT, "freqs NULL or misaligned");
  if (r->dims < 2 || r->dims > d || r->dims % 2)
    return fail(SS_ERR_INVALID_ARGUMENT, "dims %d is not an even number in 2..%d", r->dims, d);
  if (!std::isfinite(r->gain)) return fail(SS_ERR_INVALID_ARGUMENT, "gain is not finite");
  return SS_OK;
}

ss::RowsView rows_view(const ss_rows* r) {
  return {static_cast<const uint16_t*>(r->data), r->head_stride, r->token_stride};
}

ss::Turn turn_of(const ss_rotary* r, const int64_t* positions, bool transposed) {
  if (!r) return {nullptr, nullptr, 0, 0, 1.0f, 1.0f};
  return {r->freqs, positions, r->dims, r->interleaved ? 1 : 0, r->gain, transposed ? -1.0f : 1.0f};
}

void fill_spans(ss::Spans& s, int32_t n_tokens, int n_streams, const int32_t* n) {
  s.uniform = 0;
  if (!n) {
    s.uniform = n_tokens / n_streams;
    return;
  }
  int at = 0;
  for (int i = 0; i < n_streams; ++i) {
    s.start[i] = at;
    at += n[i];
  }
  s.start[n_streams] = at;
}

// How a call of attention is cut: see for_share in the kernels.  Sizes alone decide
// (lengths are known on the device): the table's width stands for every length.
ss_status plan_attend(const ss_cache* c, const ss_cache_streams* s, int32_t n_tokens, const int32_t* n_q, int32_t window,
                      ss::PagedAttendPlan& p) {
  const int G = c->desc.n_q_heads / c->desc.n_kv_heads, Hk = c->desc.n_kv_heads, S = s->n_streams, D = c->desc.head_dim;
  int most = 0;
  if (n_q) {
    for (int i = 0; i < S; ++i) most = std::max(most, n_q[i]);
  } else {
    most = n_tokens / S;
  }
  // blocks of 32 tokens that a unit of bm columns can see
  auto seen = [&](int bm) {
    const int64_t all = (int64_t)s->width + 1;
    return window ? std::min(all, cdiv((int64_t)window + cdiv(bm, G) + 1, ss::kBlockTokens) + 1) : all;
  };
  // More than 128 columns: 256 a unit, but at d = 64 (bound by the vector unit) 128 where units are short: what
  // starts and ends them weighs more there (2,000 tokens over a window of 1,000: 72 us with 256, 52; 4,096 tokens
  // over 16,384: 350 us, 365).
  const int bm = G * most <= 16 ? 16 : G * most <= 32 ? 32 : G * most <= 128 || (D == 64 && seen(256) <= 64) ? 128 : 256;
  const int round = bm <= 32 ? 1 : 2;
  p.bm = bm;
  p.round = round;
  p.per = n_q ? 0 : (int)cdiv((int64_t)G * most, bm);
  p.units = n_q ? (int)((int64_t)G * n_tokens / bm) + S : S * p.per;
  p.cols = std::min(bm, G * most);
  const int64_t work = cdiv(seen(bm), round);
  // What beginning and ending a unit counts as, in blocks (pairs).  128 streams, 28/4 heads of 128, the last 64 of one token
  // and the others of 16,000: 384 us with none, 191 with 8, 179 with 12; with 10 drafts, of 6,144: 711, 168, 151; 4,096
  // tokens from the first: 260, 150, 149.  (More makes shares of equal units end apart: 64 tokens for each of 32
  // streams of 6,144, 16/4 heads of 64: 83, 87, 90.)  Less where 31 bits would not hold the sum.
  const int64_t most_work = 0x7FFFFFFF / p.units;
  if (work + 1 > most_work)
    return fail(SS_ERR_UNSUPPORTED, "%d units of up to %lld blocks are more than 2^31", p.units, (long long)work);
  p.start = (int)std::min<int64_t>(bm <= 32 ? 12 : 8, most_work - work - 1);
  const int64_t all = (work + p.start) * p.units * Hk;
  p.min_share = 8;
  // A block a unit leaves part of the last round of blocks idle; shares fill all rounds, but their parts are
  // joined by another kernel, which costs about as much as so many blocks (pairs) of work.  Where streams may differ, one
  // that fills its table can be the only long one, and its units what everyone waits for: then a block a unit only
  // as long as no unit can be long.  (28/4 heads of 128, a block a unit and shares.  A token for each of 128 streams: one of
  // 705,000 tokens and the others of 100 5,298 us and 129, one of 16,000 124, 22, lengths spread up to that 204, 187,
  // up to 8,192 108, 108, all of 8,192 167, 170, all of 100 9, 14.  64 tokens for each of 32 streams: one of 6,144
  // 140, 57, spread up to that 150, 127, all of 6,144 186, 187, all of 100 25, 30.)
  const int64_t join_work = bm <= 32 ? 64 : 32;
  const int64_t room = bm == 256 ? 256 : bm == 128 && D == 64 ? 768 : 512, blocks = (int64_t)p.units * Hk;
  const int64_t idle = (cdiv(blocks, room) * room - blocks) * work / room;
  const int64_t short_work = bm <= 32 ? 256 : 64;
  if ((idle <= join_work && (S == 1 || work <= short_work)) || p.units > ss::kPagedUnits) {
    p.n_wg = 0;
    p.o_bytes = p.ml_bytes = p.plan_bytes = 0;
    return SS_OK;
  }
  p.n_wg = (int)std::min<int64_t>(room, cdiv(all, p.min_share));
  p.o_bytes = align256((size_t)2 * p.n_wg * p.cols * D * 4);
  p.ml_bytes = align256((size_t)2 * p.n_wg * p.cols * 8);
  p.plan_bytes = align256((size_t)(p.units + 2) * 4);
  return SS_OK;
}

ss_status check_attend(const ss_cache* c, const ss_cache_streams* s, int32_t n_tokens, const int32_t* n_q, int32_t window) {
  const ss_status st = check_streams(c, s, n_tokens, n_q, "n_q");
  if (st) return st;
  if (window < 0 || window > 1 << 30) return fail(SS_ERR_INVALID_ARGUMENT, "window %d outside 0..2^30", window);
  return SS_OK;
}

}  // namespace

extern "C" {

ss_status ss_rotary_freqs(int32_t dims, double base, double factor, double original, double fast, double slow,
                          double* freqs, float* gain) {
  if (!freqs || !gain) return fail(SS_ERR_INVALID_ARGUMENT, "freqs or gain is NULL");
  if (dims < 2 || dims > 1024 || dims % 2)
    return fail(SS_ERR_INVALID_ARGUMENT, "dims %d is not an even number in 2..1024", dims);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(SS_ERR_INVALID_ARGUMENT, "base must be above 1");
  if (!(factor >= 1.0 && factor <= 1048576.0)) return fail(SS_ERR_INVALID_ARGUMENT, "factor outside 1..2^20");
  if (!(original >= 0.0) || !std::isfinite(original)) return fail(SS_ERR_INVALID_ARGUMENT, "original must be 0 or more");
  if (!(slow >= 0.0 && fast > slow) || !std::isfinite(fast))
    return fail(SS_ERR_INVALID_ARGUMENT, "fast and slow must be 0 <= slow < fast");
  const double two_pi = 6.283185307179586476925286766559;
  const bool parts = original > 0.0 && factor > 1.0;
  for (int i = 0; i < dims / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / dims);
    double k = 1.0 / factor;
    if (parts) {
      const double c = std::min(1.0, std::max(0.0, (original * f / two_pi - slow) / (fast - slow)));
      k = c + (1.0 - c) / factor;
    }
    freqs[i] = f * k / two_pi;
  }
  *gain = parts ? (float)(1.0 + 0.1 * std::log(factor)) : 1.0f;
  return SS_OK;
}

ss_status ss_rotate(const ss_rotary* rotary, int32_t n_heads, int32_t n_tokens, int32_t head_dim, const ss_rows* x,
                    const int64_t* positions, int32_t transposed, const ss_rows* out, void* stream) {
  return guarded([&]() -> ss_status {
    if (!rotary) return fail(SS_ERR_INVALID_ARGUMENT, "rotary is NULL");
    if (n_heads < 1 || n_heads > 4096) return fail(SS_ERR_UNSUPPORTED, "n_heads %d outside 1..4096", n_heads);
    if (head_dim != 64 && head_dim != 128) return fail(SS_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", head_dim);
    ss_status st = check_tokens(n_tokens);
    if (!st) st = check_rotary(rotary, head_dim);
    if (!st) st = check_rows(x, "x");
    if (!st) st = check_written(out, n_heads, n_tokens, head_dim, "out");
    if (st) return st;
    if (!positions || !aligned(positions, 8)) return fail(SS_ERR_INVALID_ARGUMENT, "positions NULL or misaligned");
    if (out->data == x->data && (out->head_stride != x->head_stride || out->token_stride != x->token_stride))
      return fail(SS_ERR_INVALID_ARGUMENT, "out is x with other strides");
    const ss::RotateArgs a = {rows_view(x), rows_view(out), turn_of(rotary, positions, transposed != 0), n_heads, n_tokens};
    const hipError_t e = ss::launch_rotate(a, head_dim, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "rotation launch failed: %s", hipGetErrorString(e));
    return SS_OK;
  });
}

size_t ss_cache_required_bytes(const ss_cache_desc* desc) {
  if (check_desc(desc) != SS_OK) return 0;
  return layout(*desc).total;
}

ss_status ss_cache_create(const ss_cache_desc* desc, void* dev_arena, size_t arena_bytes, ss_cache** out) {
  return guarded([&]() -> ss_status {
    if (!out) return fail(SS_ERR_INVALID_ARGUMENT, "out is NULL");
    const ss_status st = check_desc(desc);
    if (st) return st;
    if (!dev_arena || !aligned(dev_arena, 256))
      return fail(SS_ERR_INVALID_ARGUMENT, "arena NULL or not 256-byte aligned");
    const size_t need = layout(*desc).total;
    if (arena_bytes < need) return fail(SS_ERR_CAPACITY, "arena %zu bytes, %zu needed", arena_bytes, need);
    *out = new ss_cache{*desc, static_cast<char*>(dev_arena)};
    return SS_OK;
  });
}

ss_status ss_cache_destroy(ss_cache* cache) {
  if (!cache) return fail(SS_ERR_INVALID_ARGUMENT, "cache is NULL");
  delete cache;
  return SS_OK;
}

ss_status ss_cache_append(ss_cache* cache, const ss_cache_streams* streams, int32_t layer, int32_t n_tokens,
                          const int32_t* n_new, const ss_rows* keys, const ss_rows* values, const ss_rotary* rotary,
                          const int64_t* positions, const ss_rows* queries, const ss_rows* queries_out, void* stream) {
  return guarded([&]() -> ss_status {
    ss_status st = check_streams(cache, streams, n_tokens, n_new, "n_new");
    if (!st) st = check_layer(cache, layer);
    if (!st) st = check_rows(keys, "keys");
    if (!st) st = check_rows(values, "values");
    if (!st && rotary) st = check_rotary(rotary, cache->desc.head_dim);
    if (st) return st;
    if (positions && (!rotary || !aligned(positions, 8)))
      return fail(SS_ERR_INVALID_ARGUMENT, "positions without rotary, or misaligned");
    if ((queries == nullptr) != (queries_out == nullptr))
      return fail(SS_ERR_INVALID_ARGUMENT, "give queries and queries_out, or neither");
    if (queries) {
      st = check_rows(queries, "queries");
      if (!st) st = check_written(queries_out, cache->desc.n_q_heads, n_tokens, cache->desc.head_dim, "queries_out");
      if (st) return st;
      if (queries_out->data == queries->data &&
          (queries_out->head_stride != queries->head_stride || queries_out->token_stride != queries->token_stride))
        return fail(SS_ERR_INVALID_ARGUMENT, "queries_out is queries with other strides");
      if (queries_out->data == keys->data || queries_out->data == values->data)
        return fail(SS_ERR_INVALID_ARGUMENT, "queries_out is keys or values");
    }
    ss::PagedAppendArgs a;
    a.c = view(cache, streams, layer);
    a.k = rows_view(keys);
    a.v = rows_view(values);
    a.q = queries ? rows_view(queries) : ss::RowsView{nullptr, 0, 0};
    a.q_out = queries ? rows_view(queries_out) : ss::RowsView{nullptr, 0, 0};
    a.turn = turn_of(rotary, positions, false);
    a.Hq = cache->desc.n_q_heads;
    a.S = streams->n_streams;
    ss::Spans spans;
    fill_spans(spans, n_tokens, a.S, n_new);
    constexpr int B = ss::kBlockTokens;
    a.items = 0;
    if (n_new) {
      for (int i = 0; i < a.S; ++i) a.items += n_new[i] > 0 ? (n_new[i] + 2 * B - 2) / B : 0;
    } else {
      a.items = a.S * ((spans.uniform + 2 * B - 2) / B);
    }
    const hipError_t e = ss::launch_paged_append(a, spans, cache->desc.head_dim, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "append launch failed: %s", hipGetErrorString(e));
    return SS_OK;
  });
}

size_t ss_cache_attend_workspace_bytes(const ss_cache* cache, const ss_cache_streams* streams, int32_t n_tokens,
                                       const int32_t* n_q, int32_t window) {
  ss::PagedAttendPlan p;
  if (check_attend(cache, streams, n_tokens, n_q, window) != SS_OK) return 0;
  if (plan_attend(cache, streams, n_tokens, n_q, window, p) != SS_OK) return 0;
  return std::max(kLeastWorkspace, p.o_bytes + p.ml_bytes + p.plan_bytes);
}

ss_status ss_cache_attend(const ss_cache* cache, const ss_cache_streams* streams, int32_t layer, int32_t n_tokens,
                          const int32_t* n_q, const ss_rows* queries, int32_t window, const ss_rows* prior_out,
                          const float* prior_lse, void* ws, size_t ws_bytes, void* stream, const ss_rows* out,
                          float* lse) {
  return guarded([&]() -> ss_status {
    ss_status st = check_attend(cache, streams, n_tokens, n_q, window);
    if (!st) st = check_layer(cache, layer);
    if (!st) st = check_rows(queries, "queries");
    if (!st) st = check_written(out, cache->desc.n_q_heads, n_tokens, cache->desc.head_dim, "out");
    if (st) return st;
    if (out->data == queries->data) return fail(SS_ERR_INVALID_ARGUMENT, "out is queries");
    if (lse && !aligned(lse, 4)) return fail(SS_ERR_INVALID_ARGUMENT, "lse misaligned");
    if ((prior_out == nullptr) != (prior_lse == nullptr))
      return fail(SS_ERR_INVALID_ARGUMENT, "give prior_out and prior_lse, or neither");
    if (prior_out) {
      st = check_rows(prior_out, "prior_out");
      if (st) return st;
      if (!aligned(prior_lse, 4)) return fail(SS_ERR_INVALID_ARGUMENT, "prior_lse misaligned");
      if (prior_out->data == out->data || prior_lse == lse)
        return fail(SS_ERR_INVALID_ARGUMENT, "out or lse is the prior's");
    }
    if (!ws || !aligned(ws, 256)) return fail(SS_ERR_WORKSPACE, "workspace NULL or not 256-byte aligned");
    ss::PagedAttendPlan p;
    st = plan_attend(cache, streams, n_tokens, n_q, window, p);
    if (st) return st;
    const size_t need = std::max(kLeastWorkspace, p.o_bytes + p.ml_bytes + p.plan_bytes);
    if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
    const ss_cache_desc& d = cache->desc;
    ss::PagedAttendArgs a;
    a.c = view(cache, streams, layer);
    a.q = rows_view(queries);
    a.out = rows_view(out);
    a.prior = prior_out ? rows_view(prior_out) : ss::RowsView{nullptr, 0, 0};
    a.prior_lse = prior_lse;
    a.lse = lse;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + p.o_bytes);
    a.plan = reinterpret_cast<int*>(static_cast<char*>(ws) + p.o_bytes + p.ml_bytes);
    a.G = d.n_q_heads / d.n_kv_heads;
    a.S = streams->n_streams;
    a.N = n_tokens;
    a.window = window;
    a.c1 = (float)(1.4426950408889634 / std::sqrt((double)d.head_dim));
    a.units = p.units;
    a.per = p.per;
    a.cols = p.cols;
    a.n_wg = p.n_wg;
    a.min_share = p.min_share;
    a.start = p.start;
    ss::Spans spans;
    fill_spans(spans, n_tokens, a.S, n_q);
    const hipError_t e = ss::launch_paged_attend(a, spans, p, d.head_dim, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "attention launch failed: %s", hipGetErrorString(e));
    return SS_OK;
  });
}

}  // extern "C"
