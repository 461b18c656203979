// C ABI of the shallow-index evidence retrieval library: argument validation,
// per-index host bookkeeping and the retrieval planner.  Every check runs before
// any HIP call, so invalid calls leave the index and the device untouched.
#include "../../include/shallowstream.h"
#include "ss_internal.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>
#include <vector>

struct ss_index {
  ss_index_desc desc;
  void* arena;
  size_t arena_bytes;
  ss::IndexDev dev;
  int64_t n_frames;          // frames appended so far: ids 0 .. n_frames - 1
  int64_t frame_base = 0;    // frames below it were dropped from the arena (ss_index_compact);
                             // per-frame arena entries are indexed by id - frame_base
  int64_t n_rows;            // rows the arena holds per (layer, KV head)
  std::vector<int64_t> off;  // arena row offsets of frames frame_base .. n_frames
  int64_t first_detail = 0;  // frames before it were folded into long-term clusters
  int32_t rpf;               // common rows per frame, 0 if mixed, -1 before the first append
  uint16_t* values = nullptr;  // [L][H_kv][max_rows][d] bf16, null without a value cache
  float* weights = nullptr;    // [L][H_kv][max_rows], with the value cache
  size_t values_bytes = 0;     // of their arena
};

namespace {

// The last failure's text: a fixed buffer, so recording an error never allocates.
thread_local char g_err[512] = "";
thread_local hipEvent_t g_ev_start = nullptr;
thread_local hipEvent_t g_ev_stop = nullptr;

ss_status fail(ss_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return st;
}

// Runs the body of an entry point; no C++ exception crosses the C ABI (host
// allocations can throw std::bad_alloc).
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

struct Layout {
  size_t keys, counts, desc, pooled, off, stats, total;
};

// Check an index shape; fills `why` on failure.
ss_status check_desc(const ss_index_desc* d) {
  if (!d) return fail(SS_ERR_INVALID_ARGUMENT, "desc is NULL");
  if (d->n_layers < 1 || d->n_layers > ss::kMaxLayers)
    return fail(SS_ERR_UNSUPPORTED, "n_layers %d outside 1..%d", d->n_layers, ss::kMaxLayers);
  if (d->n_q_heads < 1 || d->n_kv_heads < 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "head counts must be >= 1");
  if (d->n_q_heads % d->n_kv_heads != 0)
    return fail(SS_ERR_INVALID_ARGUMENT, "n_q_heads %d is not a multiple of n_kv_heads %d",
                d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads / d->n_kv_heads > ss::kMaxGroup)
    return fail(SS_ERR_UNSUPPORTED, "query heads per KV head %d > %d",
                d->n_q_heads / d->n_kv_heads, ss::kMaxGroup);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(SS_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", d->head_dim);
  if ((int64_t)d->n_kv_heads * d->head_dim > 1024)
    return fail(SS_ERR_UNSUPPORTED, "n_kv_heads * head_dim %lld > 1024",
                (long long)d->n_kv_heads * d->head_dim);
  if (d->max_frames < 1 || d->max_frames > (int64_t)1 << 30)
    return fail(SS_ERR_INVALID_ARGUMENT, "max_frames %lld outside 1..2^30", (long long)d->max_frames);
  if (d->max_rows < 1 || d->max_rows > (int64_t)0x7FFFFFFF - 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "max_rows %lld outside 1..2^31-2", (long long)d->max_rows);
  // one (layer, KV head) segment is read through a 32-bit buffer range
  if (d->max_rows * d->head_dim * 2 > ((int64_t)1 << 31) - 1)
    return fail(SS_ERR_UNSUPPORTED, "max_rows * head_dim * 2 = %lld bytes per (layer, KV head) >= 2^31",
                (long long)(d->max_rows * d->head_dim * 2));
  if (d->n_recent < 0) return fail(SS_ERR_INVALID_ARGUMENT, "n_recent must be >= 0");
  if ((int64_t)d->n_layers * d->n_q_heads > ss::kMaxListsPerStream)
    return fail(SS_ERR_UNSUPPORTED, "n_layers * n_q_heads %lld > %d",
                (long long)d->n_layers * d->n_q_heads, ss::kMaxListsPerStream);
  return SS_OK;
}

Layout layout(const ss_index_desc& d) {
  Layout L{};
  const size_t lg = (size_t)d.n_layers * d.n_kv_heads;
  size_t off = 0;
  L.keys = off;
  off = align256(off + lg * (size_t)d.max_rows * d.head_dim * 2);
  L.counts = off;
  off = align256(off + lg * (size_t)d.max_rows * 4);
  L.desc = off;
  off = align256(off + (size_t)d.max_frames * d.n_kv_heads * d.head_dim * 4);
  L.pooled = off;
  off = align256(off + (size_t)d.max_frames * lg * d.head_dim * 4);
  L.off = off;
  off = align256(off + ((size_t)d.max_frames + 1) * 4);
  L.stats = off;
  off = align256(off + 16);
  L.total = off;
  return L;
}

// The value cache's arena: values, then weights.
struct ValuesLayout {
  size_t weights, total;
};
ValuesLayout values_layout(const ss_index_desc& d) {
  const size_t rows = (size_t)d.n_layers * d.n_kv_heads * (size_t)d.max_rows;
  ValuesLayout v{};
  v.weights = align256(rows * d.head_dim * 2);
  v.total = align256(v.weights + rows * 4);
  return v;
}

bool same_shape(const ss_index_desc& a, const ss_index_desc& b) {
  return a.n_layers == b.n_layers && a.n_q_heads == b.n_q_heads && a.n_kv_heads == b.n_kv_heads &&
         a.head_dim == b.head_dim;
}

// Candidate frames [f_lo, f_hi) and rows [r_lo, r_hi) of an index: Eq.
// context_partition excludes the newest n_recent frames, and with long-history
// compression the frames already folded into clusters are not token candidates
// (the detailed history S_T of Eq. optional_context_compression).
struct Window {
  int64_t f_lo, f_hi, r_lo, r_hi;
};
// Arena row where frame f's rows start (frame_base <= f <= n_frames).
inline int64_t row_of(const ss_index* x, int64_t f) { return x->off[(size_t)(f - x->frame_base)]; }

Window candidates(const ss_index* x) {
  Window w;
  // frames leave the arena only after they left the detailed window, which
  // never reaches into the recent window: frame_base <= f_lo <= f_hi
  w.f_hi = std::max(x->frame_base, x->n_frames - x->desc.n_recent);
  w.f_lo = std::min(x->first_detail, w.f_hi);
  w.r_lo = row_of(x, w.f_lo);
  w.r_hi = row_of(x, w.f_hi);
  return w;
}

constexpr int kSampleRank = 32;      // rank r of the sample cut-off
constexpr int kFullScanRows = 4096;  // at or below this many rows the sample is the whole list
static_assert(kFullScanRows <= 16384, "a full-scan sample must fit the register select");
constexpr int kChunkRows = 4096;
constexpr int kSampleChunk = 128;

// Expected candidates per list: 6k (at least 1024), raised for very long lists
// so the sample stays within the register select (kSampleMax rows).  The count
// behaves like E Gamma(r) / r; it falls below k with probability
// P(Poisson(r k / E) >= r) and exceeds the capacity 3E with probability
// P(Poisson(3 r) <= r - 1); either case takes the exact fallback.  A smaller E
// keeps fewer tiles on the candidate path of the streaming pass and fewer
// candidates for the selection; a larger E allows a smaller r, hence a smaller
// sample (m = r n / E).  E = 6k gives r = 14, where the capacity tail binds
// (m = 3,216 of 705,600 rows per list group on the 1-hour index); against 4k
// (r = 21) it took 2 to 7 us off a call on the 1-hour, paper-settings, 10-minute
// and 16-stream workloads, and 8k was slower on all four.
constexpr int64_t kSampleMax = 16384;
int64_t expected_candidates(int64_t n, int64_t kk) {
  const int64_t r = std::min<int64_t>(kk, kSampleRank);
  return std::max<int64_t>({6 * kk, 1024, (n * r + kSampleMax - 1) / kSampleMax});
}

// P(X >= r) for X ~ Poisson(lam): the terms from r upward, in log space.
double poisson_tail(double lam, int r) {
  if (lam <= 0.0) return r <= 0 ? 1.0 : 0.0;
  double term = std::exp(-lam + r * std::log(lam) - std::lgamma(r + 1.0)), sum = 0.0;
  for (int i = r; i < r + 2000 && term > 1e-300; ++i) {
    sum += term;
    term *= lam / (i + 1);
    if (i > lam && term < 1e-20 * sum) break;   // falling terms that no longer change the sum
  }
  return sum;
}

// P(X <= r) for X ~ Poisson(lam).
double poisson_cdf(double lam, int r) {
  if (r < 0) return 0.0;
  double term = std::exp(-lam), sum = 0.0;
  for (int i = 0; i <= r; ++i) {
    sum += term;
    term *= lam / (i + 1);
  }
  return std::min(sum, 1.0);
}

// The smallest sample rank r <= min(k, 32) whose chances of too few candidates,
// P(Poisson(r k / E) >= r), and of more than the capacity (at least 3E),
// P(Poisson(3 r) <= r - 1), are both at most kFallbackOdds per list.
constexpr double kFallbackOdds = 2e-7;
int64_t sample_rank(int64_t kk, int64_t E) {
  // the second condition does not depend on the list: the first rank that meets it
  static const int first = [] {
    int r = 1;
    while (r < kSampleRank && poisson_cdf(3.0 * (double)r, r - 1) > kFallbackOdds) ++r;
    return r;
  }();
  const int64_t rmax = std::min<int64_t>(kk, kSampleRank);
  for (int64_t r = first; r < rmax; ++r)
    if (poisson_tail((double)r * (double)kk / (double)E, (int)r) <= kFallbackOdds &&
        poisson_cdf(3.0 * (double)r, (int)r - 1) <= kFallbackOdds)
      return r;
  return rmax;
}

struct StreamSizes {
  int n, f, m, r, kk;
};

// Sample plan of one list.  With m sampled rows spread evenly over n rows and the
// cut-off at the r-th largest sample score, about r n / m rows score at or above
// it (the expected candidate count E).  r from sample_rank (14 when E = 6k);
// m = n gives an exact cut (r = k) for small lists.
StreamSizes plan_stream(int64_t n, int64_t f, int top_k) {
  StreamSizes z{};
  z.n = (int)n;
  z.f = (int)f;
  z.kk = (int)std::min<int64_t>(top_k, n);
  if (n == 0) return z;
  const int64_t E = expected_candidates(n, z.kk);
  int64_t r = sample_rank(z.kk, E);
  int64_t m = std::max<int64_t>(r, (n * r + E - 1) / E);
  if (n <= kFullScanRows || (2 * m >= n && n <= kSampleMax)) {
    m = n;
    r = z.kk;
  }
  z.m = (int)m;
  z.r = (int)r;
  return z;
}

int64_t candidate_cap(int top_k, int64_t n_max) {
  const int64_t kk = std::min<int64_t>(top_k, std::max<int64_t>(n_max, 1));
  return std::max<int64_t>(3 * expected_candidates(n_max, kk), 4096);
}

ss_status check_params(const ss_retrieve_params* p, int Hk, int D) {
  if (!p) return fail(SS_ERR_INVALID_ARGUMENT, "params is NULL");
  if (p->top_k < 1 || p->top_k > ss::kMaxTopK)
    return fail(SS_ERR_UNSUPPORTED, "top_k %d outside 1..%d", p->top_k, ss::kMaxTopK);
  if (p->n_select < 1 || p->n_select > ss::kMaxSelect)
    return fail(SS_ERR_UNSUPPORTED, "n_select %d outside 1..%d", p->n_select, ss::kMaxSelect);
  if (p->pool_mult < 1) return fail(SS_ERR_INVALID_ARGUMENT, "pool_mult must be >= 1");
  if ((int64_t)p->pool_mult * p->n_select > ss::kMaxPool)
    return fail(SS_ERR_UNSUPPORTED, "pool_mult * n_select %lld > %d",
                (long long)p->pool_mult * p->n_select, ss::kMaxPool);
  if (p->head_mode != 0 && p->head_mode != 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "head_mode must be 0 or 1");
  if (p->head_mode == 1 && Hk > 8)
    return fail(SS_ERR_UNSUPPORTED, "head_mode 1 supports at most 8 KV heads");
  if (p->score_mode != 0 && p->score_mode != 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "score_mode must be 0 or 1");
  if (p->head_mode == 1 && p->score_mode == 1 &&
      ((int64_t)Hk * D > 512 || (Hk != 1 && Hk != 2 && Hk != 4 && Hk != 8)))
    return fail(SS_ERR_UNSUPPORTED,
                "head_mode 1 with attention probabilities needs n_kv_heads in {1, 2, 4, 8} and "
                "n_kv_heads * head_dim <= 512");
  return SS_OK;
}

// Builds the plan of streams [s0, s0 + S) of a validated batch (`queries` may be
// NULL when only the workspace size is wanted), on the route of short lists where
// that is the better one.
void build_plan(ss::RetrievePlan& p, ss_index* const* idx, int s0, int S, const void* const* queries,
                const int32_t* n_q, const ss_retrieve_params* prm) {
  std::memset(&p, 0, sizeof p);
  const ss_index_desc& d = idx[0]->desc;
  p.S = S;
  p.L = d.n_layers;
  p.Hq = d.n_q_heads;
  p.Hk = d.n_kv_heads;
  p.G = p.Hq / p.Hk;
  p.D = d.head_dim;
  p.head_mode = prm->head_mode;
  p.score_mode = prm->score_mode;
  p.hm_prob = prm->head_mode == 1 && prm->score_mode == 1;
  p.NL = prm->head_mode == 0 ? p.L * p.Hq : p.L;
  p.NLs = p.hm_prob ? p.L * p.Hq : p.NL;
  p.ncol = prm->head_mode == 0 ? p.G : 1;
  p.ngs = prm->head_mode == 0 ? p.Hk : 1;
  p.top_k = prm->top_k;
  p.n_select = prm->n_select;
  p.pool_mult = prm->pool_mult;
  p.pool = prm->pool_mult * prm->n_select;
  p.chunk_rows = kChunkRows;
  p.samp_chunk = kSampleChunk;
  int64_t n_max = 0;
  int hist = 1;
  for (int i = 0; i < S; ++i) {
    const ss_index* x = idx[s0 + i];
    const Window w = candidates(x);
    const int64_t rows = w.r_hi - w.r_lo, frames = w.f_hi - w.f_lo;
    const StreamSizes z = plan_stream(rows, frames, prm->top_k);
    ss::StreamPlan& sp = p.st[i];
    sp.keys = x->dev.keys + w.r_lo * d.head_dim;          // each (layer, KV head) run from r_lo
    sp.frame_off = x->dev.frame_off + (w.f_lo - x->frame_base);
    sp.desc = x->dev.desc + (w.f_lo - x->frame_base) * (int64_t)d.n_kv_heads * d.head_dim;
    sp.frame0 = w.f_lo;
    sp.hist0 = w.f_lo - x->frame_base;
    sp.row0 = w.r_lo;
    sp.kmax = x->dev.stats;
    sp.row_stride = (int32_t)x->desc.max_rows;
    sp.n = z.n;
    sp.f = z.f;
    sp.m = z.m;
    sp.r = z.r;
    sp.kk = z.kk;
    sp.nq = n_q[s0 + i];
    sp.rpf = x->rpf > 0 ? x->rpf : 0;
    double sc = 1.0 / ((double)sp.nq * std::sqrt((double)p.D));
    if (prm->head_mode == 1 && !p.hm_prob) sc /= (double)p.Hq;   // the logit mean folds 1/H_q into the query
    sp.qscale = (float)sc;
    for (int l = 0; l < p.L; ++l)
      sp.q[l] = queries ? static_cast<const uint16_t*>(queries[(size_t)(s0 + i) * p.L + l]) : nullptr;
    n_max = std::max<int64_t>(n_max, rows);
    p.k_max = std::max(p.k_max, z.kk);
    p.m_max = std::max(p.m_max, z.m);
    p.f_max = std::max(p.f_max, z.f);
    hist = (int)std::max<int64_t>(hist, x->desc.max_frames);
  }
  p.f_max = std::max(p.f_max, 1);
  p.m_samp = p.m_max = std::max(p.m_max, 1);
  // Short lists: score and keep every row instead of sampling, streaming the
  // candidates and reading the keys twice.  What it costs is writing and reading
  // the scores, so beyond 8,192 rows a batch takes it up to 3 M of them.
  // Per call, sampled / all rows, k = 64, d = 128: 112 lists of 2,048 rows 59.4 /
  // 30.6 us, 8,192 rows 45.4 / 37.5, 19,200 rows 51.8 / 47.5; 160 lists (8 KV
  // heads) of 16,384 rows 66.7 / 64.0, of 25,600 (4.1 M) 81.2 / 84.0; 448 lists of
  // 8,192 rows 84 / 65, of 19,200 107 / 110.
  // The line at 512 lists holds for every list length up to 8,192 rows on this
  // side of it; on the other it depends on the length: 896 lists of 3,920 rows 108
  // / 67 us, of 7,840 98 / 95, 1,792 of 3,920 180 / 113, of 7,840 156 / 170, 3,360
  // of 7,840 277 / 315.  A line on the scores there (shorter lists than about 4,096
  // rows in any number) would gain what these say.
  const int64_t lists = (int64_t)p.S * p.NL;
  if (prm->head_mode == 0 && prm->top_k <= ss::kAllTopK && n_max <= ss::kAllRows && p.S * p.L <= 128 &&
      lists <= 512 && (n_max <= 8192 || lists * n_max <= 3'000'000)) {
    p.all_rows = true;
    p.m_max = p.m_all = (int)((std::max<int64_t>(n_max, 1) + 15) / 16 * 16);   // whole tiles
  }
  p.cap = (int)candidate_cap(prm->top_k, n_max);
  p.dbg_hist_stride = hist;
}

ss_status check_batch(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                      const ss_retrieve_params* prm) {
  if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
  if (n_streams < 1) return fail(SS_ERR_INVALID_ARGUMENT, "n_streams must be >= 1");
  if (!n_q) return fail(SS_ERR_INVALID_ARGUMENT, "n_q is NULL");
  for (int s = 0; s < n_streams; ++s) {
    if (!idx[s]) return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] is NULL", s);
    if (!same_shape(idx[s]->desc, idx[0]->desc))
      return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] shape differs from idx[0]", s);
    if (n_q[s] < 1 || n_q[s] > 4096)
      return fail(SS_ERR_INVALID_ARGUMENT, "n_q[%d] = %d outside 1..4096", s, n_q[s]);
  }
  return check_params(prm, idx[0]->desc.n_kv_heads, idx[0]->desc.head_dim);
}

// The plan's two routes: of longer lists (sample, cut-off, streaming pass), and of
// short ones where build_plan chose that.
void take_sampled_route(ss::RetrievePlan& p) {
  p.all_rows = false;
  p.m_max = p.m_samp;
}
void take_all_rows_route(ss::RetrievePlan& p) {
  p.all_rows = true;
  p.m_max = p.m_all;
}

// Workspace bytes of a batch.  Every group needs the sampled route's (`least`);
// the size a caller should have adds room for the route of short lists, where
// that stays within kNoAllocBytes.
size_t batch_ws(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                const ss_retrieve_params* prm, bool least) {
  size_t need = 0;
  for (int s0 = 0; s0 < n_streams; s0 += ss::kMaxStreams) {
    const int S = std::min(ss::kMaxStreams, n_streams - s0);
    ss::RetrievePlan p;
    build_plan(p, idx, s0, S, nullptr, n_q, prm);
    if (p.all_rows && !least) {
      const size_t all = ss::carve_workspace(p, nullptr);
      if (all <= ss::kNoAllocBytes) need = std::max(need, all);
    }
    take_sampled_route(p);
    need = std::max(need, ss::carve_workspace(p, nullptr));
  }
  return need;
}

ss_status retrieve_common(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                          const int32_t* n_q, const ss_retrieve_params* prm, void* ws,
                          size_t ws_bytes, void* stream, int64_t* frame_ids, int32_t* votes,
                          float* mass, int32_t* n_out, const ss_debug_out* dbg) {
  ss_status st = check_batch(idx, n_streams, n_q, prm);
  if (st) return st;
  if (!queries) return fail(SS_ERR_INVALID_ARGUMENT, "queries is NULL");
  const int L = idx[0]->desc.n_layers;
  for (int i = 0; i < n_streams * L; ++i) {
    if (!queries[i]) return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] is NULL", i);
    if (!aligned(queries[i], 16)) return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] not 16-byte aligned", i);
  }
  if (!frame_ids || !votes || !mass || !n_out)
    return fail(SS_ERR_INVALID_ARGUMENT, "an output pointer is NULL");
  if (!ws || !aligned(ws, 256)) return fail(SS_ERR_WORKSPACE, "workspace NULL or not 256-byte aligned");
  // a batch of one group (the usual one) is sized by the plan it runs; of more,
  // every group before the first is enqueued
  auto too_small = [&](size_t need) {
    return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
  };
  if (n_streams > ss::kMaxStreams) {
    const size_t need = batch_ws(idx, n_streams, n_q, prm, true);
    if (ws_bytes < need) return too_small(need);
  }
  if (dbg && dbg->topk_score == nullptr && dbg->topk_pos != nullptr)
    return fail(SS_ERR_INVALID_ARGUMENT, "debug topk_pos needs topk_score");
  if (dbg && (dbg->vote_hist == nullptr) != (dbg->mass_hist == nullptr))
    return fail(SS_ERR_INVALID_ARGUMENT, "debug vote_hist and mass_hist go together");
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  for (int s0 = 0; s0 < n_streams; s0 += ss::kMaxStreams) {
    const int S = std::min(ss::kMaxStreams, n_streams - s0);
    ss::RetrievePlan p;
    build_plan(p, idx, s0, S, queries, n_q, prm);
    // the route of short lists, where the workspace has room for its scores too and
    // the streaming pass's statistics are not asked for
    const bool all = p.all_rows && !(dbg && dbg->list_stats) && ss::carve_workspace(p, nullptr) <= ws_bytes;
    take_sampled_route(p);
    const size_t need = ss::carve_workspace(p, ws);
    if (need > ws_bytes) return too_small(need);
    if (all) {
      take_all_rows_route(p);
      ss::carve_workspace(p, ws);
    }
    p.out_ids = frame_ids + (size_t)s0 * prm->n_select;
    p.out_votes = votes + (size_t)s0 * prm->n_select;
    p.out_mass = mass + (size_t)s0 * prm->n_select;
    p.out_n = n_out + s0;
    p.out_stride = prm->n_select;
    if (dbg) {
      const size_t NLt = (size_t)p.NL * prm->top_k;
      int hist = 1;
      for (int s = 0; s < n_streams; ++s) hist = (int)std::max<int64_t>(hist, idx[s]->desc.max_frames);
      p.dbg_hist_stride = hist;
      p.dbg_topk_pos = dbg->topk_pos ? dbg->topk_pos + (size_t)s0 * NLt : nullptr;
      p.dbg_topk_score = dbg->topk_score ? dbg->topk_score + (size_t)s0 * NLt : nullptr;
      p.dbg_vote_hist = dbg->vote_hist ? dbg->vote_hist + (size_t)s0 * hist : nullptr;
      p.dbg_mass_hist = dbg->mass_hist ? dbg->mass_hist + (size_t)s0 * hist : nullptr;
      p.dbg_pool = dbg->pool ? dbg->pool + (size_t)s0 * p.pool : nullptr;
      p.dbg_pool_n = dbg->pool_n ? dbg->pool_n + s0 : nullptr;
      p.dbg_list_stats = dbg->list_stats ? dbg->list_stats + (size_t)s0 * p.NL * 2 : nullptr;
    }
    p.ev_start = g_ev_start;
    p.ev_stop = g_ev_stop;
    const hipError_t e = ss::launch_retrieve(p, hs);
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "retrieve launch failed: %s", hipGetErrorString(e));
  }
  return SS_OK;
}

// Plan of one group of streams [s0, s0 + S) of a pooled-ranking batch.
void build_pooled(ss::PooledPlan& p, ss_index* const* idx, int s0, int S, const void* const* queries,
                  const int32_t* n_q, int n_select) {
  std::memset(&p, 0, sizeof p);
  const ss_index_desc& d = idx[0]->desc;
  p.S = S; p.L = d.n_layers; p.Hq = d.n_q_heads; p.Hk = d.n_kv_heads; p.G = p.Hq / p.Hk;
  p.D = d.head_dim; p.n_select = n_select;
  for (int i = 0; i < S; ++i) {
    const ss_index* x = idx[s0 + i];
    const Window w = candidates(x);
    const int64_t frames = w.f_hi - w.f_lo;
    p.F[i] = frames;
    p.frame0[i] = w.f_lo;
    p.f_max = std::max<int64_t>(p.f_max, frames);
    p.pooled[i] = x->dev.pooled + (w.f_lo - x->frame_base) * (int64_t)p.L * p.Hk * p.D;
    p.nq[i] = n_q[s0 + i];
    for (int l = 0; l < p.L; ++l)
      p.q[i * p.L + l] = queries ? static_cast<const uint16_t*>(queries[(size_t)(s0 + i) * p.L + l]) : nullptr;
  }
}

size_t pooled_ws(ss_index* const* idx, int32_t n_streams, const int32_t* n_q, int n_select) {
  size_t need = 0;
  for (int s0 = 0; s0 < n_streams; s0 += ss::kMaxStreams) {
    ss::PooledPlan p;
    build_pooled(p, idx, s0, std::min(ss::kMaxStreams, n_streams - s0), nullptr, n_q, n_select);
    need = std::max(need, ss::pooled_workspace(p, nullptr));
  }
  return need;
}

ss_status check_pooled(ss_index* const* idx, int32_t n_streams, const int32_t* n_q, int32_t n_select) {
  if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
  if (n_streams < 1) return fail(SS_ERR_INVALID_ARGUMENT, "n_streams must be >= 1");
  if (!n_q) return fail(SS_ERR_INVALID_ARGUMENT, "n_q is NULL");
  for (int s = 0; s < n_streams; ++s) {
    if (!idx[s]) return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] is NULL", s);
    if (!same_shape(idx[s]->desc, idx[0]->desc))
      return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] shape differs from idx[0]", s);
    if (n_q[s] < 1 || n_q[s] > 4096)
      return fail(SS_ERR_INVALID_ARGUMENT, "n_q[%d] = %d outside 1..4096", s, n_q[s]);
  }
  if (n_select < 1 || n_select > ss::kMaxSelect)
    return fail(SS_ERR_UNSUPPORTED, "n_select %d outside 1..%d", n_select, ss::kMaxSelect);
  return SS_OK;
}

struct ClusterLayout {
  size_t state, centroids, sizes, span, reps, total;
};

bool cluster_desc_ok(const ss_cluster_desc* d) {
  return d && d->n_layers >= 1 && d->n_layers <= ss::kMaxLayers && d->n_kv_heads >= 1 &&
         (d->head_dim == 64 || d->head_dim == 128) && (int64_t)d->n_kv_heads * d->head_dim <= 1024 &&
         d->rows_per_unit >= 1 && d->rows_per_unit <= 65536 && d->max_clusters >= 1 &&
         d->max_clusters <= ((int64_t)1 << 30) && std::isfinite(d->tau);
}

ClusterLayout cluster_layout(const ss_cluster_desc& d) {
  ClusterLayout L{};
  const size_t dim = (size_t)d.n_kv_heads * d.head_dim, M = (size_t)d.max_clusters;
  size_t off = 0;
  L.state = off;
  off = align256(off + 16);
  L.centroids = off;
  off = align256(off + M * dim * 4);
  L.sizes = off;
  off = align256(off + M * 4);
  L.span = off;
  off = align256(off + M * 16);
  L.reps = off;
  off = align256(off + M * d.n_layers * dim * d.rows_per_unit * 4);
  L.total = off;
  return L;
}

// Candidate items of one stream's evidence, or -1 for invalid parameters.
int64_t evidence_units_max(const ss_evidence_params* p, int32_t n_select, int32_t k_clusters) {
  if (!p || p->n_recent < 0 || p->n_before < 0 || p->n_after < 0) return -1;
  if (p->retrieved != 0 && p->retrieved != 1) return -1;
  if (k_clusters < 0 || k_clusters > ss::kMaxSelect) return -1;
  int64_t n = p->n_recent;
  if (p->retrieved) {
    if (n_select < 1 || n_select > ss::kMaxSelect) return -1;
    n += (int64_t)n_select * (1 + (int64_t)p->n_before + p->n_after) + k_clusters;
  }
  return n;
}

ss_status append_common(ss_index* idx, const void* const* layer_keys, const void* const* layer_values,
                        int32_t n_frames, int32_t n_tokens, const ss_compress* compress, void* stream,
                        int64_t* first_frame_id) {
  const ss_index_desc& d = idx->desc;
  if (!layer_keys) return fail(SS_ERR_INVALID_ARGUMENT, "layer_keys is NULL");
  if (n_frames < 1 || n_tokens < 1)
    return fail(SS_ERR_INVALID_ARGUMENT, "n_frames and n_tokens must be >= 1");
  if ((int64_t)n_frames * n_tokens > 0x7FFFFFFF)
    return fail(SS_ERR_UNSUPPORTED, "n_frames * n_tokens exceeds 2^31-1");
  for (int l = 0; l < d.n_layers; ++l) {
    if (!layer_keys[l]) return fail(SS_ERR_INVALID_ARGUMENT, "layer_keys[%d] is NULL", l);
    if (!aligned(layer_keys[l], 16))
      return fail(SS_ERR_INVALID_ARGUMENT, "layer_keys[%d] not 16-byte aligned", l);
  }
  for (int l = 0; layer_values && l < d.n_layers; ++l) {
    if (!layer_values[l]) return fail(SS_ERR_INVALID_ARGUMENT, "layer_values[%d] is NULL", l);
    if (!aligned(layer_values[l], 16))
      return fail(SS_ERR_INVALID_ARGUMENT, "layer_values[%d] not 16-byte aligned", l);
  }
  int rpf = n_tokens;
  if (compress) {
    if (compress->n_centroids < 1 || compress->n_centroids > ss::kMaxCentroids)
      return fail(SS_ERR_UNSUPPORTED, "n_centroids %d outside 1..%d", compress->n_centroids,
                  ss::kMaxCentroids);
    if (compress->n_iters < 0 || compress->n_iters > 100)
      return fail(SS_ERR_INVALID_ARGUMENT, "n_iters %d outside 0..100", compress->n_iters);
    if (n_tokens > ss::kMaxTokensCompress)
      return fail(SS_ERR_UNSUPPORTED, "compression supports at most %d tokens per frame",
                  ss::kMaxTokensCompress);
    rpf = std::min(compress->n_centroids, n_tokens);
  }
  const int64_t stored = idx->n_frames - idx->frame_base;
  if (stored + n_frames > d.max_frames)
    return fail(SS_ERR_CAPACITY, "%lld stored frames + %d exceeds max_frames %lld", (long long)stored,
                n_frames, (long long)d.max_frames);
  const int64_t new_rows = (int64_t)n_frames * rpf;
  if (idx->n_rows + new_rows > d.max_rows)
    return fail(SS_ERR_CAPACITY, "%lld rows + %lld exceeds max_rows %lld", (long long)idx->n_rows,
                (long long)new_rows, (long long)d.max_rows);
  // the host offsets are reserved before anything is enqueued, so that the
  // bookkeeping after the launch cannot fail and leave the index behind the
  // device state
  // (grown by doubling: reserving each call's few frames alone would copy them all each time)
  const size_t want = idx->off.size() + (size_t)n_frames;
  if (want > idx->off.capacity()) idx->off.reserve(std::max(want, 2 * idx->off.capacity()));
  ss::AppendArgs a{};
  a.L = d.n_layers;
  a.Hk = d.n_kv_heads;
  a.D = d.head_dim;
  a.n_frames = n_frames;
  a.n_tokens = n_tokens;
  a.max_rows = d.max_rows;
  a.row0 = idx->n_rows;
  a.frame0 = stored;        // per-frame arena entries sit at id - frame_base
  a.rows_per_frame = rpf;
  a.n_centroids = compress ? compress->n_centroids : 0;
  a.n_iters = compress ? compress->n_iters : 0;
  for (int l = 0; l < d.n_layers; ++l) a.src[l] = static_cast<const uint16_t*>(layer_keys[l]);
  a.dst = idx->dev;
  hipError_t e = hipSuccess;
  if (idx->n_frames == 0)   // the key-magnitude statistic starts with the first append
    e = ss::launch_zero32(reinterpret_cast<int32_t*>(idx->dev.stats), 1, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) e = ss::launch_append(a, compress != nullptr, static_cast<hipStream_t>(stream));
  if (e == hipSuccess && layer_values) {
    ss::StoreValuesArgs v{};
    v.L = d.n_layers;
    v.Hk = d.n_kv_heads;
    v.D = d.head_dim;
    v.max_rows = d.max_rows;
    v.row0 = idx->n_rows;
    v.rows = new_rows;
    for (int l = 0; l < d.n_layers; ++l) v.src[l] = static_cast<const uint16_t*>(layer_values[l]);
    v.values = idx->values;
    v.weights = idx->weights;
    e = ss::launch_store_values(v, static_cast<hipStream_t>(stream));
  }
  if (e != hipSuccess) return fail(SS_ERR_DEVICE, "append launch failed: %s", hipGetErrorString(e));
  if (first_frame_id) *first_frame_id = idx->n_frames;
  for (int f = 1; f <= n_frames; ++f) idx->off.push_back(idx->n_rows + (int64_t)f * rpf);   // reserved
  idx->n_frames += n_frames;
  idx->n_rows += new_rows;
  idx->rpf = (idx->rpf == -1 || idx->rpf == rpf) ? rpf : 0;
  return SS_OK;
}

// Own tokens of a stream in a call (0: history alone).
int own_count(const ss_own_tokens* own, int s) { return own ? own->n_own[s] : 0; }

ss_status check_attend(ss_index* const* idx, int32_t n_streams, const int32_t* n_q, const ss_own_tokens* own,
                       const ss_attend_params* prm) {
  if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
  if (n_streams < 1) return fail(SS_ERR_INVALID_ARGUMENT, "n_streams must be >= 1");
  if (!n_q) return fail(SS_ERR_INVALID_ARGUMENT, "n_q is NULL");
  if (!prm) return fail(SS_ERR_INVALID_ARGUMENT, "params is NULL");
  if (own && (!own->n_own || !own->capacity)) return fail(SS_ERR_INVALID_ARGUMENT, "own->n_own or own->capacity is NULL");
  for (int s = 0; s < n_streams; ++s) {
    if (!idx[s]) return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] is NULL", s);
    if (!same_shape(idx[s]->desc, idx[0]->desc))
      return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] shape differs from idx[0]", s);
    if (!idx[s]->values) return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] keeps no values (ss_index_attach_values)", s);
    if (n_q[s] < 1 || n_q[s] > 4096)
      return fail(SS_ERR_INVALID_ARGUMENT, "n_q[%d] = %d outside 1..4096", s, n_q[s]);
    if (!own) continue;
    const int n = own->n_own[s];
    if (n != 0 && (n < n_q[s] || n > ss::kMaxOwn))
      return fail(SS_ERR_INVALID_ARGUMENT, "n_own[%d] = %d is neither 0 nor in n_q .. %d", s, n, ss::kMaxOwn);
    if (n != 0 && (own->capacity[s] < n || own->capacity[s] > ss::kMaxOwn))
      return fail(SS_ERR_INVALID_ARGUMENT, "capacity[%d] = %d outside n_own .. %d", s, own->capacity[s], ss::kMaxOwn);
    if (own->parents && own->parents[s]) {
      if (n == 0) return fail(SS_ERR_INVALID_ARGUMENT, "stream %d has a tree but no own tokens", s);
      if (n_q[s] > ss::kMaxTree)
        return fail(SS_ERR_UNSUPPORTED, "stream %d drafts %d tokens > %d", s, n_q[s], ss::kMaxTree);
    }
  }
  if (prm->layer < 0 || prm->layer >= idx[0]->desc.n_layers)
    return fail(SS_ERR_INVALID_ARGUMENT, "layer %d outside 0..%d", prm->layer, idx[0]->desc.n_layers - 1);
  if (!std::isfinite(prm->softcap) || prm->softcap < 0.0f)
    return fail(SS_ERR_INVALID_ARGUMENT, "softcap must be 0 (none) or positive and finite");
  if (prm->softcap > 0.0f && (prm->softcap < 1e-3f || prm->softcap > 1e6f))
    return fail(SS_ERR_UNSUPPORTED, "softcap outside 1e-3 .. 1e6");
  if (prm->frames && (prm->n_listed < 1 || prm->n_listed > ss::kMaxListed))
    return fail(SS_ERR_UNSUPPORTED, "n_listed %d outside 1..%d", prm->n_listed, ss::kMaxListed);
  if (!prm->frames && (prm->n_listed != 0 || prm->kinds))
    return fail(SS_ERR_INVALID_ARGUMENT, "n_listed or kinds without frames");
  if (!aligned(prm->frames, 8) || !aligned(prm->kinds, 4) || !aligned(prm->slopes, 4))
    return fail(SS_ERR_INVALID_ARGUMENT, "misaligned device pointer");
  return SS_OK;
}

// Launch shapes of k_attend: query columns of a block, keys of a tile.
struct AttendTile {
  int columns, keys;
};
constexpr int kAttendColumns[4] = {32, 64, 128, 256};
AttendTile attend_tile(int D, int shape) {
  return {kAttendColumns[shape], shape == 0 || (shape == 1 && D == 64) ? 128 : 64};
}
constexpr int kCus = 256;
// What a call that writes no workspace asks for, and no other call.
constexpr size_t kLeastWorkspace = 256;

// Key tiles of a stream, and its items before the key axis is shared.
int64_t key_tiles(const ss::AttendStream& st, int64_t visible, const AttendTile& tile) {
  return (visible + tile.keys - 1) / tile.keys + (st.n_own + tile.keys - 1) / tile.keys;
}
int64_t column_blocks(const ss::AttendArgs& a, const ss::AttendStream& st, const AttendTile& tile) {
  return ((int64_t)a.G * st.n_q + tile.columns - 1) / tile.columns * a.Hk;
}

// Shares of the key axis: the key tiles of an item.  A CU holds two blocks, but one by LDS of
// the narrowest tiling at d = 128, and of the widest the second does not pay (52 columns of d = 64 over 1 hour
// 149 -> 122 us, 400 over 10 minutes 90 -> 103), so items run in rounds of `slots`, and a round costs its longest item: `per`
// tiles and what starting and ending an item costs (kItemTiles).  For each number of
// rounds the smallest `per` that fits it is found, and the cheapest number taken, or no
// sharing at all where that saves the second launch (kJoinTiles).  Measured, us, one /
// two / four / eight rounds: one token over 1 hour 276 / 281 / 289 / 316, 64 tokens 691
// / 706 / 736 / 793; 1,024 tokens over 10 minutes (112 column blocks): 224 items 1,593,
// 336 items 1,996, 1,008 items 1,690.
int64_t attend_share(const ss::AttendArgs& a, int D, int shape, const int64_t* visible) {
  const AttendTile tile = attend_tile(D, shape);
  const int64_t slots = shape == 3 || (shape == 0 && D == 128) ? kCus : 2 * kCus;
  const int64_t kItemTiles = tile.keys == 128 ? 2 : 4, kJoinTiles = tile.keys == 128 ? 8 : 4;
  int64_t tiles[ss::kAttendStreams], blocks_of[ss::kAttendStreams], longest_tiles = 1, whole = 0;
  for (int i = 0; i < a.S; ++i) {
    tiles[i] = key_tiles(a.st[i], visible[i], tile);
    blocks_of[i] = column_blocks(a, a.st[i], tile);
    longest_tiles = std::max(longest_tiles, tiles[i]);
    whole += blocks_of[i];
  }
  auto items_at = [&](int64_t per) {
    int64_t n = 0;
    for (int i = 0; i < a.S; ++i) n += std::max<int64_t>(1, (tiles[i] + per - 1) / per) * blocks_of[i];
    return n;
  };
  const int64_t rounds_whole = (whole + slots - 1) / slots;
  int64_t per = longest_tiles, cost = rounds_whole * (longest_tiles + kItemTiles);
  for (int64_t r = rounds_whole; r <= rounds_whole + 7; ++r) {
    int64_t lo = 1, hi = longest_tiles;             // items_at(hi) = whole <= r slots
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (items_at(mid) <= r * slots) hi = mid;
      else lo = mid + 1;
    }
    const int64_t c = r * (lo + kItemTiles) + kJoinTiles;
    if (c < cost) {
      cost = c;
      per = lo;
    }
  }
  return per;
}

// Fills the arguments of one group of streams [s0, s0 + S); pointers into the
// workspace when `ws` is given.  Returns the group's workspace bytes.
size_t plan_attend(ss::AttendArgs& a, ss::AttendPlan& p, ss::RowsArgs& rows, ss_index* const* idx, int s0, int S,
                   const int32_t* n_q, const ss_own_tokens* own, const ss_attend_params* prm, bool accumulate,
                   void* ws) {
  const ss_index_desc& d = idx[0]->desc;
  std::memset(&a, 0, sizeof a);
  std::memset(&p, 0, sizeof p);
  std::memset(&rows, 0, sizeof rows);
  a.S = rows.S = S;
  a.Hk = d.n_kv_heads;
  a.G = d.n_q_heads / d.n_kv_heads;
  p.D = d.head_dim;
  const double scale = 1.0 / std::sqrt((double)d.head_dim), log2e = 1.4426950408889634;
  a.c1 = (float)(scale * log2e);
  if (prm->softcap > 0.0f) {
    constexpr double fit[6] = {0.999999998, -0.333332833, 0.13331689, -0.0537687049, 0.0207536292, -0.00585216861};
    constexpr double near_fit[4] = {0.9999999653, -0.3333242244, 0.1329579934, -0.04895823077};
    const double cap = (double)prm->softcap, x = scale / cap;
    a.cap.x = (float)x;
    for (int k = 0; k < 6; ++k) a.cap.fit[k] = (float)(cap * log2e * fit[k]);
    // powers of x up to the seventh have to stay in range
    a.cap.near_limit = cap <= 1e3 ? (float)(0.35 / x) : 0.0f;
    for (int k = 0; k < 4; ++k) a.cap.near_fit[k] = (float)(cap * log2e * near_fit[k] * std::pow(x, 2 * k + 1));
  }
  a.slopes = prm->slopes;
  p.listed = prm->frames != nullptr;
  rows.n_listed = prm->n_listed;
  int m_max = 0;
  for (int i = 0; i < S; ++i) m_max = std::max(m_max, a.G * n_q[s0 + i]);
  p.join_rows = m_max * a.Hk;
  int64_t visible[ss::kAttendStreams];   // most rows each stream can see
  for (int i = 0; i < S; ++i) {
    const ss_index* x = idx[s0 + i];
    const int64_t f_lo = std::min(x->first_detail, x->n_frames);
    a.st[i].n_q = n_q[s0 + i];
    a.st[i].n_own = own_count(own, s0 + i);
    visible[i] = x->n_rows - row_of(x, f_lo);
    if (!p.listed) continue;
    int64_t longest = x->rpf;
    if (x->rpf <= 0) {
      longest = 0;
      for (int64_t f = f_lo; f < x->n_frames; ++f) longest = std::max(longest, row_of(x, f + 1) - row_of(x, f));
    }
    visible[i] = std::min<int64_t>(visible[i], longest * prm->n_listed);
  }
  int64_t per = 0;                       // key tiles of an item of k_attend
  if (!accumulate) {
    // The fewest columns that hold the query rows, since every column block reads the keys
    // again.  But where an item of a wide tiling has few tiles (up to 1,024 / d of 64 keys), starting it
    // and joining the parts of its many columns cost more than reading twice: two
    // waves' columns.  Us, wide / two waves: 448 columns over 67 frames of 196 rows (7 tiles) 41 / 37, over
    // 134 (13) 48 / 52; 252 over 134 (7) 40 / 37, over 300 (15) 55 / 56; 112 over 300 (8) 42 / 40, over
    // 3,600 (87) 284 / 345; d = 64, 256 over 300 (15) 42 / 40, 100 over 3,600 (87) 182 / 188.
    p.shape = 0;
    while (p.shape < 3 && kAttendColumns[p.shape] < m_max) ++p.shape;
    per = attend_share(a, p.D, p.shape, visible);
    if (p.shape > 1 && per * p.D <= 1024) {
      p.shape = 1;
      per = attend_share(a, p.D, p.shape, visible);
    }
  }
  // A bias needs each row's frame: a quotient where all frames have the same rows, else a
  // map (one token over 1 hour 260 -> 242 us without it).  k_attend's widest tiling has only
  // the map.
  p.map = p.listed;
  for (int i = 0; i < S; ++i) p.map |= prm->slopes && (idx[s0 + i]->rpf <= 0 || (!accumulate && p.shape == 3));
  size_t off = 0;
  auto take = [&](size_t bytes) -> char* {
    off = align256(off);
    char* r = ws ? static_cast<char*>(ws) + off : nullptr;
    off += bytes;
    return r;
  };
  for (int i = 0; i < S; ++i) {
    const ss_index* x = idx[s0 + i];
    ss::AttendStream& st = a.st[i];
    const int64_t f_lo = std::min(x->first_detail, x->n_frames), r_lo = row_of(x, f_lo), n = x->n_rows - r_lo;
    const int64_t base = (int64_t)prm->layer * a.Hk * x->desc.max_rows;
    const int64_t first = p.map ? 0 : r_lo;
    st.keys = x->dev.keys + (base + first) * p.D;
    st.values = x->values + (base + first) * p.D;
    st.weights = x->weights + base + first;
    st.head_stride = x->desc.max_rows * p.D;
    st.w_stride = x->desc.max_rows;
    st.row0 = (int32_t)(p.map ? r_lo : 0);
    st.n_rows = (int32_t)n;
    st.rpf = std::max(x->rpf, 1);
    st.age0 = (int32_t)(x->n_frames - f_lo);
    if (!p.map) continue;
    const size_t one = align256((size_t)(visible[i] + 1) * 4);
    char* map = take(2 * one + 256);
    ss::RowsStream& r = rows.st[i];
    r.list = p.listed ? prm->frames + (size_t)(s0 + i) * prm->n_listed : nullptr;
    r.kinds = prm->kinds ? prm->kinds + (size_t)(s0 + i) * prm->n_listed : nullptr;
    r.frame_off = x->dev.frame_off;
    r.frame_base = x->frame_base;
    r.f_lo = f_lo;
    r.f_hi = r.n_frames = x->n_frames;
    r.row0 = (int32_t)r_lo;
    r.n_rows = (int32_t)n;
    if (map) {
      r.rowmap = reinterpret_cast<int32_t*>(map);
      r.age = reinterpret_cast<float*>(map + one);
      r.n_vis = reinterpret_cast<int32_t*>(map + 2 * one);
      st.rowmap = r.rowmap;
      st.n_vis = r.n_vis;
      st.age_off = (uint32_t)one;
    }
  }

  // Rows that one block alone reads, and that the 256 MB Infinity Cache could not hold
  // until the next call, are read past the caches: 35 columns over 1 hour 246 -> 236 us,
  // one token for each of 8 streams (1.7 GB) 290 -> 257; 64 MB in turn are served from it (52
  // columns over 10 minutes of 49 rows, d 64: 33 us, past it 37).
  {
    int64_t bytes = 0;
    for (int i = 0; i < S; ++i) bytes += visible[i] * a.Hk * p.D * (accumulate ? 2 : 4);
    a.once = bytes > (int64_t)256 << 20 && m_max <= kAttendColumns[accumulate ? 2 : std::min(p.shape, 2)];
  }

  if (accumulate) {
    // A wave takes 32 keys at a time, every wave the same number of turns.  Few query
    // rows (bound by reading the keys): several short blocks for each that a CU holds, which
    // end evenly (8 / 16 / 32 / 64 a CU: 113 / 113 / 114 / 127 us for one token over 1
    // hour).  More rows: one round of the two blocks that a CU holds with 256 rows staged.
    p.shape = m_max <= 32 ? 0 : 1;
    const int64_t waves = p.shape == 0 ? 4 : 8, slots = (p.shape == 0 ? 16 : 2) * kCus;
    int64_t groups = 0;
    for (int i = 0; i < S; ++i) groups += (visible[i] + 31) / 32 * a.Hk;
    const int64_t turns = std::max<int64_t>(1, (groups + slots * waves - 1) / (slots * waves));
    int64_t blocks = 0;
    for (int i = 0; i < S; ++i) {
      ss::AttendStream& st = a.st[i];
      st.n_split = (int32_t)std::max<int64_t>(1, ((visible[i] + 31) / 32 + turns * waves - 1) / (turns * waves));
      blocks += st.n_split * a.Hk;
    }
    // Few keys and many query rows: the query rows are shared out as far as that fills
    // the round, at least 64 a share (983 tokens of 16 heads over 5,000 rows: 710 us
    // with one share).
    int64_t parts = 0;
    for (int i = 0; i < S; ++i) {
      ss::AttendStream& st = a.st[i];
      st.q_split = p.shape == 0 ? 1 : (int32_t)std::max<int64_t>(1, std::min(slots / blocks, (int64_t)a.G * st.n_q / 64));
      st.item0 = p.items;
      p.items += st.n_split * a.Hk * st.q_split;
      st.part0 = parts;
      if (st.q_split > 1) {
        parts += st.q_split * a.Hk * visible[i];
        p.add_rows = std::max(p.add_rows, a.Hk * visible[i]);
      }
    }
    a.part_o = reinterpret_cast<float*>(take((size_t)parts * 4));
    // up to 64 sums would fit the least workspace, which stands for one that is not written
    return off > 0 ? std::max(align256(off), 2 * kLeastWorkspace) : 0;
  }

  int64_t parts = 0;
  for (int i = 0; i < S; ++i) {
    ss::AttendStream& st = a.st[i];
    const int64_t M = (int64_t)a.G * st.n_q, tiles = key_tiles(st, visible[i], attend_tile(p.D, p.shape));
    st.n_split = (int32_t)std::max<int64_t>(1, (tiles + per - 1) / per);
    st.item0 = p.items;
    p.items += (int)(st.n_split * column_blocks(a, st, attend_tile(p.D, p.shape)));
    st.part0 = parts;
    p.join_parts = std::max(p.join_parts, st.n_split);
    if (st.n_split > 1) parts += st.n_split * M * a.Hk;
  }
  a.part_o = reinterpret_cast<float*>(take((size_t)parts * p.D * 4));
  a.part_ml = reinterpret_cast<float*>(take((size_t)parts * 8));
  return align256(off);
}

size_t attend_ws(ss_index* const* idx, int32_t n_streams, const int32_t* n_q, const ss_own_tokens* own,
                 const ss_attend_params* prm, bool accumulate) {
  size_t need = kLeastWorkspace;
  for (int s0 = 0; s0 < n_streams; s0 += ss::kAttendStreams) {
    ss::AttendArgs a;
    ss::AttendPlan p;
    ss::RowsArgs r;
    need = std::max(need, plan_attend(a, p, r, idx, s0, std::min(ss::kAttendStreams, n_streams - s0), n_q, own, prm,
                                      accumulate, nullptr));
  }
  return need;
}

}  // namespace

struct ss_clusters {
  ss_cluster_desc desc;
  ss::ClusterDev dev;
};

extern "C" {

size_t ss_clusters_required_bytes(const ss_cluster_desc* desc) {
  return cluster_desc_ok(desc) ? cluster_layout(*desc).total : 0;
}

ss_status ss_clusters_create(const ss_cluster_desc* desc, void* dev_arena, size_t arena_bytes, void* stream,
                             ss_clusters** out) {
  return guarded([&]() -> ss_status {
    if (!out) return fail(SS_ERR_INVALID_ARGUMENT, "out is NULL");
    if (!cluster_desc_ok(desc)) return fail(SS_ERR_INVALID_ARGUMENT, "invalid cluster description");
    if (!dev_arena || !aligned(dev_arena, 256)) return fail(SS_ERR_INVALID_ARGUMENT, "arena NULL or not 256-byte aligned");
    const ClusterLayout L = cluster_layout(*desc);
    if (arena_bytes < L.total) return fail(SS_ERR_CAPACITY, "arena %zu bytes, %zu needed", arena_bytes, L.total);
    ss_clusters* c = new (std::nothrow) ss_clusters;
    if (!c) return fail(SS_ERR_INTERNAL, "out of host memory");
    c->desc = *desc;
    char* b = static_cast<char*>(dev_arena);
    c->dev.state = reinterpret_cast<int32_t*>(b + L.state);
    c->dev.centroids = reinterpret_cast<float*>(b + L.centroids);
    c->dev.sizes = reinterpret_cast<int32_t*>(b + L.sizes);
    c->dev.span = reinterpret_cast<int64_t*>(b + L.span);
    c->dev.reps = reinterpret_cast<float*>(b + L.reps);
    const hipError_t e = ss::launch_zero32(c->dev.state, 4, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) {
      delete c;
      return fail(SS_ERR_DEVICE, "cluster state reset: %s", hipGetErrorString(e));
    }
    *out = c;
    return SS_OK;
  });
}

ss_status ss_clusters_destroy(ss_clusters* cl) {
  return guarded([&]() -> ss_status {
    delete cl;
    return SS_OK;
  });
}

size_t ss_clusters_absorb_workspace_bytes(int64_t n_frames) {
  return n_frames < 0 ? 0 : std::max<size_t>(256, ((size_t)n_frames * 8 + 255) & ~(size_t)255);
}

ss_status ss_clusters_absorb(ss_clusters* cl, ss_index* idx, int64_t frame_hi, void* ws, size_t ws_bytes,
                             void* stream) {
  return guarded([&]() -> ss_status {
    if (!cl || !idx) return fail(SS_ERR_INVALID_ARGUMENT, "cluster set or index is NULL");
    const ss_cluster_desc& c = cl->desc;
    const ss_index_desc& d = idx->desc;
    if (c.n_layers != d.n_layers || c.n_kv_heads != d.n_kv_heads || c.head_dim != d.head_dim)
      return fail(SS_ERR_INVALID_ARGUMENT, "cluster set and index shapes differ");
    const int64_t f_lo = idx->first_detail;
    // (an eviction may have left an index whose recent window reaches before f_lo)
    const int64_t f_end = std::max(f_lo, idx->n_frames - (int64_t)d.n_recent);
    if (frame_hi < f_lo || frame_hi > f_end)
      return fail(SS_ERR_INVALID_ARGUMENT, "frame_hi %lld outside %lld..%lld (frames leave in order, never from the recent window)",
                  (long long)frame_hi, (long long)f_lo, (long long)f_end);
    for (int64_t f = f_lo; f < frame_hi; ++f)
      if (row_of(idx, f + 1) - row_of(idx, f) != c.rows_per_unit)
        return fail(SS_ERR_INVALID_ARGUMENT, "frame %lld stores %lld rows, the cluster set takes %d", (long long)f,
                    (long long)(row_of(idx, f + 1) - row_of(idx, f)), c.rows_per_unit);
    const int64_t n = frame_hi - f_lo;
    if (n > 0x7FFFFFFF) return fail(SS_ERR_UNSUPPORTED, "too many frames in one call");
    if (n > 0 && (!ws || !aligned(ws, 256) || ws_bytes < ss_clusters_absorb_workspace_bytes(n)))
      return fail(SS_ERR_WORKSPACE, "absorb workspace NULL, misaligned or below %zu bytes",
                  ss_clusters_absorb_workspace_bytes(n));
    ss::AbsorbArgs a{};
    a.L = c.n_layers; a.Hk = c.n_kv_heads; a.D = c.head_dim; a.R = c.rows_per_unit;
    a.max_clusters = c.max_clusters; a.max_rows = d.max_rows; a.tau = c.tau;
    a.f_lo = f_lo; a.n_units = (int)n; a.row_lo = row_of(idx, f_lo);
    a.desc = idx->dev.desc + (f_lo - idx->frame_base) * (int64_t)d.n_kv_heads * d.head_dim;
    a.keys = idx->dev.keys;
    a.assign = static_cast<int32_t*>(ws);
    a.cl = cl->dev;
    const hipError_t e = ss::launch_absorb(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "absorb launch failed: %s", hipGetErrorString(e));
    idx->first_detail = frame_hi;
    return SS_OK;
  });
}

size_t ss_clusters_retrieve_workspace_bytes(const ss_clusters* cl) {
  if (!cl) return 0;
  ss::ClusterQueryPlan p{};
  p.Hk = cl->desc.n_kv_heads; p.D = cl->desc.head_dim; p.max_clusters = cl->desc.max_clusters;
  return ss::cluster_query_workspace(p, nullptr);
}

ss_status ss_clusters_retrieve(const ss_clusters* cl, const ss_index* idx, const void* const* queries,
                               int32_t n_q, int32_t k_clusters, void* ws, size_t ws_bytes, void* stream,
                               int64_t* cluster_ids, float* scores, int64_t* first_frame,
                               int64_t* last_frame, int32_t* n_out) {
  return guarded([&]() -> ss_status {
    if (!cl || !idx) return fail(SS_ERR_INVALID_ARGUMENT, "cluster set or index is NULL");
    const ss_index_desc& d = idx->desc;
    if (cl->desc.n_layers != d.n_layers || cl->desc.n_kv_heads != d.n_kv_heads || cl->desc.head_dim != d.head_dim)
      return fail(SS_ERR_INVALID_ARGUMENT, "cluster set and index shapes differ");
    if (n_q < 1 || n_q > 4096) return fail(SS_ERR_INVALID_ARGUMENT, "n_q %d outside 1..4096", n_q);
    if (k_clusters < 1 || k_clusters > ss::kMaxSelect)
      return fail(SS_ERR_UNSUPPORTED, "k_clusters %d outside 1..%d", k_clusters, ss::kMaxSelect);
    if (!queries || !queries[d.n_layers - 1]) return fail(SS_ERR_INVALID_ARGUMENT, "last-layer queries are NULL");
    if (!aligned(queries[d.n_layers - 1], 16)) return fail(SS_ERR_INVALID_ARGUMENT, "queries not 16-byte aligned");
    if (!cluster_ids || !scores || !first_frame || !last_frame || !n_out)
      return fail(SS_ERR_INVALID_ARGUMENT, "an output pointer is NULL");
    ss::ClusterQueryPlan p{};
    p.L = d.n_layers; p.Hq = d.n_q_heads; p.Hk = d.n_kv_heads; p.G = p.Hq / p.Hk; p.D = d.head_dim;
    p.nq = n_q; p.k = k_clusters; p.max_clusters = cl->desc.max_clusters;
    p.q_last = static_cast<const uint16_t*>(queries[d.n_layers - 1]);
    p.cl = cl->dev;
    const size_t need = ss::cluster_query_workspace(p, nullptr);
    if (!ws || !aligned(ws, 256) || ws_bytes < need)
      return fail(SS_ERR_WORKSPACE, "cluster retrieval workspace NULL, misaligned or below %zu bytes", need);
    ss::cluster_query_workspace(p, ws);
    p.out_ids = cluster_ids; p.out_scores = scores; p.out_first = first_frame; p.out_last = last_frame;
    p.out_n = n_out;
    const hipError_t e = ss::launch_cluster_query(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "cluster retrieval launch failed: %s", hipGetErrorString(e));
    return SS_OK;
  });
}

ss_status ss_clusters_export(const ss_clusters* cl, int32_t* state, float* centroids, int32_t* sizes,
                             int64_t* span, float* reps, void* stream) {
  return guarded([&]() -> ss_status {
    if (!cl) return fail(SS_ERR_INVALID_ARGUMENT, "cluster set is NULL");
    const ss_cluster_desc& c = cl->desc;
    const size_t M = (size_t)c.max_clusters, dim = (size_t)c.n_kv_heads * c.head_dim;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    struct Part { void* dst; const void* src; size_t bytes; } parts[] = {
        {state, cl->dev.state, 8},
        {centroids, cl->dev.centroids, M * dim * 4},
        {sizes, cl->dev.sizes, M * 4},
        {span, cl->dev.span, M * 16},
        {reps, cl->dev.reps, M * c.n_layers * dim * c.rows_per_unit * 4}};
    for (const Part& q : parts) {
      if (!q.dst) continue;
      const hipError_t e = hipMemcpyAsync(q.dst, q.src, q.bytes, hipMemcpyDeviceToDevice, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "cluster export: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

size_t ss_pooled_workspace_bytes(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                                  int32_t n_select) {
  if (check_pooled(idx, n_streams, n_q, n_select) != SS_OK) return 0;
  return pooled_ws(idx, n_streams, n_q, n_select);
}

ss_status ss_retrieve_pooled(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                             const int32_t* n_q, int32_t n_select, void* ws, size_t ws_bytes,
                             void* stream, int64_t* frame_ids, float* scores, int32_t* n_out) {
  return guarded([&]() -> ss_status {
    ss_status st = check_pooled(idx, n_streams, n_q, n_select);
    if (st) return st;
    if (!queries) return fail(SS_ERR_INVALID_ARGUMENT, "queries is NULL");
    const int L = idx[0]->desc.n_layers;
    for (int i = 0; i < n_streams * L; ++i) {
      if (!queries[i]) return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] is NULL", i);
      if (!aligned(queries[i], 16)) return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] not 16-byte aligned", i);
    }
    if (!frame_ids || !scores || !n_out) return fail(SS_ERR_INVALID_ARGUMENT, "an output pointer is NULL");
    if (!ws || !aligned(ws, 256)) return fail(SS_ERR_WORKSPACE, "workspace NULL or not 256-byte aligned");
    const size_t need = pooled_ws(idx, n_streams, n_q, n_select);
    if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    for (int s0 = 0; s0 < n_streams; s0 += ss::kMaxStreams) {
      ss::PooledPlan p;
      build_pooled(p, idx, s0, std::min(ss::kMaxStreams, n_streams - s0), queries, n_q, n_select);
      ss::pooled_workspace(p, ws);
      p.out_ids = frame_ids + (size_t)s0 * n_select;
      p.out_scores = scores + (size_t)s0 * n_select;
      p.out_n = n_out + s0;
      const hipError_t e = ss::launch_pooled(p, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "pooled ranking launch failed: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

int32_t ss_evidence_max_units(const ss_evidence_params* params, int32_t n_select, int32_t k_clusters) {
  const int64_t n = evidence_units_max(params, n_select, k_clusters);
  return (n < 0 || n > ss::kMaxEvidence) ? 0 : (int32_t)std::max<int64_t>(n, 1);
}

ss_status ss_assemble_evidence(ss_index* const* idx, int32_t n_streams, const int64_t* frame_ids,
                               int32_t n_select, const ss_evidence_clusters* clusters,
                               const ss_evidence_params* params, void* stream, int64_t* units, int32_t* kinds,
                               int32_t* n_units, int32_t max_units) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (n_streams < 1) return fail(SS_ERR_INVALID_ARGUMENT, "n_streams must be >= 1");
    for (int s = 0; s < n_streams; ++s)
      if (!idx[s]) return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] is NULL", s);
    const int kc = clusters ? clusters->k_clusters : 0;
    if (clusters && (kc < 1 || kc > ss::kMaxSelect))
      return fail(SS_ERR_UNSUPPORTED, "k_clusters %d outside 1..%d", kc, ss::kMaxSelect);
    const int64_t need = evidence_units_max(params, n_select, kc);
    if (need < 0) return fail(SS_ERR_INVALID_ARGUMENT, "invalid evidence parameters");
    if (need > ss::kMaxEvidence)
      return fail(SS_ERR_UNSUPPORTED, "%lld candidate items per stream > %d", (long long)need, ss::kMaxEvidence);
    if (max_units < std::max<int64_t>(need, 1) || max_units > ss::kMaxEvidence)
      return fail(SS_ERR_INVALID_ARGUMENT, "max_units %d outside %lld..%d", max_units,
                  (long long)std::max<int64_t>(need, 1), ss::kMaxEvidence);
    if (params->retrieved && !frame_ids) return fail(SS_ERR_INVALID_ARGUMENT, "frame_ids is NULL");
    if (!units || !n_units) return fail(SS_ERR_INVALID_ARGUMENT, "an output pointer is NULL");
    if (clusters && !kinds) return fail(SS_ERR_INVALID_ARGUMENT, "kinds is NULL (needed with clusters)");
    if (!aligned(units, 8) || !aligned(n_units, 4) || (kinds && !aligned(kinds, 4)) ||
        (frame_ids && !aligned(frame_ids, 8)))
      return fail(SS_ERR_INVALID_ARGUMENT, "misaligned device pointer");
    if (clusters) {
      if (!clusters->sets) return fail(SS_ERR_INVALID_ARGUMENT, "clusters->sets is NULL");
      if (params->retrieved && !clusters->cluster_ids)
        return fail(SS_ERR_INVALID_ARGUMENT, "clusters->cluster_ids is NULL");
      if (clusters->cluster_ids && !aligned(clusters->cluster_ids, 8))
        return fail(SS_ERR_INVALID_ARGUMENT, "misaligned device pointer");
      for (int s = 0; s < n_streams; ++s) {
        const ss_clusters* c = clusters->sets[s];
        if (c && (c->desc.n_layers != idx[s]->desc.n_layers || c->desc.n_kv_heads != idx[s]->desc.n_kv_heads ||
                  c->desc.head_dim != idx[s]->desc.head_dim))
          return fail(SS_ERR_INVALID_ARGUMENT, "cluster set %d and index %d shapes differ", s, s);
      }
    }
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    for (int s0 = 0; s0 < n_streams; s0 += ss::kMaxStreams) {
      ss::EvidenceArgs a{};
      a.S = std::min(ss::kMaxStreams, n_streams - s0);
      a.n_select = params->retrieved ? n_select : 0;
      a.n_recent = params->n_recent;
      a.n_before = params->n_before;
      a.n_after = params->n_after;
      a.retrieved = params->retrieved;
      a.max_units = max_units;
      for (int s = 0; s < a.S; ++s) {
        const ss_index* x = idx[s0 + s];
        a.T[s] = x->n_frames;
        a.lo[s] = std::min(x->first_detail, x->n_frames);
      }
      a.frame_ids = params->retrieved ? frame_ids + (size_t)s0 * n_select : nullptr;
      if (clusters && params->retrieved) {
        a.k_clusters = kc;
        a.cluster_ids = clusters->cluster_ids + (size_t)s0 * kc;
        for (int s = 0; s < a.S; ++s) {
          const ss_clusters* c = clusters->sets[s0 + s];
          a.cl_span[s] = c ? c->dev.span : nullptr;
          a.cl_count[s] = c ? c->dev.state : nullptr;
        }
      }
      a.units = units + (size_t)s0 * max_units;
      a.kinds = kinds ? kinds + (size_t)s0 * max_units : nullptr;
      a.n_units = n_units + s0;
      const hipError_t e = ss::launch_evidence(a, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "evidence launch failed: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

size_t ss_index_required_bytes(const ss_index_desc* desc) {
  if (check_desc(desc) != SS_OK) return 0;
  return layout(*desc).total;
}

ss_status ss_index_create(const ss_index_desc* desc, void* dev_arena, size_t arena_bytes,
                          ss_index** out) {
  return guarded([&]() -> ss_status {
    if (!out) return fail(SS_ERR_INVALID_ARGUMENT, "out is NULL");
    ss_status st = check_desc(desc);
    if (st) return st;
    if (!dev_arena) return fail(SS_ERR_INVALID_ARGUMENT, "arena is NULL");
    if (!aligned(dev_arena, 256)) return fail(SS_ERR_INVALID_ARGUMENT, "arena not 256-byte aligned");
    const Layout L = layout(*desc);
    if (arena_bytes < L.total)
      return fail(SS_ERR_CAPACITY, "arena %zu bytes, %zu needed", arena_bytes, L.total);
    ss_index* x = new (std::nothrow) ss_index();
    if (!x) return fail(SS_ERR_INTERNAL, "out of host memory");
    x->desc = *desc;
    x->arena = dev_arena;
    x->arena_bytes = arena_bytes;
    char* b = static_cast<char*>(dev_arena);
    x->dev.keys = reinterpret_cast<uint16_t*>(b + L.keys);
    x->dev.counts = reinterpret_cast<int32_t*>(b + L.counts);
    x->dev.desc = reinterpret_cast<float*>(b + L.desc);
    x->dev.pooled = reinterpret_cast<float*>(b + L.pooled);
    x->dev.stats = reinterpret_cast<uint32_t*>(b + L.stats);
    x->dev.frame_off = reinterpret_cast<int32_t*>(b + L.off);
    x->n_frames = 0;
    x->n_rows = 0;
    x->off.assign(1, 0);
    x->rpf = -1;
    *out = x;
    return SS_OK;
  });
}

ss_status ss_index_destroy(ss_index* idx) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    delete idx;
    return SS_OK;
  });
}

ss_status ss_index_info(const ss_index* idx, int64_t* n_frames, int64_t* n_rows) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (n_frames) *n_frames = idx->n_frames;
    if (n_rows) *n_rows = idx->n_rows;
    return SS_OK;
  });
}

ss_status ss_index_window(const ss_index* idx, int64_t* first_stored, int64_t* first_detail) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (first_stored) *first_stored = idx->frame_base;
    if (first_detail) *first_detail = idx->first_detail;
    return SS_OK;
  });
}

ss_status ss_index_compact(ss_index* idx, void* stream) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    const int64_t fs = idx->first_detail - idx->frame_base;
    if (fs <= 0) return SS_OK;
    const int64_t rs = row_of(idx, idx->first_detail);
    // the new host offsets first, so that nothing after the launch can fail
    std::vector<int64_t> off(idx->off.begin() + fs, idx->off.end());
    for (int64_t& v : off) v -= rs;
    ss::CompactArgs a{};
    const ss_index_desc& d = idx->desc;
    a.dev = idx->dev;
    a.L = d.n_layers; a.Hk = d.n_kv_heads; a.D = d.head_dim; a.max_rows = d.max_rows;
    a.row_shift = rs;
    a.keep_rows = idx->n_rows - rs;
    a.frame_shift = fs;
    a.keep_frames = idx->n_frames - idx->first_detail;
    hipError_t e = ss::launch_compact(a, static_cast<hipStream_t>(stream));
    if (e == hipSuccess && idx->values)
      e = ss::launch_move_values({a.L * a.Hk, a.D, a.max_rows, a.row_shift, a.keep_rows, idx->values, idx->weights},
                                 static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "compaction launch failed: %s", hipGetErrorString(e));
    idx->off.swap(off);
    idx->frame_base = idx->first_detail;
    idx->n_rows = a.keep_rows;
    return SS_OK;
  });
}

ss_status ss_index_budget_split(const ss_index* idx, uint64_t budget_bytes, int64_t* frame_hi) {
  return guarded([&]() -> ss_status {
    if (!idx || !frame_hi) return fail(SS_ERR_INVALID_ARGUMENT, "idx or frame_hi is NULL");
    const ss_index_desc& d = idx->desc;
    const uint64_t L = (uint64_t)d.n_layers, Hk = (uint64_t)d.n_kv_heads, D = (uint64_t)d.head_dim;
    const uint64_t row_bytes = (idx->values ? 2 : 1) * (2 * D + 4);
    auto bytes = [&](int64_t f) {
      const uint64_t rows = (uint64_t)(row_of(idx, f + 1) - row_of(idx, f));
      return rows * L * Hk * row_bytes + (Hk * D + L * Hk * D) * 4 + 4;
    };
    const int64_t T = idx->n_frames, lo = idx->first_detail;
    const int64_t hi = std::max(lo, T - (int64_t)d.n_recent);   // the recent window stays detailed
    uint64_t mem = 0;
    for (int64_t f = lo; f < T; ++f) mem += bytes(f);
    int64_t h = lo;
    while (h < hi && mem > budget_bytes) mem -= bytes(h++);
    *frame_hi = h;
    return SS_OK;
  });
}

ss_status ss_index_append(ss_index* idx, const void* const* layer_keys, int32_t n_frames,
                          int32_t n_tokens, const ss_compress* compress, void* stream,
                          int64_t* first_frame_id) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (idx->values)
      return fail(SS_ERR_INVALID_ARGUMENT, "the index keeps values: append through ss_index_append_kv");
    return append_common(idx, layer_keys, nullptr, n_frames, n_tokens, compress, stream, first_frame_id);
  });
}

size_t ss_values_required_bytes(const ss_index_desc* desc) {
  if (check_desc(desc) != SS_OK) return 0;
  return values_layout(*desc).total;
}

ss_status ss_index_attach_values(ss_index* idx, void* dev_arena, size_t arena_bytes) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (idx->values) return fail(SS_ERR_INVALID_ARGUMENT, "the index keeps values already");
    if (idx->n_frames != 0) return fail(SS_ERR_INVALID_ARGUMENT, "values can only be attached to an empty index");
    if (!dev_arena || !aligned(dev_arena, 256))
      return fail(SS_ERR_INVALID_ARGUMENT, "arena NULL or not 256-byte aligned");
    const ValuesLayout v = values_layout(idx->desc);
    if (arena_bytes < v.total) return fail(SS_ERR_CAPACITY, "arena %zu bytes, %zu needed", arena_bytes, v.total);
    idx->values = static_cast<uint16_t*>(dev_arena);
    idx->weights = reinterpret_cast<float*>(static_cast<char*>(dev_arena) + v.weights);
    idx->values_bytes = v.total;
    return SS_OK;
  });
}

ss_status ss_index_append_kv(ss_index* idx, const void* const* layer_keys, const void* const* layer_values,
                             int32_t n_frames, int32_t n_tokens, void* stream, int64_t* first_frame_id) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    if (!idx->values) return fail(SS_ERR_INVALID_ARGUMENT, "the index keeps no values (ss_index_attach_values)");
    if (!layer_values) return fail(SS_ERR_INVALID_ARGUMENT, "layer_values is NULL");
    return append_common(idx, layer_keys, layer_values, n_frames, n_tokens, nullptr, stream, first_frame_id);
  });
}

size_t ss_attend_workspace_bytes(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                                 const ss_own_tokens* own, const ss_attend_params* params) {
  if (check_attend(idx, n_streams, n_q, own, params) != SS_OK) return 0;
  return attend_ws(idx, n_streams, n_q, own, params, false);
}

ss_status ss_attend(ss_index* const* idx, int32_t n_streams, const void* const* queries, const int32_t* n_q,
                    const ss_own_tokens* own, const ss_attend_params* params, void* ws, size_t ws_bytes,
                    void* stream, void* const* out, float* const* lse) {
  return guarded([&]() -> ss_status {
    const ss_status st = check_attend(idx, n_streams, n_q, own, params);
    if (st) return st;
    if (!queries || !out) return fail(SS_ERR_INVALID_ARGUMENT, "queries or out is NULL");
    for (int s = 0; s < n_streams; ++s) {
      if (!queries[s] || !aligned(queries[s], 16))
        return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] NULL or not 16-byte aligned", s);
      if (!out[s] || !aligned(out[s], 16))
        return fail(SS_ERR_INVALID_ARGUMENT, "out[%d] NULL or not 16-byte aligned", s);
      if (lse && (!lse[s] || !aligned(lse[s], 4)))
        return fail(SS_ERR_INVALID_ARGUMENT, "lse[%d] NULL or misaligned", s);
      for (int t = 0; t < n_streams; ++t)
        if (out[s] == queries[t]) return fail(SS_ERR_INVALID_ARGUMENT, "out[%d] is queries[%d]", s, t);
      for (int t = 0; t < s; ++t)
        if (out[s] == out[t] || (lse && lse[s] == lse[t]))
          return fail(SS_ERR_INVALID_ARGUMENT, "streams %d and %d have one output", t, s);
      if (own_count(own, s) == 0) continue;
      if (!own->keys || !own->values || !own->keys[s] || !own->values[s] || !aligned(own->keys[s], 16) ||
          !aligned(own->values[s], 16))
        return fail(SS_ERR_INVALID_ARGUMENT, "own keys or values of stream %d NULL or not 16-byte aligned", s);
      if (own->parents && !aligned(own->parents[s], 4))
        return fail(SS_ERR_INVALID_ARGUMENT, "parents[%d] misaligned", s);
    }
    if (!ws || !aligned(ws, 256)) return fail(SS_ERR_WORKSPACE, "workspace NULL or not 256-byte aligned");
    // a batch of one group is sized by the plan it runs; of more, every group before the first is enqueued
    size_t need = n_streams > ss::kAttendStreams ? attend_ws(idx, n_streams, n_q, own, params, false) : 0;
    if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    for (int s0 = 0; s0 < n_streams; s0 += ss::kAttendStreams) {
      ss::AttendArgs a;
      ss::AttendPlan p;
      ss::RowsArgs r;
      need = std::max(kLeastWorkspace, plan_attend(a, p, r, idx, s0, std::min(ss::kAttendStreams, n_streams - s0), n_q, own,
                                               params, false, ws));
      if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
      for (int i = 0; i < a.S; ++i) {
        ss::AttendStream& t = a.st[i];
        const int s = s0 + i;
        t.q = static_cast<const uint16_t*>(queries[s]);
        t.out = static_cast<uint16_t*>(out[s]);
        t.lse = lse ? lse[s] : nullptr;
        if (t.n_own == 0) continue;
        t.own_k = static_cast<const uint16_t*>(own->keys[s]);
        t.own_v = static_cast<const uint16_t*>(own->values[s]);
        t.own_cap = own->capacity[s];
        t.parents = own->parents ? own->parents[s] : nullptr;
      }
      hipError_t e = p.map ? ss::launch_rows(r, hs) : hipSuccess;
      if (e == hipSuccess) e = ss::launch_attend(a, p, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "attention launch failed: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

size_t ss_attend_accumulate_workspace_bytes(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                                            const ss_attend_params* params) {
  if (check_attend(idx, n_streams, n_q, nullptr, params) != SS_OK) return 0;
  return attend_ws(idx, n_streams, n_q, nullptr, params, true);
}

ss_status ss_attend_accumulate(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                               const int32_t* n_q, const float* const* lse, const ss_attend_params* params,
                               float decay, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> ss_status {
    const ss_status st = check_attend(idx, n_streams, n_q, nullptr, params);
    if (st) return st;
    if (!(decay >= 0.0f && decay <= 1.0f)) return fail(SS_ERR_INVALID_ARGUMENT, "decay outside 0..1");
    if (!queries || !lse) return fail(SS_ERR_INVALID_ARGUMENT, "queries or lse is NULL");
    for (int s = 0; s < n_streams; ++s) {
      if (!queries[s] || !aligned(queries[s], 16))
        return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] NULL or not 16-byte aligned", s);
      if (!lse[s] || !aligned(lse[s], 4)) return fail(SS_ERR_INVALID_ARGUMENT, "lse[%d] NULL or misaligned", s);
      for (int t = 0; t < s; ++t)
        if (idx[t] == idx[s])
          return fail(SS_ERR_INVALID_ARGUMENT, "idx[%d] and idx[%d] are one index: their weights would be added at once",
                      t, s);
    }
    if (!ws || !aligned(ws, 256)) return fail(SS_ERR_WORKSPACE, "workspace NULL or not 256-byte aligned");
    size_t need = n_streams > ss::kAttendStreams ? attend_ws(idx, n_streams, n_q, nullptr, params, true) : 0;
    if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    for (int s0 = 0; s0 < n_streams; s0 += ss::kAttendStreams) {
      ss::AttendArgs a;
      ss::AttendPlan p;
      ss::RowsArgs r;
      need = std::max(kLeastWorkspace, plan_attend(a, p, r, idx, s0, std::min(ss::kAttendStreams, n_streams - s0), n_q,
                                               nullptr, params, true, ws));
      if (ws_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", ws_bytes, need);
      for (int i = 0; i < a.S; ++i) {
        a.st[i].q = static_cast<const uint16_t*>(queries[s0 + i]);
        a.st[i].lse = const_cast<float*>(lse[s0 + i]);   // read only
      }
      hipError_t e = p.map ? ss::launch_rows(r, hs) : hipSuccess;
      if (e == hipSuccess) e = ss::launch_accumulate(a, p, decay, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "weight accumulation launch failed: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

ss_status ss_index_evict(const ss_index* src, ss_index* dst, int64_t frame_hi, int32_t keep_rows, void* stream) {
  return guarded([&]() -> ss_status {
    if (!src || !dst) return fail(SS_ERR_INVALID_ARGUMENT, "src or dst is NULL");
    if (src == dst) return fail(SS_ERR_INVALID_ARGUMENT, "src and dst are one index");
    const ss_index_desc &d = src->desc, &e = dst->desc;
    if (!same_shape(d, e)) return fail(SS_ERR_INVALID_ARGUMENT, "src and dst shapes differ");
    if (!src->values || !dst->values)
      return fail(SS_ERR_INVALID_ARGUMENT, "src or dst keeps no values (ss_index_attach_values)");
    auto overlap = [](const void* a, size_t an, const void* b, size_t bn) {
      const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
      return x < y + bn && y < x + an;
    };
    if (overlap(src->arena, layout(d).total, dst->arena, layout(e).total) ||
        overlap(src->arena, layout(d).total, dst->values, dst->values_bytes) ||
        overlap(src->values, src->values_bytes, dst->arena, layout(e).total) ||
        overlap(src->values, src->values_bytes, dst->values, dst->values_bytes))
      return fail(SS_ERR_INVALID_ARGUMENT, "the arenas of src and dst overlap");
    if (keep_rows < 1) return fail(SS_ERR_INVALID_ARGUMENT, "keep_rows must be >= 1");
    const int64_t f_lo = src->first_detail, f_end = std::max(f_lo, src->n_frames - (int64_t)d.n_recent);
    if (frame_hi < f_lo || frame_hi > f_end)
      return fail(SS_ERR_INVALID_ARGUMENT, "frame_hi %lld outside %lld..%lld (the recent window stays whole)",
                  (long long)frame_hi, (long long)f_lo, (long long)f_end);
    const int64_t frames = src->n_frames - f_lo;
    if (frames > e.max_frames)
      return fail(SS_ERR_CAPACITY, "%lld frames exceed dst's max_frames %lld", (long long)frames, (long long)e.max_frames);
    std::vector<int64_t> off((size_t)frames + 1, 0);
    int32_t rpf = -1;
    for (int64_t i = 0; i < frames; ++i) {
      int64_t n = row_of(src, f_lo + i + 1) - row_of(src, f_lo + i);
      if (f_lo + i < frame_hi) n = std::min<int64_t>(n, keep_rows);
      off[(size_t)i + 1] = off[(size_t)i] + n;
      rpf = (rpf == -1 || rpf == (int32_t)n) ? (int32_t)n : 0;
    }
    if (off.back() > e.max_rows)
      return fail(SS_ERR_CAPACITY, "%lld rows exceed dst's max_rows %lld", (long long)off.back(), (long long)e.max_rows);
    ss::EvictArgs a{};
    a.L = d.n_layers;
    a.Hk = d.n_kv_heads;
    a.D = d.head_dim;
    a.n_frames = frames;
    a.n_thin = frame_hi - f_lo;
    a.keep = keep_rows;
    a.rpf = src->rpf > 0 ? src->rpf : 0;
    a.src_row0 = row_of(src, f_lo);
    a.src_max_rows = d.max_rows;
    a.dst_max_rows = e.max_rows;
    a.src = src->dev;
    const int64_t f0 = f_lo - src->frame_base;
    a.src.frame_off += f0;
    a.src.desc += f0 * d.n_kv_heads * d.head_dim;
    a.src.pooled += f0 * d.n_layers * d.n_kv_heads * d.head_dim;
    a.dst = dst->dev;
    a.src_values = src->values;
    a.dst_values = dst->values;
    a.src_weights = src->weights;
    a.dst_weights = dst->weights;
    const hipError_t he = ss::launch_evict(a, static_cast<hipStream_t>(stream));
    if (he != hipSuccess) return fail(SS_ERR_DEVICE, "eviction launch failed: %s", hipGetErrorString(he));
    dst->n_frames = src->n_frames;
    dst->frame_base = dst->first_detail = f_lo;
    dst->n_rows = off.back();
    dst->off.swap(off);
    dst->rpf = rpf;
    return SS_OK;
  });
}

size_t ss_retrieve_workspace_bytes(ss_index* const* idx, int32_t n_streams, const int32_t* n_q,
                                   const ss_retrieve_params* params) {
  if (check_batch(idx, n_streams, n_q, params) != SS_OK) return 0;
  return batch_ws(idx, n_streams, n_q, params, false);
}

ss_status ss_retrieve(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                      const int32_t* n_q, const ss_retrieve_params* params, void* ws,
                      size_t ws_bytes, void* stream, int64_t* frame_ids, int32_t* votes,
                      float* mass, int32_t* n_out) {
  return guarded([&]() -> ss_status {
    return retrieve_common(idx, n_streams, queries, n_q, params, ws, ws_bytes, stream, frame_ids,
                           votes, mass, n_out, nullptr);
  });
}

ss_status ss_retrieve_noalloc(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                              const int32_t* n_q, const ss_retrieve_params* params, void* stream,
                              int64_t* frame_ids, int32_t* votes, float* mass, int32_t* n_out) {
  return guarded([&]() -> ss_status {
    ss_status st = check_batch(idx, n_streams, n_q, params);
    if (st) return st;
    const size_t need = batch_ws(idx, n_streams, n_q, params, true);
    if (need > ss::kNoAllocBytes)
      return fail(SS_ERR_WORKSPACE,
                  "this batch needs a %zu-byte workspace, above the %zu bytes of the library-owned one: "
                  "call ss_retrieve with a caller workspace, or split the batch",
                  need, ss::kNoAllocBytes);
    void* ws = nullptr;
    const hipError_t e = ss::noalloc_workspace(&ws);
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "library workspace lookup failed: %s", hipGetErrorString(e));
    return retrieve_common(idx, n_streams, queries, n_q, params, ws, ss::kNoAllocBytes, stream, frame_ids,
                           votes, mass, n_out, nullptr);
  });
}

ss_status ss_retrieve_debug(ss_index* const* idx, int32_t n_streams, const void* const* queries,
                            const int32_t* n_q, const ss_retrieve_params* params, void* ws,
                            size_t ws_bytes, void* stream, int64_t* frame_ids, int32_t* votes,
                            float* mass, int32_t* n_out, const ss_debug_out* dbg) {
  return guarded([&]() -> ss_status {
    if (!dbg) return fail(SS_ERR_INVALID_ARGUMENT, "dbg is NULL");
    return retrieve_common(idx, n_streams, queries, n_q, params, ws, ws_bytes, stream, frame_ids,
                           votes, mass, n_out, dbg);
  });
}

size_t ss_debug_scores_workspace_bytes(const ss_index* idx) {
  if (!idx) return 0;
  const ss_index_desc& d = idx->desc;
  return align256((size_t)d.n_layers * d.n_kv_heads * 2 * (d.head_dim / 32) * 64 * 16);
}

ss_status ss_debug_scores(const ss_index* idx, const void* const* queries, int32_t n_q,
                          int32_t layer, int32_t q_head, int32_t head_mode, int64_t row0,
                          int64_t n_rows, float* out, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    const ss_index_desc& d = idx->desc;
    if (!queries) return fail(SS_ERR_INVALID_ARGUMENT, "queries is NULL");
    for (int l = 0; l < d.n_layers; ++l)
      if (!queries[l] || !aligned(queries[l], 16))
        return fail(SS_ERR_INVALID_ARGUMENT, "queries[%d] NULL or not 16-byte aligned", l);
    if (n_q < 1 || n_q > 4096) return fail(SS_ERR_INVALID_ARGUMENT, "n_q %d outside 1..4096", n_q);
    if (head_mode != 0 && head_mode != 1) return fail(SS_ERR_INVALID_ARGUMENT, "head_mode must be 0 or 1");
    if (head_mode == 1 && d.n_kv_heads > 8)
      return fail(SS_ERR_UNSUPPORTED, "head_mode 1 supports at most 8 KV heads");
    if (layer < 0 || layer >= d.n_layers) return fail(SS_ERR_INVALID_ARGUMENT, "layer out of range");
    if (head_mode == 0 && (q_head < 0 || q_head >= d.n_q_heads))
      return fail(SS_ERR_INVALID_ARGUMENT, "q_head out of range");
    if (row0 < 0 || n_rows < 0 || row0 + n_rows > idx->n_rows)
      return fail(SS_ERR_INVALID_ARGUMENT, "rows [%lld, %lld) outside the %lld stored rows",
                  (long long)row0, (long long)(row0 + n_rows), (long long)idx->n_rows);
    if (!out && n_rows > 0) return fail(SS_ERR_INVALID_ARGUMENT, "out is NULL");
    if (!ws || !aligned(ws, 256) || ws_bytes < ss_debug_scores_workspace_bytes(idx))
      return fail(SS_ERR_WORKSPACE, "debug-scores workspace too small or misaligned");
    ss::RetrievePlan p;
    std::memset(&p, 0, sizeof p);
    p.S = 1;
    p.L = d.n_layers;
    p.Hq = d.n_q_heads;
    p.Hk = d.n_kv_heads;
    p.G = p.Hq / p.Hk;
    p.D = d.head_dim;
    p.head_mode = head_mode;
    p.NL = head_mode == 0 ? p.L * p.Hq : p.L;
    p.ncol = head_mode == 0 ? p.G : 1;
    p.ngs = head_mode == 0 ? p.Hk : 1;
    p.chunk_rows = kChunkRows;
    p.qB = static_cast<uint32_t*>(ws);
    ss::StreamPlan& sp = p.st[0];
    sp.keys = idx->dev.keys;
    sp.row_stride = (int32_t)d.max_rows;
    sp.nq = n_q;
    double sc = 1.0 / ((double)n_q * std::sqrt((double)p.D));
    if (head_mode == 1) sc /= (double)p.Hq;
    sp.qscale = (float)sc;
    for (int l = 0; l < p.L; ++l) sp.q[l] = static_cast<const uint16_t*>(queries[l]);
    const hipError_t e =
        ss::launch_debug_scores(p, layer, q_head, row0, n_rows, out, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(SS_ERR_DEVICE, "debug scores launch failed: %s", hipGetErrorString(e));
    return SS_OK;
  });
}

ss_status ss_index_export(const ss_index* idx, void* rows_dev, int32_t* counts_dev, float* desc_dev,
                          int64_t* frame_offsets_host, void* stream) {
  return guarded([&]() -> ss_status {
    if (!idx) return fail(SS_ERR_INVALID_ARGUMENT, "idx is NULL");
    const ss_index_desc& d = idx->desc;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const size_t lg = (size_t)d.n_layers * d.n_kv_heads;
    if (frame_offsets_host)
      std::memcpy(frame_offsets_host, idx->off.data(), idx->off.size() * sizeof(int64_t));
    if (idx->n_rows > 0 && rows_dev) {
      const size_t rb = (size_t)idx->n_rows * d.head_dim * 2;
      const hipError_t e = hipMemcpy2DAsync(rows_dev, rb, idx->dev.keys, (size_t)d.max_rows * d.head_dim * 2,
                                            rb, lg, hipMemcpyDeviceToDevice, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "export rows: %s", hipGetErrorString(e));
    }
    if (idx->n_rows > 0 && counts_dev) {
      const size_t rb = (size_t)idx->n_rows * 4;
      const hipError_t e = hipMemcpy2DAsync(counts_dev, rb, idx->dev.counts, (size_t)d.max_rows * 4, rb, lg,
                                            hipMemcpyDeviceToDevice, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "export counts: %s", hipGetErrorString(e));
    }
    const int64_t stored = idx->n_frames - idx->frame_base;
    if (stored > 0 && desc_dev) {
      const hipError_t e = hipMemcpyAsync(desc_dev, idx->dev.desc,
                                          (size_t)stored * d.n_kv_heads * d.head_dim * 4,
                                          hipMemcpyDeviceToDevice, hs);
      if (e != hipSuccess) return fail(SS_ERR_DEVICE, "export descriptors: %s", hipGetErrorString(e));
    }
    return SS_OK;
  });
}

ss_status ss_debug_sample_plan(int64_t n_rows, int32_t top_k, int32_t* out) {
  return guarded([&]() -> ss_status {
    if (!out) return fail(SS_ERR_INVALID_ARGUMENT, "out is NULL");
    if (n_rows < 0 || n_rows > (int64_t)0x7FFFFFFF - 1)
      return fail(SS_ERR_INVALID_ARGUMENT, "n_rows %lld outside 0..2^31-2", (long long)n_rows);
    if (top_k < 1 || top_k > ss::kMaxTopK)
      return fail(SS_ERR_UNSUPPORTED, "top_k %d outside 1..%d", top_k, ss::kMaxTopK);
    const StreamSizes z = plan_stream(n_rows, 0, top_k);
    out[0] = z.m;
    out[1] = z.r;
    out[2] = (int32_t)candidate_cap(top_k, n_rows);
    out[3] = z.kk > 0 ? (int32_t)expected_candidates(n_rows, z.kk) : 0;
    return SS_OK;
  });
}

ss_status ss_set_profile_events(void* ev_start, void* ev_stop) {
  return guarded([&]() -> ss_status {
    if ((ev_start == nullptr) != (ev_stop == nullptr))
      return fail(SS_ERR_INVALID_ARGUMENT, "give both events or neither");
    g_ev_start = static_cast<hipEvent_t>(ev_start);
    g_ev_stop = static_cast<hipEvent_t>(ev_stop);
    return SS_OK;
  });
}

const char* ss_status_string(ss_status s) {
  switch (s) {
    case SS_OK: return "ok";
    case SS_ERR_INVALID_ARGUMENT: return "invalid argument";
    case SS_ERR_UNSUPPORTED: return "unsupported";
    case SS_ERR_CAPACITY: return "capacity exceeded";
    case SS_ERR_WORKSPACE: return "workspace too small";
    case SS_ERR_DEVICE: return "device error";
    case SS_ERR_INTERNAL: return "internal error";
    default: return "unknown status";
  }
}

const char* ss_last_error(void) { return g_err; }

int32_t ss_version(void) { return 1; }

}  // extern "C"
