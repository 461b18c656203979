// Internal declarations of the paged cache: its C-ABI layer (ss_paged_api.cpp) and
// its gfx950 kernels (ss_paged.hip).  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ss {

constexpr int kBlockTokens = 32;      // tokens of a page
constexpr int kPagedStreams = 512;    // streams of a call
constexpr int kPagedTokens = 1 << 16; // new tokens (queries) of a call
constexpr int kPagedUnits = 1536;     // units of a KV head that are cut into shares (more are not)
constexpr int kPagedWidth = (1 << 26) - 2;   // pages of a stream: tokens, up to the end of its open block, in 31 bits

// Which tokens of a call are a stream's.  Kernels of small calls take the one or the other: 2 KB more of
// arguments cost a launch some 0.4 us.
struct EvenSpans {
  int uniform;                        // tokens of every stream
};
struct Spans {
  int uniform;                        // 0: by start
  int start[kPagedStreams + 1];
};

// One layer of a cache, and where each stream's rows lie.
struct PagedDev {
  uint8_t *k8, *v8;                   // [n_pages][H_kv][32 d] e4m3
  float *ks, *vs;                     // [n_pages][H_kv]
  uint16_t *ok, *ov;                  // [n_slots][2][H_kv][32 d] bf16
  const int32_t *tables, *lengths, *slots;
  int width, n_slots, n_pages, Hk;
};

// Rows [heads][tokens][d]: elements from one head and from one token to the next.
struct RowsView {
  const uint16_t* p;
  int64_t hs, ts;
};

struct Turn {
  const double* freqs;                // turns a position, [dims / 2]
  const int64_t* positions;           // one a token of the call, or null
  int dims, interleaved;              // dims 0: no rotation
  float gain, sign;
};

struct RotateArgs {
  RowsView x, out;
  Turn turn;
  int heads, N;
};
hipError_t launch_rotate(const RotateArgs& a, int D, hipStream_t st);

struct PagedAppendArgs {
  PagedDev c;
  RowsView k, v, q, q_out;            // q.p null: no queries
  Turn turn;
  int Hq, S, items;                   // items: blocks that the new tokens can touch, of all streams
};
hipError_t launch_paged_append(const PagedAppendArgs& a, const Spans& spans, int D, hipStream_t st);

struct PagedAttendArgs {
  PagedDev c;
  RowsView q, out, prior;             // prior.p null: none
  const float* prior_lse;
  float* lse;
  float* part_o;                      // partial sums [2 blocks][cols][d] and their (maximum, sum)
  float* part_ml;
  int* plan;                          // share, units' work before each
  int G, S, N, window;
  float c1;                           // log2(e) / sqrt(d)
  int units, per, cols;               // units of a KV head; of a stream (0: ragged); columns kept of a unit
  int n_wg, min_share;                // blocks; 0: a block a unit, nothing to join
  int start;                          // work that beginning a unit counts as
};
struct PagedAttendPlan {
  int bm, round;                      // columns of a unit, blocks that its work is counted in
  int units, per, cols, n_wg, min_share, start;
  size_t o_bytes, ml_bytes, plan_bytes;
};
hipError_t launch_paged_attend(const PagedAttendArgs& a, const Spans& spans, const PagedAttendPlan& p, int D,
                               hipStream_t st);

}  // namespace ss

// Records an entry point's failure as the last one of this thread; returns `st`.
int32_t ss_fail_text(int32_t st, const char* text);
