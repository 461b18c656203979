// gfx950 (MI355X) kernels of attention over the stored history: the rows a call
// sees (k_rows), attention for questions and drafted trees (k_attend, k_join),
// the weight that it gives each row (k_accumulate), the value cache's append
// (k_store_values) and eviction by weight (k_evict).
//
// Attention reads keys and values row-major from the arena, in one pass with the
// running maximum and sum of a softmax.  All matrix products are 32x32x16 bf16
// MFMAs with fp32 accumulation:
//   S^T = K Q^T   A: 32 keys, B: 32 query columns, chained over d;
//   O^T = V^T P^T A: 32 dimensions, B: the same 32 columns, chained over keys.
// A query is a column of both, so its maximum, sum and rescaling live in the two
// lanes that hold that column, and P^T's B operand is S^T's own registers rounded
// to bf16: register r of lane half h holds key 8 (r / 4) + 4 h + r % 4, and the
// k order of the second product is free as long as A uses it too.  V^T's A
// operand is read from the row-major tile by the transposing LDS read, four keys
// of one dimension at a time, which is that same order.
// P is rounded to bf16 for the second product (its sum is taken before): a
// rounding of at most 2^-8 of each term, like the rounding of the values
// themselves; maxima, sums and the output stay fp32 until the one rounding at
// the end.
#include "ss_internal.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace ss {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#define SS_LDS __attribute__((address_space(3)))

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}

// The other half's value of the same column.
__device__ __forceinline__ float other_half(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// One wave's direct load from global memory to LDS, 16 or 4 bytes a lane: lane l's
// piece lands at lds + 16 l (4 l).  Written as asm because the compiler makes every
// later LDS read wait for all such loads; the waits are counted by hand below.  No
// register but m0 is written, and the caller waits before the pieces are read.
// (base and lds are the same in every lane; readfirstlane keeps them in scalar registers.)
__device__ __forceinline__ const void* in_scalar(const void* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return reinterpret_cast<const void*>((uint64_t)hi << 32 | lo);
}
// ONCE: not kept in the caches.
template <bool ONCE>
__device__ __forceinline__ void load_lds16(const void* base, uint32_t off, uint32_t lds) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(
                     __builtin_amdgcn_readfirstlane(lds)),
                 "v"(off), "s"(in_scalar(base))
                 : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
                 "v"(off), "s"(in_scalar(base))
                 : "m0", "memory");
}
__device__ __forceinline__ void load_lds4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
               "v"(off), "s"(in_scalar(base))
               : "m0", "memory");
}
// At most N of this wave's loads are still under way, and its LDS reads are done;
// with BAR all waves of the block have come this far.
template <int N, bool BAR>
__device__ __forceinline__ void wait_loads() {
  if constexpr (BAR)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// tanh through exp; below 1 by the continued fraction x / (1 + x^2 / (3 + x^2 / (5 +
// ...))) cut after 11 (off by less than 2^-31 there), which keeps small scores' relative
// precision.
__device__ __forceinline__ float tanh_any(float x) {
  const float y = x * x;
  const float p = fmaf(y, fmaf(y, 21.0f, 1260.0f), 10395.0f);
  const float q = fmaf(y, fmaf(y, y + 210.0f, 4725.0f), 10395.0f);
  const float e = exp2_fast(fabsf(x) * (-2.0f * kLog2e));
  const float t = (1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e);
  return fabsf(x) < 1.0f ? x * p * __builtin_amdgcn_rcpf(q) : copysignf(t, x);
}
// v[i] <- cap tanh(v[i] x) in units of log 2, x = scale / cap: by polynomials of least
// maximum error in z^2, z = v x, for tanh(z) / z: of degree 3 where all of a wave's |z|
// are below 0.35 (off by 2^-24.7 at most), of degree 5 below 0.6 (2^-28.3).  Scores far
// below their cap are the usual case.
template <int N>
__device__ __forceinline__ float top_of(const float (&v)[N]) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]));
  return top;
}
template <int N>
__device__ __forceinline__ bool near_cap(const float (&v)[N], const CapArgs& a) {
  return !__any(!(top_of(v) < a.near_limit));
}
__device__ __forceinline__ float near_factor(float v, const CapArgs& a) {
  const float y = v * v;
  return fmaf(y, fmaf(y, fmaf(y, a.near_fit[3], a.near_fit[2]), a.near_fit[1]), a.near_fit[0]);
}
template <int N>
__device__ __forceinline__ void cap_scores(float (&v)[N], const CapArgs& a) {
  if (near_cap(v, a)) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= near_factor(v[i], a);
  } else if (!__any(!(top_of(v) * a.x < 0.6f))) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = v[i] * a.x, y = z * z;
      v[i] = z * fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, a.fit[5], a.fit[4]), a.fit[3]), a.fit[2]), a.fit[1]), a.fit[0]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = a.fit[0] * tanh_any(v[i] * a.x);
  }
}

// ---------------------------------------------------------------------------
// k_rows: the rows that a call sees, when they are not simply the detailed ones.
// With a list of frames: the listed frames of the detailed window, each once, in
// temporal order, their rows laid end to end; without (a bias over frames of several
// sizes needs the rows' ages): every detailed row.  rowmap[j] is the j-th row's place in the arena run,
// age[j] the frames from it to the end of the stream.
// Each block of a list orders it anew (up to 512 entries by comparing all pairs, up to
// 4,096 by sorting in LDS) and writes its share of the frames, so one launch does; a
// wave writes a frame.  Bound by three dependent trips to memory: 70 listed frames of
// 196 rows take about 7 us.
// ---------------------------------------------------------------------------
constexpr int kRowsThreads = 512;

__global__ __launch_bounds__(kRowsThreads) void k_rows(RowsArgs a) {
  const RowsStream& st = a.st[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int kWaves = kRowsThreads / 64;
  if (a.n_listed == 0) {
    for (int64_t f = st.f_lo + blockIdx.x * kWaves + wave; f < st.f_hi; f += (int64_t)gridDim.x * kWaves) {
      const int r0 = st.frame_off[f - st.frame_base], r1 = st.frame_off[f + 1 - st.frame_base];
      const float age = (float)(st.n_frames - f);
      for (int r = r0 + lane; r < r1; r += 64) {
        st.rowmap[r - st.row0] = r;
        st.age[r - st.row0] = age;
      }
    }
    if (blockIdx.x == 0 && tid == 0) st.n_vis[0] = st.n_rows;
    return;
  }
  __shared__ __align__(16) int ids[kMaxListed];   // stored frame of each entry; no frame: INT_MAX
  __shared__ __align__(16) int pre[kMaxListed];   // its rows, or the rows before it
  __shared__ int part[kWaves];
  int P2 = 1;
  while (P2 < a.n_listed) P2 <<= 1;
  auto entry = [&](int i) -> int {
    if (i >= a.n_listed || (st.kinds && st.kinds[i] != 0)) return 0x7FFFFFFF;
    const int64_t f = st.list[i];
    return f >= st.f_lo && f < st.f_hi ? (int)(f - st.frame_base) : 0x7FFFFFFF;
  };
  if (P2 <= kRowsThreads) {
    // a thread an entry: an earlier entry of the same frame takes its rows away, and the
    // rows before it are those of all smaller frames; no sorting
    __shared__ int first_row[kRowsThreads], place[kRowsThreads];
    const int f = entry(tid);
    int r0 = 0, n = 0;
    if (f != 0x7FFFFFFF) {
      r0 = st.frame_off[f];
      n = st.frame_off[f + 1] - r0;
    }
    ids[tid] = f;
    __syncthreads();
    const int4* ids4 = reinterpret_cast<const int4*>(ids);
    const int4* pre4 = reinterpret_cast<const int4*>(pre);
    const int quads = (a.n_listed + 3) / 4;          // entries behind the last have no frame and no rows
    bool again = false;
#pragma unroll 4
    for (int j = 0; j < quads; ++j) {
      const int4 x = ids4[j];
      again |= (x.x == f & 4 * j < tid) | (x.y == f & 4 * j + 1 < tid) | (x.z == f & 4 * j + 2 < tid) |
               (x.w == f & 4 * j + 3 < tid);
    }
    if (again) n = 0;
    pre[tid] = n;
    first_row[tid] = r0;
    __syncthreads();
    int before = 0;
#pragma unroll 4
    for (int j = 0; j < quads; ++j) {
      const int4 x = ids4[j], y = pre4[j];
      before += (x.x < f ? y.x : 0) + (x.y < f ? y.y : 0) + (x.z < f ? y.z : 0) + (x.w < f ? y.w : 0);
    }
    place[tid] = before;
    int all = before + n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) all = max(all, __shfl_xor(all, d));
    if (lane == 0) part[wave] = all;
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
#pragma unroll
      for (int w = 1; w < kWaves; ++w) all = max(all, part[w]);
      st.n_vis[0] = all;
    }
    for (int i = blockIdx.x * kWaves + wave; i < a.n_listed; i += gridDim.x * kWaves) {
      const float age = (float)(st.n_frames - (ids[i] + st.frame_base));
      for (int r = lane; r < pre[i]; r += 64) {
        st.rowmap[place[i] + r] = first_row[i] + r;
        st.age[place[i] + r] = age;
      }
    }
    return;
  }
  for (int i = tid; i < P2; i += kRowsThreads) ids[i] = entry(i);
  for (int k = 2; k <= P2; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int i = tid; i < P2; i += kRowsThreads) {
        const int o = i ^ j;
        if (o > i) {
          const int x = ids[i], y = ids[o];
          if ((x > y) == ((i & k) == 0)) {
            ids[i] = y;
            ids[o] = x;
          }
        }
      }
    }
  __syncthreads();
  // rows before each distinct frame: a run of entries per thread, then the threads' sums
  const int run = (P2 + kRowsThreads - 1) / kRowsThreads;
  auto rows_of = [&](int i) -> int {
    const int f = ids[i];
    if (f == 0x7FFFFFFF || (i > 0 && ids[i - 1] == f)) return 0;
    return st.frame_off[f + 1] - st.frame_off[f];
  };
  int sum = 0;
  for (int i = tid * run; i < min(P2, (tid + 1) * run); ++i) sum += rows_of(i);
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  int at = upto - sum, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) at += part[w];
    all += part[w];
  }
  for (int i = tid * run; i < min(P2, (tid + 1) * run); ++i) {
    pre[i] = at;
    at += rows_of(i);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) st.n_vis[0] = all;
  for (int i = blockIdx.x * kWaves + wave; i < P2; i += gridDim.x * kWaves) {
    const int n = rows_of(i);
    if (n == 0) continue;
    const int r0 = st.frame_off[ids[i]], j0 = pre[i];
    const float age = (float)(st.n_frames - (ids[i] + st.frame_base));
    for (int r = lane; r < n; r += 64) {
      st.rowmap[j0 + r] = r0 + r;
      st.age[j0 + r] = age;
    }
  }
}

// ---------------------------------------------------------------------------
// Where the 16-byte pieces of a staged row lie: piece p of row r at p ^ swizzle(r), so
// that the lanes that read LDS in one clock (256 bytes) meet different banks: 16
// rows at one piece for the keys, four rows at four pieces for the values.
template <int D>
__device__ __forceinline__ int key_swizzle(int r) {
  return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int value_swizzle(int r) {
  return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
}

// k_attend<D, WQ, WK, BN, NS, MAP>: one item = (stream, KV head, block of 32 WQ
// query columns, share of the key tiles).  WQ waves along the columns x WK along
// the keys; a tile of BN keys and values is staged in LDS, up to NS tiles at a time.
// The M = G n_q query rows of a KV head are one run of memory, so column c is
// token c % n_q of head c / n_q.  The tiles of a stream are those of its visible
// rows and then those of the question's own tokens.
// MAP: rows come through rowmap, with their ages; without, row j is row j, and a bias
// takes its age from the frames' one size.
//
// What bounds it.  Few columns: reading keys and values (one token over 705,600 rows of 4
// KV heads, d 128: 219 to 240 us, 6.0 to 6.6 TB/s; WQ = 1: each wave loads what it reads, no
// barriers).
// Many columns: the matrix unit and the power that the card may draw under it (1,024 tokens of 28 heads over
// 117,600 rows: 1.44 to 1.54 ms, 1.1 to 1.2 PFLOP/s by card; a block's tile of 64 keys x 256 columns takes
// 3,200 clocks, 2,048 of them matrix work: it is busy for 62% of the clocks, a large library product for 70%, both
// at 1.6 to 1.75 GHz).
// Between, blocks of four waves, two a CU: one's softmax runs beside the other's products and
// loads (56 columns over 705,600 rows, 4 KV heads, d 128: 251 us with one block of eight, 224; 112
// columns 303 -> 284; at d 64 one block of eight waves and tiles of 128 keys keep up to 64 columns: 125 us, 140).
// 32 columns a wave keep O^T, the queries, a tile's scores and two steps of LDS reads in
// 200 registers, so that two waves fit a SIMD and can take turns.
template <int D, int WQ, int WK, int BN, int NS, bool MAP>
struct AttendShape {
  static constexpr int NW = WQ * WK, BM = 32 * WQ, RB = D * 2, CH = D / 8, RPI = 64 / CH;
  static constexpr int NI = BN * RB / 1024 / NW;      // 1 KB loads of keys (of values) per wave and tile
  static constexpr int SUB = BN / (32 * WK);          // 32-key groups per wave and tile
  static constexpr bool BAR = WQ > 1;                 // waves share tiles; with WQ = 1 each loads what it reads
  static constexpr int KB = BN * RB;                  // bytes of a key tile
  static constexpr int NG = BN / 32;
  static constexpr int META = MAP ? 8 * NG * 256 : 0; // ring of row places and ages
  static constexpr int ANC = (kMaxTree / 32) * BM * 4;
  static constexpr int MERGE = WK > 1 ? WQ * (WK - 1) * (32 * (D + 4) + 64) * 4 : 0;
  static constexpr int RING = 2 * NS * KB;
  static constexpr int LDS = (RING > MERGE ? RING : MERGE) + META + ANC;
  static constexpr int NL = 2 * NI + (MAP ? 1 : 0);   // loads a wave issues for a tile
  static_assert(NI >= 1 && NI * 1024 * NW == BN * RB && SUB >= 1 && NG <= NW && LDS <= 160 * 1024);
  static_assert(NS == 2 || (NS == 4 && NW == 8));
};

template <int D, int WQ, int WK, int BN, int NS, bool MAP>
__global__ __launch_bounds__(64 * WQ * WK, 2) void k_attend(AttendArgs a) {
  using T = AttendShape<D, WQ, WK, BN, NS, MAP>;
  constexpr int NW = T::NW, BM = T::BM, RB = T::RB, CH = T::CH, RPI = T::RPI, NI = T::NI, SUB = T::SUB, NL = T::NL;
  constexpr int KST = D / 16, DT = D / 32;
  constexpr bool PP = NS == 4;                          // two groups of waves take turns
  constexpr int MERGE_AT = (T::RING > T::MERGE ? T::RING : T::MERGE);
  __shared__ __align__(1024) unsigned char smem[T::LDS];
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(SS_LDS unsigned char*)smem);
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wq = wave % WQ, wk = wave / WQ;

  // the item: consecutive ones share keys (column blocks fastest) and stay on one XCD
  int item = blockIdx.x;
  {
    const int n = gridDim.x, per = n / 8;
    if (item < per * 8) item = (item & 7) * per + (item >> 3);
  }
  int s = 0;
  while (s + 1 < a.S && item >= a.st[s + 1].item0) ++s;
  const AttendStream& st = a.st[s];
  const int M = a.G * st.n_q, mbs = (M + BM - 1) / BM;
  item -= st.item0;
  const int mb = item % mbs;
  item /= mbs;
  const int split = item % st.n_split, hk = item / st.n_split;

  const int n_vis = MAP ? __builtin_amdgcn_readfirstlane(*st.n_vis) : st.n_rows;
  const int Th = (n_vis + BN - 1) / BN;
  // own tiles: up to the last token that a column of this block sees
  const int c_lo = mb * BM, c_hi = min(M, c_lo + BM) - 1;
  const int i_lo = c_lo % st.n_q;
  const int i_hi = (i_lo + (c_hi - c_lo) >= st.n_q) ? st.n_q - 1 : i_lo + (c_hi - c_lo);
  const int own_end = st.n_own > 0 ? st.n_own - st.n_q + i_hi + 1 : 0;
  const int Tt = Th + (own_end + BN - 1) / BN;
  // this item's tiles: split, split + n_split, ...; the items of a KV head, side by side in
  // time, so read one dense window of it.  t below counts them.
  constexpr int t0 = 0;
  const int t1 = split < Tt ? (Tt - split + st.n_split - 1) / st.n_split : 0;

  const unsigned char* kh = reinterpret_cast<const unsigned char*>(st.keys + hk * st.head_stride);
  const unsigned char* vh = reinterpret_cast<const unsigned char*>(st.values + hk * st.head_stride);
  const unsigned char* ko = reinterpret_cast<const unsigned char*>(st.own_k + (int64_t)hk * st.own_cap * D);
  const unsigned char* vo = reinterpret_cast<const unsigned char*>(st.own_v + (int64_t)hk * st.own_cap * D);

  // arguments that the loop needs, kept in registers (they would be read again behind every barrier)
  auto keep = [](auto x) {
    asm volatile("" : "+v"(x));
    if constexpr (sizeof(x) == 4) return (decltype(x))__builtin_amdgcn_readfirstlane((int)x);
    else return (decltype(x))in_scalar(x);
  };
  const int n_own = keep(st.n_own), draft0 = keep(st.n_own - st.n_q);   // own tokens before draft0 are seen by every query
  // and those before own_full by every column of this block
  const int own_full = keep(st.parents ? st.n_own - st.n_q : st.n_own - st.n_q + (i_lo + (c_hi - c_lo) >= st.n_q ? 0 : i_lo) + 1);
  const int32_t* rowmap = keep(st.rowmap);
  const uint32_t age_off = keep(st.age_off);
  const int n_split = keep(st.n_split);
  const int rpf = keep(st.rpf), age0 = keep(st.age0);
  const bool once = keep((int)a.once) != 0;
  auto tile_of = [&](int t) { return split + t * n_split; };

  // this lane's query column (behind the last one: that one again, not written)
  const int c = c_lo + wq * 32 + c32, cc = min(c, M - 1);
  const int qi = cc % st.n_q;
  const float slope2 = a.slopes ? a.slopes[hk * a.G + cc / st.n_q] * kLog2e : 0.0f;
  u32x4 qf[KST];
  {
    const uint16_t* q = st.q + ((int64_t)hk * M + cc) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < KST; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }

  // ancestors of the drafted tokens of this block's columns, bit e of word w: draft 32 w + e
  uint32_t* anc = reinterpret_cast<uint32_t*>(smem + MERGE_AT + T::META);
  const bool tree = st.parents != nullptr;
  if (tree && t1 > 0 && tile_of(t1 - 1) >= Th) {
    int* par = reinterpret_cast<int*>(smem);          // before the ring is used
    for (int i = tid; i < st.n_q; i += 64 * NW) par[i] = st.parents[i];
    const int words = (st.n_q + 31) / 32;
    for (int i = tid; i < words * BM; i += 64 * NW) anc[i] = 0;
    __syncthreads();
    if (tid < BM) {
      int i = min(c_lo + tid, M - 1) % st.n_q;
      while (i >= 0) {                                 // parents lie before their children: at most n_q steps
        anc[(i >> 5) * BM + tid] |= 1u << (i & 31);
        const int p = par[i];
        i = p < i ? p : -1;
      }
    }
    __syncthreads();
  }

  f32x16 O[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) O[i] = f32x16{};
  float m = neg_inf(), l = 0.0f;

  auto meta_at = [&](int t, int g) -> uint32_t { return (uint32_t)(MERGE_AT + ((t & 7) * T::NG + g) * 256); };
  auto load_meta = [&](int t) {
    const int g = wave % T::NG;
    const int j = max(0, min(tile_of(t) * BN + g * 32 + c32, n_vis - 1));
    // lanes 0..31 the rows' places, 32..63 their ages
    const uint32_t off = (uint32_t)j * 4u + (half ? age_off : 0u);
    load_lds4(rowmap, off, lds0 + meta_at(t, g));
  };
  auto issue = [&](int t) {
    const int tile = tile_of(t);
    const bool hist = tile < Th;
    const unsigned char* kb = hist ? kh : ko;
    const unsigned char* vb = hist ? vh : vo;
    const int n = hist ? n_vis : n_own, j0 = (hist ? tile : tile - Th) * BN;
    const uint32_t buf = lds0 + (uint32_t)((t - t0) % NS) * 2u * T::KB;
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      const int idx = wave * NI + k, r = idx * RPI + lane / CH, pos = lane % CH;
      int j = min(j0 + r, n - 1);
      if (MAP && hist) j = *reinterpret_cast<const int*>(smem + meta_at(t, r >> 5) + (r & 31) * 4);
      const uint32_t row = (uint32_t)j * RB;
      const uint32_t ko_ = row + ((pos ^ key_swizzle<D>(r)) << 4), vo_ = row + ((pos ^ value_swizzle<D>(r)) << 4);
      if (WQ < 8 && once) {
        load_lds16<true>(kb, ko_, buf + idx * 1024);
        load_lds16<true>(vb, vo_, buf + T::KB + idx * 1024);
      } else {
        load_lds16<false>(kb, ko_, buf + idx * 1024);
        load_lds16<false>(vb, vo_, buf + T::KB + idx * 1024);
      }
    }
    if (MAP) load_meta(t + 2);
  };

  // LDS places of this lane's operands in the first buffer; rows 32 apart, and 8 apart
  // for the values, have the same swizzle and differ by constants
  const int kr = wk * 32 + c32;
  uint32_t k_at[KST];
#pragma unroll
  for (int i = 0; i < KST; ++i) k_at[i] = lds0 + kr * RB + (((2 * i + half) ^ key_swizzle<D>(kr)) << 4);
  // dimensions 32 dt + c32, keys 16 w + 8 x + 4 half + 0..3 of a group
  const int vr = wk * 32 + 4 * half + ((lane & 15) >> 2), vd = 16 * (c32 >> 4) + (lane & 3) * 4;
  uint32_t v_at[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
    v_at[i] = lds0 + T::KB + vr * RB + ((((32 * i + vd) >> 3) ^ value_swizzle<D>(vr)) << 4) + (vd & 7) * 2;

  u32x4 pb[SUB * 2];      // p as the second product's B operand
  f32x16 S[SUB];
  // Both products run in steps of up to four fragments (16 bytes a lane each), the next
  // step's read from LDS while this one's are multiplied: 128 clocks of the matrix unit
  // cover the reads' latency.  Without that order the compiler waits for each read.
  constexpr int VS = SUB * 2, VF = DT;                       // steps and fragments of the second product
  constexpr int KF = KST * SUB < 4 ? KST * SUB : 4, KS = KST * SUB / KF;   // and of the first
  constexpr int FR = VF > KF ? VF : KF;
  u32x4 fr[2][FR];
  uint32_t kb_at[KST], vb_at[DT];
  auto key_buffer = [&](int t) {
    const uint32_t buf = (uint32_t)((t - t0) % NS) * 2u * T::KB;
#pragma unroll
    for (int i = 0; i < KST; ++i) {
      kb_at[i] = k_at[i] + buf;
      asm("" : "+v"(kb_at[i]));            // one address, the groups by constant offsets
    }
  };
  auto value_buffer = [&](int t) {
    const uint32_t buf = (uint32_t)((t - t0) % NS) * 2u * T::KB;
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      vb_at[i] = v_at[i] + buf;
      asm("" : "+v"(vb_at[i]));
    }
  };
  auto read_keys = [&](int step, u32x4 (&f)[FR]) {
#pragma unroll
    for (int x = 0; x < KF; ++x) {
      const int n = step * KF + x, i = n / SUB, u = n % SUB;
      f[x] = *((const SS_LDS u32x4*)(uintptr_t)kb_at[i] + u * WK * 32 * RB / 16);
    }
  };
  auto multiply_keys = [&](int step, const u32x4 (&f)[FR]) {
#pragma unroll
    for (int x = 0; x < KF; ++x) {
      const int n = step * KF + x, i = n / SUB, u = n % SUB;
      S[u] = mfma32(f[x], qf[i], i == 0 ? f32x16{} : S[u]);
    }
  };
  auto read_values = [&](int step, u32x4 (&f)[FR]) {
    const int u = step >> 1, w = step & 1;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (SS_LDS s16x4*)(uintptr_t)vb_at[dt] + (u * WK * 32 + 16 * w + 8 * x) * RB / 8));
        f[dt][2 * x] = y[0];
        f[dt][2 * x + 1] = y[1];
      }
  };
  auto multiply_values = [&](int step, const u32x4 (&f)[FR]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] = mfma32(f[dt], pb[step], O[dt]);
  };
  // S^T of a tile whose first step is in fr[first]
  auto scores_from = [&](int first) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (k + 1 < KS) read_keys(k + 1, fr[(first + k + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
      multiply_keys(k, fr[(first + k) & 1]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // O^T += V^T P^T with the first step in fr[0]; more(k) goes with step k
  auto values_from = [&](auto&& more) {
#pragma unroll
    for (int k = 0; k < VS; ++k) {
      if (k + 1 < VS) read_values(k + 1, fr[(k + 1) & 1]);
      more(k);
      __builtin_amdgcn_sched_barrier(0);
      multiply_values(k, fr[k & 1]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto softmax = [&](int t) {
    const int tile = tile_of(t);
    const bool hist = tile < Th;
    const int j0 = (hist ? tile : tile - Th) * BN;
    float sv[SUB * 16];
#pragma unroll
    for (int i = 0; i < SUB * 16; ++i) sv[i] = S[i >> 4][i & 15];
    // scores in units of log 2: value * cs
    float cs = a.c1;
    if (a.cap.x > 0.0f) {
      cap_scores(sv, a.cap);
      cs = 1.0f;
    }
    if (MAP && a.slopes) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const float* age = reinterpret_cast<const float*>(smem + meta_at(t, wk + u * WK) + 128);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 ag = hist ? *reinterpret_cast<const f32x4*>(age + 8 * q4 + 4 * half) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) sv[u * 16 + q4 * 4 + e] = fmaf(-slope2, ag[e], sv[u * 16 + q4 * 4 + e] * cs);
        }
      }
      cs = 1.0f;
    } else if (!MAP && WQ < 8 && a.slopes) {      // (the widest tiling takes the map: its loop is 1.3% shorter for it)
      // frames of rpf rows: a group of 32 keys starts at row `rem` of its frame.  Each score meets its own
      // frame's bias (that of the group's first frame and a step back would round at the larger one)
      const float inv = 1.0f / (float)rpf, slope = hist ? slope2 : 0.0f;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const int jb = j0 + (wk + u * WK) * 32, f0 = jb / rpf, rem = jb - f0 * rpf + 4 * half;
        const float age = (float)(age0 - f0), b0 = -slope * age, b1 = -slope * (age - 1.0f);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int x = rem + 8 * (i >> 2) + (i & 3);          // below rpf + 32
          const float b = rpf >= 32 ? (x >= rpf ? b1 : b0) : -slope * (age - floorf(((float)x + 0.5f) * inv));
          sv[u * 16 + i] = fmaf(sv[u * 16 + i], cs, b);
        }
      }
      cs = 1.0f;
    }
    // keys that not every column sees (2,048 tokens of 16 heads over 392 rows and themselves: 140 us with
    // every own tile masked, 61)
    if (j0 + BN > (hist ? n_vis : own_full)) {
      // this lane's first key, and the last one that it sees, from there
      const int jb = j0 + wk * 32 + 4 * half, last = (hist ? n_vis : tree ? own_end : draft0 + qi + 1) - 1 - jb;
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (u * WK * 32 + 8 * (i >> 2) + (i & 3) > last) sv[u * 16 + i] = neg_inf();
      if (tree && !hist) {
        // bits of 32 keys from two words; what lies before the drafts is seen, what lies behind them masked above
        const int words = (n_own - draft0 + 31) >> 5;
        auto word = [&](int k) -> uint32_t { return k < 0 ? ~0u : anc[min(k, words - 1) * BM + wq * 32 + c32]; };
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int e = j0 + (wk + u * WK) * 32 - draft0;
          const uint32_t bits = __builtin_amdgcn_alignbit(word((e >> 5) + 1), word(e >> 5), e & 31) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(bits >> (8 * (i >> 2) + (i & 3)) & 1u)) sv[u * 16 + i] = neg_inf();
        }
      }
    }
    // p of all scores against the subtracted maximum, packed as pb; returns their sum
    auto form = [&](float mu) -> float {
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < SUB * 2; ++w) {
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = exp2_fast(fmaf(sv[w * 8 + e], cs, -mu));
          sum[e & 3] += x;
          p[e] = (__bf16)x;
        }
        pb[w] = __builtin_bit_cast(u32x4, p);
      }
      return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    // The subtracted maximum m moves only when it has to: as long as a lane's p add up
    // to at most 2^13, fp32 sums and bf16 p are as good against an older, smaller m, and
    // a tile needs neither its maximum nor a rescaling.  The first tile that a column
    // sees, and one that outgrows m, forms its p anew.
    float sum = form(m == neg_inf() ? 0.0f : m);
    if (__any(!(sum <= 8192.0f) || m == neg_inf())) {
      float top = sv[0];
#pragma unroll
      for (int i = 1; i < SUB * 16; ++i) top = fmaxf(top, sv[i]);
      top = fmaxf(top, other_half(top)) * cs;
      const float mn = fmaxf(m, top);
      const float al = m == neg_inf() ? 0.0f : exp2_fast(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int i = 0; i < DT; ++i) O[i] *= al;
      sum = form(m == neg_inf() ? 0.0f : m);
    }
    l += sum;
    if constexpr (PP) {       // formed here, not behind the barrier
#pragma unroll
      for (int w = 0; w < SUB * 2; ++w) asm volatile("" : "+v"(pb[w]));
      asm volatile("" : "+v"(l));
    }
  };

  if (t0 < t1) {
    if (MAP) {
      load_meta(t0);
      load_meta(t0 + 1);
      if (PP) load_meta(t0 + 2);
      wait_loads<0, T::BAR>();
    }
    issue(t0);
    if constexpr (PP) {
      // The two waves of a SIMD (w and w + 4) take turns: while one forms its softmax on
      // the vector unit, the other keeps the matrix unit busy, half an iteration behind.
      // A barrier ends each half.  Half 2t + 1 (first group: products of tile t, second:
      // softmax of tile t) begins with tile t + 1 in LDS and all readers of tile t - 1
      // done, whose buffer tile t + 3 then takes: each group orders its part of it at
      // the start of its next softmax (between the products it cost 4% more).
      auto end_even = [&](int t) {      // of half 2t: tile t + 1 has come, t + 2 may be under way
        if (t + 2 < t1) wait_loads<NL, true>();
        else wait_loads<0, true>();
      };
      if (t0 + 1 < t1) issue(t0 + 1);
      if (t0 + 2 < t1) issue(t0 + 2);
      if (t0 + 2 < t1) wait_loads<2 * NL, true>();
      else wait_loads<0, true>();
      key_buffer(t0);
      read_keys(0, fr[0]);
      scores_from(0);
      const bool second = wave >= 4;
      const int fill = second ? 3 : 2;
      if (second) end_even(t0);
      for (int t = t0; t < t1; ++t) {
        // first: half 2t begins here, second: half 2t + 1
        if (t + fill < t1 && t + fill > t0 + 2) issue(t + fill);
        softmax(t);
        value_buffer(t);
        read_values(0, fr[0]);
        if (second) wait_loads<63, true>();
        else end_even(t);
        // (behind the last tile the scores are those of an old buffer, and not used)
        key_buffer(t + 1);
        __builtin_amdgcn_s_setprio(1);
        values_from([&](int k) {
          if (k == VS - 1) read_keys(0, fr[VS & 1]);
        });
        scores_from(VS & 1);
        __builtin_amdgcn_s_setprio(0);
        if (second) end_even(t + 1);
        else wait_loads<63, true>();
      }
      if (!second) wait_loads<63, true>();
    } else {
      for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) {
          wait_loads<63, T::BAR>();         // every reader is done with the buffer that is filled next
          issue(t + 1);
          wait_loads<NL, T::BAR>();
        } else {
          wait_loads<0, T::BAR>();
        }
        key_buffer(t);
        read_keys(0, fr[0]);
        scores_from(0);
        value_buffer(t);
        read_values(0, fr[0]);
        softmax(t);
        values_from([](int) {});
      }
    }
  }
  l += other_half(l);

  // the waves along the keys hand their parts to the first of them
  if constexpr (WK > 1) {
    constexpr int OS = D + 4;
    wait_loads<0, true>();                 // the ring is no longer read
    float* mo = reinterpret_cast<float*>(smem);
    float* ml = mo + WQ * (WK - 1) * 32 * OS;
    if (wk > 0) {
      const int slot = (wk - 1) * WQ + wq;
      float* o = mo + (slot * 32 + c32) * OS + 4 * half;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<f32x4*>(o + 32 * dt + 8 * q4) =
              f32x4{O[dt][q4 * 4], O[dt][q4 * 4 + 1], O[dt][q4 * 4 + 2], O[dt][q4 * 4 + 3]};
      if (half == 0) {
        ml[slot * 64 + c32] = m;
        ml[slot * 64 + 32 + c32] = l;
      }
    }
    __syncthreads();
    if (wk > 0) return;
    float mt = m;
#pragma unroll
    for (int x = 0; x < WK - 1; ++x) mt = fmaxf(mt, ml[(x * WQ + wq) * 64 + c32]);
    const float mu = mt == neg_inf() ? 0.0f : mt;
    float w0 = exp2_fast(m - mu);
    l *= w0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] *= w0;
#pragma unroll
    for (int x = 0; x < WK - 1; ++x) {
      const int slot = x * WQ + wq;
      const float w = exp2_fast(ml[slot * 64 + c32] - mu);
      l = fmaf(ml[slot * 64 + 32 + c32], w, l);
      const float* o = mo + (slot * 32 + c32) * OS + 4 * half;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(o + 32 * dt + 8 * q4);
#pragma unroll
          for (int e = 0; e < 4; ++e) O[dt][q4 * 4 + e] = fmaf(v[e], w, O[dt][q4 * 4 + e]);
        }
    }
    m = mt;
  }

  if (c >= M) return;
  if (st.n_split == 1) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    uint16_t* o = st.out + ((int64_t)hk * M + c) * D + 4 * half;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (__bf16)(O[dt][q4 * 4 + e] * inv);
        *reinterpret_cast<bf16x4*>(o + 32 * dt + 8 * q4) = v;
      }
    if (half == 0 && st.lse) st.lse[(int64_t)hk * M + c] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : neg_inf();
  } else {
    const int64_t part = st.part0 + ((int64_t)hk * st.n_split + split) * M + c;
    float* o = a.part_o + part * D + 4 * half;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4*>(o + 32 * dt + 8 * q4) =
            f32x4{O[dt][q4 * 4], O[dt][q4 * 4 + 1], O[dt][q4 * 4 + 2], O[dt][q4 * 4 + 3]};
    if (half == 0) {
      a.part_ml[part * 2] = m;
      a.part_ml[part * 2 + 1] = l;
    }
  }
}

// k_join: the parts of one query row, brought to one maximum and added in a fixed
// order: GPR groups of D / 4 lanes share a row's parts (8 where there are many, 1 where
// a few: then a block takes several rows).
template <int D, int GPR>
__global__ __launch_bounds__(256) void k_join(AttendArgs a) {
  const AttendStream& st = a.st[blockIdx.y];
  const int M = a.G * st.n_q, n = st.n_split;
  constexpr int L4 = D / 4, ROWS = 256 / L4 / GPR;
  const int tid = threadIdx.x, g = tid / L4 % GPR, d4 = (tid % L4) * 4;
  const int row = blockIdx.x * ROWS + tid / (L4 * GPR);
  if (n == 1 || blockIdx.x * ROWS >= a.Hk * M) return;      // the whole block
  const bool live = row < a.Hk * M;
  const int hk = row / M, c = row % M;
  const int64_t p0 = live ? st.part0 + (int64_t)hk * n * M + c : 0;
  float mt = neg_inf();
  for (int i = tid % (L4 * GPR); live && i < n; i += L4 * GPR) mt = fmaxf(mt, a.part_ml[(p0 + (int64_t)i * M) * 2]);
  constexpr int WIDE = L4 * GPR < 64 ? L4 * GPR : 64;
#pragma unroll
  for (int x = WIDE / 2; x > 0; x >>= 1) mt = fmaxf(mt, __shfl_xor(mt, x));
  if constexpr (L4 * GPR > 64) {
    __shared__ float sm[4];
    constexpr int NWV = L4 * GPR / 64;
    if ((tid & 63) == 0) sm[tid >> 6] = mt;
    __syncthreads();
    const int w0 = tid / (L4 * GPR) * NWV;
#pragma unroll
    for (int x = 0; x < NWV; ++x) mt = fmaxf(mt, sm[w0 + x]);
  }
  const float mu = mt == neg_inf() ? 0.0f : mt;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.0f;
#pragma unroll 4
  for (int i = g; live && i < n; i += GPR) {
    const int64_t p = p0 + (int64_t)i * M;
    const float w = exp2_fast(a.part_ml[p * 2] - mu);
    l = fmaf(a.part_ml[p * 2 + 1], w, l);
    o += *reinterpret_cast<const f32x4*>(a.part_o + p * D + d4) * w;
  }
  if constexpr (GPR > 1) {
    __shared__ __align__(16) float so[256 / L4][D];
    __shared__ float sl[256 / L4];
    *reinterpret_cast<f32x4*>(&so[tid / L4][d4]) = o;
    if (tid % L4 == 0) sl[tid / L4] = l;
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int x = 1; x < GPR; ++x) {
      o += *reinterpret_cast<const f32x4*>(&so[tid / L4 + x][d4]);
      l += sl[tid / L4 + x];
    }
  }
  if (!live) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  bf16x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[e] * inv);
  *reinterpret_cast<bf16x4*>(st.out + (int64_t)row * D + d4) = v;
  if (d4 == 0 && st.lse) st.lse[row] = l > 0.0f ? (mt + __builtin_amdgcn_logf(l)) * kLn2 : neg_inf();
}

// ---------------------------------------------------------------------------
// k_accumulate<D, PM, NW, MAP>: w[row] = decay w[row] + sum over the M = G n_q
// query rows of a KV head of exp(s - lse).  S = Q K^T with the keys as columns: a
// wave keeps 32 keys in registers as the B operand, straight from memory, and
// walks the query rows, staged in LDS PM at a time; a row's sum then stays in the
// two lanes that hold it, added in one order, so nothing is atomic.  Where the keys
// alone do not fill the card, the query rows are shared out too: each share's sums go
// to the workspace and k_add adds them in order.
// One token: bound by reading the keys, which a block without a map takes through LDS in
// whole lines (705,600 rows of 4 KV heads, d 128: 116 to 119 us, 6.1 TB/s).  More: by cap,
// bias and exp on the vector unit for 59% of the time (32 tokens of 28 heads, 117,600 rows, 105 M scores: 56
// us); the rest are products and LDS reads that a wave does not overlap with them.
template <int D, int PM, int NW, bool MAP>
__global__ __launch_bounds__(64 * NW) void k_accumulate(AttendArgs a, float decay) {
  constexpr int RB = D * 2, CH = D / 8, KST = D / 16;
  __shared__ __align__(1024) unsigned char sq[PM * RB];
  __shared__ __align__(16) float s_lse[PM];
  __shared__ __align__(16) float s_slope[PM];
  // Few query rows: the pass is bound by reading the keys, which then come through LDS in
  // whole lines, two groups of 32 a wave, one under way while the other is multiplied.
  constexpr bool STAGED = !MAP && NW == 4;
  constexpr int NI = 32 * RB / 1024, RPI = 64 / CH;
  __shared__ __align__(1024) unsigned char sk[STAGED ? NW * 2 * 32 * RB : 16];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int item = blockIdx.x, s = 0;
  while (s + 1 < a.S && item >= a.st[s + 1].item0) ++s;
  const AttendStream& st = a.st[s];
  item -= st.item0;
  const int share = item % st.q_split;
  item /= st.q_split;
  const int split = item % st.n_split, hk = item / st.n_split;
  const int M = a.G * st.n_q;
  // this share's query rows: whole groups of 32
  const int M32 = (M + 31) / 32;
  const int m0 = (int)((int64_t)M32 * share / st.q_split) * 32;
  const int m1 = min(M, (int)((int64_t)M32 * (share + 1) / st.q_split) * 32);
  const int n_vis = MAP ? __builtin_amdgcn_readfirstlane(*st.n_vis) : st.n_rows;
  // groups of 32 keys: NW at a time, the items of a KV head in turn (one dense window)
  const int T = (n_vis + 31) / 32, step = st.n_split * NW;
  if (split * NW >= T) return;                           // the whole block
  const uint16_t* kh = st.keys + hk * st.head_stride;
  float* wh = st.weights + (int64_t)hk * st.w_stride;
  const float* ages = reinterpret_cast<const float*>(reinterpret_cast<const char*>(st.rowmap) + st.age_off);

  for (int p0 = m0; p0 < m1; p0 += PM) {
    const int np = min(PM, m1 - p0), np32 = (np + 31) & ~31;
    if (p0 > m0) __syncthreads();
    for (int i = tid; i < np32 * CH; i += 64 * NW) {
      const int r = i / CH, ch = i % CH;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (r < np) v = *reinterpret_cast<const u32x4*>(st.q + ((int64_t)hk * M + p0 + r) * D + ch * 8);
      *reinterpret_cast<u32x4*>(sq + r * RB + ((ch ^ (r & (CH - 1))) << 4)) = v;
    }
    for (int r = tid; r < np32; r += 64 * NW) {
      // a row that saw nothing (-inf) and padding give nothing
      float x = r < np ? st.lse[(int64_t)hk * M + p0 + r] * kLog2e : neg_inf();
      s_lse[r] = x == neg_inf() ? -neg_inf() : x;
      if (a.slopes) s_slope[r] = r < np ? a.slopes[hk * a.G + (p0 + r) / st.n_q] * kLog2e : 0.0f;
    }
    __syncthreads();
    const float dk = p0 > m0 ? 1.0f : (st.q_split > 1 ? 0.0f : decay);
    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(SS_LDS unsigned char*)sk) + wave * 2 * 32 * RB;
    auto issue = [&](int t, int b) {
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        const int r = k * RPI + lane / CH, jr = min(t * 32 + r, n_vis - 1);
        const uint32_t at = (uint32_t)jr * RB + ((lane % CH ^ key_swizzle<D>(r)) << 4), to = ring + b * 32 * RB + k * 1024;
        if (a.once) load_lds16<true>(kh, at, to);
        else load_lds16<false>(kh, at, to);
      }
    };
    int b = 0;
    if (STAGED && split * NW + wave < T) issue(split * NW + wave, 0);
    for (int t = split * NW + wave; t < T; t += step, b ^= 1) {
      const int j = min(t * 32 + c32, n_vis - 1);
      const int row = MAP ? st.rowmap[j] : j;
      const float age = !a.slopes ? 0.0f : MAP ? ages[j] : (float)(st.age0 - j / st.rpf);
      u32x4 kf[KST];
      if constexpr (STAGED) {
        if (t + step < T) {
          wait_loads<63, false>();            // the other buffer has been read
          issue(t + step, b ^ 1);
          wait_loads<NI, false>();
        } else {
          wait_loads<0, false>();
        }
#pragma unroll
        for (int i = 0; i < KST; ++i)
          kf[i] = *(const SS_LDS u32x4*)(uintptr_t)(ring + b * 32 * RB + c32 * RB +
                                                    (((2 * i + half) ^ key_swizzle<D>(c32)) << 4));
      } else {
#pragma unroll
        for (int i = 0; i < KST; ++i)
          kf[i] = *reinterpret_cast<const u32x4*>(kh + (int64_t)row * D + 16 * i + 8 * half);
      }
      float sum = 0.0f;
      for (int q0 = 0; q0 < np32; q0 += 32) {
        const int r = q0 + c32;
        f32x16 S = f32x16{};
#pragma unroll
        for (int i = 0; i < KST; ++i) {
          const u32x4 q = *reinterpret_cast<const u32x4*>(sq + r * RB + (((2 * i + half) ^ (r & (CH - 1))) << 4));
          S = mfma32(q, kf[i], S);
        }
        float sv[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) sv[i] = S[i];
        // adds exp of sv * factor(i) - lse (and the bias)
        auto add = [&](auto factor) {
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            f32x4 z = *reinterpret_cast<const f32x4*>(&s_lse[q0 + 8 * q4 + 4 * half]);
            if (a.slopes) {
              const f32x4 sl = *reinterpret_cast<const f32x4*>(&s_slope[q0 + 8 * q4 + 4 * half]);
#pragma unroll
              for (int e = 0; e < 4; ++e) z[e] = fmaf(sl[e], age, z[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += exp2_fast(fmaf(sv[q4 * 4 + e], factor(q4 * 4 + e), -z[e]));
          }
        };
        if (a.cap.x == 0.0f) {
          add([&](int) { return a.c1; });
        } else if (near_cap(sv, a.cap)) {
          add([&](int i) { return near_factor(sv[i], a.cap); });    // its last product is the fma's
        } else {
          cap_scores(sv, a.cap);
          add([](int) { return 1.0f; });
        }
      }
      sum += other_half(sum);
      if (half == 0 && t * 32 + c32 < n_vis) {
        float* w = st.q_split > 1 ? a.part_o + st.part0 + ((int64_t)share * a.Hk + hk) * n_vis + j : wh + row;
        *w = dk == 0.0f ? sum : fmaf(dk, *w, sum);
      }
    }
  }
}

// w[row] = decay w[row] + the shares' sums, in their order.
__global__ __launch_bounds__(256) void k_add(AttendArgs a, bool map, float decay) {
  const AttendStream& st = a.st[blockIdx.y];
  if (st.q_split == 1) return;
  const int n_vis = map ? *st.n_vis : st.n_rows;
  const int64_t n = (int64_t)a.Hk * n_vis;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int j = (int)(i % n_vis);
    float sum = 0.0f;
    for (int q = 0; q < st.q_split; ++q) sum += a.part_o[st.part0 + q * n + i];
    float* w = st.weights + (i / n_vis) * st.w_stride + (map ? st.rowmap[j] : j);
    *w = decay == 0.0f ? sum : fmaf(decay, *w, sum);
  }
}

// w *= decay for every detailed row (with a list of frames the sums reach only some).
__global__ __launch_bounds__(256) void k_decay(AttendArgs a, float decay) {
  const AttendStream& st = a.st[blockIdx.y];
  const int64_t n = (int64_t)a.Hk * st.n_rows;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float* w = st.weights + (i / st.n_rows) * st.w_stride + st.row0 + i % st.n_rows;
    *w = decay == 0.0f ? 0.0f : *w * decay;
  }
}

// ---------------------------------------------------------------------------
// k_store_values: the values of appended frames, and zeros for their weights.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_store_values(StoreValuesArgs a) {
  const int64_t per = a.rows * (a.D / 8);               // 16-byte pieces of one (layer, KV head)
  const int lh = blockIdx.y, l = lh / a.Hk, h = lh % a.Hk;
  const u32x4* src = reinterpret_cast<const u32x4*>(a.src[l]) + h * per;
  u32x4* dst = reinterpret_cast<u32x4*>(a.values + ((int64_t)lh * a.max_rows + a.row0) * a.D);
  float* w = a.weights + (int64_t)lh * a.max_rows + a.row0;
  const int64_t step = (int64_t)gridDim.x * 256, i0 = blockIdx.x * 256ll + threadIdx.x;
  for (int64_t i = i0; i < per; i += 4 * step) {
    u32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < per) v[k] = __builtin_nontemporal_load(src + i + k * step);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < per) dst[i + k * step] = v[k];
  }
  for (int64_t i = i0; i < a.rows; i += step) w[i] = 0.0f;
}

// k_move_values: values and weights of the rows that stay move to the start of their run,
// in place.  Pieces o, o + shift, o + 2 shift, ... each take the place of the one before;
// one thread walks such a chain in order, four reads ahead, and no two threads meet.
template <class U>
__device__ __forceinline__ void move_down(U* run, int64_t shift, int64_t keep) {
  const int64_t step = (int64_t)gridDim.x * 256, len = min(shift, keep);
  for (int64_t o = blockIdx.x * 256ll + threadIdx.x; o < len; o += step)
    for (int64_t k = o; k < keep; k += 4 * shift) {
      U x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k + i * shift < keep) x[i] = run[k + (i + 1) * shift];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k + i * shift < keep) run[k + i * shift] = x[i];
    }
}
__global__ __launch_bounds__(256) void k_move_values(MoveValuesArgs a) {
  const int64_t row0 = blockIdx.y * a.max_rows, unit = a.D / 8;       // 16-byte pieces of a row
  move_down(reinterpret_cast<u32x4*>(a.values + row0 * a.D), a.row_shift * unit, a.keep_rows * unit);
  move_down(a.weights + row0, a.row_shift, a.keep_rows);
}

// ---------------------------------------------------------------------------
// Eviction.  k_evict_offsets: the row offsets of the thinned frames, one block (frames
// of one size need none: their offsets are products).
// k_evict: a wave takes one (frame, layer, KV head).  The cut is the largest key
// u with at least `keep` rows at or above it, found bit by bit over the weights'
// order-preserving 32-bit image; rows above it stay, and of the rows at it the
// first ones.  The kept rows are then copied, 16 bytes a lane, past the caches (1 hour to
// 32 rows a frame: 388 us, 5.3 TB/s read and written; through the caches 417 to 430).
// A launch holds fewer than 2^32 threads, so more than kEvictItems items (4.5 times 1 hour of
// 4 layers and 4 KV heads) take several launches; a loop over the items in the kernel
// made 418 us 444.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void k_evict_offsets(EvictArgs a) {
  __shared__ int64_t wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t base = 0;
  if (tid == 0) a.dst.frame_off[0] = 0;
  for (int64_t f0 = 0; f0 < a.n_frames; f0 += 1024) {
    const int64_t f = f0 + tid;
    int64_t v = 0;
    if (f < a.n_frames) {
      v = a.src.frame_off[f + 1] - a.src.frame_off[f];
      if (f < a.n_thin) v = min(v, (int64_t)a.keep);
    }
    for (int x = 1; x < 64; x <<= 1) {
      const int64_t o = __shfl_up(v, x);
      if (lane >= x) v += o;
    }
    if (lane == 63) wsum[wave] = v;
    __syncthreads();
    int64_t before = base;
    for (int x = 0; x < wave; ++x) before += wsum[x];
    if (f < a.n_frames) a.dst.frame_off[f + 1] = (int32_t)(before + v);
    for (int x = 0; x < 16; ++x) base += wsum[x];
    __syncthreads();
  }
}

constexpr int64_t kEvictItems = 1 << 18;

__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w + 0.0f);          // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

template <int D>
__global__ __launch_bounds__(256) void k_evict(EvictArgs a) {
  constexpr int CH = D / 8, RPW = 64 / CH;               // 16-byte pieces of a row; rows per wave and step
  __shared__ int s_row[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int LH = a.L * a.Hk;
  const int64_t items = a.n_frames * LH;
  if ((int64_t)blockIdx.x >= a.item_blocks) {
    // the frames' descriptors and mean keys, and the key statistic
    const int64_t nb = gridDim.x - a.item_blocks, i0 = ((int64_t)blockIdx.x - a.item_blocks) * 256 + tid;
    const int64_t nd = a.n_frames * a.Hk * D / 4, np = nd * a.L;
    const u32x4* sd = reinterpret_cast<const u32x4*>(a.src.desc);
    const u32x4* sp = reinterpret_cast<const u32x4*>(a.src.pooled);
    for (int64_t i = i0; i < nd + np; i += nb * 256) {
      if (i < nd) reinterpret_cast<u32x4*>(a.dst.desc)[i] = sd[i];
      else reinterpret_cast<u32x4*>(a.dst.pooled)[i - nd] = sp[i - nd];
    }
    if (i0 == 0) a.dst.stats[0] = a.src.stats[0];
    return;
  }
  const int64_t it = a.item0 + (int64_t)blockIdx.x * 4 + wave;
  if (it >= items) return;
  const int64_t f = it / LH;
  const int lh = (int)(it % LH);
  const int64_t r0 = a.rpf > 0 ? a.src_row0 + f * a.rpf : a.src.frame_off[f];
  const int64_t n = a.rpf > 0 ? a.rpf : a.src.frame_off[f + 1] - r0;
  const int64_t keep = f < a.n_thin ? min(n, (int64_t)a.keep) : n;
  int64_t o0;
  if (a.rpf > 0) {
    o0 = min(f, a.n_thin) * min(a.rpf, (int64_t)a.keep) + max(f - a.n_thin, (int64_t)0) * a.rpf;
    if (lh == 0 && lane == 0) {
      if (f == 0) a.dst.frame_off[0] = 0;
      a.dst.frame_off[f + 1] = (int32_t)(o0 + keep);
    }
  } else {
    o0 = a.dst.frame_off[f];
  }
  const int64_t s0 = (int64_t)lh * a.src_max_rows + r0, d0 = (int64_t)lh * a.dst_max_rows + o0;
  const float* w = a.src_weights + s0;
  uint32_t cut = 0;
  int64_t ties = n;                                      // rows at the cut that stay (keep == n: all)
  if (keep < n) {
    constexpr int kReg = 8;
    uint32_t key[kReg];
    const bool in_reg = n <= 64 * kReg;
    if (in_reg) {
#pragma unroll
      for (int i = 0; i < kReg; ++i) key[i] = i * 64 + lane < n ? weight_key(w[i * 64 + lane]) : 0u;
    }
    // rows with a key of at least u (u > 0: padding does not count)
    auto count = [&](uint32_t u) -> int64_t {
      int64_t c = 0;
      if (in_reg) {
#pragma unroll
        for (int i = 0; i < kReg; ++i)
          if (i * 64 < n) c += __popcll(__ballot(key[i] >= u));
      } else {
        for (int64_t i = 0; i < n; i += 64) c += __popcll(__ballot(i + lane < n && weight_key(w[i + lane]) >= u));
      }
      return c;
    };
    for (int b = 31; b >= 0; --b) {
      const uint32_t u = cut | (1u << b);
      if (count(u) >= keep) cut = u;
    }
    ties = keep - (cut == 0xFFFFFFFFu ? 0 : count(cut + 1u));
  }
  int64_t out = 0, tied = 0;
  for (int64_t i = 0; i < n; i += 64) {
    bool stay = i + lane < n;
    if (keep < n) {
      const uint32_t k = stay ? weight_key(w[i + lane]) : 0u;
      const uint64_t eq = __ballot(stay && k == cut);
      const int64_t rank = tied + __popcll(eq & ((1ull << lane) - 1));
      stay = stay && (k > cut || (k == cut && rank < ties));
      tied += __popcll(eq);
    }
    const uint64_t mask = __ballot(stay);
    const int c = __popcll(mask);
    if (stay) {
      const int at = __popcll(mask & ((1ull << lane) - 1));
      s_row[wave][at] = (int)(i + lane);
      a.dst_weights[d0 + out + at] = w[i + lane];
      a.dst.counts[d0 + out + at] = a.src.counts[s0 + i + lane];
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int sub = lane / CH, ch = lane % CH;
    for (int x = sub; x < c; x += 4 * RPW) {
      u32x4 k[4], v[4];
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (x + y * RPW < c) {
          const int64_t r = s0 + s_row[wave][x + y * RPW];
          k[y] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.src.keys + r * D + ch * 8));
          v[y] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.src_values + r * D + ch * 8));
        }
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (x + y * RPW < c) {
          const int64_t r = d0 + out + x + y * RPW;
          __builtin_nontemporal_store(k[y], reinterpret_cast<u32x4*>(a.dst.keys + r * D + ch * 8));
          __builtin_nontemporal_store(v[y], reinterpret_cast<u32x4*>(a.dst_values + r * D + ch * 8));
        }
    }
    __builtin_amdgcn_wave_barrier();
    out += c;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int D, int WQ, int WK, int BN, int NS>
hipError_t attend_go(const AttendArgs& a, bool map, int items, hipStream_t st) {
  if (map)
    hipLaunchKernelGGL((k_attend<D, WQ, WK, BN, NS, true>), dim3(items), dim3(64 * WQ * WK), 0, st, a);
  else
    hipLaunchKernelGGL((k_attend<D, WQ, WK, BN, NS, false>), dim3(items), dim3(64 * WQ * WK), 0, st, a);
  return hipGetLastError();
}

template <int D>
hipError_t attend_impl(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  hipError_t e;
  switch (p.shape) {
    case 0: e = attend_go<D, 1, 4, 128, 2>(a, p.map, p.items, st); break;
    case 1:
      if constexpr (D == 128) e = attend_go<D, 2, 2, 64, 2>(a, p.map, p.items, st);
      else e = attend_go<D, 2, 4, 128, 2>(a, p.map, p.items, st);
      break;
    case 2: e = attend_go<D, 4, 1, 64, 2>(a, p.map, p.items, st); break;
    default: e = attend_go<D, 8, 1, 64, 4>(a, p.map, p.items, st); break;
  }
  if (e != hipSuccess) return e;
  if (p.join_parts > 4) hipLaunchKernelGGL((k_join<D, 8>), dim3(cdiv(p.join_rows * 8, 1024 / D), a.S), dim3(256), 0, st, a);
  else if (p.join_parts > 1) hipLaunchKernelGGL((k_join<D, 1>), dim3(cdiv(p.join_rows, 1024 / D), a.S), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int D>
hipError_t accumulate_impl(const AttendArgs& a, const AttendPlan& p, float decay, hipStream_t st) {
  if (p.shape == 0) {
    if (p.map) hipLaunchKernelGGL((k_accumulate<D, 32, 4, true>), dim3(p.items), dim3(256), 0, st, a, decay);
    else hipLaunchKernelGGL((k_accumulate<D, 32, 4, false>), dim3(p.items), dim3(256), 0, st, a, decay);
  } else {
    if (p.map) hipLaunchKernelGGL((k_accumulate<D, 256, 8, true>), dim3(p.items), dim3(512), 0, st, a, decay);
    else hipLaunchKernelGGL((k_accumulate<D, 256, 8, false>), dim3(p.items), dim3(512), 0, st, a, decay);
  }
  if (p.add_rows > 0)
    hipLaunchKernelGGL(k_add, dim3((unsigned)std::min<int64_t>(cdiv(p.add_rows, 256), 4096), a.S), dim3(256), 0, st, a, p.map,
                       decay);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rows(const RowsArgs& a, hipStream_t st) {
  int64_t most = 0;
  for (int s = 0; s < a.S; ++s) most = std::max<int64_t>(most, a.st[s].f_hi - a.st[s].f_lo);
  if (a.n_listed > 0) most = std::min<int64_t>(most, a.n_listed);
  const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(most, kRowsThreads / 64), a.n_listed > 0 ? 32 : 512));
  hipLaunchKernelGGL(k_rows, dim3(blocks, a.S), dim3(kRowsThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  return p.D == 128 ? attend_impl<128>(a, p, st) : attend_impl<64>(a, p, st);
}

hipError_t launch_accumulate(const AttendArgs& a, const AttendPlan& p, float decay, hipStream_t st) {
  if (p.listed && decay != 1.0f) {
    int64_t most = 1;
    for (int s = 0; s < a.S; ++s) most = std::max<int64_t>(most, (int64_t)a.Hk * a.st[s].n_rows);
    hipLaunchKernelGGL(k_decay, dim3((unsigned)std::min<int64_t>(cdiv(most, 1024), 4096), a.S), dim3(256), 0, st, a, decay);
    decay = 1.0f;
  }
  if (p.items == 0) return hipGetLastError();
  return p.D == 128 ? accumulate_impl<128>(a, p, decay, st) : accumulate_impl<64>(a, p, decay, st);
}

hipError_t launch_store_values(const StoreValuesArgs& a, hipStream_t st) {
  const int64_t pieces = a.rows * (a.D / 8);
  const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(pieces, 1024), 1024));
  hipLaunchKernelGGL(k_store_values, dim3(blocks, a.L * a.Hk), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_move_values(const MoveValuesArgs& a, hipStream_t st) {
  const int64_t pieces = std::min(a.row_shift, a.keep_rows) * (a.D / 8);
  if (pieces <= 0) return hipSuccess;
  const int blocks = (int)std::min<int64_t>(cdiv(pieces, 256), 4096);
  hipLaunchKernelGGL(k_move_values, dim3(blocks, a.lh), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_evict(EvictArgs a, hipStream_t st) {
  if (a.n_frames == 0) a.rpf = 0;
  if (a.rpf <= 0) {
    hipLaunchKernelGGL(k_evict_offsets, dim3(1), dim3(1024), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t items = a.n_frames * a.L * a.Hk;
  // the first launch also copies what is kept of the frames themselves
  int64_t copy = std::max<int64_t>(1, std::min<int64_t>(cdiv(a.n_frames * a.Hk * a.D * (1 + a.L) / 4, 1024), 4096));
  for (a.item0 = 0; a.item0 < items || copy > 0; a.item0 += kEvictItems, copy = 0) {
    a.item_blocks = cdiv(std::min(items - a.item0, kEvictItems), 4);
    const dim3 grid((unsigned)(a.item_blocks + copy));
    if (a.D == 128) hipLaunchKernelGGL((k_evict<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_evict<64>), grid, dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ss
