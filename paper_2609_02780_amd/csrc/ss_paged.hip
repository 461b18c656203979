// gfx950 (MI355X) kernels of rotary positions (k_rotate), of appending to a paged
// cache (k_paged_append) and of attention over it (k_paged_few, k_paged_many,
// k_paged_join).
//
// A page holds a block of 32 tokens of one KV head in the order in which the matrix
// unit takes it, so that a wave's loads are runs of 1 KB and nothing crosses lanes:
//   keys    [d / 16][32 tokens][16]:  A of S^T = K Q^T (32x32x16): lane l takes 16
//           elements of token l % 32 at piece 2 j + l / 32, eight for each of two steps;
//   values  [d / 32][2][32][16]:  A of O^T = V^T P^T: lane l takes, for dimension
//           32 c + l % 32, the 16 tokens whose scores its half of S^T holds,
//           8 g + 4 (l / 32) + e, in the order of groups g = 0, 2, 1, 3.
// Elements are e4m3 with a scale for each page, or bf16 in an open block.  e4m3 is
// exact in bf16, so the products are bf16 MFMAs with fp32 sums; a key scale meets the
// scores, a value scale joins the exponent of p.
#include "ss_paged.h"

#include <algorithm>

namespace ss {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int B = kBlockTokens;

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

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

// Eight e4m3 as bf16 (exact).
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
               __builtin_bit_cast(uint32_t, d)};
}

__device__ __forceinline__ float bf16_at(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ int span_start(const Spans& s, int i) { return s.uniform ? i * s.uniform : s.start[i]; }

// A stream's tokens, by what its table can hold.
__device__ __forceinline__ int stream_length(const PagedDev& c, int s) {
  return max(0, min(c.lengths[s], c.width * B + (B - 1)));
}

// ---------------------------------------------------------------------------
// Rotation.  cos and sin of up to 32 tokens are formed once for all heads of a block:
// the angle in turns, position * (f / 2 pi), in 64 bits (a far position times a
// frequency loses what matters in 32), its fraction in 32.
// ---------------------------------------------------------------------------
constexpr int kMaxPairs = 64;
struct Angles {
  float2 cs[B][kMaxPairs + 1];       // gain cos, gain sin
};

// Rows [r0, r1) of the table; token r's position is positions[first + r] or pos0 + r.
__device__ __forceinline__ void fill_angles(Angles& g, const Turn& t, int r0, int r1, int first, int64_t pos0) {
  const int half = t.dims >> 1, n = (r1 - r0) * half;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int r = r0 + i / half, j = i % half;
    const int64_t pos = t.positions ? t.positions[first + r] : pos0 + r;
    const double turns = (double)pos * t.freqs[j];
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    g.cs[r][j] = make_float2(t.gain * c, t.gain * t.sign * s);
  }
}

// Elements 16 p .. 16 p + 15 of a row at x, rotated by the angles cs.
__device__ __forceinline__ void turned(const uint16_t* x, int p, const float2* cs, const Turn& t, float (&y)[16]) {
  const int i0 = 16 * p, half = t.dims >> 1;
  const u32x4* v = reinterpret_cast<const u32x4*>(x + i0);
  const u32x4 a = v[0], b = v[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(a[i] << 16);
    y[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    y[8 + 2 * i] = __uint_as_float(b[i] << 16);
    y[8 + 2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
  }
  if (i0 >= t.dims) return;
  if (t.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + 2 * i < t.dims) {
        const float2 w = cs[i0 / 2 + i];
        const float e = y[2 * i], o = y[2 * i + 1];
        y[2 * i] = e * w.x - o * w.y;
        y[2 * i + 1] = o * w.x + e * w.y;
      }
    }
  } else if ((half & 7) == 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int at = i0 + 8 * k;
      if (at >= t.dims) break;
      const bool low = at < half;
      const u32x4 o = *reinterpret_cast<const u32x4*>(x + (low ? at + half : at - half));
      const float2* w = cs + (low ? at : at - half);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = i & 1 ? __uint_as_float(o[i / 2] & 0xFFFF0000u) : __uint_as_float(o[i / 2] << 16);
        const float sn = low ? -w[i].y : w[i].y;
        y[8 * k + i] = y[8 * k + i] * w[i].x + z * sn;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = i0 + i;
      if (at < t.dims) {
        const bool low = at < half;
        const float2 w = cs[low ? at : at - half];
        y[i] = y[i] * w.x + bf16_at(x[low ? at + half : at - half]) * (low ? -w.y : w.y);
      }
    }
  }
}

__device__ __forceinline__ void store16(uint16_t* p, const float (&y)[16]) {
  bf16x8 a, b;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = (__bf16)y[i];
    b[i] = (__bf16)y[8 + i];
  }
  reinterpret_cast<bf16x8*>(p)[0] = a;
  reinterpret_cast<bf16x8*>(p)[1] = b;
}

// k_rotate: a block takes 32 tokens and some of the heads; a thread 16 elements of a row.
constexpr int kRotateHeads = 4;
template <int D>
__global__ __launch_bounds__(2 * D) void k_rotate(RotateArgs a) {
  constexpr int P = D / 16;
  __shared__ Angles g;
  const int t0 = blockIdx.x * B, n = min(B, a.N - t0);
  fill_angles(g, a.turn, 0, n, t0, t0);
  __syncthreads();
  const int r = threadIdx.x / P, p = threadIdx.x % P;
  if (r >= n) return;
  const int h1 = min(a.heads, (int)(blockIdx.y + 1) * kRotateHeads);
  for (int h = blockIdx.y * kRotateHeads; h < h1; ++h) {
    float y[16];
    turned(a.x.p + h * a.x.hs + (int64_t)(t0 + r) * a.x.ts, p, g.cs[r], a.turn, y);
    store16(const_cast<uint16_t*>(a.out.p) + h * a.out.hs + (int64_t)(t0 + r) * a.out.ts + 16 * p, y);
  }
}

// ---------------------------------------------------------------------------
// k_paged_append: a block takes the tokens of one cache block of a stream and one KV
// head (its keys and values) or some query heads.  Rows of a full block are rounded to
// e4m3 with one scale; rows of the stream's open blocks stay bf16.
// ---------------------------------------------------------------------------
constexpr float kLeastMax = 0x1p-100f;    // 448 / it stays finite

template <int D>
__device__ __forceinline__ float block_max(float v, float* part) {
  constexpr int W = 2 * D / 64;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) v = fmaxf(v, __shfl_xor(v, x));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < W; ++w) v = fmaxf(v, part[w]);
  return v;
}

__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d) {
  int r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

template <int D>
__global__ __launch_bounds__(2 * D) void k_paged_append(PagedAppendArgs a) {
  constexpr int P = D / 16;
  __shared__ Angles g;
  __shared__ __align__(16) uint16_t vt[B][D + 8];
  __shared__ float part[8];
  const int tid = threadIdx.x, r = tid / P, p = tid % P;
  // the stream and which of its touched blocks: (n + 62) / 32 at most, wherever the old tokens end
  int s, k;
  if (a.spans.uniform) {
    const int per = (a.spans.uniform + 2 * B - 2) / B;
    s = blockIdx.x / per;
    k = blockIdx.x % per;
  } else {
    s = 0;
    int first = 0;
    for (;; ++s) {
      const int n = a.spans.start[s + 1] - a.spans.start[s];
      const int per = n > 0 ? (n + 2 * B - 2) / B : 0;
      if ((int)blockIdx.x < first + per) break;
      first += per;
    }
    k = blockIdx.x - first;
  }
  const int start = span_start(a.spans, s), n = span_start(a.spans, s + 1) - start;
  const int L = stream_length(a.c, s), old = L - n, b0 = max(old, 0) / B, last = (L - 1) / B;
  int b = b0 + k;
  if (L == 0 || b > last) return;
  const int slot = a.c.slots[s];
  const bool has_slot = (unsigned)slot < (unsigned)a.c.n_slots;
  // A token's open rows lie in buffer block & 1.  Where the last block's buffer is the one that
  // the first block reads, the first block's own thread block writes it, after reading.
  const bool shared = last > b0 && ((last - b0) & 1) == 0;
  const bool keys = (int)blockIdx.y < a.c.Hk;
  for (int job = 0; job < 2; ++job) {
    if (job == 1) {
      if (!(shared && b == b0 && keys)) return;
      b = last;
      __syncthreads();
    }
    const int t0 = max(max(old, 0), B * b), t1 = min(L, B * (b + 1));    // new tokens of this block
    if (a.turn.dims) fill_angles(g, a.turn, t0 - B * b, t1 - B * b, start + B * b - old, (int64_t)B * b);
    __syncthreads();
    const int t = B * b + r;
    const bool fresh = t >= t0 && t < t1;
    const int64_t row = start + t - old;                                   // of the call's tokens
    if (!keys) {
      const int h0 = (blockIdx.y - a.c.Hk) * kRotateHeads, h1 = min(a.Hq, h0 + kRotateHeads);
      if (!fresh) return;
      for (int h = h0; h < h1; ++h) {
        float y[16];
        turned(a.q.p + h * a.q.hs + row * a.q.ts, p, g.cs[r], a.turn, y);
        store16(const_cast<uint16_t*>(a.q_out.p) + h * a.q_out.hs + row * a.q_out.ts + 16 * p, y);
      }
      return;
    }
    const int h = blockIdx.y;
    const bool full = job == 0 && t1 == B * (b + 1);
    const bool stays = has_slot && (job == 1 || (b == last && !shared) || (b == last && b == b0) ||
                                    (b == b0 && ((last - b0) & 1) == 1));
    const int64_t open_at = (((int64_t)slot * 2 + (b & 1)) * a.c.Hk + h) * B * D;
    float y[16], v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = v[i] = 0.0f;
    if (fresh) {
      turned(a.k.p + h * a.k.hs + row * a.k.ts, p, g.cs[r], a.turn, y);
      const u32x4* src = reinterpret_cast<const u32x4*>(a.v.p + h * a.v.hs + row * a.v.ts + 16 * p);
      const u32x4 x0 = src[0], x1 = src[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x0[i] << 16);
        v[2 * i + 1] = __uint_as_float(x0[i] & 0xFFFF0000u);
        v[8 + 2 * i] = __uint_as_float(x1[i] << 16);
        v[8 + 2 * i + 1] = __uint_as_float(x1[i] & 0xFFFF0000u);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = (float)(__bf16)y[i];
    } else if (full && t < t0 && has_slot) {
      const uint16_t* ko = a.c.ok + open_at + (p * B + r) * 16;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        y[i] = bf16_at(ko[i]);
        const int d = 16 * p + i, gq = r >> 3, w = (gq >> 1) | ((gq & 1) << 1);
        v[i] = bf16_at(a.c.ov[open_at + (((d >> 5) * 2 + ((r >> 2) & 1)) * 32 + (d & 31)) * 16 + w * 4 + (r & 3)]);
      }
    }
    if (full) {
      float km = 0.0f, vm = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        km = fmaxf(km, fabsf(y[i]));
        vm = fmaxf(vm, fabsf(v[i]));
        vt[r][16 * p + i] = to_bf16(v[i]);
      }
      km = fmaxf(block_max<D>(km, part), kLeastMax);
      vm = fmaxf(block_max<D>(vm, part), kLeastMax);
      const int page = a.c.tables[(int64_t)s * a.c.width + b];
      if ((unsigned)page < (unsigned)a.c.n_pages && (has_slot || t0 == B * b)) {
        const int64_t at = ((int64_t)page * a.c.Hk + h);
        const float ki = 448.0f / km, vi = 448.0f / vm;
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack8(y[4 * i] * ki, y[4 * i + 1] * ki, y[4 * i + 2] * ki, y[4 * i + 3] * ki);
        *reinterpret_cast<u32x4*>(a.c.k8 + at * B * D + (p * B + r) * 16) = w;
        // values: a thread takes 16 tokens of one dimension
        const int m = tid & 31, half = (tid >> 5) & 1, d = (tid >> 6) * 32 + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = 8 * ((i >> 1) | ((i & 1) << 1)) + 4 * half;
          w[i] = pack8(bf16_at(vt[tok][d]) * vi, bf16_at(vt[tok + 1][d]) * vi, bf16_at(vt[tok + 2][d]) * vi,
                       bf16_at(vt[tok + 3][d]) * vi);
        }
        *reinterpret_cast<u32x4*>(a.c.v8 + at * B * D + tid * 16) = w;
        if (tid == 0) {
          a.c.ks[at] = km / 448.0f;
          a.c.vs[at] = vm / 448.0f;
        }
      }
    }
    if (stays && fresh) {
      store16(a.c.ok + open_at + (p * B + r) * 16, y);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 16 * p + i, gq = r >> 3, w = (gq >> 1) | ((gq & 1) << 1);
        a.c.ov[open_at + (((d >> 5) * 2 + ((r >> 2) & 1)) * 32 + (d & 31)) * 16 + w * 4 + (r & 3)] = to_bf16(v[i]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Attention.  A unit is a stream's run of BM query columns (column c: token c / G, head c % G of
// its KV head); its work are the blocks that some column sees.  All units' work, laid end to
// end over the KV heads, is cut into equal shares, one a thread block, so streams of any
// lengths fill the card alike.  A block's first and last unit may be parts, joined by k_paged_join.
// ---------------------------------------------------------------------------
struct Unit {
  int s, n, start, L, c0, M;         // its columns c0 .. min(c0 + BM, M) - 1
  int b_lo, count;                   // first block, and how many (at least 1: someone writes the outputs); 0: no unit
};
__device__ __forceinline__ int unit_first(const PagedAttendArgs& a, int s, int bm) {
  return a.per ? s * a.per : a.G * a.spans.start[s] / bm + s;
}
__device__ __forceinline__ Unit unit_of(const PagedAttendArgs& a, int u, int bm, int round) {
  Unit x;
  if (a.per) {
    x.s = u / a.per;
  } else {
    int lo = 0, hi = a.S - 1;        // the last stream that begins at u or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (unit_first(a, mid, bm) <= u) lo = mid;
      else hi = mid - 1;
    }
    x.s = lo;
  }
  x.start = span_start(a.spans, x.s);
  x.n = span_start(a.spans, x.s + 1) - x.start;
  x.M = a.G * x.n;
  x.c0 = (u - unit_first(a, x.s, bm)) * bm;
  x.L = 0;
  x.b_lo = x.count = 0;
  if (x.c0 >= x.M) return x;
  x.L = stream_length(a.c, x.s);
  const int p_lo = x.L - x.n + x.c0 / a.G;                                   // the first and the last column's tokens
  const int p_hi = x.L - x.n + (min(x.M, x.c0 + bm) - 1) / a.G;
  const int lowest = a.window > 0 ? max(0, p_lo - a.window + 1) : 0;
  x.b_lo = lowest / B / round * round;
  x.count = p_hi < 0 ? 1 : max(1, (p_hi / B - x.b_lo + round) / round);
  return x;
}

// pre[u]: the work before unit u (pre[units]: all of it).
template <int T>
__device__ __forceinline__ void plan_units(const PagedAttendArgs& a, int bm, int round, int* pre) {
  __shared__ int part[T / 64];
  const int tid = threadIdx.x, run = (a.units + T - 1) / T, u0 = min(a.units, tid * run), u1 = min(a.units, u0 + run);
  int sum = 0;
  for (int u = u0; u < u1; ++u) sum += unit_of(a, u, bm, round).count;
  int upto = sum;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int v = __shfl_up(upto, x);
    if ((tid & 63) >= x) upto += v;
  }
  if ((tid & 63) == 63) part[tid >> 6] = upto;
  __syncthreads();
  int at = upto - sum;
#pragma unroll
  for (int w = 0; w < T / 64; ++w)
    if (w < (tid >> 6)) at += part[w];
  for (int u = u0; u < u1; ++u) {
    pre[u] = at;
    at += unit_of(a, u, bm, round).count;
  }
  if (tid == T - 1) pre[a.units] = at;
  __syncthreads();
}

// The share of a block, the same in k_paged_join.
__device__ __forceinline__ int64_t share_of(const PagedAttendArgs& a, int64_t all) {
  return max((all + a.n_wg - 1) / a.n_wg, (int64_t)a.min_share);
}

// Calls work(kv head, unit, first of its blocks, how many, slot of the part or -1) for a block's share.
template <int T, class F>
__device__ __forceinline__ void for_share(const PagedAttendArgs& a, int bm, int round, int* pre, F&& work) {
  const int wg = blockIdx.x;
  if (a.n_wg == 0) {
    const Unit x = unit_of(a, wg % a.units, bm, round);
    if (x.count) work(wg / a.units, x, 0, x.count, -1);
    return;
  }
  plan_units<T>(a, bm, round, pre);
  const int64_t one = pre[a.units], all = one * a.c.Hk, share = share_of(a, all);
  if (wg == 0) {
    if (threadIdx.x == 0) a.plan[0] = (int)share;
    for (int u = threadIdx.x; u <= a.units; u += T) a.plan[1 + u] = pre[u];
  }
  int64_t x = wg * share;
  const int64_t end = min(all, x + share);
  for (bool begin = true; x < end; begin = false) {
    const int hk = (int)(x / one), y = (int)(x % one);
    int lo = 0, hi = a.units - 1;                        // the last unit whose work begins at y or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pre[mid] <= y) lo = mid;
      else hi = mid - 1;
    }
    const int u = uniform(lo), first = uniform(y - pre[u]), whole = uniform(pre[u + 1] - pre[u]);
    const int cnt = uniform((int)min((int64_t)(whole - first), end - x));
    work(uniform(hk), unit_of(a, u, bm, round), first, cnt, cnt == whole ? -1 : 2 * wg + (begin ? 0 : 1));
    x += cnt;
  }
}

// The end of a column: o, its sum against maximum m (in units of log 2) and the normaliser l,
// joined with the prior's.  `at` is its place among the tokens, h its head, d the first of o's elements.
__device__ __forceinline__ void finish(const PagedAttendArgs& a, int h, int at, int d, f32x4 o, float m, float l) {
  float scale;
  if (a.prior.p) {
    const float pl = a.prior_lse[(int64_t)h * a.N + at] * kLog2e;
    const float top = fmaxf(m, pl);
    const float wa = m == neg_inf() ? 0.0f : exp2_fast(m - top), wb = pl == neg_inf() ? 0.0f : exp2_fast(pl - top);
    l = l * wa + wb;
    m = top;
    o *= wa;
    if (wb > 0.0f) {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(a.prior.p + h * a.prior.hs + at * a.prior.ts + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(wb, (float)x[e], o[e]);
    }
  }
  scale = l > 0.0f ? 1.0f / l : 0.0f;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * scale);
  *reinterpret_cast<bf16x4*>(const_cast<uint16_t*>(a.out.p) + h * a.out.hs + at * a.out.ts + d) = y;
  if (d == 0 && a.lse) a.lse[(int64_t)h * a.N + at] = l > 0.0f ? (m + log2_fast(l)) * kLn2 : neg_inf();
}

// Scores of 32 N keys by a lane's column -> p as the second product's operand.
// v: sums of products; cs, lvs: for each block of 32 keys the score's and the value's
// scale (the latter's log 2), rvs: 1 / value scale.  m moves only when it has to: as
// long as a lane's p add up to at most 2^13, fp32 sums and bf16 p are as good against
// an older, smaller m.  O is rescaled when m moves.
template <int N, int DT>
__device__ __forceinline__ void softmax_step(float (&v)[N * 16], const float (&lvs)[N], const float (&rvs)[N], float& m,
                                             float& l, f32x16 (&O)[DT], u32x4 (&pb)[N * 2]) {
  auto form = [&](float mu) -> float {
    float all = 0.0f;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float off = lvs[u] - mu;
      float p[16], sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = exp2_fast(v[u * 16 + i] + off);
        sum[i & 3] += p[i];
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        bf16x8 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = (__bf16)p[4 * w + e];
          x[4 + e] = (__bf16)p[4 * w + 8 + e];
        }
        pb[u * 2 + w] = __builtin_bit_cast(u32x4, x);
      }
      all = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), rvs[u], all);
    }
    return all;
  };
  float sum = form(m == neg_inf() ? 0.0f : m);
  if (__any(!(sum <= 8192.0f) || m == neg_inf())) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N * 16; ++i) top = fmaxf(top, v[i]);
    top = fmaxf(top, other_half(top));
    const float mn = fmaxf(m, top);
    const float al = m == neg_inf() ? 0.0f : exp2_fast(m - mn);
    m = mn;
    l *= al;
#pragma unroll
    for (int i = 0; i < DT; ++i) O[i] *= al;
    sum = form(m == neg_inf() ? 0.0f : m);
  }
  l += sum;
}

// A lane's 16 keys of block b that its column (token `last`, the first seen `lowest`) does not see.
__device__ __forceinline__ void hide(float* v, int b, int half, int last, int lowest) {
  const int j0 = b * B + 4 * half;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = j0 + 8 * (i >> 2) + (i & 3);
    if (j > last || j < lowest) v[i] = neg_inf();
  }
}

// A lane's pieces of an open block: rows from cnt on are zero.
template <int D>
__device__ __forceinline__ u32x4 open_key(const uint16_t* base, int i, int lane, int cnt) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(base + (((i >> 1) * 2 + (lane >> 5)) * B + (lane & 31)) * 16 + 8 * (i & 1));
  return (lane & 31) < cnt ? x : u32x4{0, 0, 0, 0};
}
template <int D>
__device__ __forceinline__ u32x4 open_value(const uint16_t* base, int c, int t, int lane, int cnt) {
  u32x4 x = *reinterpret_cast<const u32x4*>(base + (c * 64 + lane) * 16 + 8 * t);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // words 0, 1: tokens 8 t + 4 half + 0..3; words 2, 3: 16 on
    const int tok = 8 * t + 16 * (i >> 1) + 4 * (lane >> 5) + 2 * (i & 1);
    x[i] &= (tok < cnt ? 0xFFFFu : 0u) | (tok + 1 < cnt ? 0xFFFF0000u : 0u);
  }
  return x;
}

// k_paged_few: units of up to 32 columns (decoded tokens, a few drafts).  The four waves of a
// block take its 32-token blocks in turn, each straight from memory to registers, and join
// at the end of a unit.
template <int D>
__global__ __launch_bounds__(256, 2) void k_paged_few(PagedAttendArgs a) {
  constexpr int KST = D / 16, NC = D / 32, OS = D + 4, W = 4;
  __shared__ __align__(16) float mo[W][32][OS];
  __shared__ float ml[W][2][32];
  __shared__ int pre[kPagedUnits + 1];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31, wave = uniform(tid >> 6);
  for_share<256>(a, 32, 1, pre, [&](int hk, const Unit& un, int first, int cnt, int slot) {
    const int M = un.M, cc = min(c32, M - 1), tok = cc / a.G, head = hk * a.G + cc - tok * a.G;
    const int last = un.L - un.n + tok, lowest = a.window > 0 ? last - a.window + 1 : 0;
    const int full = uniform(un.L / B), b_at = uniform(un.b_lo + first);
    const int n = (cnt - wave + W - 1) / W;                 // this wave's blocks: b_at + wave + W i
    const int p_lo = uniform(un.L - un.n), w_lo = uniform(a.window > 0 ? max(0, un.L - a.window) : 0);
    u32x4 qf[KST];
    {
      const uint16_t* q = a.q.p + head * a.q.hs + (int64_t)(un.start + tok) * a.q.ts;
#pragma unroll
      for (int i = 0; i < KST; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + ((i >> 1) * 2 + half) * 16 + 8 * (i & 1));
    }
    f32x16 O[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) O[i] = f32x16{};
    float m = neg_inf(), l = 0.0f;

    auto step = [&](const u32x4 (&kf)[KST], const u32x4 (&vf)[NC][2], float cs, float lvs, float rvs, int b) {
      f32x16 S = f32x16{};
#pragma unroll
      for (int i = 0; i < KST; ++i) S = mfma32(kf[i], qf[i], S);
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = S[i] * cs;
      // (w_lo: the first token that the last column sees; what lies before it, another may see)
      if (b * B + B - 1 > p_lo || b * B < w_lo) hide(v, b, half, last, lowest);
      const float lv[1] = {lvs}, rv[1] = {rvs};
      u32x4 pb[2];
      softmax_step<1, NC>(v, lv, rv, m, l, O, pb);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) O[c] = mfma32(vf[c][t], pb[t], O[c]);
    };

    for (int i0 = 0; i0 < n; i0 += 64) {
      // pages and scales of the next 64 blocks, one a lane
      int id = -1;
      float ksv = 0.0f, vsv = 1.0f;
      {
        const int b = b_at + wave + W * (i0 + lane);
        if (i0 + lane < n && b < full) id = a.c.tables[(int64_t)un.s * a.c.width + b];
        if ((unsigned)id >= (unsigned)a.c.n_pages) id = -1;
        if (id >= 0) {
          ksv = a.c.ks[(int64_t)id * a.c.Hk + hk] * a.c1;
          vsv = a.c.vs[(int64_t)id * a.c.Hk + hk];
        }
      }
      const float lvv = log2_fast(vsv), rvv = 1.0f / vsv;
      const int k1 = min(64, n - i0);
      u32x4 kq[NC], vq[NC];
      auto load = [&](int k) {
        const int pid = max(0, __builtin_amdgcn_readlane(id, k));
        const int64_t at = ((int64_t)pid * a.c.Hk + hk) * (B * D);
#pragma unroll
        for (int c = 0; c < NC; ++c) kq[c] = *(reinterpret_cast<const u32x4*>(a.c.k8 + at) + c * 64 + lane);
#pragma unroll
        for (int c = 0; c < NC; ++c) vq[c] = *(reinterpret_cast<const u32x4*>(a.c.v8 + at) + c * 64 + lane);
      };
      load(0);
      for (int k = 0; k < k1; ++k) {
        u32x4 kf[KST], vf[NC][2];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          kf[2 * c] = widen(kq[c][0], kq[c][1]);
          kf[2 * c + 1] = widen(kq[c][2], kq[c][3]);
          vf[c][0] = widen(vq[c][0], vq[c][1]);
          vf[c][1] = widen(vq[c][2], vq[c][3]);
        }
        if (k + 1 < k1) load(k + 1);
        if (__builtin_amdgcn_readlane(id, k) < 0) continue;
        auto at = [&](float x) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), k)); };
        step(kf, vf, at(ksv), at(lvv), at(rvv), b_at + wave + W * (i0 + k));
      }
    }
    const int open_rows = un.L - full * B;
    if (open_rows > 0 && b_at + cnt - 1 == full && wave == ((cnt - 1) & (W - 1))) {
      const int sl = uniform(a.c.slots[un.s]);
      if ((unsigned)sl < (unsigned)a.c.n_slots) {
        const int64_t at = (((int64_t)sl * 2 + (full & 1)) * a.c.Hk + hk) * (B * D);
        u32x4 kf[KST], vf[NC][2];
#pragma unroll
        for (int i = 0; i < KST; ++i) kf[i] = open_key<D>(a.c.ok + at, i, lane, open_rows);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int t = 0; t < 2; ++t) vf[c][t] = open_value<D>(a.c.ov + at, c, t, lane, open_rows);
        step(kf, vf, a.c1, 0.0f, 1.0f, full);
      }
    }
    l += other_half(l);

    __syncthreads();                  // the unit before is read
    if (c32 < M) {
      float* o = &mo[wave][c32][4 * half];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<f32x4*>(o + 32 * c + 8 * q4) =
              f32x4{O[c][q4 * 4], O[c][q4 * 4 + 1], O[c][q4 * 4 + 2], O[c][q4 * 4 + 3]};
      if (half == 0) {
        ml[wave][0][c32] = m;
        ml[wave][1][c32] = l;
      }
    }
    __syncthreads();
    for (int i = tid; i < M * (D / 4); i += 256) {
      const int c = i / (D / 4), d = i % (D / 4) * 4;
      float top = ml[0][0][c];
#pragma unroll
      for (int w = 1; w < W; ++w) top = fmaxf(top, ml[w][0][c]);
      const float mu = top == neg_inf() ? 0.0f : top;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float z = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float e = exp2_fast(ml[w][0][c] - mu);
        z = fmaf(ml[w][1][c], e, z);
        const f32x4 x = *reinterpret_cast<const f32x4*>(&mo[w][c][d]);
        o += x * e;
      }
      if (slot < 0) {
        finish(a, hk * a.G + c % a.G, un.start + c / a.G, d, o, top, z);
      } else {
        const int64_t at = (int64_t)slot * a.cols + c;
        *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = o;
        if (d == 0) {
          a.part_ml[2 * at] = top;
          a.part_ml[2 * at + 1] = z;
        }
      }
    }
  });
}

// k_paged_many: units of 32 WQ columns, 32 a wave.  The waves stage tiles of two blocks (64
// tokens) together: 8-bit pieces from memory to registers a tile ahead, widened once into
// LDS, where a fragment is a run of 1 KB.
template <int D, int WQ>
__global__ __launch_bounds__(64 * WQ, 2) void k_paged_many(PagedAttendArgs a) {
  constexpr int KST = D / 16, NC = D / 32, BM = 32 * WQ, SUBS = WQ / 4, NCH = NC / SUBS;
  constexpr int KB = 2 * KST * 64, TB = 2 * KB;        // 16-byte pieces of a tile's keys, of a tile
  static_assert(NCH >= 1);
  __shared__ __align__(16) u32x4 ring[2][TB];
  __shared__ float4 meta[2][2];                         // score scale, log 2 and inverse of the value scale, valid
  __shared__ int pre[kPagedUnits + 1];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31, wave = uniform(tid >> 6);
  const int su = (wave >> 1) & 1, sub = wave >> 2;      // staging: block su of a tile, its keys or its values
  const bool values = wave & 1;
  for_share<64 * WQ>(a, BM, 2, pre, [&](int hk, const Unit& un, int first, int cnt, int slot) {
    const int c = un.c0 + wave * 32 + c32, cc = min(c, un.M - 1), tok = cc / a.G, head = hk * a.G + cc - tok * a.G;
    const int last = un.L - un.n + tok, lowest = a.window > 0 ? last - a.window + 1 : 0;
    const int full = uniform(un.L / B), open_rows = uniform(un.L % B), b_at = uniform(un.b_lo + 2 * first);
    // tokens that every column of the unit sees: w_lo .. p_lo
    const int p_lo = uniform(un.L - un.n + un.c0 / a.G);
    const int w_lo = uniform(a.window > 0 ? un.L - un.n + (min(un.M, un.c0 + BM) - 1) / a.G - a.window + 1 : 0);
    const int sl = uniform(a.c.slots[un.s]);
    const bool has_slot = (unsigned)sl < (unsigned)a.c.n_slots;
    const int32_t* table = a.c.tables + (int64_t)un.s * a.c.width;
    u32x4 qf[KST];
    {
      const uint16_t* q = a.q.p + head * a.q.hs + (int64_t)(un.start + tok) * a.q.ts;
#pragma unroll
      for (int i = 0; i < KST; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + ((i >> 1) * 2 + half) * 16 + 8 * (i & 1));
    }
    f32x16 O[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) O[i] = f32x16{};
    float m = neg_inf(), l = 0.0f;

    u32x4 raw[NCH];
    float rk = 0.0f, rv = 1.0f;
    int rid = -1;
    // this wave's pieces of tile t, to registers
    auto fetch = [&](int t) {
      const int b = b_at + 2 * t + su;
      rid = b < full ? uniform(table[b]) : -1;
      if ((unsigned)rid >= (unsigned)a.c.n_pages) rid = -1;
      if (rid < 0) return;
      const int64_t at = (int64_t)rid * a.c.Hk + hk;
      const u32x4* src = reinterpret_cast<const u32x4*>((values ? a.c.v8 : a.c.k8) + at * (B * D)) + sub * NCH * 64 + lane;
#pragma unroll
      for (int i = 0; i < NCH; ++i) raw[i] = src[i * 64];
      rk = a.c.ks[at];
      rv = a.c.vs[at];
    };
    // and widened to LDS
    auto stage = [&](int t) {
      const int b = b_at + 2 * t + su;
      u32x4* buf = ring[t & 1];
      const bool open = b == full && open_rows > 0 && has_slot;
      const int64_t at = (((int64_t)(has_slot ? sl : 0) * 2 + (full & 1)) * a.c.Hk + hk) * (B * D);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int ch = sub * NCH + i;
        u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
        if (rid >= 0) {
          x = widen(raw[i][0], raw[i][1]);
          y = widen(raw[i][2], raw[i][3]);
        } else if (open) {
          if (values) {
            x = open_value<D>(a.c.ov + at, ch, 0, lane, open_rows);
            y = open_value<D>(a.c.ov + at, ch, 1, lane, open_rows);
          } else {
            x = open_key<D>(a.c.ok + at, 2 * ch, lane, open_rows);
            y = open_key<D>(a.c.ok + at, 2 * ch + 1, lane, open_rows);
          }
        }
        u32x4* to = buf + (values ? KB : 0) + (su * KST + 2 * ch) * 64 + lane;
        to[0] = x;
        to[64] = y;
      }
      if (!values && sub == 0 && lane == 0)
        meta[t & 1][su] = rid >= 0 ? make_float4(rk * a.c1, log2_fast(rv), 1.0f / rv, 1.0f)
                                   : make_float4(a.c1, 0.0f, 1.0f, open ? 1.0f : 0.0f);
    };

    __syncthreads();                  // the unit before is read
    fetch(0);
    stage(0);
    if (cnt > 1) fetch(1);
    __syncthreads();
    for (int t = 0; t < cnt; ++t) {
      const u32x4* buf = ring[t & 1] + lane;
      f32x16 S[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        S[u] = f32x16{};
#pragma unroll
        for (int i = 0; i < KST; ++i) S[u] = mfma32(buf[(u * KST + i) * 64], qf[i], S[u]);
      }
      float v[32], lv[2], rs[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float4 x = meta[t & 1][u];
        lv[u] = x.y;
        rs[u] = x.z;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[u * 16 + i] = S[u][i] * x.x;
        const int b = b_at + 2 * t + u;
        if (b * B + B - 1 > p_lo || b * B < w_lo) hide(v + u * 16, b, half, last, lowest);
        if (x.w == 0.0f) {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[u * 16 + i] = neg_inf();
        }
      }
      u32x4 pb[4];
      softmax_step<2, NC>(v, lv, rs, m, l, O, pb);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int i = 0; i < NC; ++i) O[i] = mfma32(buf[KB + (u * KST + 2 * i + w) * 64], pb[u * 2 + w], O[i]);
      if (t + 1 < cnt) {
        stage(t + 1);
        if (t + 2 < cnt) fetch(t + 2);
      }
      __syncthreads();
    }
    l += other_half(l);
    if (c >= un.M) return;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 o = {O[i][q4 * 4], O[i][q4 * 4 + 1], O[i][q4 * 4 + 2], O[i][q4 * 4 + 3]};
        const int d = 32 * i + 8 * q4 + 4 * half;
        if (slot < 0) {
          finish(a, head, un.start + tok, d, o, m, l);
        } else {
          const int64_t at = (int64_t)slot * a.cols + (c - un.c0);
          *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = o;
          if (d == 0) {
            a.part_ml[2 * at] = m;
            a.part_ml[2 * at + 1] = l;
          }
        }
      }
  });
}

// k_paged_join: the parts of a unit's columns, brought to one maximum and added in order.
template <int D>
__global__ __launch_bounds__(256) void k_paged_join(PagedAttendArgs a, int bm, int round) {
  constexpr int L4 = D / 4, ROWS = 256 / L4;
  const int hk = blockIdx.x / a.units, u = blockIdx.x % a.units;
  const int64_t share = a.plan[0], one = a.plan[1 + a.units];
  const int64_t x0 = hk * one + a.plan[1 + u], x1 = hk * one + a.plan[2 + u];
  if (x0 == x1) return;
  const int64_t g0 = x0 / share, g1 = (x1 - 1) / share;
  if (g0 == g1) return;
  const Unit un = unit_of(a, u, bm, round);
  const int c = blockIdx.y * ROWS + threadIdx.x / L4, d = threadIdx.x % L4 * 4;
  if (c >= min(bm, un.M - un.c0)) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = neg_inf(), l = 0.0f;
  for (int64_t g = g0; g <= g1; ++g) {
    const int64_t at = (2 * g + (g * share >= x0 ? 0 : 1)) * a.cols + c;
    const float pm = a.part_ml[2 * at], pl = a.part_ml[2 * at + 1];
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + at * D + d);
    const float top = fmaxf(m, pm), mu = top == neg_inf() ? 0.0f : top;
    const float wa = exp2_fast(m - mu), wb = exp2_fast(pm - mu);
    o = o * wa + x * wb;
    l = l * wa + pl * wb;
    m = top;
  }
  const int col = un.c0 + c;
  finish(a, hk * a.G + col % a.G, un.start + col / a.G, d, o, m, l);
}

template <int D>
hipError_t attend_impl(const PagedAttendArgs& a, const PagedAttendPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)(a.n_wg ? a.n_wg : a.units * a.c.Hk));
  if (p.shape == 0) hipLaunchKernelGGL((k_paged_few<D>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_paged_many<D, 4>), grid, dim3(256), 0, st, a);
  if (a.n_wg) {
    const int bm = p.shape == 0 ? 32 : 128, rows = 256 / (D / 4);
    hipLaunchKernelGGL((k_paged_join<D>), dim3((unsigned)(a.units * a.c.Hk), (unsigned)((a.cols + rows - 1) / rows)),
                       dim3(256), 0, st, a, bm, p.shape == 0 ? 1 : 2);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int D, hipStream_t st) {
  const dim3 grid((unsigned)((a.N + B - 1) / B), (unsigned)((a.heads + kRotateHeads - 1) / kRotateHeads));
  if (D == 128) hipLaunchKernelGGL((k_rotate<128>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_rotate<64>), grid, dim3(128), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, int D, hipStream_t st) {
  const int qg = a.q.p ? (a.Hq + kRotateHeads - 1) / kRotateHeads : 0;
  const dim3 grid((unsigned)a.items, (unsigned)(a.c.Hk + qg));
  if (D == 128) hipLaunchKernelGGL((k_paged_append<128>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_paged_append<64>), grid, dim3(128), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_attend(const PagedAttendArgs& a, const PagedAttendPlan& p, int D, hipStream_t st) {
  return D == 128 ? attend_impl<128>(a, p, st) : attend_impl<64>(a, p, st);
}

}  // namespace ss
