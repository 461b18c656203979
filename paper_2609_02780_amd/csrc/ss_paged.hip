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
// exact in bf16 and in fp16, so the products are MFMAs of these with fp32 sums (bf16 where
// reading the pages bounds, fp16 where the products do); a key scale meets the scores, a
// value scale joins the exponent of p.
#include "ss_paged.h"

#include <algorithm>
#include <type_traits>

namespace ss {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
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

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}

// A page's 16-byte pieces, read once (past the caches); of no page zeros, without a trip to memory.
constexpr int kAuxNT = 2;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_bytes(const uint8_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 load_shared(__amdgpu_buffer_rsrc_t r, int at) {     // other blocks read it too
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
}
__device__ __forceinline__ u32x4 load_piece(__amdgpu_buffer_rsrc_t r, int at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kAuxNT));
}

__device__ __forceinline__ f32x16 mfma_half(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Eight e4m3 as fp16 (exact).
__device__ __forceinline__ u32x4 widen_half(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
               __builtin_bit_cast(uint32_t, d)};
}

// Eight e4m3 times a power of two as bf16 (exact).
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
               __builtin_bit_cast(uint32_t, d)};
}

__device__ __forceinline__ float bf16_at(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ int span_start(const Spans& s, int i) { return s.uniform ? i * s.uniform : s.start[i]; }
__device__ __forceinline__ int span_start(const EvenSpans& s, int i) { return i * s.uniform; }

// A stream's tokens, by what its table can hold.
__device__ __forceinline__ int stream_length(const PagedDev& c, int s) {
  return max(0, min(c.lengths[s], c.width * B + (B - 1)));
}

// ---------------------------------------------------------------------------
// Rotation.  cos and sin of a block's tokens are formed once for all its heads: the angle
// in turns, position * (f / 2 pi), in 64 bits (a far position times a frequency loses what
// matters in 32), less the nearest quarter turn, still in 64, and of the rest the Taylor series of sine and
// cosine (x up to pi / 4).  Queries, which are rounded to bf16 and multiplied, take it in 32 bits, cut behind x^9 and
// x^10 (off by less than 2^-28); keys that are cached, which a rounding the other way would keep so, in 64 bits, cut
// behind x^13 and x^12 (2^-41; an append of 8,192 tokens 31.8 -> 32.9 us), then rounded to fp32 and from there to bf16
// (two roundings: one element in some 2^17, all but half way between two bf16, goes the other way).  (64 bits for all: 1,777
// tokens of 16 heads 7.6 -> 9.1 us.  The hardware's sine and cosine, off by 2^-22.9, save nothing that the rows' traffic
// does not cover.)
//
// A thread takes 16 elements of a row as two groups of 8, so that what it loads is what it
// writes: both elements of eight pairs (i, i + dims / 2) where the groups lie on 16 bytes; else
// 16 side by side, where pairs of neighbours are.  (Other odd sizes read the other elements one by one.)
// ---------------------------------------------------------------------------
constexpr int kMaxPairs = 64;
template <class T> struct PairOf;
template <> struct PairOf<float> { using type = float2; };
template <> struct PairOf<double> { using type = double2; };
template <int ROWS, class T>
struct Angles {
  typename PairOf<T>::type cs[ROWS][kMaxPairs * 32 / ROWS + 1];      // gain cos, gain sin; 64 rows of d = 64, 32 of d = 128
};

// cos and sin of x quarters of a turn, |x| <= 1 / 2.
__device__ __forceinline__ void cos_sin(double quarters, float& c, float& s) {
  const float x = (float)quarters * 1.57079632679489662f, z = x * x;
  c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
}
__device__ __forceinline__ void cos_sin(double quarters, double& c, double& s) {
  const double x = quarters * 1.57079632679489662, z = x * x;
  c = fma(z, fma(z, fma(z, fma(z, fma(z, fma(z, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24),
                 -0.5), 1.0);
  s = fma(x * z, fma(z, fma(z, fma(z, fma(z, fma(z, 1.0 / 6227020800, -1.0 / 39916800), 1.0 / 362880), -1.0 / 5040),
                            1.0 / 120), -1.0 / 6), x);
}
// Rows [r0, r1) of the table; token r's position is positions[first + r] or pos0 + r.
template <int ROWS, class T>
__device__ __forceinline__ void fill_angles(Angles<ROWS, T>& g, const Turn& t, int r0, int r1, int first, int64_t pos0) {
  const int half = t.dims >> 1, lg = 32 - __clz(half - 1);      // 2^lg threads a token
  const int j = threadIdx.x & ((1 << lg) - 1);
  if (j >= half) return;
  const double f = t.freqs[j];
  for (int r = r0 + (threadIdx.x >> lg); r < r1; r += blockDim.x >> lg) {
    const int64_t pos = t.positions ? t.positions[first + r] : pos0 + r;
    const double quarters = (double)pos * f * 4.0, q = rint(quarters);
    T c, s;
    cos_sin(quarters - q, c, s);
    const int k = (int)(q - 4.0 * floor(q * 0.25));               // quarter turns, 0 .. 3
    if (k & 1) {
      const T y = c;
      c = -s;
      s = y;
    }
    if (k & 2) {
      c = -c;
      s = -s;
    }
    g.cs[r][j] = {t.gain * c, t.gain * t.sign * s};
  }
}

// The two groups of item p: elements e0 .. e0 + 7 and e1 .. e1 + 7.
struct Groups {
  int e0, e1;
};
__device__ __forceinline__ Groups groups_of(const Turn& t, int p) {
  const int half = t.dims >> 1;
  if (!t.interleaved && (half & 7) == 0 && 8 * p < half) return {8 * p, half + 8 * p};
  return {16 * p, 16 * p + 8};
}
struct Raw {
  u32x4 a, b;
};
__device__ __forceinline__ Raw load_groups(const uint16_t* x, Groups g) {
  return {*reinterpret_cast<const u32x4*>(x + g.e0), *reinterpret_cast<const u32x4*>(x + g.e1)};
}
__device__ __forceinline__ void as_floats(const Raw& v, float (&y)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(v.a[i] << 16);
    y[2 * i + 1] = __uint_as_float(v.a[i] & 0xFFFF0000u);
    y[8 + 2 * i] = __uint_as_float(v.b[i] << 16);
    y[8 + 2 * i + 1] = __uint_as_float(v.b[i] & 0xFFFF0000u);
  }
}
// x: the row (read again only where its pairs lie across 16 bytes).
template <class T2>
__device__ __forceinline__ void turn_groups(const uint16_t* x, const Raw& v, Groups g, const T2* cs, const Turn& t,
                                            float (&y)[16]) {
  using T = decltype(cs->x);
  as_floats(v, y);
  const int half = t.dims >> 1;
  if (g.e0 >= t.dims) return;
  if (t.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (g.e0 + 2 * i < t.dims) {
        const T2 w = cs[g.e0 / 2 + i];
        const T e = y[2 * i], o = y[2 * i + 1];
        y[2 * i] = (float)(e * w.x - o * w.y);
        y[2 * i + 1] = (float)(o * w.x + e * w.y);
      }
    }
  } else if ((half & 7) == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T2 w = cs[g.e0 + i];
      const T e = y[i], o = y[8 + i];
      y[i] = (float)(e * w.x - o * w.y);
      y[8 + i] = (float)(o * w.x + e * w.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = g.e0 + i;
      if (at < t.dims) {
        const bool low = at < half;
        const T2 w = cs[low ? at : at - half];
        const T e = y[i], o = bf16_at(x[low ? at + half : at - half]);
        y[i] = (float)(e * w.x + o * (low ? -w.y : w.y));
      }
    }
  }
}
__device__ __forceinline__ bf16x8 eight(const float* y) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)y[i];
  return v;
}
__device__ __forceinline__ void store_groups(uint16_t* p, Groups g, const float (&y)[16]) {
  *reinterpret_cast<bf16x8*>(p + g.e0) = eight(y);
  *reinterpret_cast<bf16x8*>(p + g.e1) = eight(y + 8);
}

// Rotates row `at` of heads h0 .. h1 - 1 (at most N): all loads first.
// x and out may be one: a thread writes what it has read, and where another reads it too (pairs across 16 bytes),
// `apart` orders the two.
template <int N>
__device__ __forceinline__ void turn_heads(const RowsView& x, const RowsView& out, int64_t at, int h0, int h1, int p,
                                           bool live, const float2* cs, const Turn& t, bool apart) {
  const Groups g = groups_of(t, p);
  Raw v[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (live && h0 + i < h1) v[i] = load_groups(x.p + (h0 + i) * x.hs + at * x.ts, g);
  __syncthreads();                                 // the angles are there
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int h = h0 + i;
    float y[16];
    if (live && h < h1) turn_groups(x.p + h * x.hs + at * x.ts, v[i], g, cs, t, y);
    if (apart) __syncthreads();
    if (live && h < h1) store_groups(const_cast<uint16_t*>(out.p) + h * out.hs + at * out.ts, g, y);
  }
}
__device__ __forceinline__ bool pairs_across(const Turn& t) { return t.dims > 0 && !t.interleaved && ((t.dims >> 1) & 7) != 0; }

// k_rotate: a block takes 32 tokens (64 at d = 64) and H heads.  Bound by reading and writing the
// rows: 8,192 tokens of 28 heads of 128 (118 MB), 21 us, 5.6 TB/s, a little above the rate of a large copy.
template <int D, int H>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a) {
  constexpr int P = D / 16, ROWS = 256 / P;
  __shared__ Angles<ROWS, float> g;
  const int t0 = blockIdx.x * ROWS, n = min(ROWS, a.N - t0), r = threadIdx.x / P;
  fill_angles(g, a.turn, 0, n, t0, t0);
  turn_heads<H>(a.x, a.out, t0 + r, blockIdx.y * H, min(a.heads, (int)(blockIdx.y + 1) * H), threadIdx.x % P, r < n,
                g.cs[r], a.turn, pairs_across(a.turn));
}

// ---------------------------------------------------------------------------
// k_paged_append: a block takes the tokens of one cache block of a stream and one KV
// head (its keys and values) or some query heads.  Rows of a full block are rounded to
// e4m3 with one scale; rows of the stream's open blocks stay bf16.  Bound by reading and writing
// rows: 8,192 tokens of 4 KV heads with the rotation of 28 query heads (143 MB), 32.9 us, 4.3 TB/s; a token of
// each of 64 streams 6.2 us, of one 3.3.
// ---------------------------------------------------------------------------
constexpr float kLeastMax = 0x1p-100f;    // 448 / it stays finite

__device__ __forceinline__ uint32_t pack8(float a, float b, float c, float d) {
  int r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

// Where element e of token r lies in a block of values.
__device__ __forceinline__ int value_place(int r, int e) {
  const int w = ((r >> 4) & 1) | ((r >> 3) & 1) << 1;
  return (((e >> 5) * 2 + ((r >> 2) & 1)) * 32 + (e & 31)) * 16 + w * 4 + (r & 3);
}

template <int D, int H, class SP>
__global__ __launch_bounds__(2 * D) void k_paged_append(PagedAppendArgs a, SP spans) {
  constexpr int P = D / 16;
  __shared__ Angles<32, double> g;
  __shared__ __align__(16) uint16_t vt[B][D + 8];
  __shared__ float part[8];
  const int tid = threadIdx.x, p = tid % P;
  // the stream and which of its touched blocks: (n + 62) / 32 at most, wherever the old tokens end
  int s, k;
  if (std::is_same_v<SP, EvenSpans>) {
    const int per = (spans.uniform + 2 * B - 2) / B;
    s = blockIdx.x / per;
    k = blockIdx.x % per;
  } else {
    s = 0;
    int first = 0;
    for (;; ++s) {
      const int n = span_start(spans, s + 1) - span_start(spans, s);
      const int per = n > 0 ? (n + 2 * B - 2) / B : 0;
      if ((int)blockIdx.x < first + per) break;
      first += per;
    }
    k = blockIdx.x - first;
  }
  const int start = span_start(spans, s), n = span_start(spans, s + 1) - start;
  const int L = stream_length(a.c, s), old = L - n, b0 = max(old, 0) / B, last = (L - 1) / B;
  int b = b0 + k;
  if (L == 0 || b > last) return;
  const int slot = a.c.slots[s];
  const bool has_slot = (unsigned)slot < (unsigned)a.c.n_slots;
  const bool keys = (int)blockIdx.y < a.c.Hk;
  if (!keys) {
    const int t0 = max(max(old, 0), B * b), t1 = min(L, B * (b + 1)), i = tid / P;
    auto& gq = reinterpret_cast<Angles<32, float>&>(g);
    if (a.turn.dims) fill_angles(gq, a.turn, t0 - B * b, t1 - B * b, start + B * b - old, (int64_t)B * b);
    const int h0 = (blockIdx.y - a.c.Hk) * H;
    turn_heads<H>(a.q, a.q_out, start + (t0 - old) + i, h0, min(a.Hq, h0 + H), p, t0 + i < t1,
                  gq.cs[(t0 - B * b + i) & 31], a.turn, pairs_across(a.turn));
    return;
  }
  // A token's open rows lie in buffer block & 1.  Where the last block's buffer is the one that
  // the first block reads, the first block's own thread block writes it, after reading.
  const bool shared = last > b0 && ((last - b0) & 1) == 0;
  const int h = blockIdx.y, r = tid / P;
  const Groups e = groups_of(a.turn, p);
  for (int job = 0; job < 2; ++job) {
    if (job == 1) {
      if (!(shared && b == b0)) return;
      b = last;
      __syncthreads();
    }
    const int t0 = max(max(old, 0), B * b), t1 = min(L, B * (b + 1));    // new tokens of this block
    const int t = B * b + r;
    const bool fresh = t >= t0 && t < t1;
    const int64_t row = start + t - old;                                   // of the call's tokens
    const uint16_t *kp = a.k.p + h * a.k.hs + row * a.k.ts, *vp = a.v.p + h * a.v.hs + row * a.v.ts;
    const bool full = job == 0 && t1 == B * (b + 1);
    const bool stays = has_slot && (job == 1 || (b == last && !shared) || (b == last && b == b0) ||
                                    (b == b0 && ((last - b0) & 1) == 1));
    const int64_t open_at = (((int64_t)slot * 2 + (b & 1)) * a.c.Hk + h) * B * D;
    Raw kr, vr;
    if (fresh) {
      kr = load_groups(kp, e);
      vr = load_groups(vp, {16 * p, 16 * p + 8});
    }
    if (a.turn.dims) fill_angles(g, a.turn, t0 - B * b, t1 - B * b, start + B * b - old, (int64_t)B * b);
    __syncthreads();
    float y[16], v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = v[i] = 0.0f;
    // bytes of a page (elements of an open block) from one piece of keys, 16 elements, to the next: 32 tokens of 16
    const int k0 = ((e.e0 >> 4) * B + r) * 16 + (e.e0 & 15), k1 = ((e.e1 >> 4) * B + r) * 16 + (e.e1 & 15);
    if (fresh) {
      turn_groups(kp, kr, e, g.cs[r], a.turn, y);
      as_floats(vr, v);
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = (float)(__bf16)y[i];
    } else if (full && t < t0 && has_slot) {
      kr = {*reinterpret_cast<const u32x4*>(a.c.ok + open_at + k0), *reinterpret_cast<const u32x4*>(a.c.ok + open_at + k1)};
      as_floats(kr, y);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = bf16_at(a.c.ov[open_at + value_place(r, 16 * p + i)]);
    }
    if (full) {
      float km = 0.0f, vm = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        km = fmaxf(km, fabsf(y[i]));
        vm = fmaxf(vm, fabsf(v[i]));
      }
      *reinterpret_cast<bf16x8*>(&vt[r][16 * p]) = eight(v);
      *reinterpret_cast<bf16x8*>(&vt[r][16 * p + 8]) = eight(v + 8);
      // the block's maxima, both at once (the barriers also show vt)
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) {
        km = fmaxf(km, __shfl_xor(km, x));
        vm = fmaxf(vm, __shfl_xor(vm, x));
      }
      if ((tid & 63) == 0) {
        part[2 * (tid >> 6)] = km;
        part[2 * (tid >> 6) + 1] = vm;
      }
      __syncthreads();
      km = vm = kLeastMax;
#pragma unroll
      for (int w = 0; w < 2 * D / 64; ++w) {
        km = fmaxf(km, part[2 * w]);
        vm = fmaxf(vm, part[2 * w + 1]);
      }
      const int page = a.c.tables[(int64_t)s * a.c.width + b];
      if ((unsigned)page < (unsigned)a.c.n_pages && (has_slot || t0 == B * b)) {
        const int64_t at = ((int64_t)page * a.c.Hk + h);
        const float ki = 448.0f / km, vi = 448.0f / vm;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack8(y[4 * i] * ki, y[4 * i + 1] * ki, y[4 * i + 2] * ki, y[4 * i + 3] * ki);
        uint8_t* kd = a.c.k8 + at * B * D;
        *reinterpret_cast<u32x2*>(kd + k0) = u32x2{w[0], w[1]};
        *reinterpret_cast<u32x2*>(kd + k1) = u32x2{w[2], w[3]};
        // values: a thread takes 16 tokens of one dimension
        const int m = tid & 31, half = (tid >> 5) & 1, d = (tid >> 6) * 32 + m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = 8 * ((i >> 1) | ((i & 1) << 1)) + 4 * half;
          w[i] = pack8(bf16_at(vt[tok][d]) * vi, bf16_at(vt[tok + 1][d]) * vi, bf16_at(vt[tok + 2][d]) * vi,
                       bf16_at(vt[tok + 3][d]) * vi);
        }
        *reinterpret_cast<u32x4*>(a.c.v8 + at * B * D + tid * 16) = u32x4{w[0], w[1], w[2], w[3]};
        if (tid == 0) {
          a.c.ks[at] = km / 448.0f;
          a.c.vs[at] = vm / 448.0f;
        }
      }
    }
    if (stays && fresh) {
      *reinterpret_cast<bf16x8*>(a.c.ok + open_at + k0) = eight(y);
      *reinterpret_cast<bf16x8*>(a.c.ok + open_at + k1) = eight(y + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) a.c.ov[open_at + value_place(r, 16 * p + i)] = to_bf16(v[i]);
    }
  }
}

// ---------------------------------------------------------------------------
// Attention.  A unit is a stream's run of BM query columns (column c: token c / G, head c % G of
// its KV head); its work are the blocks that some column sees, behind `start` places that stand for
// what beginning and ending a unit takes (without them a thread block that got the idle streams of a padded
// batch was the last by far).  All units' work, laid end to end over the KV heads, is cut into equal shares,
// one a thread block, so streams of any lengths fill the card alike; where no unit can be long, or units are
// more than kPagedUnits, each is a thread block's.  A block's first and last unit may be parts, joined by
// k_paged_join.
// ---------------------------------------------------------------------------
struct Unit {
  int s, n, start, L, c0, M;         // its columns c0 .. min(c0 + BM, M) - 1
  int b_lo, count;                   // first block, and how many (at least 1: someone writes the outputs); 0: no unit
};
// Where the streams' tokens begin, and their lengths, in LDS: one trip to memory for all.
struct Streams {
  int start[kPagedStreams + 1], length[kPagedStreams];
};
template <bool LENGTHS, class SP>
__device__ __forceinline__ void load_streams(const PagedAttendArgs& a, const SP& spans, Streams& t) {
  for (int i = threadIdx.x; i <= a.S; i += blockDim.x) {
    t.start[i] = span_start(spans, i);
    if (LENGTHS && i < a.S) t.length[i] = stream_length(a.c, i);
  }
  __syncthreads();
}
__device__ __forceinline__ int unit_first(const PagedAttendArgs& a, const Streams& t, int s, int bm) {
  return a.per ? s * a.per : a.G * t.start[s] / bm + s;
}
// A unit's columns, which take no lengths.
__device__ __forceinline__ Unit columns_of(const PagedAttendArgs& a, const Streams& t, int u, int bm) {
  Unit x;
  if (a.per) {
    x.s = u / a.per;
  } else {
    int lo = 0, hi = a.S - 1;        // the last stream that begins at u or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (unit_first(a, t, mid, bm) <= u) lo = mid;
      else hi = mid - 1;
    }
    x.s = lo;
  }
  x.start = t.start[x.s];
  x.n = t.start[x.s + 1] - x.start;
  x.M = a.G * x.n;
  x.c0 = (u - unit_first(a, t, x.s, bm)) * bm;
  x.L = 0;
  x.b_lo = x.count = 0;
  return x;
}
__device__ __forceinline__ Unit unit_of(const PagedAttendArgs& a, const Streams& t, int u, int bm, int round) {
  Unit x = columns_of(a, t, u, bm);
  if (x.c0 >= x.M) return x;
  x.L = t.length[x.s];
  const int p_lo = x.L - x.n + x.c0 / a.G;                                   // the first and the last column's tokens
  const int p_hi = x.L - x.n + (min(x.M, x.c0 + bm) - 1) / a.G;
  const int lowest = a.window > 0 ? max(0, p_lo - a.window + 1) : 0;
  x.b_lo = round == 2 ? (lowest / B) & ~1 : lowest / B;
  x.count = p_hi < 0 ? 1 : max(1, round == 2 ? (p_hi / B - x.b_lo + 2) >> 1 : p_hi / B - x.b_lo + 1);
  return x;
}

// A unit's work; that of no unit is none.
__device__ __forceinline__ int work_of(const PagedAttendArgs& a, const Unit& x) { return x.count > 0 ? a.start + x.count : 0; }

// pre[u]: the work before unit u (pre[units]: all of it).
template <int T>
__device__ __forceinline__ void plan_units(const PagedAttendArgs& a, const Streams& t, int bm, int round, int* pre) {
  __shared__ int part[T / 64];
  const int tid = threadIdx.x, run = (a.units + T - 1) / T, u0 = min(a.units, tid * run), u1 = min(a.units, u0 + run);
  int sum = 0;
  for (int u = u0; u < u1; ++u) sum += work_of(a, unit_of(a, t, u, bm, round));
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
    at += work_of(a, unit_of(a, t, u, bm, round));
  }
  if (tid == T - 1) pre[a.units] = at;
  __syncthreads();
}

// The share of a block, the same in k_paged_join.
__device__ __forceinline__ int64_t share_of(const PagedAttendArgs& a, int64_t all) {
  return max((all + a.n_wg - 1) / a.n_wg, (int64_t)a.min_share);
}

// Calls work(kv head, unit, first of its blocks, how many, slot of the part or -1) for a block's share.
template <int T, class SP, class F>
__device__ __forceinline__ void for_share(const PagedAttendArgs& a, const SP& spans, int bm, int round, int* pre, F&& work) {
  int wg = blockIdx.x;
  // neighbouring shares, which read the same pages, on one XCD (blocks go round them)
  if (a.n_wg != 0 && wg < a.n_wg / 8 * 8) wg = (wg & 7) * (a.n_wg / 8) + (wg >> 3);
  int64_t one = 1, x = 0, end = 1;
  __shared__ Streams streams;
  load_streams<true>(a, spans, streams);
  if (a.n_wg != 0) {
    plan_units<T>(a, streams, bm, round, pre);
    one = pre[a.units];
    const int64_t all = one * a.c.Hk, share = share_of(a, all);
    if (wg == 0) {
      if (threadIdx.x == 0) a.plan[0] = (int)share;
      for (int u = threadIdx.x; u <= a.units; u += T) a.plan[1 + u] = pre[u];
    }
    x = wg * share;
    end = min(all, x + share);
  }
  for (int side = 0; x < end; side = 1) {                // (one call of work: it is inlined)
    // (a block a unit: a head's on few XCDs, the last units, which may see the most, first)
    int hk = wg % a.c.Hk, u = a.units - 1 - wg / a.c.Hk, first = 0, y = 0;
    if (a.n_wg != 0) {
      hk = (int)(x / one);
      y = (int)(x % one);
      int lo = 0, hi = a.units - 1;                      // the last unit whose work begins at y or before
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pre[mid] <= y) lo = mid;
        else hi = mid - 1;
      }
      u = lo;
      y -= pre[u];
    }
    u = uniform(u);
    const Unit un = unit_of(a, streams, u, bm, round);
    int cnt = un.count, slot = -1;
    if (a.n_wg == 0) {
      if (cnt == 0) return;
      x = end;
    } else {
      // places y .. to - 1 of the unit; a share that ends among the first `start` leaves all blocks to the next
      const int to = (int)min((int64_t)(a.start + un.count), y + (end - x));
      x += to - y;
      first = max(0, y - a.start);
      cnt = max(0, to - a.start) - first;
      if (cnt == 0) return;
      if (cnt != un.count) slot = 2 * wg + side;
    }
    work(uniform(hk), un, uniform(first), uniform(cnt), uniform(slot));
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
  if (d == 0 && a.lse) {
    // (the exponent of l apart: where values are tiny m and log2 l are far from 0 on either side, and steps there wide)
    float z = neg_inf();
    if (l > 0.0f) z = (m + (float)__builtin_amdgcn_frexp_expf(l) + log2_fast(__builtin_amdgcn_frexp_mantf(l))) * kLn2;
    a.lse[(int64_t)h * a.N + at] = z;
  }
}

// exp2 of scores against m, as the second product's operand takes them.  v: scores in units of log 2; lvs: log 2
// of the block's value scale, which p takes on (so values need no scaling), rvs: 1 / that scale.
// m moves only when it has to: as long as a lane's p add up to at most 2^13, fp32 sums and bf16 p are
// as good against an older, smaller m.  O is rescaled when m moves.  form(mu) forms all p against mu and
// returns their sum without the value scale; top(): the largest score of the column.
template <class Form, class Top, class Scale>
__device__ __forceinline__ void running_softmax(float& m, float& l, Form&& form, Top&& top, Scale&& rescale) {
  float sum = form(m == neg_inf() ? 0.0f : m);
  if (__any(!(sum <= 8192.0f) || m == neg_inf())) {
    const float mn = fmaxf(m, top());
    const float al = m == neg_inf() ? 0.0f : exp2_fast(m - mn);
    m = mn;
    l *= al;
    rescale(al);
    sum = form(m == neg_inf() ? 0.0f : m);
  }
  l += sum;
}

// The same for p in fp16: form(mu) returns the sum of p with the value scale, which has to stay in its range, and the
// one without; top() is the largest of the scores with it.
template <class Form, class Top, class Scale>
__device__ __forceinline__ void running_softmax_half(float& m, float& l, Form&& form, Top&& top, Scale&& rescale) {
  float2 sum = form(m == neg_inf() ? 0.0f : m);
  if (__any(!(sum.x <= 32768.0f) || m == neg_inf())) {
    const float mn = fmaxf(m, top() - 9.0f);
    const float al = m == neg_inf() ? 0.0f : exp2_fast(m - mn);
    m = mn;
    l *= al;
    rescale(al);
    sum = form(m == neg_inf() ? 0.0f : m);
  }
  l += sum.y;
}

// A value scale is cut in two: p takes what lies in 2^-60 .. 2^60, the conversion of the
// codes the rest, a power of two (blocks of zeros have the least scale, and their p must still count).
struct ValueScale {
  float log2, inverse, codes;
};
// (a scale below what the library writes, 0 among them, as that)
__device__ __forceinline__ float at_least(float scale) { return fmaxf(scale, 0x1p-109f); }
__device__ __forceinline__ ValueScale cut_scale(float scale) {
  const float vs = at_least(scale);
  const int e = (int)(__float_as_uint(vs) >> 23) - 127;
  const int k = e < -60 ? e + 60 : e > 60 ? e - 60 : 0;
  const float in_p = vs * __uint_as_float((uint32_t)(127 - k) << 23);
  return {log2_fast(in_p), 1.0f / in_p, __uint_as_float((uint32_t)(127 + k) << 23)};
}

// A lane's pieces of an open block: rows from cnt on are zero.
__device__ __forceinline__ u32x4 open_key(const uint16_t* base, int piece, int token, int x, int cnt) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(base + (piece * B + token) * 16 + 8 * x);
  return token < cnt ? v : u32x4{0, 0, 0, 0};
}
// 8 tokens of one dimension: words 2 y and 2 y + 1 of [c][h][m].
__device__ __forceinline__ u32x4 open_masked(u32x4 v, int h, int y, int cnt) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = 8 * y + 16 * (i >> 1) + 4 * h + 2 * (i & 1);
    v[i] &= (tok < cnt ? 0xFFFFu : 0u) | (tok + 1 < cnt ? 0xFFFF0000u : 0u);
  }
  return v;
}
__device__ __forceinline__ u32x4 open_value(const uint16_t* base, int c, int h, int m, int y, int cnt) {
  return open_masked(*reinterpret_cast<const u32x4*>(base + ((c * 2 + h) * 32 + m) * 16 + 8 * y), h, y, cnt);
}
// The largest magnitude of eight bf16, as bits, and the power of two that lifts it to 2^7 (2^least and less: as that).
__device__ __forceinline__ uint32_t largest(u32x4 v) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(v[i] & 0x7FFFu, (v[i] >> 16) & 0x7FFFu));
  return top;
}
__device__ __forceinline__ int exponent_of(uint32_t top, int least) { return max((int)(top >> 7) - 127, least) - 7; }
// Eight bf16 times 2^-e as fp16.
__device__ __forceinline__ u32x4 halves(u32x4 v, int e) {
  f16x8 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = (_Float16)ldexpf(__uint_as_float(v[i] << 16), -e);
    x[2 * i + 1] = (_Float16)ldexpf(__uint_as_float(v[i] & 0xFFFF0000u), -e);
  }
  return __builtin_bit_cast(u32x4, x);
}

__device__ __forceinline__ float of_lane(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// k_paged_few: units of up to C columns (decoded tokens, a few drafts).  The W waves of a
// block take its 32-token blocks in turn, each straight from memory to registers, and join
// at the end of a unit.  Bound by reading the pages, so p is kept in two bf16 parts (16 bits
// of it): the second product twice costs nothing (the matrix unit is busy for 12% of the clocks).
// A token over 705,634 (723 MB) 113 us, 6.4 TB/s; for each of 64 streams (560 MB) 89 us, 6.3 TB/s; three for each of
// 16 streams 36.
// C = 16: 16x16x32 products.  Lane l = 16 g + r of S^T holds tokens 16 t + 4 g + e of column r;
// a load of 16 bytes a lane brings piece 4 j + g of token 16 t + r, or the values of dimension
// 32 c + 16 (g / 2) + r for half g & 1, of which the lanes 32 apart swap a half.
template <int D, int C, int W, class SP>
__global__ __launch_bounds__(64 * W, W == 4 ? 2 : 1) void k_paged_few(PagedAttendArgs a, SP spans) {
  constexpr bool WIDE = C == 32;
  constexpr int NL = D / 32;                     // 16-byte loads of a block's keys (values)
  constexpr int KST = WIDE ? D / 16 : D / 32;    // steps of the first product
  constexpr int NO = D / C, NV = C / 2, OS = D + 4, AHEAD = 1;
  using acc_t = std::conditional_t<WIDE, f32x16, f32x4>;
  __shared__ __align__(16) float mo[W][C][OS];
  __shared__ float ml[W][2][C];
  __shared__ int pre[kPagedUnits + 1];
  const int tid = threadIdx.x, lane = tid & 63, g = lane / C, r = lane % C, wave = uniform(tid >> 6);
  // token of score i in its block
  auto token_of = [&](int i) { return (WIDE ? 8 : 16) * (i >> 2) + 4 * g + (i & 3); };
  auto mma = [](u32x4 x, u32x4 y, acc_t z) -> acc_t {
    if constexpr (WIDE) return mfma32(x, y, z);
    else return mfma16(x, y, z);
  };
  // byte offsets of this lane's pieces in a page
  auto key_at = [&](int i) { return WIDE ? i * 1024 + lane * 16 : (4 * (i % (D / 64)) + g) * 512 + (16 * (i / (D / 64)) + r) * 16; };
  const int value_lane = WIDE ? lane * 16 : ((g & 1) * 32 + 16 * (g >> 1) + r) * 16;
  for_share<64 * W>(a, spans, C, 1, pre, [&](int hk, const Unit& un, int first, int cnt, int slot) {
    const int M = un.M, cc = min(r, M - 1), tok = cc / a.G, head = hk * a.G + cc - tok * a.G;
    const int last = un.L - un.n + tok, lowest = a.window > 0 ? last - a.window + 1 : 0;
    const int full = uniform(un.L / B), b_at = uniform(un.b_lo + first);
    const int n = (cnt - wave + W - 1) / W;                 // this wave's blocks: b_at + wave + W i
    // tokens that every column sees: w_lo .. p_lo
    const int p_lo = uniform(un.L - un.n), w_lo = uniform(a.window > 0 ? max(0, un.L - a.window) : 0);
    const int open_rows = un.L - full * B;
    const bool opens = open_rows > 0 && b_at + cnt - 1 == full && wave == ((cnt - 1) & (W - 1));   // the open block is this wave's
    const int sl = opens ? a.c.slots[un.s] : -1;
    u32x4 qf[KST];
    {
      const uint16_t* q = a.q.p + head * a.q.hs + (int64_t)(un.start + tok) * a.q.ts;
#pragma unroll
      for (int i = 0; i < KST; ++i)
        qf[i] = *reinterpret_cast<const u32x4*>(q + ((i >> 1) * (64 / C) + g) * 16 + 8 * (i & 1));
    }
    acc_t O[NO];
#pragma unroll
    for (int i = 0; i < NO; ++i) O[i] = acc_t{};
    float m = neg_inf(), l = 0.0f;

    // kf(i): keys WIDE [step], else [t][step]; vf(i): values [NO][1 or 2 steps]; more() once the keys are used
    constexpr int NK = WIDE ? KST : 2 * KST, NVF = WIDE ? 2 * NO : NO;
    auto step = [&](auto&& kf, auto&& vf, auto&& more, float cs, float lvs, float rvs, int b) {
      float v[NV];
      if constexpr (WIDE) {
        acc_t S = acc_t{};
#pragma unroll
        for (int i = 0; i < KST; ++i) S = mma(kf(i), qf[i], S);
        more();
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = S[i];
      } else {
        acc_t S[2] = {acc_t{}, acc_t{}};
#pragma unroll
        for (int i = 0; i < KST; ++i)
#pragma unroll
          for (int t = 0; t < 2; ++t) S[t] = mma(kf(t * KST + i), qf[i], S[t]);
        more();
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = S[i >> 2][i & 3];
      }
      if (b * B + B - 1 > p_lo || b * B < w_lo) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int j = b * B + token_of(i);
          if (j > last || j < lowest) v[i] = neg_inf();
        }
      }
      // words of p: groups of four tokens 0, 2 (and 1, 3) of WIDE, 0, 1 of the others
      u32x4 hi[NV / 8], lo[NV / 8];
      running_softmax(
          m, l,
          [&](float mu) {
            const float off = lvs - mu;
            float sum[4];
#pragma unroll
            for (int w = 0; w < NV / 8; ++w) {
              bf16x8 x, y;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int i = WIDE ? 4 * w + (e & 3) + 8 * (e >> 2) : e;
                const float p = exp2_fast(fmaf(v[i], cs, off));
                sum[e & 3] = w == 0 && e < 4 ? p : sum[e & 3] + p;
                x[e] = (__bf16)p;
                y[e] = (__bf16)(p - (float)x[e]);
              }
              hi[w] = __builtin_bit_cast(u32x4, x);
              lo[w] = __builtin_bit_cast(u32x4, y);
            }
            return ((sum[0] + sum[1]) + (sum[2] + sum[3])) * rvs;
          },
          [&]() {
            float top = v[0];
#pragma unroll
            for (int i = 1; i < NV; ++i) top = fmaxf(top, v[i]);
            top *= cs;
            if constexpr (!WIDE) top = fmaxf(top, __shfl_xor(top, 16));
            return fmaxf(top, other_half(top));
          },
          [&](float al) {
#pragma unroll
            for (int i = 0; i < NO; ++i) O[i] *= al;
          });
#pragma unroll
      for (int i = 0; i < NO; ++i)
#pragma unroll
        for (int w = 0; w < NV / 8; ++w) {
          const u32x4 x = vf(i * (NV / 8) + w);
          O[i] = mma(x, hi[w], O[i]);
          O[i] = mma(x, lo[w], O[i]);
        }
    };

    // The open block, its loads all at once.  It comes last, when the pages' registers are free (beside the first page's
    // loads its own cost 64 streams 3%).
    auto open_step = [&]() {
      const int at_slot = uniform(sl);
      if ((unsigned)at_slot >= (unsigned)a.c.n_slots) return;
      const int64_t at = (((int64_t)at_slot * 2 + (full & 1)) * a.c.Hk + hk) * (B * D);
      u32x4 kr[NK], vr[NVF];
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int t = WIDE ? 0 : i / KST, st = WIDE ? i : i % KST;
        kr[i] = open_key(a.c.ok + at, (st >> 1) * (64 / C) + g, 16 * t + r, st & 1, open_rows);
      }
#pragma unroll
      for (int i = 0; i < NVF; ++i)
        vr[i] = WIDE ? open_value(a.c.ov + at, i >> 1, g, r, i & 1, open_rows)
                     : open_value(a.c.ov + at, i >> 1, g & 1, 16 * (i & 1) + r, g >> 1, open_rows);
      step([&](int i) { return kr[i]; }, [&](int i) { return vr[i]; }, []() {}, a.c1, 0.0f, 1.0f, full);
    };

    for (int i0 = 0; i0 < n; i0 += 64) {
      // pages and scales of the next 64 blocks, one a lane
      int id = -1;
      float ksv = 0.0f;
      ValueScale vsv = {0.0f, 1.0f, 1.0f};
      {
        const int b = b_at + wave + W * (i0 + lane);
        if (i0 + lane < n && b < full) id = a.c.tables[(int64_t)un.s * a.c.width + b];
        if ((unsigned)id >= (unsigned)a.c.n_pages) id = -1;
      }
      const int k1 = min(64, n - i0);
      // AHEAD blocks ahead; behind the last one nothing is read, without a branch, so that waits are counted
      u32x4 kq[AHEAD][NL], vq[AHEAD][NL];
      auto page = [&](int k, int64_t& at) -> int {
        const int pid = k < k1 ? __builtin_amdgcn_readlane(id, k & 63) : -1;
        at = ((int64_t)max(0, pid) * a.c.Hk + hk) * (B * D);
        return pid < 0 ? 0 : B * D;
      };
      auto load_keys = [&](int64_t at, int bytes, u32x4 (&kr)[NL]) {
        const auto p = page_bytes(a.c.k8 + at, bytes);
#pragma unroll
        for (int i = 0; i < NL; ++i) kr[i] = load_piece(p, key_at(i));
      };
      auto load_values = [&](int64_t at, int bytes, u32x4 (&vr)[NL]) {
        const auto p = page_bytes(a.c.v8 + at, bytes);
#pragma unroll
        for (int i = 0; i < NL; ++i) vr[i] = load_piece(p, i * 1024 + value_lane);
      };
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        int64_t at;
        const int bytes = page(k, at);
        load_keys(at, bytes, kq[k]);
        load_values(at, bytes, vq[k]);
      }
      if (id >= 0) {
        ksv = at_least(a.c.ks[(int64_t)id * a.c.Hk + hk]) * a.c1;
        vsv = cut_scale(a.c.vs[(int64_t)id * a.c.Hk + hk]);
      }
      auto one = [&](int k, u32x4 (&kr)[NL], u32x4 (&vr)[NL]) {
        const float codes = of_lane(vsv.codes, k);
        int64_t at;
        const int bytes = page(k + AHEAD, at);
        if (__builtin_amdgcn_readlane(id, k) >= 0) {
          u32x4 half[2];
          step([&](int i) { return widen(kr[i >> 1][2 * (i & 1)], kr[i >> 1][2 * (i & 1) + 1], 1.0f); },
               [&](int i) {
                 const u32x4& x = vr[i >> 1];
                 if constexpr (WIDE) {
                   return widen(x[2 * (i & 1)], x[2 * (i & 1) + 1], codes);
                 } else {
                   if ((i & 1) == 0) {
                     const auto y = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
                     const auto z = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
                     half[0] = widen(y[0], z[0], codes);
                     half[1] = widen(y[1], z[1], codes);
                   }
                   return half[i & 1];
                 }
               },
               [&]() { load_keys(at, bytes, kr); }, of_lane(ksv, k), of_lane(vsv.log2, k), of_lane(vsv.inverse, k),
               b_at + wave + W * (i0 + k));
        } else {
          load_keys(at, bytes, kr);
        }
        load_values(at, bytes, vr);
      };
      for (int k = 0; k < k1; k += AHEAD) {
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
          if (k + x >= k1) break;
          one(k + x, kq[x], vq[x]);
        }
      }
    }
    open_step();
    if constexpr (!WIDE) l += __shfl_xor(l, 16);
    l += other_half(l);

    __syncthreads();                  // the unit before is read
    if (r < M) {
      float* o = &mo[wave][r][4 * g];
#pragma unroll
      for (int i = 0; i < NO; ++i)
#pragma unroll
        for (int q4 = 0; q4 < (WIDE ? 4 : 1); ++q4)
          *reinterpret_cast<f32x4*>(o + C * i + 8 * q4) =
              f32x4{O[i][q4 * 4], O[i][q4 * 4 + 1], O[i][q4 * 4 + 2], O[i][q4 * 4 + 3]};
      if (g == 0) {
        ml[wave][0][r] = m;
        ml[wave][1][r] = l;
      }
    }
    __syncthreads();
    for (int i = tid; i < M * (D / 4); i += 64 * W) {
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

// A lane's 16 keys of block b that its column (token `last`, the first seen `lowest`) does not see.
__device__ __forceinline__ void hide(float* v, int b, int half, int last, int lowest) {
  const int j0 = b * B + 4 * half;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = j0 + 8 * (i >> 2) + (i & 3);
    if (j > last || j < lowest) v[i] = neg_inf();
  }
}

// All waves of the block have come this far, and their LDS traffic is done (loads from memory may be under way).
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// k_paged_many: units of 32 WQ columns, 32 a wave.  The waves stage tiles of two blocks (64
// tokens) together: 8-bit pieces from memory to registers a tile ahead, widened once into
// LDS, where a fragment is a run of 1 KB.
// The products are of fp16: e4m3 is exact in it, and its 11 bits of p are off by an eighth of what bf16's 8 are,
// at the same cost.  What is bf16, queries and open rows, is brought into its range by a power of two that
// lifts the largest of a column (a block) to 2^7: exact, but for elements 2^21 times smaller.  p's range is kept by
// what m is: the largest score with its value scale, less 9, so that p reaches up to 2^9 (2^15 before m moves) and its
// steps are at most 2^-33 of the largest (less 12, m moves too often; less 6, 8 and 9 take the same time).  Value
// scales count as 2^-64 .. 2^40, so that fp32 holds the sums without them beside each other; the values of a block
// with a smaller one (values below 2^-55) count as zeros.
// WQ = 8: the two waves of a SIMD (w and w + 4) take turns: while one forms its softmax on the
// vector unit, the other keeps the matrix unit busy, half an iteration behind.  WQ = 4 (33 to 128
// columns): two blocks a CU, whose phases fall beside each other by themselves.
// Bound by the matrix unit (busy for 62% of the clocks) and the clock that the card's power leaves it: 4,096 tokens,
// the last of 16,384, 28 heads of 128: 739 us, 1.14 PFLOP/s.  At d = 64 by the vector unit's exponentials.
template <int D, int WQ>
__global__ __launch_bounds__(64 * WQ, D == 64 && WQ == 4 ? 3 : 2) void k_paged_many(PagedAttendArgs a, Spans spans) {
  constexpr bool TURNS = WQ == 8;
  constexpr int KST = D / 16, NC = D / 32, BM = 32 * WQ, SUBS = WQ / 4, NCH = NC / SUBS, NS = TURNS ? 4 : 2;
  constexpr int KB = 2 * KST * 64, TB = 2 * KB;        // 16-byte pieces of a tile's keys, of a tile
  static_assert(NCH >= 1);
  __shared__ __align__(16) u32x4 ring[NS][TB];
  __shared__ __align__(16) float2 meta[2][64][2];   // of a tile's blocks, 64 tiles at a time: key scale (0: not seen;
                                                    // negative: values count as zeros), log 2 of the value scale
  __shared__ int open_power[2];       // of the open block's keys, of its values
  __shared__ int pre[kPagedUnits + 1];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, c32 = lane & 31, wave = uniform(tid >> 6);
  const int su = (wave >> 1) & 1, sub = wave >> 2;      // staging: block su of a tile, its keys or its values
  const bool values = wave & 1;
  for_share<64 * WQ>(a, spans, BM, 2, pre, [&](int hk, const Unit& un, int first, int cnt, int slot) {
    const int c = un.c0 + wave * 32 + c32, cc = min(c, un.M - 1), tok = cc / a.G, head = hk * a.G + cc - tok * a.G;
    const int last = un.L - un.n + tok, lowest = a.window > 0 ? last - a.window + 1 : 0;
    const int full = uniform(un.L / B), open_rows = uniform(un.L % B), b_at = uniform(un.b_lo + 2 * first);
    // tokens that every column of the unit sees: w_lo .. p_lo
    const int p_lo = uniform(un.L - un.n + un.c0 / a.G);
    const int w_lo = uniform(a.window > 0 ? un.L - un.n + (min(un.M, un.c0 + BM) - 1) / a.G - a.window + 1 : 0);
    // the first block that one of them sees: a tile's other block may lie before it, and hold anything
    const int b_first = uniform(a.window > 0 ? max(0, p_lo - a.window + 1) / B : 0);
    const int sl = uniform(a.c.slots[un.s]);
    const bool has_slot = (unsigned)sl < (unsigned)a.c.n_slots;
    const int32_t* table = a.c.tables + (int64_t)un.s * a.c.width;
    u32x4 qf[KST];
    {
      const uint16_t* q = a.q.p + head * a.q.hs + (int64_t)(un.start + tok) * a.q.ts;
#pragma unroll
      for (int i = 0; i < KST; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + ((i >> 1) * 2 + half) * 16 + 8 * (i & 1));
    }
    float qs;                          // what the column's scores are multiplied by
    {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < KST; ++i) top = max(top, largest(qf[i]));
      top = max(top, __float_as_uint(other_half(__uint_as_float(top))));
      const int e = exponent_of(top, -100);
#pragma unroll
      for (int i = 0; i < KST; ++i) qf[i] = halves(qf[i], e);
      qs = ldexpf(a.c1, e);
    }
    f32x16 O[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) O[i] = f32x16{};
    float m = neg_inf(), l = 0.0f;

    // (kept in registers: read again from the arguments in every tile they cost a trip each)
    const uint8_t* pages = (values ? a.c.v8 : a.c.k8) + hk * (B * D);
    int page_stride = a.c.Hk * (B * D);
    asm volatile("" : "+s"(pages), "+s"(page_stride));
    int ids = -1;                      // a lane the page of one of 64 tiles
    auto open_piece = [&](int ch, int x) {
      const int64_t at = (((int64_t)sl * 2 + (full & 1)) * a.c.Hk + hk) * (B * D);
      return values ? open_value(a.c.ov + at, ch, half, c32, x, open_rows)
                    : open_key(a.c.ok + at, 2 * ch + half, c32, x, open_rows);
    };
    constexpr int kMostScale = 40;
    auto held = [&](float log2) { return fminf(fmaxf(log2, -64.0f), (float)kMostScale); };
    // pages and scales of tiles t .. t + 63; the scales may be used behind the next barrier
    auto look_up = [&](int t) {
      const int b = b_at + 2 * (t + lane) + su;
      ids = t + lane < cnt && b >= b_first && b < full ? table[b] : -1;
      if ((unsigned)ids >= (unsigned)a.c.n_pages) ids = -1;
    };
    auto look_up_scales = [&](int t) {
      if (values || sub != 0) return;
      float2 x = {0.0f, 0.0f};                               // (an open block's: put_open)
      if (ids >= 0) {
        const float ks = at_least(a.c.ks[(int64_t)ids * a.c.Hk + hk]), vs = at_least(a.c.vs[(int64_t)ids * a.c.Hk + hk]);
        x = make_float2(vs < 0x1p-64f ? -ks : ks, held(log2_fast(vs)));
      }
      meta[(t >> 6) & 1][lane][su] = x;
    };
    // this wave's pieces of tile t, to registers; of no page, or behind the last tile, none are read
    auto fetch = [&](int t, u32x4 (&raw)[NCH]) {
      if ((t & 63) == 0 && t > 0) {
        look_up(t);
        look_up_scales(t);
      }
      const int id = __builtin_amdgcn_readlane(ids, t & 63);
      const auto p = page_bytes(pages + (int64_t)max(0, id) * page_stride, id < 0 ? 0 : B * D);
#pragma unroll
      for (int i = 0; i < NCH; ++i) raw[i] = load_shared(p, (sub * NCH + i) * 1024 + lane * 16);
    };
    // and widened to LDS, piece by piece (2 NCH)
    auto put = [&](int t, const u32x4 (&raw)[NCH], int i) {
      u32x4* to = ring[t % NS] + (values ? KB : 0) + (su * KST + 2 * sub * NCH) * 64 + lane;
      to[64 * i] = widen_half(raw[i >> 1][2 * (i & 1)], raw[i >> 1][2 * (i & 1) + 1]);
    };
    // an open block comes from its slot instead
    auto put_open = [&](int t) {
      if (t >= cnt || b_at + 2 * t + su != full || open_rows == 0 || !has_slot) return;
      u32x4* to = ring[t % NS] + (values ? KB : 0) + (su * KST + 2 * sub * NCH) * 64 + lane;
      const int e = open_power[values];
#pragma unroll
      for (int i = 0; i < 2 * NCH; ++i) to[64 * i] = halves(open_piece(sub * NCH + (i >> 1), i & 1), e);
      if (sub == 0 && lane == 0) {
        float2& x = meta[(t >> 6) & 1][t & 63][su];
        if (values) x.y = held((float)e);
        else x.x = ldexpf(1.0f, e);
      }
    };
    auto stage = [&](int t, const u32x4 (&raw)[NCH]) {
#pragma unroll
      for (int i = 0; i < 2 * NCH; ++i) put(t, raw, i);
      put_open(t);
    };

    u32x4 pb[4];            // p as the second product's operand
    f32x16 S[2];
    // Both products run in steps of four fragments, the next step's read from LDS while this one's
    // are multiplied; without that order the compiler waits for each read.
    constexpr int KF = 4, KS = 2 * KST / KF, VF = NC, VS = 4, FR = KF > VF ? KF : VF;
    u32x4 fr[2][FR];
    auto read_keys = [&](int t, int step, u32x4 (&f)[FR]) {
      const u32x4* buf = ring[t % NS] + lane;
#pragma unroll
      for (int x = 0; x < KF; ++x) {
        const int n = step * KF + x, i = n >> 1, u = n & 1;
        f[x] = buf[(u * KST + i) * 64];
      }
    };
    auto multiply_keys = [&](int step, const u32x4 (&f)[FR]) {
#pragma unroll
      for (int x = 0; x < KF; ++x) {
        const int n = step * KF + x, i = n >> 1, u = n & 1;
        S[u] = mfma_half(f[x], qf[i], i == 0 ? f32x16{} : S[u]);
      }
    };
    auto read_values = [&](int t, int step, u32x4 (&f)[FR]) {
      const u32x4* buf = ring[t % NS] + KB + lane;
#pragma unroll
      for (int i = 0; i < NC; ++i) f[i] = buf[((step >> 1) * KST + 2 * i + (step & 1)) * 64];
    };
    // S^T of tile t, whose first step is in fr[at]
    auto scores = [&](int t, int at) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if (k + 1 < KS) read_keys(t, k + 1, fr[(at + k + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
        multiply_keys(k, fr[(at + k) & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // O^T += V^T P^T of tile t, whose first step is in fr[0]; more() goes with the last step.  The pieces of tile
    // `next` are widened between the products, whose time on the matrix unit covers them (in the softmax's
    // half of an iteration they cost their full 600 clocks).
    auto add_values = [&](int t, int next, const u32x4 (&raw)[NCH], auto&& more) {
      constexpr int GAP = VS * NC / (2 * NCH);
#pragma unroll
      for (int k = 0; k < VS; ++k) {
        if (k + 1 < VS) read_values(t, k + 1, fr[(k + 1) & 1]);
        else more();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          O[i] = mfma_half(fr[k & 1][i], pb[k], O[i]);
          const int n = k * NC + i + 1;
          if (n % GAP == 0) {
            put(next, raw, n / GAP - 1);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto softmax = [&](int t, const float4& mt) {
      float cs[2], lv[2], rs[2], v[32];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float2 x = u ? make_float2(mt.z, mt.w) : make_float2(mt.x, mt.y);
        cs[u] = fmaxf(fabsf(x.x) * qs, 0x1p-126f);          // (above 0: -inf times it stays -inf)
        lv[u] = x.y;
        rs[u] = exp2_fast(-x.y);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[u * 16 + i] = S[u][i];
        const int b = b_at + 2 * t + u;
        if (b * B + B - 1 > p_lo || b * B < w_lo) hide(v + u * 16, b, half, last, lowest);
        if (__any(x.x == 0.0f)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[u * 16 + i] = neg_inf();
        }
      }
      running_softmax_half(
          m, l,
          [&](float mu) {
            float2 all = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const float off = lv[u] - mu;
              float sum[4];
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                f16x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const float p = exp2_fast(fmaf(v[u * 16 + 4 * w + (e & 3) + 8 * (e >> 2)], cs[u], off));
                  sum[e & 3] = w == 0 && e < 4 ? p : sum[e & 3] + p;     // (0 + p costs a prompt 3%)
                  x[e] = (_Float16)p;
                }
                pb[u * 2 + w] = __builtin_bit_cast(u32x4, x);
              }
              const float one = (sum[0] + sum[1]) + (sum[2] + sum[3]);
              all.x += one;
              all.y = fmaf(one, rs[u], all.y);
            }
            return all;
          },
          [&]() {
            float top[2] = {v[0], v[16]};
#pragma unroll
            for (int i = 1; i < 16; ++i) {
              top[0] = fmaxf(top[0], v[i]);
              top[1] = fmaxf(top[1], v[16 + i]);
            }
            const float x = fmaxf(fmaf(top[0], cs[0], lv[0]), fmaf(top[1], cs[1], lv[1]));
            return fmaxf(x, other_half(x));
          },
          [&](float al) {
#pragma unroll
            for (int i = 0; i < NC; ++i) O[i] *= al;
          });
      if (__any(mt.x < 0.0f)) pb[0] = pb[1] = u32x4{0, 0, 0, 0};
      if (__any(mt.z < 0.0f)) pb[2] = pb[3] = u32x4{0, 0, 0, 0};
      if constexpr (TURNS) {       // formed here, not behind the barrier
#pragma unroll
        for (int w = 0; w < 4; ++w) asm volatile("" : "+v"(pb[w]));
        asm volatile("" : "+v"(l));
      }
    };

    // the first tiles' loads, under way while the unit before is read to its end and the scales are looked up (ragged
    // prompts 55.4 -> 53.5 us)
    constexpr int AHEAD = TURNS ? 2 : 1;      // a tile is staged so many iterations before its softmax, fetched one more
    u32x4 first_raw[AHEAD][NCH], raw[NCH];
    look_up(0);
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) fetch(t, first_raw[t]);
    fetch(AHEAD, raw);
    meet();                           // the unit before is read
    look_up_scales(0);
    if (wave < 2 && b_at + 2 * cnt > full && open_rows > 0 && has_slot) {
      u32x4 x[2 * NC];
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i) x[i] = open_piece(i >> 1, i & 1);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i) top = max(top, largest(x[i]));
#pragma unroll
      for (int i = 32; i > 0; i >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, i));
      // (the values' power within what their scale is held to: 2^48 is lifted to 2^8)
      if (lane == 0) open_power[wave] = values ? min(exponent_of(top, -57), kMostScale) : exponent_of(top, -100);
    }
    meet();
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) stage(t, first_raw[t]);
    meet();
    if constexpr (TURNS) {
      // Halves of an iteration: half 2t is the first group's softmax of tile t beside the second group's
      // products of tile t - 1, half 2t + 1 the other way round.  The first group writes its part of tile T
      // in half 2T - 3, the second in 2T - 2; its buffer's last tile, T - 4, is read until half 2T - 6, and
      // T itself from half 2T - 1 on.
      const bool second = wave >= 4;
      read_keys(0, 0, fr[0]);
      scores(0, 0);
      if (second) meet();
      for (int t = 0; t < cnt; ++t) {
        const float4 mt = *reinterpret_cast<const float4*>(meta[(t >> 6) & 1][t & 63]);
        __builtin_amdgcn_sched_barrier(0);
        softmax(t, mt);
        read_values(t, 0, fr[0]);
        meet();
        // (behind the last tile the scores are those of an old buffer, and not used)
        __builtin_amdgcn_s_setprio(1);
        add_values(t, t + AHEAD, raw, [&]() { read_keys(t + 1, 0, fr[VS & 1]); });
        put_open(t + AHEAD);
        fetch(t + AHEAD + 1, raw);
        scores(t + 1, VS & 1);
        __builtin_amdgcn_s_setprio(0);
        meet();
      }
      if (!second) meet();
    } else {
      for (int t = 0; t < cnt; ++t) {
        const float4 mt = *reinterpret_cast<const float4*>(meta[(t >> 6) & 1][t & 63]);
        read_keys(t, 0, fr[0]);
        __builtin_amdgcn_sched_barrier(0);
        scores(t, 0);
        softmax(t, mt);
        read_values(t, 0, fr[0]);
        // (the next buffer's last reader passed the barrier at the end of tile t - 1)
        add_values(t, t + AHEAD, raw, []() {});
        put_open(t + AHEAD);
        fetch(t + AHEAD + 1, raw);
        meet();
      }
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

// k_paged_join: the parts of a unit's columns, brought to one maximum and added in a fixed order.  Eight
// groups of d / 4 lanes share a column's parts.  Bound by its trips to memory: 129 parts of a token 5.3 us, 33 parts
// of each of 448 columns 9.6.
template <int D, class SP>
__global__ __launch_bounds__(2 * D) void k_paged_join(PagedAttendArgs a, SP spans, int bm) {
  constexpr int L4 = D / 4, NG = 8;
  const int hk = blockIdx.x / a.units, u = blockIdx.x % a.units, c = blockIdx.y;
  const int64_t share = a.plan[0], one = a.plan[1 + a.units];
  const int64_t x0 = hk * one + a.plan[1 + u], x1 = hk * one + a.plan[2 + u];
  if (x0 == x1) return;
  const int g0 = (int)((x0 + a.start) / share), g1 = (int)((x1 - 1) / share);
  if (g0 == g1) return;
  __shared__ Streams streams;
  load_streams<false>(a, spans, streams);
  const Unit un = columns_of(a, streams, u, bm);
  if (c >= min(bm, un.M - un.c0)) return;
  __shared__ __align__(16) f32x4 so[NG][L4];
  __shared__ float sm[NG], sl[NG];
  const int grp = threadIdx.x / L4, d4 = threadIdx.x % L4;
  // a block's part of this unit lies in its first slot when its share begins in the unit
  auto part = [&](int g) { return (2 * (int64_t)g + ((int64_t)g * share >= x0 ? 0 : 1)) * a.cols + c; };
  // a group's parts AT at a time: all loads under way before the first is used
  constexpr int AT = 8;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.0f, m = neg_inf();
  for (int g = g0 + grp; g <= g1; g += NG * AT) {
    f32x4 po[AT];
    float pm[AT], pl[AT], top = m;
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int64_t at = part(min(g + NG * i, g1));
      pm[i] = a.part_ml[2 * at];
      pl[i] = a.part_ml[2 * at + 1];
      po[i] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + 4 * d4);
    }
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      if (g + NG * i > g1) pm[i] = neg_inf();
      top = fmaxf(top, pm[i]);
    }
    const float mu = top == neg_inf() ? 0.0f : top, w0 = exp2_fast(m - mu);
    o *= w0;
    l *= w0;
    m = top;
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const float w = exp2_fast(pm[i] - mu);
      l = fmaf(pl[i], w, l);
      o += po[i] * w;
    }
  }
  if (d4 == 0) sm[grp] = m;
  __syncthreads();
  float top = sm[0];
#pragma unroll
  for (int x = 1; x < NG; ++x) top = fmaxf(top, sm[x]);
  {
    const float w = exp2_fast(m - (top == neg_inf() ? 0.0f : top));
    o *= w;
    l *= w;
  }
  so[grp][d4] = o;
  if (d4 == 0) sl[grp] = l;
  __syncthreads();
  if (grp > 0) return;
#pragma unroll
  for (int x = 1; x < NG; ++x) {
    o += so[x][d4];
    l += sl[x];
  }
  const int col = un.c0 + c;
  finish(a, hk * a.G + col % a.G, un.start + col / a.G, 4 * d4, o, top, l);
}

// The same where units have many columns and few parts: a group of d / 4 lanes a column (a prompt's 4,096 tokens of 28
// heads: 20 us).
template <int D>
__global__ __launch_bounds__(256) void k_paged_join_many(PagedAttendArgs a, Spans spans, int bm) {
  constexpr int L4 = D / 4, ROWS = 256 / L4;
  const int hk = blockIdx.x / a.units, u = blockIdx.x % a.units;
  const int64_t share = a.plan[0], one = a.plan[1 + a.units];
  const int64_t x0 = hk * one + a.plan[1 + u], x1 = hk * one + a.plan[2 + u];
  if (x0 == x1) return;
  const int g0 = (int)((x0 + a.start) / share), g1 = (int)((x1 - 1) / share);
  if (g0 == g1) return;
  __shared__ Streams streams;
  load_streams<false>(a, spans, streams);
  const Unit un = columns_of(a, streams, u, bm);
  const int c = blockIdx.y * ROWS + threadIdx.x / L4, d = threadIdx.x % L4 * 4;
  if (c >= min(bm, un.M - un.c0)) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = neg_inf(), l = 0.0f;
#pragma unroll 2
  for (int g = g0; g <= g1; ++g) {
    const int64_t at = (2 * (int64_t)g + (g * share >= x0 ? 0 : 1)) * a.cols + c;
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

// The kernels of few columns, with the spans that they take.
template <int D, class SP>
hipError_t few_impl(const PagedAttendArgs& a, const SP& spans, const PagedAttendPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)(a.n_wg ? a.n_wg : a.units * a.c.Hk));
  // where blocks are few, eight waves each share a unit's pages
  const bool wide = a.n_wg == 0 && grid.x <= 256;
  if (p.bm == 16 && wide) hipLaunchKernelGGL((k_paged_few<D, 16, 8, SP>), grid, dim3(512), 0, st, a, spans);
  else if (p.bm == 16) hipLaunchKernelGGL((k_paged_few<D, 16, 4, SP>), grid, dim3(256), 0, st, a, spans);
  else if (wide) hipLaunchKernelGGL((k_paged_few<D, 32, 8, SP>), grid, dim3(512), 0, st, a, spans);
  else hipLaunchKernelGGL((k_paged_few<D, 32, 4, SP>), grid, dim3(256), 0, st, a, spans);
  if (a.n_wg)
    hipLaunchKernelGGL((k_paged_join<D, SP>), dim3((unsigned)(a.units * a.c.Hk), (unsigned)a.cols), dim3(2 * D), 0, st, a,
                       spans, p.bm);
  return hipGetLastError();
}

template <int D>
hipError_t attend_impl(const PagedAttendArgs& a, const Spans& spans, const PagedAttendPlan& p, hipStream_t st) {
  if (p.bm <= 32)
    return spans.uniform ? few_impl<D>(a, EvenSpans{spans.uniform}, p, st) : few_impl<D>(a, spans, p, st);
  const unsigned rows = (unsigned)(a.units * a.c.Hk);
  const dim3 grid(a.n_wg ? (unsigned)a.n_wg : rows);
  if (p.bm == 128) hipLaunchKernelGGL((k_paged_many<D, 4>), grid, dim3(256), 0, st, a, spans);
  else hipLaunchKernelGGL((k_paged_many<D, 8>), grid, dim3(512), 0, st, a, spans);
  if (a.n_wg > 4 * (int64_t)rows) {                 // many parts a unit
    hipLaunchKernelGGL((k_paged_join<D, Spans>), dim3(rows, (unsigned)a.cols), dim3(2 * D), 0, st, a, spans, p.bm);
  } else if (a.n_wg) {
    const int per = 256 / (D / 4);
    hipLaunchKernelGGL((k_paged_join_many<D>), dim3(rows, (unsigned)((a.cols + per - 1) / per)), dim3(256), 0, st, a,
                       spans, p.bm);
  }
  return hipGetLastError();
}

template <int D, class SP>
hipError_t append_impl(const PagedAppendArgs& a, const SP& spans, int h, hipStream_t st) {
  const dim3 grid((unsigned)a.items, (unsigned)(a.c.Hk + (a.q.p ? (a.Hq + h - 1) / h : 0)));
  if (h == 4) hipLaunchKernelGGL((k_paged_append<D, 4, SP>), grid, dim3(2 * D), 0, st, a, spans);
  else hipLaunchKernelGGL((k_paged_append<D, 1, SP>), grid, dim3(2 * D), 0, st, a, spans);
  return hipGetLastError();
}

}  // namespace

// Heads that a block rotates: four share its angles and have their loads under way together, where such
// blocks fill the card; else one (1,777 tokens of 16 heads: 7.0 us with four, 6.4; 8,192 of 28: 21, 26.8).
static int heads_a_block(int64_t token_blocks, int heads) { return token_blocks * ((heads + 3) / 4) >= 256 ? 4 : 1; }

hipError_t launch_rotate(const RotateArgs& a, int D, hipStream_t st) {
  const int rows = 256 / (D / 16), blocks = (a.N + rows - 1) / rows, h = heads_a_block(blocks, a.heads);
  const dim3 grid((unsigned)blocks, (unsigned)((a.heads + h - 1) / h));
  if (D == 128 && h == 4) hipLaunchKernelGGL((k_rotate<128, 4>), grid, dim3(256), 0, st, a);
  else if (D == 128) hipLaunchKernelGGL((k_rotate<128, 1>), grid, dim3(256), 0, st, a);
  else if (h == 4) hipLaunchKernelGGL((k_rotate<64, 4>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_rotate<64, 1>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, const Spans& spans, int D, hipStream_t st) {
  const int h = heads_a_block(a.items, a.Hq);
  const EvenSpans even = {spans.uniform};
  if (spans.uniform) return D == 128 ? append_impl<128>(a, even, h, st) : append_impl<64>(a, even, h, st);
  return D == 128 ? append_impl<128>(a, spans, h, st) : append_impl<64>(a, spans, h, st);
}

hipError_t launch_paged_attend(const PagedAttendArgs& a, const Spans& spans, const PagedAttendPlan& p, int D,
                               hipStream_t st) {
  return D == 128 ? attend_impl<128>(a, spans, p, st) : attend_impl<64>(a, spans, p, st);
}

}  // namespace ss
