// Rotary positions, appends to caches of 16, 32 and 4 bits, and loads from the
// 4-bit cache, gfx950.
//
// One kernel body serves all of them.  The heads of all rows are one list; a wave
// takes one or two times as many as its 64 lanes hold, issues all their loads,
// works out the angles of the rows that they belong to, a lane per frequency, in
// 64 bits, into LDS of its own, and turns and writes them.  Waves neither loop
// nor wait for each other: the work is bound by memory (about 3 flops per
// element against 4 or 8 bytes), and waves that come and go keep more reads in
// flight than longer-lived ones that prefetch, because a wave's loads and stores
// retire in order (65,536 rows of 4 KV heads packed: in a loop over items, which
// waited for its own stores, 105 us; without the loop 82 us).  Where all of a head
// turns in halves, a lane holds both dims of its pairs, so that no partner is
// loaded a second time (72 us), and a head's codes leave in one piece (70 us).  The
// vector work beside the loads counts: no checks before the turn, packing from
// bf16 pairs, divisions of small numbers in fp32 (67 us), and LDS for 6 waves per
// SIMD instead of 5 (64 us; the kernel as it stands 60.6 us, 5.1 TB/s, where a copy
// of that size reaches 5.2).  16,384 rows of 16 heads of 80 in fp32: 32.2 us, 6.1 TB/s
// with lines written in two parts; 17,024 rows of 36 heads of 128 in bf16: 59.1 us, 5.3
// TB/s; 65,536 rows loaded from 4 bits: 31.8 us, 5.7 TB/s.
// 64-bit arithmetic fits under the loads (v_fma_f64 issues at the rate of an
// fp32 one on this chip), and it makes the rounding to 4 bits reproducible: no
// fp32 error of an angle or a product can move a value over a border between
// two codes.
#include <algorithm>

#include "mx.h"

namespace conduit {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;  // dims of a lane
constexpr int kWaves = kThreads / 64;
// Heads of a wave in units of what its lanes hold, where a row has as many: their
// angles are shared.  17,024 rows of 36 heads: 1 unit 67 us, 2 units 62; with 64 of
// 128 dims that turn 85 and 74; in fp32, whole heads, 107 and 111 us (twice the
// registers), so 1 there.  With few rows 1 keeps more waves busy.
constexpr int kMany = 2;
constexpr int64_t kManyFrom = 8192;  // units of work from which on
constexpr int kDppQuad0011 = 0x50, kDppQuad2233 = 0xFA;  // lane i of four <- that of the four
constexpr int kDppShl4 = 0x104;  // lane i <- lane i + 4 of its 16
typedef double f64x2 __attribute__((ext_vector_type(2)));

// (cos, sin) of a = p * f: a is reduced by the nearest multiple of pi/2 (two-part
// constant, fused multiply-adds), then Taylor series on [-pi/4, pi/4], whose
// first omitted terms are below 5e-17.
__device__ __forceinline__ f64x2 cos_sin(double a) {
  // (1.5 * 2^52 leaves the integer in the low bits; |a| < 2^41.01)
  const double shifted = __builtin_fma(a, 0.63661977236758134308, 6755399441055744.0);
  const double k = shifted - 6755399441055744.0;
  double r = __builtin_fma(-k, 1.57079632679489655800e+00, a);
  r = __builtin_fma(-k, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = -1.0 / 1307674368000.0;                        // 1/15!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);              // 1/13!
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;                        // 1/16!
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);            // 1/14!
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int q = (int)__builtin_bit_cast(uint64_t, shifted) & 3;  // k mod 4
  const double cc = q & 1 ? s : c, ss = q & 1 ? c : s;
  return f64x2{q == 1 || q == 2 ? -cc : cc, q >= 2 ? -ss : ss};
}

// 8 elements as loaded, and their values.
template <typename T>
struct Raw {
  u32x4 w[sizeof(T) / 2];
};
// (fp32: the second four are `gap` elements after the first)
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T *p, int gap = 4) {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = ld16(p + gap * i);
  return r;
}
__device__ __forceinline__ void expand(const Raw<u16> &r, float (&x)[kVec]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __builtin_bit_cast(float, r.w[0][j] << 16);
    x[2 * j + 1] = __builtin_bit_cast(float, r.w[0][j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void expand(const Raw<float> &r, float (&x)[kVec]) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const uint32_t w = r.w[j / 4][j % 4];  // (a copy: a bit cast of the vector's element itself reads element 0)
    x[j] = __builtin_bit_cast(float, w);
  }
}
// What is written here is read by another kernel, if at all soon by other XCDs:
// streaming stores keep it out of the L2's way (65,536 rows loaded from 4 bits:
// 33 us against 49 us with ordinary stores).
__device__ __forceinline__ void st16_stream(void *p, u32x4 v) {
  __builtin_nontemporal_store(v, static_cast<u32x4 *>(p));
}
// Eight of a lane's elements.  fp32: either store writes 16 bytes of every 32, which
// reach memory in parts, so where four lanes hold 32 dims side by side (gap 0) they
// trade first and a store writes 64 bytes side by side (16,384 rows of 16 heads of
// 80 of which 40 dims turn: 46 us, 36 us so); otherwise the second four go `gap`
// elements on.
__device__ __forceinline__ void store_words(u16 *p, const u32x4 (&w)[1], int) { st16_stream(p, w[0]); }
__device__ __forceinline__ void store_words(float *p, const u32x4 (&w)[2], int gap) {
  if (gap) {
    st16_stream(p, w[0]);
    st16_stream(p + gap, w[1]);
    return;
  }
  const int l = threadIdx.x & 3;
  u32x4 a, b;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t x = w[0][j], y = w[1][j];
    const uint32_t xa = dpp_mov<kDppQuad0011>(0u, x), ya = dpp_mov<kDppQuad0011>(0u, y);
    const uint32_t xb = dpp_mov<kDppQuad2233>(0u, x), yb = dpp_mov<kDppQuad2233>(0u, y);
    a[j] = l & 1 ? ya : xa;
    b[j] = l & 1 ? yb : xb;
  }
  st16_stream(p - 4 * l, a);
  st16_stream(p - 4 * l + 16, b);
}
template <typename T>
__device__ __forceinline__ void store_raw(T *p, const Raw<T> &r, int gap) {
  store_words(p, r.w, gap);
}
__device__ __forceinline__ void store(u16 *p, const float (&x)[kVec], int gap) {
  u32x4 r[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x2 b = {static_cast<__bf16>(x[2 * j]), static_cast<__bf16>(x[2 * j + 1])};
    r[0][j] = __builtin_bit_cast(uint32_t, b);
  }
  store_words(p, r, gap);
}
__device__ __forceinline__ void store(float *p, const float (&x)[kVec], int gap) {
  const u32x4 r[2] = {__builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}),
                      __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]})};
  store_words(p, r, gap);
}
__device__ __forceinline__ float one(const u16 *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float one(const float *p) { return *p; }

// A result in fp32, kept as such: the compiler must not merge this rounding with
// the one to bf16 that follows (two roundings and one differ near ties).
__device__ __forceinline__ float to_f32(double x) {
  float r = (float)x;
  asm("" : "+v"(r));
  return r;
}

// The turn, in place.  x[0] holds dims [o, o + 8) of a head, cs the row's cosines
// and sines.  FULL: x[1] holds their partners, dims [o + half, o + half + 8), and
// the second four of either may be `gap` dims after the first.
// Otherwise y holds the partners (halves; dims from 2 half on have none), or the
// pairs lie side by side in x[0] (adjacent).
template <bool FULL, int NV>
__device__ __forceinline__ void turn(float (&x)[NV][kVec], const float (&y)[kVec], int o, int half, bool adjacent,
                                     const f64x2 *cs, int gap) {
  if constexpr (FULL) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const f64x2 t = cs[o + j % 4 + j / 4 * gap];
      const double a = x[0][j], b = x[1][j];
      x[0][j] = to_f32(__builtin_fma(a, t[0], -(b * t[1])));
      x[1][j] = to_f32(__builtin_fma(b, t[0], a * t[1]));
    }
    return;
  }
  if (o >= 2 * half) return;
  if (adjacent) {
#pragma unroll
    for (int j = 0; j < kVec / 2; ++j) {
      if (o / 2 + j < half) {
        const f64x2 t = cs[o / 2 + j];
        const double a = x[0][2 * j], b = x[0][2 * j + 1];
        x[0][2 * j] = to_f32(__builtin_fma(a, t[0], -(b * t[1])));
        x[0][2 * j + 1] = to_f32(__builtin_fma(b, t[0], a * t[1]));
      }
    }
    return;
  }
  const bool first = o < half;
  const f64x2 *f = cs + (first ? o : o - half);
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const f64x2 t = f[j];
    const double m = (double)y[j] * t[1];
    x[0][j] = to_f32(__builtin_fma((double)x[0][j], t[0], first ? -m : m));
  }
}

// The same where a half is not a multiple of 8 dims: partners one by one.
template <typename T>
__device__ __forceinline__ void turn_single(float (&x)[kVec], int o, int half, const f64x2 *cs, const T *head) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const int i = o + j;
    if (i >= 2 * half) continue;
    const bool first = i < half;
    const f64x2 t = cs[first ? i : i - half];
    const double m = (double)one(head + (first ? i + half : i - half)) * t[1];
    x[j] = to_f32(__builtin_fma((double)x[j], t[0], first ? -m : m));
  }
}

// 8 values of a 4-bit row: a dword of codes and its block's scale byte.
__device__ __forceinline__ void unpack(uint32_t codes, int scale, float (&x)[kVec]) {
  const float s = __builtin_bit_cast(float, (uint32_t)scale << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3);
  const bf16x2 r[4] = {a, b, c, d};
#pragma unroll
  for (int j = 0; j < 4; ++j) x[2 * j] = (float)r[j][0], x[2 * j + 1] = (float)r[j][1];
}

// A lane's 8 values of a row to be packed: their bits as fp32 or, in pairs, as bf16.
__device__ __forceinline__ void pack_bits(const float (&x)[kVec], uint32_t (&w)[4], u16) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x2 b = {static_cast<__bf16>(x[2 * j]), static_cast<__bf16>(x[2 * j + 1])};
    w[j] = __builtin_bit_cast(uint32_t, b);
  }
}
__device__ __forceinline__ void pack_bits(const float (&x)[kVec], uint32_t (&w)[8], float) {
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = __builtin_bit_cast(uint32_t, x[j]);
}
template <typename T>
__device__ __forceinline__ void raw_bits(const Raw<T> &r, uint32_t (&w)[2 * sizeof(T)]) {
#pragma unroll
  for (int j = 0; j < (int)(2 * sizeof(T)); ++j) w[j] = r.w[j / 4][j % 4];
}

// Largest magnitude of 32 dims, 8 of them in each of 4 consecutive lanes, as the
// bits of an fp32 number.
__device__ __forceinline__ uint32_t largest_bits(const uint32_t (&w)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, w[j] & 0x7fffffffu);
  m = max(m, dpp_mov<kDppXor1>(0u, m));
  return max(m, dpp_mov<kDppXor2>(0u, m));
}
__device__ __forceinline__ uint32_t largest_bits(const uint32_t (&w)[4]) {
  uint32_t hi = 0, lo = 0;  // (of both halves the upper is enough with the lower below it)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi = max(hi, w[j] & 0x7fffffffu);
    lo = max(lo, w[j] << 16 & 0x7fffffffu);
  }
  uint32_t m = max(hi, lo) & 0xffff0000u;
  m = max(m, dpp_mov<kDppXor1>(0u, m));
  return max(m, dpp_mov<kDppXor2>(0u, m));
}

// Its scale byte: the smallest s with max|x| <= 1.5 * 2^(s - 125) (the maximum's
// exponent, one more when its mantissa is above 1.5).
__device__ __forceinline__ int block_scale(uint32_t m) {
  const int s = (int)((m + 0x3fffffu) >> 23) - 2;
  return min(max(s, kMxScaleMin), kMxScaleMax);
}

__device__ __forceinline__ uint32_t pack(const uint32_t (&w)[8], int scale) {
  const float s = __builtin_bit_cast(float, (uint32_t)scale << 23);
  float x[kVec];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t y = w[j];
    x[j] = __builtin_bit_cast(float, y);
  }
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}
__device__ __forceinline__ uint32_t pack(const uint32_t (&w)[4], int scale) {
  const float s = __builtin_bit_cast(float, (uint32_t)scale << 23);
  bf16x2 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t y = w[j];
    x[j] = __builtin_bit_cast(bf16x2, y);
  }
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x[0], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x[1], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x[2], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x[3], s, 3);
}

__device__ __forceinline__ float scalar(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}
// x / d for 0 <= x < d + 128, or x < 512 with d <= 128 (inv: about 1 / d).
__device__ __forceinline__ int small_div(int x, int d, float inv) {
  return d > 128 ? x >= d : (int)((x + 0.5f) * inv);
}

// How a head is shared out over lanes.
enum HeadShape {
  kVectors = 0,  // 8 dims a lane, partners loaded as well where there are any
  kPairs = 1,    // all of the head turns, halves, two heads a row or more: 8 dims of each half a lane
  kSingles = 2   // 8 dims a lane, partners one by one: halves that 8 does not divide (kRowTurn only)
};

// A head's lanes are lanes of one wave, so a call in place reads every partner
// before it writes (loads of a wave precede its stores).
// (6 waves per SIMD, where the compiler would use 2 registers too many for them:
// 17,024 rows of 36 heads of which 64 dims turn, 78 us, 76 us so.)
template <typename T, RowMode MODE, int K, HeadShape SHAPE>
__global__ __launch_bounds__(kThreads, K == 1                                                         ? 4
                                       : MODE == kRowAppend && SHAPE == kVectors && sizeof(T) == 2 ? 6
                                                                                                   : 1)
void rows_kernel(RowParams p) {
  constexpr bool kToKv = MODE == kRowAppend || MODE == kRowLoadMx, kMx = MODE == kRowAppendMx || MODE == kRowLoadMx;
  constexpr bool kFull = SHAPE == kPairs;
  constexpr int NV = kFull ? 2 : 1;  // vectors of 8 dims of a lane
  // K = 1: at most 64 / lanes rows of 4 * NV * lanes frequencies each, with two heads
  // a row and more (kPairs) half as many and one; K > 1: two rows of up to 128.
  // (24 KB at most, which 6 workgroups of a CU fit; with 32 KB and 5 of them 65,536
  // rows packed took 67 us instead of 64.)
  __shared__ f64x2 s_cs[kWaves][K == 1 && kFull ? 384 : 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = p.rope.half, D = p.head_dim;
  const int lanes = D / (kVec * NV), heads = 64 / lanes;  // lanes of a head, heads of the wave's lanes
  // fp32, all of a head turning: a lane's 8 dims are 4 and, a quarter of the head on,
  // 4 more, so that a store writes a head's dims side by side (the turn of 16,384
  // rows of 16 heads of 80 writes 109 MB for its 84, and 130 with 8 side by side: 38.2 and
  // 41.8 us over four inputs).
  constexpr bool kSplit = sizeof(T) == 4 && kFull && (MODE == kRowTurn || MODE == kRowAppend);
  const int gap = kSplit ? half / 2 : 4, store_gap = kSplit ? gap : lanes % 4 ? 4 : 0;
  const int sub = (int)((lane + 0.5f) * __builtin_amdgcn_rcpf((float)lanes));
  const int o = (lane - sub * lanes) * (kSplit ? 4 : kVec);
  const int units = p.n_q_heads + p.n_kv_heads;           // query heads, then KV heads, of a row
  const int total = p.n * units;
  const bool adjacent = p.rope.adjacent != 0;
  const bool partners = SHAPE == kVectors && !adjacent && half > 0;
  const int partner = o < half ? o + half : o < 2 * half ? o - half : o;
  auto dims = [&](int i) __attribute__((always_inline)) { return o + i * half; };  // first dim of vector i
  f64x2 *cs = s_cs[wave];
  const int first = (blockIdx.x * kWaves + wave) * (heads * K);  // heads of this wave: [first, first + heads * K)
  if (first >= total) return;
  const int row0 = (int)((uint32_t)first / (uint32_t)units), unit0 = first - row0 * units;
  const float inv_units = scalar(__builtin_amdgcn_rcpf((float)units));
  auto row_of = [&](int i) __attribute__((always_inline)) { return small_div(unit0 + i, units, inv_units); };
  const int last = min(heads * K, total - first) - 1;    // of this wave's heads
  const int rows = __builtin_amdgcn_readfirstlane(row_of(last)) + 1;

  struct In {
    int32_t row, unit;         // of the lane
    int32_t at, from, page, mx_page;
    bool live;
    Raw<T> x[NV], y, v[NV];
    uint32_t xc[NV], yc, vc[NV];  // 4-bit rows
    int32_t xs[NV], ys, vs[NV];
  };
  In in[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    In &c = in[k];
    const int u = min(k * heads + min(sub, heads - 1), last), r = row_of(u);  // (past the end: loads the last head)
    c.row = row0 + r;
    c.unit = unit0 + u - r * units;
    if constexpr (MODE != kRowTurn) {
      c.at = c.from = p.pos[c.row];
      if constexpr (MODE == kRowLoadMx) c.from = p.src_pos[c.row];
    }
    if constexpr (MODE != kRowLoadMx) {
      const bool query = MODE == kRowTurn || c.unit < p.n_q_heads;
      const int h = query ? c.unit : c.unit - p.n_q_heads;
      const T *src =
          static_cast<const T *>(query ? p.q : p.k_new) + c.row * (query ? p.q_stride : p.k_new_stride) + h * D;
#pragma unroll
      for (int i = 0; i < NV; ++i) c.x[i] = load_raw<T>(src + dims(i), gap);
      c.y = c.x[0];
      if (partners) c.y = load_raw<T>(src + partner);
      if constexpr (MODE != kRowTurn) {
        const T *vsrc = static_cast<const T *>(p.v_new) + c.row * p.v_new_stride + h * D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          c.v[i] = c.x[i];
          if (!query) c.v[i] = load_raw<T>(vsrc + dims(i), gap);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    In &c = in[k];
    if constexpr (MODE != kRowTurn) {
      c.live = true;
      if constexpr (kToKv) c.live = c.live && (uint32_t)c.at < (uint32_t)p.n_ctx;
      if constexpr (kMx) c.live = c.live && (uint32_t)c.from < (uint32_t)p.mx.n_ctx;
      if (!c.live) c.at = c.from = 0;  // (a row that is left out: token 0, not written)
      if constexpr (kToKv)
        if (p.pages.table) c.page = p.pages.table[c.at >> p.pages.shift];
      if constexpr (kMx) c.mx_page = mx_page(p.mx, c.row / p.mx.rows_per_seq, c.from);
    }
    if constexpr (MODE == kRowLoadMx) {
      const int64_t slot = ((int64_t)c.unit << p.mx.shift) + (c.from & ((1 << p.mx.shift) - 1));
      const int64_t co = c.mx_page * p.mx.code_stride + slot * (D / 2);
      const int64_t so = c.mx_page * p.mx.scale_stride + slot * (D / kMxBlock);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        c.xc[i] = *reinterpret_cast<const uint32_t *>(p.mx.k + co + dims(i) / 2);
        c.vc[i] = *reinterpret_cast<const uint32_t *>(p.mx.v + co + dims(i) / 2);
        c.xs[i] = p.mx.k_scale[so + dims(i) / kMxBlock];
        c.vs[i] = p.mx.v_scale[so + dims(i) / kMxBlock];
      }
      c.yc = c.xc[0];
      c.ys = c.xs[0];
      if (partners) {
        c.yc = *reinterpret_cast<const uint32_t *>(p.mx.k + co + partner / 2);
        c.ys = p.mx.k_scale[so + partner / kMxBlock];
      }
    }
  }
  // The rows' angles.
  const int n_angles = rows * half;
  const float inv_half = scalar(__builtin_amdgcn_rcpf((float)half));
  for (int e = lane; e < n_angles; e += 64) {
    const int r = (int)((e + 0.5f) * inv_half), f = e - r * half;
    // (the positions on all axes, so that none waits for the frequency's axis)
    const int32_t *pos = p.rope.pos + row0 + r;
    int32_t at[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) at[a] = a < p.rope.n_axes ? pos[a * p.rope.pos_stride] : 0;
    const int axis = p.rope.axis[f];
    f64x2 t = cos_sin((double)(axis < 2 ? axis ? at[1] : at[0] : axis == 2 ? at[2] : at[3]) *
                      (double)p.rope.inv_freq[f]);
    if (p.rope.inverse) t[1] = -t[1];
    cs[e] = t;
  }
  // (this wave's LDS accesses stay in order in the hardware)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

#pragma unroll
  for (int k = 0; k < K; ++k) {
    const In &c = in[k];
    if (sub >= heads || k * heads + sub > last) return;
    const f64x2 *rcs = cs + (c.row - row0) * half;
    float x[NV][kVec], y[kVec], v[NV][kVec];
    if constexpr (MODE == kRowLoadMx) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        unpack(c.xc[i], c.xs[i], x[i]);
        unpack(c.vc[i], c.vs[i], v[i]);
      }
      unpack(c.yc, c.ys, y);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) expand(c.x[i], x[i]);
      expand(c.y, y);
    }
    if constexpr (SHAPE == kSingles)
      turn_single<T>(x[0], o, half, rcs, static_cast<const T *>(p.q) + c.row * p.q_stride + c.unit * D);
    else
      turn<kFull>(x, y, o, half, adjacent, rcs, gap);
    if (MODE == kRowTurn || c.unit < p.n_q_heads) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        store(static_cast<T *>(p.q_out) + c.row * p.q_out_stride + c.unit * D + dims(i), x[i], store_gap);
      continue;
    }
    const int h = c.unit - p.n_q_heads;
    if constexpr (kToKv) {
      if (!c.live) continue;
      int64_t row = c.at;
      if (p.pages.table)
        row = ((int64_t)min(max(c.page, 0), p.pages.n_pages - 1) << p.pages.shift) |
              (c.at & ((1 << p.pages.shift) - 1));
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        store(static_cast<T *>(p.k) + row * p.k_stride + h * D + dims(i), x[i], store_gap);
        T *vd = static_cast<T *>(p.v) + row * p.v_stride + h * D + dims(i);
        if constexpr (MODE == kRowAppend)
          store_raw(vd, c.v[i], store_gap);
        else
          store(vd, v[i], store_gap);
      }
    }
    if constexpr (MODE == kRowAppendMx) {
      int ks[NV], vs[NV];
      uint32_t kc[NV], vc[NV];
      // a head with an infinity or a NaN among its keys or values (no turn makes a
      // finite pair of one that is not): the key is NaN, the value 0
      bool bad = false;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        uint32_t kw[2 * sizeof(T)], vw[2 * sizeof(T)];
        pack_bits(x[i], kw, T{});
        raw_bits<T>(c.v[i], vw);
        const uint32_t km = largest_bits(kw), vm = largest_bits(vw);
        ks[i] = block_scale(km);
        vs[i] = block_scale(vm);
        kc[i] = pack(kw, ks[i]);
        vc[i] = pack(vw, vs[i]);
        bad = bad || max(km, vm) >= 0x7f800000u;
      }
      if (__ballot(bad) >> (sub * lanes) & ((1ull << lanes) - 1)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          ks[i] = kMxScaleNan;
          vs[i] = kMxScaleMin;
          kc[i] = vc[i] = 0;
        }
      }
      const int64_t held = ((int64_t)c.row * p.n_kv_heads + h) * D;
      const int64_t slot = ((int64_t)h << p.mx.shift) + (c.from & ((1 << p.mx.shift) - 1));  // of the page
      const int64_t co = c.mx_page * p.mx.code_stride + slot * (D / 2);
      const int64_t so = c.mx_page * p.mx.scale_stride + slot * (D / kMxBlock);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int d = dims(i);
        if (p.k_out) {
          unpack(kc[i], ks[i], y);
          store(static_cast<T *>(p.k_out) + held + d, y, store_gap);
        }
        if (p.v_out) {
          unpack(vc[i], vs[i], y);
          store(static_cast<T *>(p.v_out) + held + d, y, store_gap);
        }
      }
      if (!c.live) continue;
      if constexpr (kFull) {
        // Neighbouring lanes swap a dword, so that a lane writes 8 bytes and a
        // head's codes go out in one piece; its scales are put together in its
        // first lane.
        const bool odd = o & kVec;
        const int64_t at = co + (odd ? half + o - kVec : o) / 2;
        auto codes = [&](uint8_t *pool, const uint32_t (&x)[NV]) __attribute__((always_inline)) {
          const uint32_t other = dpp_mov<kDppXor1>(0u, odd ? x[0] : x[1]);
          *reinterpret_cast<uint2 *>(pool + at) = odd ? make_uint2(other, x[1]) : make_uint2(x[0], other);
        };
        auto scales = [&](uint8_t *pool, const int (&x)[NV]) __attribute__((always_inline)) {
          if (lanes == 8) {  // blocks 0 and 2 in the first quad, 1 and 3 in the second
            const uint32_t mine = x[0] | x[1] << 16, next = dpp_mov<kDppShl4>(0u, mine);
            if (o == 0) *reinterpret_cast<uint32_t *>(pool + so) = mine | next << 8;
          } else if (o == 0) {
            *reinterpret_cast<uint16_t *>(pool + so) = (uint16_t)(x[0] | x[1] << 8);
          }
        };
        codes(p.mx.k, kc);
        codes(p.mx.v, vc);
        scales(p.mx.k_scale, ks);
        scales(p.mx.v_scale, vs);
      } else {
        *reinterpret_cast<uint32_t *>(p.mx.k + co + o / 2) = kc[0];
        *reinterpret_cast<uint32_t *>(p.mx.v + co + o / 2) = vc[0];
        if (o % kMxBlock == 0) {
          p.mx.k_scale[so + o / kMxBlock] = (uint8_t)ks[0];
          p.mx.v_scale[so + o / kMxBlock] = (uint8_t)vs[0];
        }
      }
    }
  }
}

template <typename T, int K, HeadShape SHAPE>
void launch_mode(const RowParams &p, RowMode mode, dim3 grid, hipStream_t s) {
  if (mode == kRowTurn)
    rows_kernel<T, kRowTurn, K, SHAPE><<<grid, kThreads, 0, s>>>(p);
  else if constexpr (SHAPE != kSingles) {
    if (mode == kRowAppend)
      rows_kernel<T, kRowAppend, K, SHAPE><<<grid, kThreads, 0, s>>>(p);
    else if (mode == kRowAppendMx)
      rows_kernel<T, kRowAppendMx, K, SHAPE><<<grid, kThreads, 0, s>>>(p);
    else if constexpr (SHAPE == kVectors || sizeof(T) == 2)
      rows_kernel<T, kRowLoadMx, K, SHAPE><<<grid, kThreads, 0, s>>>(p);
  }
}

template <typename T, int K>
void launch_shape(const RowParams &p, RowMode mode, HeadShape shape, dim3 grid, hipStream_t s) {
  if (shape == kVectors)
    launch_mode<T, K, kVectors>(p, mode, grid, s);
  else if (shape == kSingles)
    launch_mode<T, K, kSingles>(p, mode, grid, s);
  else if constexpr (K == 1 || sizeof(T) == 2)
    launch_mode<T, K, kPairs>(p, mode, grid, s);
}

}  // namespace

hipError_t launch_rows(const RowParams &p, RowMode mode, bool bf16, hipStream_t s) {
  static const char *const names[] = {"rotary", "append", "append_mx", "load_mx"};
  ProfScope ps(names[mode], s);
  const int half = p.rope.half;
  const int units = p.n_q_heads + p.n_kv_heads;
  // (fp32 rows loaded from 4 bits: 8 dims a lane let four lanes trade pieces of one
  // run of dims instead of two; 65,536 rows 58 us, in pairs 71)
  const bool pairs = 2 * half == p.head_dim && units > 1 && (bf16 || mode != kRowLoadMx);
  const HeadShape shape = p.rope.adjacent || !half ? kVectors
                          : half % kVec           ? kSingles
                          : pairs                 ? kPairs
                                                  : kVectors;
  const int heads = 64 / (p.head_dim / (kVec * (shape == kPairs ? 2 : 1)));
  const int64_t total = (int64_t)p.n * units;
  const bool many = units >= kMany * heads && total >= kManyFrom * heads && (bf16 || shape != kPairs);
  const int k = many ? kMany : 1;
  const dim3 grid((unsigned)((total + heads * k * kWaves - 1) / (heads * k * kWaves)));
  if (bf16)
    many ? launch_shape<u16, kMany>(p, mode, shape, grid, s) : launch_shape<u16, 1>(p, mode, shape, grid, s);
  else
    many ? launch_shape<float, kMany>(p, mode, shape, grid, s) : launch_shape<float, 1>(p, mode, shape, grid, s);
  return hipGetLastError();
}

}  // namespace conduit
