// What kernels over rows of heads share (rotary.hip, append_byte.hip): a lane's 8 dims
// as loaded and stored, and angles in 64 bits.
#pragma once

#include "mx.h"

namespace conduit {
namespace {

constexpr int kVec = 8;  // dims of a lane
constexpr int kDppQuad0011 = 0x50, kDppQuad2233 = 0xFA;  // lane i of four <- that of the four
typedef double f64x2 __attribute__((ext_vector_type(2)));

// (cos, sin) of a = p * f: a is reduced by the nearest multiple of pi/2 (two-part
// constant, fused multiply-adds), then Taylor series on [-pi/4, pi/4], whose
// first omitted terms are below 5e-17.  SCALAR: constants in scalar registers (in a kernel with
// a loop around, where they would be held in 30 vector registers).
template <bool SCALAR = false>
__device__ __forceinline__ f64x2 cos_sin(double a) {
  auto k_ = [](double x) __attribute__((always_inline)) {
    if constexpr (SCALAR) asm("" : "+s"(x));
    return x;
  };
  // (1.5 * 2^52 leaves the integer in the low bits; |a| < 2^41.01)
  const double shifted = __builtin_fma(a, 0.63661977236758134308, 6755399441055744.0);
  const double k = shifted - 6755399441055744.0;
  double r = __builtin_fma(-k, 1.57079632679489655800e+00, a);
  r = __builtin_fma(-k, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = k_(-1.0 / 1307674368000.0);                        // 1/15!
  s = __builtin_fma(s, z, k_(1.0 / 6227020800.0));              // 1/13!
  s = __builtin_fma(s, z, k_(-1.0 / 39916800.0));
  s = __builtin_fma(s, z, k_(1.0 / 362880.0));
  s = __builtin_fma(s, z, k_(-1.0 / 5040.0));
  s = __builtin_fma(s, z, k_(1.0 / 120.0));
  s = __builtin_fma(s, z, k_(-1.0 / 6.0));
  s = __builtin_fma(s * z, r, r);
  double c = k_(1.0 / 20922789888000.0);                        // 1/16!
  c = __builtin_fma(c, z, k_(-1.0 / 87178291200.0));            // 1/14!
  c = __builtin_fma(c, z, k_(1.0 / 479001600.0));
  c = __builtin_fma(c, z, k_(-1.0 / 3628800.0));
  c = __builtin_fma(c, z, k_(1.0 / 40320.0));
  c = __builtin_fma(c, z, k_(-1.0 / 720.0));
  c = __builtin_fma(c, z, k_(1.0 / 24.0));
  c = __builtin_fma(c, z, k_(-0.5));
  c = __builtin_fma(c, z, k_(1.0));
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

}  // namespace
}  // namespace conduit
