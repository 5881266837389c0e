// Rotary positions, appends to caches of 16, 32 and 4 bits, and loads from the
// 4-bit cache, gfx950.
//
// One kernel body serves all of them: a workgroup takes a few consecutive
// rows.  First its threads compute the rows' sines and cosines, one (row,
// frequency) each, in 64 bits into LDS; every head of a row then uses them.
// Then each wave takes heads of these rows, a lane 8 dims of a head (16 bytes in
// bf16): it loads them and their partners in the pairs, turns them, and writes
// them where they go.  The work is bound by memory (each element read and
// written once; partners come from L1): about 3 flops per element against 4 or
// 8 bytes.  64-bit arithmetic is therefore free here (v_fma_f64 issues at the
// rate of an fp32 one on this chip), and it makes the rounding to 4 bits
// reproducible: no fp32 error of an angle or a product can move a value over a
// border between two codes.
#include "mx.h"

namespace conduit {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;  // dims of a lane
typedef double f64x2 __attribute__((ext_vector_type(2)));

// (cos, sin) of a = p * f: a is reduced by the nearest multiple of pi/2 (two-part
// constant, fused multiply-adds), then Taylor series on [-pi/4, pi/4], whose
// first omitted terms are below 5e-17.
__device__ __forceinline__ f64x2 cos_sin(double a) {
  const double k = __builtin_rint(a * 0.63661977236758134308);
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
  // quadrant: k mod 4 (|k| < 2^41, exact)
  const int q = (int)(k - 4.0 * __builtin_floor(k * 0.25));
  const double cc = q & 1 ? s : c, ss = q & 1 ? c : s;
  return f64x2{q == 1 || q == 2 ? -cc : cc, q >= 2 ? -ss : ss};
}

template <typename T>
struct Elem;
template <>
struct Elem<u16> {
  static __device__ __forceinline__ void load(const u16 *p, float (&x)[kVec]) {
    const u32x4 r = ld16(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __builtin_bit_cast(float, r[j] << 16);
      x[2 * j + 1] = __builtin_bit_cast(float, r[j] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float one(const u16 *p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ void store(u16 *p, const float (&x)[kVec]) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x2 b = {static_cast<__bf16>(x[2 * j]), static_cast<__bf16>(x[2 * j + 1])};
      r[j] = __builtin_bit_cast(uint32_t, b);
    }
    st16(p, r);
  }
  static __device__ __forceinline__ float rounded(float x) { return bf16_to_f32(f32_to_bf16(x)); }
};
template <>
struct Elem<float> {
  static __device__ __forceinline__ void load(const float *p, float (&x)[kVec]) {
    const f32x4 a = __builtin_bit_cast(f32x4, ld16(p)), b = __builtin_bit_cast(f32x4, ld16(p + 4));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
  }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
  static __device__ __forceinline__ void store(float *p, const float (&x)[kVec]) {
    st16(p, __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}));
    st16(p + 4, __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}));
  }
  static __device__ __forceinline__ float rounded(float x) { return x; }
};

// Dims [o, o + 8) of a head turned in place: x holds them, partner(i) gives dims
// [i, i + 8) of the same head, cs the row's cosines and sines.
template <class Partner>
__device__ __forceinline__ void turn(float (&x)[kVec], int o, int half, bool adjacent, const f64x2 *cs,
                                     Partner &&partner) {
  if (o >= 2 * half) return;
  if (adjacent) {
#pragma unroll
    for (int j = 0; j < kVec / 2; ++j) {
      if (o / 2 + j < half) {
        const f64x2 t = cs[o / 2 + j];
        const double a = x[2 * j], b = x[2 * j + 1];
        x[2 * j] = (float)__builtin_fma(a, t[0], -(b * t[1]));
        x[2 * j + 1] = (float)__builtin_fma(a, t[1], b * t[0]);
      }
    }
    return;
  }
  const bool first = o < half;
  const int f = first ? o : o - half;
  float y[kVec];
  partner(first ? o + half : o - half, y);
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const f64x2 t = cs[f + j];
    const double m = (double)y[j] * t[1];
    x[j] = (float)__builtin_fma((double)x[j], t[0], first ? -m : m);
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
    const double m = (double)Elem<T>::one(head + (first ? i + half : i - half)) * t[1];
    x[j] = (float)__builtin_fma((double)x[j], t[0], first ? -m : m);
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

// Scale byte of a block of 32 dims, 8 of them in each of 4 consecutive lanes:
// the smallest s with max|x| <= 1.5 * 2^(s - 125), from the bits of the
// maximum (its exponent, one more when its mantissa is above 1.5).
__device__ __forceinline__ int block_scale(const float (&x)[kVec]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < kVec; ++j) m = max(m, __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffffu);
  m = max(m, dpp_mov<kDppXor1>(0u, m));
  m = max(m, dpp_mov<kDppXor2>(0u, m));
  const int s = (int)((m + 0x3fffffu) >> 23) - 2;
  return min(max(s, kMxScaleMin), kMxScaleMax);
}

__device__ __forceinline__ uint32_t pack(const float (&x)[kVec], int scale) {
  const float s = __builtin_bit_cast(float, (uint32_t)scale << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}

__device__ __forceinline__ bool any_not_finite(const float (&x)[kVec]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < kVec; ++j) m = max(m, __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffffu);
  return m >= 0x7f800000u;
}

// SINGLE: halves whose length is not a multiple of 8 (kRowTurn only).
// Work unit of a lane group: one query head, or one KV head's keys and values.
// A group is head_dim / 8 lanes and never straddles two waves, so that a call
// in place reads every partner before it writes (loads of a wave precede its
// stores).
template <typename T, RowMode MODE, bool SINGLE>
__global__ __launch_bounds__(kThreads) void rows_kernel(RowParams p) {
  extern __shared__ f64x2 s_cs[];  // [rows of the block][half]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = p.rope.half;
  const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
  const int rows = (int)min((int64_t)p.rows_per_block, p.n - row0);
  for (int e = tid; e < rows * half; e += kThreads) {
    const int r = e / half, f = e - r * half;
    const int at = p.rope.pos[p.rope.axis[f] * p.rope.pos_stride + row0 + r];
    f64x2 t = cos_sin((double)at * (double)p.rope.inv_freq[f]);
    if (p.rope.inverse) t[1] = -t[1];
    s_cs[e] = t;
  }
  __syncthreads();

  const int D = p.head_dim, lanes = D / kVec;      // lanes of a head
  const int heads = 64 / lanes;                    // heads of a wave
  const int sub = lane / lanes, o = (lane - sub * lanes) * kVec;
  const int units = p.n_q_heads + p.n_kv_heads;    // of a row
  const bool adjacent = p.rope.adjacent != 0;
  if (sub >= heads) return;
  for (int u = wave * heads + sub; u < rows * units; u += kThreads / 64 * heads) {
    const int r = u / units, unit = u - r * units;
    const int64_t row = row0 + r;
    const f64x2 *cs = s_cs + r * half;
    float x[kVec];
    if (unit < p.n_q_heads) {
      const T *src = static_cast<const T *>(p.q) + row * p.q_stride + unit * D;
      Elem<T>::load(src + o, x);
      if constexpr (SINGLE)
        turn_single<T>(x, o, half, cs, src);
      else
        turn(x, o, half, adjacent, cs, [&](int i, float (&y)[kVec]) { Elem<T>::load(src + i, y); });
      Elem<T>::store(static_cast<T *>(p.q_out) + row * p.q_out_stride + unit * D + o, x);
      continue;
    }
    if constexpr (MODE == kRowTurn) continue;
    const int h = unit - p.n_q_heads;
    if constexpr (MODE == kRowAppend) {
      const int at = p.pos[row];
      if ((uint32_t)at >= (uint32_t)p.n_ctx) continue;
      const int64_t dst = kv_row(p.pages, at);
      const T *src = static_cast<const T *>(p.k_new) + row * p.k_new_stride + h * D;
      const T *vs = static_cast<const T *>(p.v_new) + row * p.v_new_stride + h * D + o;
      T *vd = static_cast<T *>(p.v) + dst * p.v_stride + h * D + o;
      const u32x4 va = ld16(vs);
      if constexpr (sizeof(T) == 4) st16(vd + 4, ld16(vs + 4));
      Elem<T>::load(src + o, x);
      turn(x, o, half, adjacent, cs, [&](int i, float (&y)[kVec]) { Elem<T>::load(src + i, y); });
      Elem<T>::store(static_cast<T *>(p.k) + dst * p.k_stride + h * D + o, x);
      st16(vd, va);
    }
    if constexpr (MODE == kRowAppendMx) {
      const T *src = static_cast<const T *>(p.k_new) + row * p.k_new_stride + h * D;
      float v[kVec];
      Elem<T>::load(static_cast<const T *>(p.v_new) + row * p.v_new_stride + h * D + o, v);
      Elem<T>::load(src + o, x);
      const bool bad = any_not_finite(x) || any_not_finite(v);
      turn(x, o, half, adjacent, cs, [&](int i, float (&y)[kVec]) { Elem<T>::load(src + i, y); });
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = Elem<T>::rounded(x[j]);
      int ks = block_scale(x), vsc = block_scale(v);
      uint32_t kc = pack(x, ks), vc = pack(v, vsc);
      // a head with an infinity or a NaN among its keys or values (before or
      // after the turn): the key is NaN, the value 0
      const uint64_t bads = __ballot(bad || any_not_finite(x));
      if (bads >> (sub * lanes) & (lanes == 16 ? 0xffffull : 0xffull)) {
        ks = kMxScaleNan;
        vsc = kMxScaleMin;
        kc = vc = 0;
      }
      if (p.k_out) {
        float y[kVec];
        unpack(kc, ks, y);
        Elem<T>::store(static_cast<T *>(p.k_out) + (row * p.n_kv_heads + h) * D + o, y);
      }
      if (p.v_out) {
        float y[kVec];
        unpack(vc, vsc, y);
        Elem<T>::store(static_cast<T *>(p.v_out) + (row * p.n_kv_heads + h) * D + o, y);
      }
      const int at = p.pos[row];
      if ((uint32_t)at >= (uint32_t)p.mx.n_ctx) continue;
      const int64_t page = mx_page(p.mx, (int)(row / p.mx.rows_per_seq), at);
      const int64_t slot = ((int64_t)h << p.mx.shift) + (at & ((1 << p.mx.shift) - 1));  // of the page
      const int64_t co = page * p.mx.code_stride + slot * (D / 2) + o / 2;
      const int64_t so = page * p.mx.scale_stride + slot * (D / kMxBlock) + o / kMxBlock;
      *reinterpret_cast<uint32_t *>(p.mx.k + co) = kc;
      *reinterpret_cast<uint32_t *>(p.mx.v + co) = vc;
      if (o % kMxBlock == 0) {
        p.mx.k_scale[so] = (uint8_t)ks;
        p.mx.v_scale[so] = (uint8_t)vsc;
      }
    }
    if constexpr (MODE == kRowLoadMx) {
      const int from = p.src_pos[row], at = p.pos[row];
      if ((uint32_t)from >= (uint32_t)p.mx.n_ctx || (uint32_t)at >= (uint32_t)p.n_ctx) continue;
      const int64_t page = mx_page(p.mx, (int)(row / p.mx.rows_per_seq), from);
      const int64_t slot = ((int64_t)h << p.mx.shift) + (from & ((1 << p.mx.shift) - 1));
      const int64_t co = page * p.mx.code_stride + slot * (D / 2);
      const int64_t so = page * p.mx.scale_stride + slot * (D / kMxBlock);
      auto key = [&](int i, float (&y)[kVec]) {
        unpack(*reinterpret_cast<const uint32_t *>(p.mx.k + co + i / 2), p.mx.k_scale[so + i / kMxBlock], y);
      };
      float v[kVec];
      unpack(*reinterpret_cast<const uint32_t *>(p.mx.v + co + o / 2), p.mx.v_scale[so + o / kMxBlock], v);
      key(o, x);
      turn(x, o, half, adjacent, cs, key);
      const int64_t dst = kv_row(p.pages, at);
      Elem<T>::store(static_cast<T *>(p.k) + dst * p.k_stride + h * D + o, x);
      Elem<T>::store(static_cast<T *>(p.v) + dst * p.v_stride + h * D + o, v);
    }
  }
}

template <typename T>
void launch_mode(const RowParams &p, RowMode mode, dim3 grid, size_t lds, hipStream_t s) {
  if (mode == kRowTurn && !p.rope.adjacent && p.rope.half % kVec)
    rows_kernel<T, kRowTurn, true><<<grid, kThreads, lds, s>>>(p);
  else if (mode == kRowTurn)
    rows_kernel<T, kRowTurn, false><<<grid, kThreads, lds, s>>>(p);
  else if (mode == kRowAppend)
    rows_kernel<T, kRowAppend, false><<<grid, kThreads, lds, s>>>(p);
  else if (mode == kRowAppendMx)
    rows_kernel<T, kRowAppendMx, false><<<grid, kThreads, lds, s>>>(p);
  else
    rows_kernel<T, kRowLoadMx, false><<<grid, kThreads, lds, s>>>(p);
}

}  // namespace

hipError_t launch_rows(const RowParams &p_in, RowMode mode, bool bf16, hipStream_t s) {
  static const char *const names[] = {"rotary", "append", "append_mx", "load_mx"};
  ProfScope ps(names[mode], s);
  RowParams p = p_in;
  // Rows of a workgroup: up to 8 share one pass over the angles' code and keep
  // its LDS at 16 KB or less; fewer while there are not enough workgroups for
  // every CU to hold several.
  p.rows_per_block = (int32_t)min(8, max(1, p.n / 1024));
  const dim3 grid((p.n + p.rows_per_block - 1) / p.rows_per_block);
  const size_t lds = (size_t)p.rows_per_block * p.rope.half * sizeof(f64x2);
  if (bf16)
    launch_mode<u16>(p, mode, grid, lds, s);
  else
    launch_mode<float>(p, mode, grid, lds, s);
  return hipGetLastError();
}

}  // namespace conduit
