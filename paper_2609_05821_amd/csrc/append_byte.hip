// New rows into the 8-bit cache, quantised as they are written, gfx950.
//
// 16 tokens and a head share a scale, so the unit of work is a run: the rows of a
// call that go to one block of 16 tokens.  A wave takes a run's keys and values of one
// head whole, 16 dims a lane and 16 tokens (2,048 elements at head_dim 128): their
// largest magnitudes need no exchange beyond the wave, and the codes are written once.
//   scale    s = the smallest with max|x| <= 448 2^(s - 127) over the rows written, and no
//            less than the block's while it keeps other tokens.  A power of two: codes
//            keep their 4 significant bits when it rises (but for those that fall below
//            the smallest normal code), and it can only rise by what the rows need.
//   kept     tokens of the block that the call does not write are read and rounded again
//            only when the scale rises.
// Which rows begin a run is found from the positions: a workgroup looks at `window` rows,
// at the row before them that goes anywhere, and at the rows after that may belong to
// its last run.  Angles are computed in 64 bits, once per run, and shared by its heads
// through LDS.  Queries are turned by workgroups of their own in the same launch.
#include <algorithm>
#include <cfloat>

#include "rows.h"

namespace conduit {
namespace {

constexpr int kMaxWaves = 4;  // heads of a run that a workgroup takes side by side
// Rows of a window: 1 keeps the chip busy with few rows (the rows that continue a
// run leave at once), 16 saves those workgroups where there are many.
constexpr int kWindow = 16;
constexpr int kWindowFrom = 4096;
constexpr int kQueryRows = 4;  // rows of a workgroup that turns queries (1 below kWindowFrom rows)

// A lane's 16 dims of a head: two vectors of 8, which turn together where they are
// the two halves of pairs (t >= 0: the first of 8 frequencies).
struct LaneDims {
  int at[2];
  int t;
};
template <int D>
__device__ __forceinline__ LaneDims lane_dims(int l, int half, bool adjacent) {
  const int turning = adjacent ? 0 : half / kVec;  // lanes that hold pairs in halves
  if (l < turning) return {{kVec * l, half + kVec * l}, kVec * l};
  const int base = 2 * kVec * turning + kVec * (l - turning);
  return {{base, base + kVec * (D / 16 - turning)}, -1};
}

template <int D>
__device__ __forceinline__ void turn(float (&x)[2][kVec], const LaneDims &d, int half, bool adjacent, const f64x2 *cs) {
  if (d.t >= 0) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const f64x2 t = cs[d.t + j];
      const double a = x[0][j], b = x[1][j];
      x[0][j] = to_f32(__builtin_fma(a, t[0], -(b * t[1])));
      x[1][j] = to_f32(__builtin_fma(b, t[0], a * t[1]));
    }
  } else if (adjacent) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (d.at[i] >= 2 * half) continue;  // (rot_dim is a multiple of 16, so of a vector)
#pragma unroll
      for (int j = 0; j < kVec / 2; ++j) {
        const f64x2 t = cs[d.at[i] / 2 + j];
        const double a = x[i][2 * j], b = x[i][2 * j + 1];
        x[i][2 * j] = to_f32(__builtin_fma(a, t[0], -(b * t[1])));
        x[i][2 * j + 1] = to_f32(__builtin_fma(b, t[0], a * t[1]));
      }
    }
  }
}

// Cosines and sines of row `row` at frequency f.
__device__ __forceinline__ f64x2 angle(const RopeTable &rope, int row, int f) {
  const int32_t *pos = rope.pos + row;
  int32_t at[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) at[a] = a < rope.n_axes ? pos[a * rope.pos_stride] : 0;
  const int axis = rope.axis[f];
  return cos_sin((double)(axis < 2 ? axis ? at[1] : at[0] : axis == 2 ? at[2] : at[3]) * (double)rope.inv_freq[f]);
}

// x as a cache of T would hold it.
__device__ __forceinline__ void as_held(const float (&x)[kVec], Raw<u16> &r) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x2 b = {static_cast<__bf16>(x[2 * j]), static_cast<__bf16>(x[2 * j + 1])};
    r.w[0][j] = __builtin_bit_cast(uint32_t, b);
  }
}
__device__ __forceinline__ void as_held(const float (&x)[kVec], Raw<float> &r) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) r.w[j / 4][j % 4] = __builtin_bit_cast(uint32_t, x[j]);
}

// Largest magnitude, as the bits of an fp32 number (infinities and NaNs are the largest).
__device__ __forceinline__ uint32_t largest_bits(const Raw<u16> &r) {
  uint32_t hi = 0, lo = 0;  // (of both halves the upper is enough with the lower below it)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = r.w[0][j];
    hi = max(hi, w & 0x7fffffffu);
    lo = max(lo, w << 16 & 0x7fffffffu);
  }
  return max(hi, lo) & 0xffff0000u;
}
__device__ __forceinline__ uint32_t largest_bits(const Raw<float> &r) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < kVec; ++j) m = max(m, (uint32_t)r.w[j / 4][j % 4] & 0x7fffffffu);
  return m;
}

// The smallest scale byte that holds magnitudes up to m: 448 = 1.75 * 2^8, so the
// exponent less 8, one more where the mantissa is above 1.75.
__device__ __forceinline__ int needed_scale(uint32_t m) {
  return min(max((int)((m + 0x1fffffu) >> 23) - 8, kByteScaleMin), kByteScaleMax);
}

typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float scale) {
  i16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint2 encode8(const float (&x)[kVec], float scale) {
  return make_uint2(encode4(x[0], x[1], x[2], x[3], scale), encode4(x[4], x[5], x[6], x[7], scale));
}
__device__ __forceinline__ void decode8(uint2 c, float scale, float (&x)[kVec]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w = i ? c.y : c.x;
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    x[4 * i] = lo[0], x[4 * i + 1] = lo[1], x[4 * i + 2] = hi[0], x[4 * i + 3] = hi[1];
  }
}

// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float two_to(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// Queries of rows [row0, row0 + n): the workgroup's threads go over the heads' lanes.
template <typename T, int D>
__device__ __forceinline__ void turn_queries(const RowParams &p, int row0, int n, f64x2 *cs) {
  constexpr int LR = D / 16;
  const int half = p.rope.half, tid = threadIdx.x;
  const bool adjacent = p.rope.adjacent != 0;
  for (int e = tid; e < n * half; e += blockDim.x) cs[e] = angle(p.rope, row0 + e / half, e % half);
  __syncthreads();
  const int items = n * p.n_q_heads * LR;
  const LaneDims d = lane_dims<D>(tid % LR, half, adjacent);  // (blockDim is a multiple of LR)
  const int gap = half / kVec % 4 && !adjacent ? 4 : 0;
  constexpr int K = 2;
  for (int e0 = tid; e0 < items; e0 += K * blockDim.x) {
    Raw<T> raw[K][2];
    int row[K], at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int unit = min(e0 + k * (int)blockDim.x, items - LR + tid % LR) / LR;
      row[k] = unit / p.n_q_heads;
      at[k] = (unit - row[k] * p.n_q_heads) * D;
      const T *src = static_cast<const T *>(p.q) + (int64_t)(row0 + row[k]) * p.q_stride + at[k];
#pragma unroll
      for (int i = 0; i < 2; ++i) raw[k][i] = load_raw<T>(src + d.at[i]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (e0 + k * (int)blockDim.x >= items) break;
      float x[2][kVec];
#pragma unroll
      for (int i = 0; i < 2; ++i) expand(raw[k][i], x[i]);
      turn<D>(x, d, half, adjacent, cs + row[k] * half);
      T *dst = static_cast<T *>(p.q_out) + (int64_t)(row0 + row[k]) * p.q_out_stride + at[k];
#pragma unroll
      for (int i = 0; i < 2; ++i) store(dst + d.at[i], x[i], gap);
    }
  }
}

// Workgroups [0, n_runs): windows of rows, for up to 4 KV heads each.  The others: queries.
template <typename T, int D>
__global__ __launch_bounds__(64 * kMaxWaves) void append_byte_kernel(ByteAppendParams a, int window, int n_runs,
                                                                   int query_rows) {
  constexpr int LR = D / 16;        // lanes of a token's head
  constexpr int RP = 64 / LR;       // tokens that the lanes hold
  constexpr int SL = kByteBlock / RP;  // tokens of a lane
  __shared__ f64x2 s_cs[kByteBlock * D / 2];
  __shared__ int s_row[kMaxWaves][kByteBlock];  // the run's row of each token of the block, or -1
  const RowParams &p = a.rows;
  if ((int)blockIdx.x >= n_runs) {
    const int row0 = ((int)blockIdx.x - n_runs) * query_rows;
    turn_queries<T, D>(p, row0, min(query_rows, p.n - row0), s_cs);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int waves = blockDim.x >> 6, head_groups = (p.n_kv_heads + waves - 1) / waves;
  const int row0 = (int)blockIdx.x / head_groups * window;
  const int h = (int)blockIdx.x % head_groups * waves + wave;
  const int r = p.mx.rows_per_seq, half = p.rope.half;
  const bool adjacent = p.rope.adjacent != 0;

  // The window's rows and 64 - window more, and the 64 before them.
  const int i = row0 + lane;
  const int at = i < p.n ? p.pos[i] : -1;
  const int back = row0 - 64 + lane;
  const int back_at = back >= 0 ? p.pos[back] : -1;
  const bool live = (uint32_t)at < (uint32_t)p.mx.n_ctx;
  const int block = at >> 4, seq = (int)((uint32_t)min(i, p.n - 1) / (uint32_t)r);
  static_assert(kByteBlock == 16, "blocks of positions");
  const uint64_t lives = __ballot(live), in_window = (1ull << window) - 1;  // (window < 64)
  const uint64_t before = lives & ((1ull << lane) - 1);
  const int prev = before ? 63 - __builtin_clzll(before) : lane;
  const int prev_block = __shfl(block, prev, 64), prev_seq = __shfl(seq, prev, 64);  // (by all lanes)
  const bool continues = before && prev_block == block && prev_seq == seq;
  uint64_t leaders = __ballot(live && !continues) & in_window;
  if (lives & in_window) {
    // does the window's first row that goes anywhere continue a run?
    const int f = __builtin_ctzll(lives & in_window);
    const int f_block = __builtin_amdgcn_readlane(block, f), start = __builtin_amdgcn_readlane(seq, f) * r;
    int j = back, j_at = back_at;
    for (int base = row0; base > start; base -= 64) {
      if (base < row0) {
        j = base - 64 + lane;
        j_at = j >= start ? p.pos[j] : -1;
      }
      const uint64_t there = __ballot(j >= start && (uint32_t)j_at < (uint32_t)p.mx.n_ctx);
      if (there) {
        if (__builtin_amdgcn_readlane(j_at, 63 - __builtin_clzll(there)) >> 4 == f_block) leaders &= ~(1ull << f);
        break;
      }
    }
  }
  // Rows that are left out are held by nobody, but may be asked for.
  uint64_t outs = p.k_out || p.v_out ? __ballot(i < p.n && !live) & in_window : 0;

  const int l = lane % LR;
  const LaneDims d = lane_dims<D>(l, half, adjacent);
  const int gap = half / kVec % 4 && !adjacent ? 4 : 0;
  while (leaders | outs) {
    const int first = __builtin_ctzll(leaders | outs);
    const bool out = outs >> first & 1;
    leaders &= ~(1ull << first);
    outs &= ~(1ull << first);
    const int run_block = __builtin_amdgcn_readlane(block, first), run_seq = __builtin_amdgcn_readlane(seq, first);
    int *rows = s_row[wave];

    // The run's rows.
    const bool member = out ? lane == first : live && lane >= first && block == run_block && seq == run_seq;
    wave_lds_fence();
    if (lane < kByteBlock) rows[lane] = -1;
    wave_lds_fence();
    if (member) rows[out ? 0 : at & (kByteBlock - 1)] = i;
    wave_lds_fence();
    if (!out && !__ballot(live && lane > first && !member) && rows[kByteBlock - 1] < 0) {
      // no other row among these 64: the run may go on behind them
      const int end = min((int64_t)(run_seq + 1) * r, (int64_t)p.n);
      for (int base = row0 + 64; base < end; base += 256) {
        int x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = base + 64 * k + lane < end ? p.pos[base + 64 * k + lane] : -1;
        bool other = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if ((uint32_t)x[k] >= (uint32_t)p.mx.n_ctx) continue;
          if (x[k] >> 4 == run_block) rows[x[k] & (kByteBlock - 1)] = base + 64 * k + lane;
          else other = true;
        }
        if (__ballot(other)) break;
      }
      wave_lds_fence();
    }
    const uint32_t written = (uint32_t)__ballot(rows[lane & (kByteBlock - 1)] >= 0) & 0xffffu;

    // The lane's tokens on their way, and where the block lies.
    int row[SL];
    Raw<T> kr[SL][2], vr[SL][2];
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      row[t] = h < p.n_kv_heads ? rows[lane / LR + RP * t] : -1;
      if (row[t] >= 0) {
        const T *k = static_cast<const T *>(p.k_new) + row[t] * p.k_new_stride + h * D;
        const T *v = static_cast<const T *>(p.v_new) + row[t] * p.v_new_stride + h * D;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          kr[t][x] = load_raw<T>(k + d.at[x]);
          vr[t][x] = load_raw<T>(v + d.at[x]);
        }
      }
    }
    const int token0 = out ? 0 : run_block * kByteBlock;
    const int64_t page = mx_page(p.mx, run_seq, token0);
    const int64_t slot = ((int64_t)min(h, p.n_kv_heads - 1) << p.mx.shift) + (token0 & ((1 << p.mx.shift) - 1));
    const int64_t codes = page * p.mx.code_stride + slot * D;
    const int64_t scale = page * p.mx.scale_stride + slot / kByteBlock;
    // tokens that the block keeps
    const int held = out          ? 0
                     : a.n_held ? min(max(a.n_held[run_seq], 0), p.mx.n_ctx)
                                  : token0 + 31 - __builtin_clz(written);
    const uint32_t kept = ~written & ((1u << min(max(held - token0, 0), kByteBlock)) - 1);
    const int k_was = p.mx.k_scale[scale], v_was = p.mx.v_scale[scale];

    // The run's angles.
    if (half) {
      __syncthreads();
      for (int e = tid; e < kByteBlock * half; e += blockDim.x) {
        const int t = e / half;
        if (rows[t] >= 0) s_cs[e] = angle(p.rope, rows[t], e - t * half);
      }
      __syncthreads();
    }

    bool bad[SL];  // a token with an infinity or a NaN among its keys or values: NaN keys, zero values
    uint32_t km = 0, vm = 0;
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      uint32_t m = 0, n = 0;
      if (row[t] >= 0) {
        if (half) {
          float x[2][kVec];
          expand(kr[t][0], x[0]);
          expand(kr[t][1], x[1]);
          turn<D>(x, d, half, adjacent, s_cs + (lane / LR + RP * t) * half);
          as_held(x[0], kr[t][0]);
          as_held(x[1], kr[t][1]);
        }
        m = max(largest_bits(kr[t][0]), largest_bits(kr[t][1]));
        n = max(largest_bits(vr[t][0]), largest_bits(vr[t][1]));
      }
      const uint64_t any = __ballot(max(m, n) >= 0x7f800000u);
      bad[t] = any >> (lane - l) & ((1ull << LR) - 1);
      km = max(km, bad[t] ? 0 : m);
      vm = max(vm, bad[t] ? 0 : n);
    }
    auto most = [](uint32_t x, uint32_t y) { return max(x, y); };
    km = wave_reduce(km, 0u, most);
    vm = wave_reduce(vm, 0u, most);
    if (h >= p.n_kv_heads) continue;

    auto finish = [&](const Raw<T> (&raw)[SL][2], uint32_t m, int was, uint8_t *pool, uint8_t *scales, void *held_out,
                      bool keys) __attribute__((always_inline)) {
      int now = needed_scale(m);
      was = min(max(was, kByteScaleMin), kByteScaleMax);
      if (kept) now = max(now, was);
      const float s = two_to(now - 127);
      const bool rises = kept && now > was;
      const float step = two_to(min(now - was, 64));
#pragma unroll
      for (int t = 0; t < SL; ++t) {
        const int token = lane / LR + RP * t;
        uint2 c[2];
        if (row[t] >= 0) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float x[kVec];
            expand(raw[t][y], x);
            if (m > 0x7f600000u)  // above 448 * 2^(246 - 127): the largest code
#pragma unroll
              for (int j = 0; j < kVec; ++j) x[j] = fminf(fmaxf(x[j], -0x1.cp127f), 0x1.cp127f);
            c[y] = encode8(x, s);
            if (bad[t]) c[y] = keys ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu) : make_uint2(0, 0);
          }
          if (held_out) {
            T *dst = static_cast<T *>(held_out) + ((int64_t)row[t] * p.n_kv_heads + h) * D;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float z[kVec];
              decode8(c[y], s, z);
              store(dst + d.at[y], z, gap);
            }
          }
        } else if (rises && kept >> token & 1) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float z[kVec];
            decode8(*reinterpret_cast<const uint2 *>(pool + codes + token * D + d.at[y]), 1.f, z);
            c[y] = encode8(z, step);
          }
        } else {
          continue;
        }
        if (out) continue;
#pragma unroll
        for (int y = 0; y < 2; ++y) *reinterpret_cast<uint2 *>(pool + codes + token * D + d.at[y]) = c[y];
      }
      if (!out && lane == 0) scales[scale] = (uint8_t)now;
    };
    finish(kr, km, k_was, p.mx.k, p.mx.k_scale, p.k_out, true);
    finish(vr, vm, v_was, p.mx.v, p.mx.v_scale, p.v_out, false);
  }
}

template <typename T, int D>
void launch(const ByteAppendParams &a, hipStream_t s) {
  const RowParams &p = a.rows;
  const bool many = p.n >= kWindowFrom;
  const int window = many ? kWindow : 1, query_rows = many ? kQueryRows : 1;
  const int waves = std::min(p.n_kv_heads, kMaxWaves), groups = (p.n_kv_heads + waves - 1) / waves;
  const int n_runs = (p.n + window - 1) / window * groups;
  const int grid = n_runs + (p.n_q_heads ? (p.n + query_rows - 1) / query_rows : 0);
  append_byte_kernel<T, D><<<grid, 64 * waves, 0, s>>>(a, window, n_runs, query_rows);
}

}  // namespace

hipError_t launch_append_byte(const ByteAppendParams &a, bool bf16, hipStream_t s) {
  ProfScope ps("append_byte", s);
  if (a.rows.head_dim == 128)
    bf16 ? launch<u16, 128>(a, s) : launch<float, 128>(a, s);
  else
    bf16 ? launch<u16, 64>(a, s) : launch<float, 64>(a, s);
  return hipGetLastError();
}

}  // namespace conduit
