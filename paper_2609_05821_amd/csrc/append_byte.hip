// New rows into the 8-bit cache, quantised as they are written, gfx950.
//
// 16 tokens and a head share a scale, so the unit of work is a run: the rows of a
// call that go to one block of 16 tokens.  A wave takes a run's keys or values of one
// head whole, 16 dims a lane and 16 tokens (2,048 elements at head_dim 128): their
// largest magnitude needs no exchange beyond the wave, and the codes are written once.
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
//
// Bound by memory where there are many rows, by the chain of loads before the first store
// (positions, page and what the block holds, rows, angles) where there are few.  Measured, 4 KV heads
// of 128: a prompt of 17,024 bf16 rows with 28 query heads, keys and queries turned, 63 us, 4.7 TB/s
// (a copy of 4 GiB: 4.5); 65,536 fp32 rows 92 us, 3.7 TB/s; 1,638 rows here and there with their
// queries 14 us, 2.0 TB/s; 64 tokens of as many sequences 7 us.
#include <algorithm>
#include <cfloat>

#include "rows.h"

namespace conduit {
namespace {

// Heads of a run that a workgroup takes side by side, two waves each: one has the keys,
// the other the values.
constexpr int kMaxHeads = 4;
constexpr int kMaxWaves = 2 * kMaxHeads;
// Rows of a window.  Fewer keep the chip busy with few rows (rows that continue a run leave at once) and take
// their runs of one or two rows side by side, a wave each, before the longer ones; windows of 16 have
// workgroups of their own for such runs; with many rows these are left out, and the code for them, whose
// registers leave fewer waves.  Rows of a prompt, and rows here and there over ten times as many tokens,
// keys, values and 28 query heads over 4, in us:
//   rows                                    1,638      2,200      4,000      8,000      20,000
//   windows of 4                            13   14    18   18    28   28    52   58
//   16, short runs apart                    12   21    12   22    18   23    32   46    88  115
//   16, short runs like others                                                          74  119
// (100 rows in windows of 2 and of 4: 9 10 and 10 11; 400: 9 11 and 10 12; 1,000: 14 13 and 10 12.)
constexpr int kWindow = 16, kWindowFew = 4, kWindowLeast = 2;
constexpr int kWindowFewFrom = 512, kWindowFrom = 2048, kManyFrom = 8192;
// Rows of a workgroup that turns queries, and from how many rows on.  With the most, whose angles fill the LDS
// of a block's, a launch has fewer than 2^32 threads for all rows, heads and dims that a call takes (up to 0.8 of that);
// two a workgroup pass it at 2^24 rows of 4 heads, and the launch then leaves queries out without an error.  (2^22
// rows, 4 heads of 64 each: 2 rows a workgroup 7.0 ms, 16 rows 3.3.)
constexpr int kQueryRows = 2, kQueryRowsFrom = 512;
constexpr int kQueryRowsMost = kByteBlock, kQueryRowsMostFrom = 1 << 22;

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
      __builtin_amdgcn_sched_barrier(0);  // (angles of one pair in registers at a time)
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
        __builtin_amdgcn_sched_barrier(0);
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
  const int32_t x = axis < 2 ? axis ? at[1] : at[0] : axis == 2 ? at[2] : at[3];
  return cos_sin<true>((double)x * (double)rope.inv_freq[f]);
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

// Queries of rows [row0, row0 + n): the workgroup's threads go over the heads' lanes, the first
// loads on their way before the angles are worked out.
template <typename T, int D>
__device__ __forceinline__ void turn_queries(const RowParams &p, int row0, int n, f64x2 *cs) {
  constexpr int LR = D / 16;
  const int half = p.rope.half, tid = threadIdx.x;
  const bool adjacent = p.rope.adjacent != 0;
  const int items = n * p.n_q_heads * LR;
  const LaneDims d = lane_dims<D>(tid % LR, half, adjacent);  // (the threads are a multiple of LR)
  const int gap = half / kVec % 4 && !adjacent ? 4 : 0;
  Raw<T> raw[2];
  int row = 0, at = 0;
  auto fetch = [&](int item) __attribute__((always_inline)) {
    const int unit = min(item, items - 1) / LR;
    row = unit / p.n_q_heads;
    at = (unit - row * p.n_q_heads) * D;
    const T *src = static_cast<const T *>(p.q) + (int64_t)(row0 + row) * p.q_stride + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) raw[i] = load_raw<T>(src + d.at[i]);
  };
  fetch(tid);
  for (int e = tid; e < n * half; e += blockDim.x) cs[e] = angle(p.rope, row0 + e / half, e % half);
  __syncthreads();
  for (int e = tid; e < items;) {
    float x[2][kVec];
#pragma unroll
    for (int i = 0; i < 2; ++i) expand(raw[i], x[i]);
    turn<D>(x, d, half, adjacent, cs + row * half);
    T *dst = static_cast<T *>(p.q_out) + (int64_t)(row0 + row) * p.q_out_stride + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) store(dst + d.at[i], x[i], gap);
    e += blockDim.x;
    if (e < items) fetch(e);
  }
}

// Workgroups [0, n_runs): windows of rows, for up to 4 KV heads each.  The next n_brief: the windows' runs of
// one or two rows (0: they are among the first).  The others: queries.
// BRIEF: with a path of their own for runs of one or two rows.
template <typename T, int D, bool BRIEF>
__global__ __launch_bounds__(64 * kMaxWaves, BRIEF || (sizeof(T) == 4 && D == 128) ? 4 : 6)
void append_byte_kernel(ByteAppendParams a, int window, int n_runs, int n_brief, int query_rows) {
  constexpr int LR = D / 16;        // lanes of a token's head
  constexpr int RP = 64 / LR;       // tokens that the lanes hold
  constexpr int SL = kByteBlock / RP;  // tokens of a lane
  __shared__ f64x2 s_cs[kByteBlock * D / 2];
  __shared__ int s_row[kMaxWaves][kByteBlock];  // the run's row of each token of the block, or -1
  __shared__ uint64_t s_bad[2][kMaxWaves][SL];  // lanes whose token is not finite there
  const RowParams &p = a.rows;
  if ((int)blockIdx.x >= n_runs + n_brief) {
    const int row0 = ((int)blockIdx.x - n_runs - n_brief) * query_rows;
    turn_queries<T, D>(p, row0, min(query_rows, p.n - row0), s_cs);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = blockDim.x >> 7, head_groups = (p.n_kv_heads + heads - 1) / heads;
  const bool for_brief = BRIEF && (int)blockIdx.x >= n_runs;
  const int row0 = (for_brief ? (int)blockIdx.x - n_runs : (int)blockIdx.x / head_groups) * window;
  const int h = (int)blockIdx.x % head_groups * heads + (wave >> 1);
  const bool keys = !(wave & 1);
  const int r = p.mx.rows_per_seq, half = p.rope.half;
  const bool adjacent = p.rope.adjacent != 0;

  // The window's rows and 64 - window more, and the 64 before them.
  const int i = row0 + lane;
  const int at = i < p.n ? p.pos[i] : -1;
  const int back = row0 - 64 + lane;
  const int back_at = back >= 0 ? p.pos[back] : -1;
  const int seq = (int)((uint32_t)min(i, p.n - 1) / (uint32_t)r);
  const int held_at = a.n_held ? a.n_held[seq] : 0;
  const bool live = (uint32_t)at < (uint32_t)p.mx.n_ctx;
  const int block = at >> 4;
  // (what a run needs to know is asked for a row a lane, before the runs are known)
  const int page_at = mx_page(p.mx, seq, live ? at : 0);
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
  // A run: its rows (the row of each token of its block, or -1), the tokens that they are, and
  // what the block keeps.
  int *rows = s_row[wave];
  struct Run {
    bool out;
    int seq, token0, page;
    uint32_t written, kept;
  };
  // Where the run lies whose first row is lane `first`'s, and what its block keeps.
  auto place_run = [&](Run &x, int first) __attribute__((always_inline)) {
    x.token0 = x.out ? 0 : __builtin_amdgcn_readlane(block, first) * kByteBlock;
    x.page = __builtin_amdgcn_readlane(page_at, first);
    const int held = x.out          ? 0
                     : a.n_held ? min(max(__builtin_amdgcn_readlane(held_at, first), 0), p.mx.n_ctx)
                                    : x.token0 + 31 - __builtin_clz(x.written);
    x.kept = ~x.written & ((1u << min(max(held - x.token0, 0), kByteBlock)) - 1);
  };
  auto run_of = [&](int first) __attribute__((always_inline)) {
    Run x;
    x.out = outs >> first & 1;
    x.seq = __builtin_amdgcn_readlane(seq, first);
    const int run_block = __builtin_amdgcn_readlane(block, first);
    const bool member = x.out ? lane == first : live && lane >= first && block == run_block && seq == x.seq;
    wave_lds_fence();
    if (lane < kByteBlock) rows[lane] = -1;
    wave_lds_fence();
    if (member) atomicMax(&rows[x.out ? 0 : at & (kByteBlock - 1)], i);
    wave_lds_fence();
    if (!x.out && !__ballot(live && lane > first && !member)) {
      // no other row among these 64: the run may go on behind them (also one that has its last token, which
      // a later row may have again)
      const int end = min((int64_t)(x.seq + 1) * r, (int64_t)p.n);
      for (int base = row0 + 64; base < end; base += 256) {
        int y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = base + 64 * k + lane < end ? p.pos[base + 64 * k + lane] : -1;
        bool other = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if ((uint32_t)y[k] >= (uint32_t)p.mx.n_ctx) continue;
          if (y[k] >> 4 == run_block) atomicMax(&rows[y[k] & (kByteBlock - 1)], base + 64 * k + lane);
          else other = true;
        }
        if (__ballot(other)) break;
      }
      wave_lds_fence();
    }
    x.written = (uint32_t)__ballot(rows[lane & (kByteBlock - 1)] >= 0) & 0xffffu;
    place_run(x, first);
    return x;
  };
  // Codes and scale byte of a run's block for one head.
  struct Place {
    uint8_t *codes, *scale;
  };
  auto place = [&](const Run &x, int head, bool k) __attribute__((always_inline)) {
    const int64_t slot = ((int64_t)head << p.mx.shift) + (x.token0 & ((1 << p.mx.shift) - 1));
    return Place{(k ? p.mx.k : p.mx.v) + x.page * p.mx.code_stride + slot * D,
                 (k ? p.mx.k_scale : p.mx.v_scale) + x.page * p.mx.scale_stride + slot / kByteBlock};
  };
  auto encode = [&](const Raw<T> &raw, uint32_t m, float s, bool bad, bool k) __attribute__((always_inline)) {
    float x[kVec];
    expand(raw, x);
    if (m > 0x7f600000u)  // above 448 * 2^(246 - 127): the largest code
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = fminf(fmaxf(x[j], -0x1.cp127f), 0x1.cp127f);
    const uint2 c = encode8(x, s);
    return !bad ? c : k ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu) : make_uint2(0, 0);
  };
  auto give_back = [&](T *held, int row, int head, const uint2 (&c)[2], float s) __attribute__((always_inline)) {
    T *dst = held + ((int64_t)row * p.n_kv_heads + head) * D;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      float z[kVec];
      decode8(c[y], s, z);
      store(dst + d.at[y], z, gap);
    }
  };
  auto again = [&](uint2 c, float step) __attribute__((always_inline)) {
    float z[kVec];
    decode8(c, 1.f, z);
    return encode8(z, step);
  };

  // Runs of one or two rows (and rows that are left out): a wave each, side by side.
  uint64_t brief = 0;
  int second = lane;  // the lane of the run's other row
  if constexpr (BRIEF) {
    const uint64_t all_leaders = __ballot(live && !continues), later = lane < 63 ? all_leaders >> (lane + 1) : 0;
    const int next = later ? lane + 1 + __builtin_ctzll(later) : 64;
    const uint64_t own = lives >> lane & (next < 64 ? (1ull << (next - lane)) - 1 : ~0ull);
    if (__builtin_popcountll(own) == 2) second = lane + 63 - __builtin_clzll(own);
    brief = (__ballot(__builtin_popcountll(own) <= 2 && (next < 64 || row0 + 64 >= p.n)) & leaders) | outs;
  }
  if (BRIEF && (n_brief ? for_brief : (int)blockIdx.x % head_groups == 0)) {  // (one workgroup for all heads)
    constexpr int kUnits = 64 / LR;  // heads' keys or values side by side
    const int n_units = 2 * p.n_kv_heads;
    f64x2 *cs = s_cs + 2 * wave * half;
    uint64_t todo = brief;
    for (int skip = wave; skip > 0; --skip) todo &= todo - 1;
    while (todo) {
      const int first = __builtin_ctzll(todo);
      Run x;
      x.out = outs >> first & 1;
      for (int skip = 2 * heads; skip > 0; --skip) todo &= todo - 1;
      // (one row, or the later of two with one position: the same twice)
      const int other = x.out ? first : __builtin_amdgcn_readlane(second, first);
      int token[2] = {0, 0}, row[2] = {row0 + first, row0 + other};
      if (!x.out) {
        token[0] = __builtin_amdgcn_readlane(at, first) & (kByteBlock - 1);
        token[1] = __builtin_amdgcn_readlane(at, other) & (kByteBlock - 1);
        if (token[0] == token[1]) row[0] = row[1];
      }
      x.written = 1u << token[0] | 1u << token[1];
      place_run(x, first);
      for (int u0 = 0; u0 < n_units; u0 += kUnits) {
        const int u = min(u0 + lane / LR, n_units - 1), head = u >> 1;
        const bool k = !(u & 1), valid = u0 + lane / LR < n_units;
        const T *src = static_cast<const T *>(k ? p.k_new : p.v_new) + head * D;
        const int64_t stride = k ? p.k_new_stride : p.v_new_stride;
        Raw<T> raw[2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int z = 0; z < 2; ++z) raw[y][z] = load_raw<T>(src + row[y] * stride + d.at[z]);
        const Place at_place = place(x, head, k);
        const int was = min(max((int)*at_place.scale, kByteScaleMin), kByteScaleMax);
        if (half && !u0) {
          for (int e = lane; e < 2 * half; e += 64) {
            const int y = e >= half;
            cs[e] = angle(p.rope, y ? row[1] : row[0], y ? e - half : e);
          }
          wave_lds_fence();
        }
        bool bad[2];
        uint32_t m = 0;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          if (half && k) {
            float z[2][kVec];
            expand(raw[y][0], z[0]);
            expand(raw[y][1], z[1]);
            turn<D>(z, d, half, adjacent, cs + y * half);
            as_held(z[0], raw[y][0]);
            as_held(z[1], raw[y][1]);
          }
          const uint32_t largest = max(largest_bits(raw[y][0]), largest_bits(raw[y][1]));
          const uint64_t any = __ballot(largest >= 0x7f800000u);  // of a head's keys and values
          bad[y] = any >> (lane & ~(2 * LR - 1)) & ((1ull << (2 * LR)) - 1);
          m = max(m, bad[y] ? 0 : largest);
        }
        m = max(m, dpp_mov<kDppXor1>(0u, m));
        m = max(m, dpp_mov<kDppXor2>(0u, m));
        if (LR == 8) m = max(m, dpp_mov<kDppHalfMirror>(0u, m));
        if (!valid) continue;
        int now = needed_scale(m);
        if (x.kept) now = max(now, was);
        const float s = two_to(now - 127);
        T *held_out = static_cast<T *>(k ? p.k_out : p.v_out);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          if (y && token[1] == token[0]) continue;
          const uint2 c[2] = {encode(raw[y][0], m, s, bad[y], k), encode(raw[y][1], m, s, bad[y], k)};
          if (held_out) give_back(held_out, row[y], head, c, s);
          if (x.out) continue;
#pragma unroll
          for (int z = 0; z < 2; ++z) *reinterpret_cast<uint2 *>(at_place.codes + token[y] * D + d.at[z]) = c[z];
        }
        if (x.out) continue;
        if (x.kept && now > was) {
          // four of the kept tokens on their way at a time
          const float step = two_to(min(now - was, 64));
          for (int t0 = 0; t0 < kByteBlock; t0 += 4) {
            uint2 c[4][2];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int z = 0; z < 2; ++z)
                c[t][z] = *reinterpret_cast<const uint2 *>(at_place.codes + (t0 + t) * D + d.at[z]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
              if (x.kept >> (t0 + t) & 1)
#pragma unroll
                for (int z = 0; z < 2; ++z)
                  *reinterpret_cast<uint2 *>(at_place.codes + (t0 + t) * D + d.at[z]) = again(c[t][z], step);
          }
        }
        if (l == 0) *at_place.scale = (uint8_t)now;
      }
    }
  }
  if (for_brief) return;
  leaders &= ~brief;
  outs &= ~brief;

  for (int turn_of = 0; leaders | outs; turn_of ^= 1) {
    const int first = __builtin_ctzll(leaders | outs);
    const Run run = run_of(first);
    leaders &= ~(1ull << first);
    outs &= ~(1ull << first);

    // The lane's tokens on their way, and where the block lies.
    int row[SL];
    Raw<T> raw[SL][2];
    const T *src = static_cast<const T *>(keys ? p.k_new : p.v_new) + h * D;
    const int64_t stride = keys ? p.k_new_stride : p.v_new_stride;
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      row[t] = h < p.n_kv_heads ? rows[lane / LR + RP * t] : -1;
      if (row[t] >= 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) raw[t][x] = load_raw<T>(src + row[t] * stride + d.at[x]);
      }
    }
    const Place at_place = place(run, min(h, p.n_kv_heads - 1), keys);
    const int was = min(max((int)*at_place.scale, kByteScaleMin), kByteScaleMax);

    // The run's angles.
    if (half) {
      __syncthreads();
      for (int e = tid; e < kByteBlock * half; e += blockDim.x) {
        const int t = e / half;
        if (rows[t] >= 0) s_cs[e] = angle(p.rope, rows[t], e - t * half);
      }
      __syncthreads();
    }

    uint32_t largest[SL];
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      largest[t] = 0;
      if (row[t] >= 0) {
        if (half && keys) {
          float x[2][kVec];
          expand(raw[t][0], x[0]);
          expand(raw[t][1], x[1]);
          turn<D>(x, d, half, adjacent, s_cs + (lane / LR + RP * t) * half);
          as_held(x[0], raw[t][0]);
          as_held(x[1], raw[t][1]);
        }
        largest[t] = max(largest_bits(raw[t][0]), largest_bits(raw[t][1]));
      }
      const uint64_t any = __ballot(largest[t] >= 0x7f800000u);
      if (lane == 0) s_bad[turn_of][wave][t] = any;
    }
    __syncthreads();
    // A token with an infinity or a NaN among its keys or values has NaN keys and zero values,
    // and no say in the scale.
    bool bad[SL];
    uint32_t m = 0;
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      const uint64_t any = s_bad[turn_of][wave][t] | s_bad[turn_of][wave ^ 1][t];
      bad[t] = any >> (lane - l) & ((1ull << LR) - 1);
      m = max(m, bad[t] ? 0 : largest[t]);
    }
    m = wave_reduce(m, 0u, [](uint32_t x, uint32_t y) { return max(x, y); });
    if (h >= p.n_kv_heads) continue;

    int now = needed_scale(m);
    if (run.kept) now = max(now, was);
    const float s = two_to(now - 127);
    const bool rises = run.kept && now > was;
    const float step = two_to(min(now - was, 64));
    T *held_out = static_cast<T *>(keys ? p.k_out : p.v_out);
#pragma unroll
    for (int t = 0; t < SL; ++t) {
      const int token = lane / LR + RP * t;
      uint2 c[2];
      if (row[t] >= 0) {
        c[0] = encode(raw[t][0], m, s, bad[t], keys);
        c[1] = encode(raw[t][1], m, s, bad[t], keys);
        if (held_out) give_back(held_out, row[t], h, c, s);
        if (run.out) continue;
      } else if (rises && run.kept >> token & 1) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
          c[y] = again(*reinterpret_cast<const uint2 *>(at_place.codes + token * D + d.at[y]), step);
      } else {
        continue;
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) *reinterpret_cast<uint2 *>(at_place.codes + token * D + d.at[y]) = c[y];
    }
    if (!run.out && lane == 0) *at_place.scale = (uint8_t)now;
  }
}

template <typename T, int D>
void launch(const ByteAppendParams &a, hipStream_t s) {
  const RowParams &p = a.rows;
  const bool many = p.n >= kManyFrom;
  const int window = p.n >= kWindowFrom ? kWindow : p.n >= kWindowFewFrom ? kWindowFew : kWindowLeast;
  const int query_rows = p.n >= kQueryRowsMostFrom ? kQueryRowsMost : p.n >= kQueryRowsFrom ? kQueryRows : 1;
  const int heads = std::min(p.n_kv_heads, kMaxHeads), groups = (p.n_kv_heads + heads - 1) / heads;
  const int windows = (p.n + window - 1) / window, n_runs = windows * groups;
  const int n_brief = many || window < kWindow ? 0 : windows;
  const int grid = n_runs + n_brief + (p.n_q_heads ? (p.n + query_rows - 1) / query_rows : 0);
  if (many)
    append_byte_kernel<T, D, false><<<grid, 128 * heads, 0, s>>>(a, window, n_runs, n_brief, query_rows);
  else
    append_byte_kernel<T, D, true><<<grid, 128 * heads, 0, s>>>(a, window, n_runs, n_brief, query_rows);
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
