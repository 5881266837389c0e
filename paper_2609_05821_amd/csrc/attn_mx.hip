// Causal attention over a 4-bit KV cache, gfx950.
//
// Few (row, head) pairs per KV head (generated or drafted tokens) read a whole
// cache for little arithmetic, so the kernel is built around the loads: every
// wave works on 32-key steps of its own, keys and values go from memory to
// registers in 16-byte loads that are contiguous over the wave (the pool keeps
// a head's tokens side by side), the next step's are in flight while this
// one's are used, and no barrier is needed before the end of a range.
//   S^T = K Q^T  v_mfma_f32_16x16x32_bf16, 16 keys x 16 pairs.  Lane (key, g) holds
//                a quarter of the key's dims (at head_dim 128 one block with its
//                scale); v_cvt_scalef32_pk_bf16_fp4 makes two exact bf16 values a
//                lane from them, and the query is held in the same order of dims.
//   softmax      online, in the log2 domain; a lane holds one pair's column, so
//                the running maximum and sum need no exchange between lanes unless
//                the maximum rises by more than kSlack.
//   O^T += V^T P^T   values are unpacked to bf16 in LDS (each wave its own tile)
//                and read back with transposing reads; the probabilities are the
//                other operand as they lie in the S^T accumulators.
// The work of a call is the list of all key steps of all (sequence, row block,
// KV head) blocks.  Workgroups take equal contiguous parts of it, whatever the
// sequences' lengths; a block that ends up in more than one part is merged by
// a second launch.  Every workgroup derives the list from the positions itself.
#include <algorithm>

#include "mx.h"

namespace conduit {
namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kMInit = -1e30f;  // initial running maximum (log2 units)
// The running maximum moves when a step exceeds it by more than this many log2
// units; probabilities stay below 2^8.  Exact: sum and output share it.
constexpr float kSlack = 8.f;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kWaveKeys = 32;
constexpr int kStep = kWaves * kWaveKeys;  // keys of a workgroup step
constexpr int kMaxSeqBlocks = 4096;        // sequence blocks whose prefix sums fit LDS

template <int NS>
struct Parts {
  bf16x8 v[NS];
};

// x as the exact sum of NS bf16 parts (NS = 1: rounded).
template <int NS>
__device__ __forceinline__ void split_parts(const float (&x)[8], Parts<NS> &out) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const __bf16 b = static_cast<__bf16>(r[j]);
      out.v[s][j] = b;
      if (s + 1 < NS) r[j] -= (float)b;
    }
}

__device__ __forceinline__ bf16x8 unpack8(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float scale_of(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

// Orders this wave's LDS writes before its reads (and the other way round) for
// the compiler; the hardware keeps a wave's LDS accesses in order.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ int wave_max_i(int x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = max(x, __shfl_xor(x, o, 64));
  return x;
}
__device__ __forceinline__ int wave_min_i(int x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = min(x, __shfl_xor(x, o, 64));
  return x;
}

// Keys 0 .. n - 1 that a row at position `pos` may see, n <= n_ctx.
__device__ __forceinline__ int keys_seen(int pos, int n_ctx) { return min(max(pos, -1), n_ctx - 1) + 1; }

// Key steps of sequence block sb for one KV head.
__device__ __forceinline__ int block_steps(const MxAttnParams &p, int sb, int pairs) {
  const int s = sb / p.blocks_per_seq, rb = sb - s * p.blocks_per_seq, r = p.mx.rows_per_seq;
  const int lo = rb * pairs / p.group, hi = min((rb * pairs + pairs - 1) / p.group, r - 1);
  int n = 0;
  for (int i = lo; i <= hi; ++i) n = max(n, keys_seen(p.pos[(int64_t)s * r + i], p.mx.n_ctx));
  return (n + kStep - 1) / kStep;
}

// Workgroups that share `total` steps: no fewer than kMinSteps each.
constexpr int kMinSteps = 2;
__device__ __forceinline__ int workers(int n_workers, int total) { return min(n_workers, max(1, total / kMinSteps)); }
__device__ __forceinline__ int part_begin(int w, int total, int n) { return (int)((int64_t)w * total / n); }

// One 32-key step of a wave in registers.
template <int D>
struct Step {
  static constexpr int kKW = D / 32;      // dwords of a lane per 16 keys
  static constexpr int kVL = D / 64;      // 16-byte value loads of a lane
  uint32_t k[2][kKW];
  u32x4 v[kVL];
  int ks[2], vs[kVL];
};

template <int D>
__device__ __forceinline__ void load_step(const MxCache &c, int seq, int h, int key0, int lane, Step<D> &st) {
  const int64_t page = mx_page(c, seq, key0);
  const int64_t slot = ((int64_t)h << c.shift) + (key0 & ((1 << c.shift) - 1));
  const uint8_t *k = c.k + page * c.code_stride + slot * (D / 2);
  const uint8_t *v = c.v + page * c.code_stride + slot * (D / 2);
  const uint8_t *ks = c.k_scale + page * c.scale_stride + slot * (D / kMxBlock);
  const uint8_t *vs = c.v_scale + page * c.scale_stride + slot * (D / kMxBlock);
  const int key = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint8_t *at = k + (16 * j + key) * (D / 2) + g * (D / 8);
    if constexpr (D == 128) {
      const u32x4 x = ld16(at);
#pragma unroll
      for (int i = 0; i < 4; ++i) st.k[j][i] = x[i];
    } else {
      const uint2 x = *reinterpret_cast<const uint2 *>(at);
      st.k[j][0] = x.x;
      st.k[j][1] = x.y;
    }
    st.ks[j] = ks[(16 * j + key) * (D / kMxBlock) + g * (D / 4) / kMxBlock];
  }
#pragma unroll
  for (int i = 0; i < Step<D>::kVL; ++i) {
    st.v[i] = ld16(v + i * 1024 + lane * 16);
    st.vs[i] = vs[i * 64 + lane];
  }
}

// MT: groups of 16 pairs of a block.  NS: exact bf16 parts of queries and
// probabilities (1: bf16 tensors, 3: fp32).
template <int D, int MT, int NS>
__global__ __launch_bounds__(kThreads) void attn_mx_kernel(MxAttnParams p) {
  constexpr int kPairs = 16 * MT;
  constexpr int C = D / 32;            // MFMA steps over the dims
  constexpr int DT = D / 16;           // 16-dim tiles of O^T
  constexpr int VP = D + 16;           // value row pitch: 8 rows of a transposing read cover the 64 banks once
  constexpr int kTile = kWaveKeys * VP * 2;  // bytes of a wave's value tile
  constexpr int OP = D + 4;            // pitch of the output rows exchanged at the end (they reuse the tile)
  static_assert(16 * OP * 4 <= kTile, "output rows fit the tile");
  __shared__ __attribute__((aligned(16))) uint8_t s_tile[kWaves][kTile];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ int s_sum[kWaves];
  extern __shared__ int s_prefix[];    // [seq blocks + 1] with shared-out steps

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int hkv = p.mx.n_kv_heads, r = p.mx.rows_per_seq, G = p.group;
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  u16 *tile = reinterpret_cast<u16 *>(s_tile[wave]);
  float *tile_o = reinterpret_cast<float *>(s_tile[wave]);

  // This workgroup's part [t, t_end) of the step list, or block blockIdx.x.
  int t = 0, t_end = 1, part0 = 0;
  if (p.n_workers) {
    int total = 0;
    for (int b0 = 0; b0 < n_sb; b0 += kThreads) {
      const int sb = b0 + tid;
      const int own = sb < n_sb ? block_steps(p, sb, kPairs) * hkv : 0;
      const int incl = (int)wave_inclusive_sum((uint32_t)own);
      __syncthreads();
      if (lane == 63) s_sum[wave] = incl;
      __syncthreads();
      int before = total;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s_sum[w];
        total += s_sum[w];
      }
      if (sb < n_sb) s_prefix[sb] = before + incl - own;
    }
    if (tid == 0) s_prefix[n_sb] = total;
    __syncthreads();
    if (blockIdx.x == 0)
      for (int i = tid; i <= n_sb; i += kThreads) p.prefix[i] = s_prefix[i];
    const int n = workers(p.n_workers, total);
    if ((int)blockIdx.x >= n) return;
    t = part0 = part_begin(blockIdx.x, total, n);
    t_end = part_begin(blockIdx.x + 1, total, n);
  }

  while (t < t_end) {
    int sb, h, first, last, steps = 0;  // block, and its steps [first, last) of this segment
    if (p.n_workers) {
      int lo = 0, hi = n_sb - 1;        // the block that holds step t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s_prefix[mid + 1] > t) hi = mid;
        else lo = mid + 1;
      }
      sb = __builtin_amdgcn_readfirstlane(lo);
      steps = (s_prefix[sb + 1] - s_prefix[sb]) / hkv;
      h = (t - s_prefix[sb]) / steps;
      first = t - s_prefix[sb] - h * steps;
      last = min(steps, first + t_end - t);
      h = __builtin_amdgcn_readfirstlane(h);
      first = __builtin_amdgcn_readfirstlane(first);
      last = __builtin_amdgcn_readfirstlane(last);
      steps = __builtin_amdgcn_readfirstlane(steps);
    } else {
      sb = blockIdx.x / hkv;
      h = blockIdx.x - sb * hkv;
      first = 0;
      last = INT32_MAX;
    }
    const int seq = sb / p.blocks_per_seq, rb = sb - seq * p.blocks_per_seq;
    const int n_pairs = min(kPairs, r * G - rb * kPairs);
    const int64_t row_base = (int64_t)seq * r;

    // Queries and key counts of the lane's columns.  Columns past the block
    // see every key (nothing to mask) and are not written.
    Parts<NS> q[MT][C];
    int seen[MT];
    int most = 0, least = INT32_MAX;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int j = 16 * mt + col, pair = rb * kPairs + j;
      seen[mt] = INT32_MAX;
      if (j < n_pairs) {
        const int row = pair / G;
        seen[mt] = keys_seen(p.pos[row_base + row], p.mx.n_ctx);
        most = max(most, seen[mt]);
        least = min(least, seen[mt]);
        const int64_t at = ((row_base + row) * p.n_q_heads + h * G + pair % G) * D + g * (D / 4);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if constexpr (NS == 1) {
            q[mt][c].v[0] = as_bf16x8(ld16(static_cast<const u16 *>(p.q) + at + 8 * c));
          } else {
            const float *src = static_cast<const float *>(p.q) + at + 8 * c;
            const f32x4 a = __builtin_bit_cast(f32x4, ld16(src)), b = __builtin_bit_cast(f32x4, ld16(src + 4));
            const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            split_parts<NS>(x, q[mt][c]);
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int s = 0; s < NS; ++s) q[mt][c].v[s] = bf16x8{};
      }
    }
    most = __builtin_amdgcn_readfirstlane(wave_max_i(most));
    least = __builtin_amdgcn_readfirstlane(wave_min_i(least));
    last = min(last, (most + kStep - 1) / kStep);

    f32x4 o[MT][DT];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = kMInit;
      l[mt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[mt][dt] = f32x4{};
    }

    auto use = [&](Step<D> &st, int key0) __attribute__((always_inline)) {
      // values: a lane's 16 bytes are one block of one key
      constexpr int LPK = D / 32;  // lanes of a key
      if (key0 + kWaveKeys > most) {
        // keys past every row of the block: their values must not reach the
        // product as NaN or infinity (their probabilities are 0)
#pragma unroll
        for (int i = 0; i < Step<D>::kVL; ++i)
          if (key0 + i * (64 / LPK) + lane / LPK >= most) {
            st.v[i] = u32x4{};
            st.vs[i] = 127;
          }
      }
#pragma unroll
      for (int i = 0; i < Step<D>::kVL; ++i) {
        u16 *dst = tile + (i * (64 / LPK) + lane / LPK) * VP + (lane % LPK) * 32;
        const float s = scale_of(st.vs[i]);
#pragma unroll
        for (int x = 0; x < 4; ++x) st16(dst + 8 * x, __builtin_bit_cast(u32x4, unpack8(st.v[i][x], s)));
      }
      // S^T of the two 16-key halves
      f32x4 s[MT][2];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s[mt][0] = s[mt][1] = f32x4{};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float sc = scale_of(st.ks[j]);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const bf16x8 kop = unpack8(st.k[j][c], sc);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int x = 0; x < NS; ++x)
              s[mt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop, q[mt][c].v[x], s[mt][j], 0, 0, 0);
        }
      }
      wave_lds_fence();
      Parts<NS> pr[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[mt][i >> 2][i & 3] * p.scale_log2;
        if (key0 + kWaveKeys > least) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = key0 + 16 * (i >> 2) + 4 * g + (i & 3) < seen[mt] ? x[i] : kNegInf;
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
        if (__any(top > m[mt] + kSlack)) {
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float mn = fmaxf(m[mt], top), a = fast_exp2(m[mt] - mn);
          m[mt] = mn;
          l[mt] *= a;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[mt][dt] *= a;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = fast_exp2(x[i] - m[mt]);
          l[mt] += x[i];
        }
        split_parts<NS>(x, pr[mt]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const u16 *at = tile + (4 * g + (col >> 2)) * VP + 16 * dt + 4 * (col & 3);
        const short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(at));
        const short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(at + 16 * VP));
        const bf16x8 vop = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int x = 0; x < NS; ++x)
            o[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, pr[mt].v[x], o[mt][dt], 0, 0, 0);
      }
      wave_lds_fence();
    };

    // Two register sets take turns, so that a step is loaded while the one
    // before it is used.
    {
      Step<D> a, b;
      int key0 = first * kStep + wave * kWaveKeys;
      const int end = min(most, last * kStep);  // (last * kStep < n_ctx + kStep <= 2^30 + kStep)
      if (key0 < end) load_step<D>(p.mx, seq, h, key0, lane, a);
      while (key0 < end) {
        if (key0 + kStep < end) load_step<D>(p.mx, seq, h, key0 + kStep, lane, b);
        use(a, key0);
        key0 += kStep;
        if (key0 >= end) break;
        if (key0 + kStep < end) load_step<D>(p.mx, seq, h, key0 + kStep, lane, a);
        use(b, key0);
        key0 += kStep;
      }
    }

    // The four waves' results, 16 pairs at a time.
    const bool whole = !p.n_workers || (first == 0 && last == steps);
    const int slot = 2 * blockIdx.x + (t == part0 ? 0 : 1);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float lt = l[mt];
      lt += __shfl_xor(lt, 16, 64);
      lt += __shfl_xor(lt, 32, 64);
      __syncthreads();
      if (g == 0) {
        s_m[wave][col] = m[mt];
        s_l[wave][col] = lt;
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<f32x4 *>(tile_o + col * OP + 16 * dt + 4 * g) = o[mt][dt];
      __syncthreads();
      const int j = tid >> 4, pair = rb * kPairs + 16 * mt + j;
      if (16 * mt + j < n_pairs) {
        float M = s_m[0][j], L = 0.f, a[kWaves];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][j]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          a[w] = fast_exp2(s_m[w][j] - M);
          L += a[w] * s_l[w][j];
        }
        const int64_t gp = (row_base + pair / G) * p.n_q_heads + h * G + pair % G;
        const float inv = whole ? (L == 0.f ? 0.f : 1.f / L) : 1.f;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const int e = (tid & 15) * 4 + 64 * i;
          f32x4 x{};
#pragma unroll
          for (int w = 0; w < kWaves; ++w)
            x += a[w] * *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(s_tile[w]) + j * OP + e);
          x *= inv;
          if (!whole) {
            *reinterpret_cast<f32x4 *>(p.part_o + ((int64_t)slot * kPairs + 16 * mt + j) * D + e) = x;
          } else if constexpr (NS == 1) {
            ushort4 y = {f32_to_bf16(x[0]), f32_to_bf16(x[1]), f32_to_bf16(x[2]), f32_to_bf16(x[3])};
            *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) = y;
          } else {
            *reinterpret_cast<f32x4 *>(static_cast<float *>(p.o_out) + gp * D + e) = x;
          }
        }
        if ((tid & 15) == 0) {
          if (!whole)
            p.part_ml[(int64_t)slot * kPairs + 16 * mt + j] = make_float2(M, L);
          else if (p.lse_out)
            p.lse_out[gp] = L == 0.f ? kNegInf : (M + __log2f(L)) * kLn2;
        }
      }
    }
    __syncthreads();  // the tiles are free again
    if (!p.n_workers) break;
    t += last - first;
  }
}

// Merge of the blocks that more than one workgroup worked on, and the outputs
// of blocks without keys: one workgroup per (row, head) pair, groups of lanes
// taking turns at the parts.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void attn_mx_merge_kernel(MxAttnParams p, int pairs) {
  constexpr int L4 = D / 4;          // lanes of a part
  constexpr int kGroups = 256 / L4;
  __shared__ float s_m[kGroups], s_l[kGroups];
  __shared__ f32x4 s_o[kGroups][L4];
  const int64_t gp = blockIdx.x;
  const int64_t row = gp / p.n_q_heads;
  const int head = (int)(gp - row * p.n_q_heads), h = head / p.group;
  const int seq = (int)(row / p.mx.rows_per_seq);
  const int pair = (int)(row - (int64_t)seq * p.mx.rows_per_seq) * p.group + head - h * p.group;
  const int rb = pair / pairs, j = pair - rb * pairs, sb = seq * p.blocks_per_seq + rb;
  const int total = p.prefix[p.n_seqs * p.blocks_per_seq], n = workers(p.n_workers, total);
  const int base = p.prefix[sb], steps = (p.prefix[sb + 1] - base) / p.mx.n_kv_heads;
  const int t0 = base + h * steps, t1 = t0 + steps;
  const int grp = threadIdx.x / L4, e = (threadIdx.x % L4) * 4;
  float M = kMInit, L = 0.f;
  f32x4 o{};
  if (steps > 0) {
    // the workgroup that holds step x is the last whose part begins at or before it
    const int w0 = (int)((((int64_t)t0 + 1) * n - 1) / total), w1 = (int)(((int64_t)t1 * n - 1) / total);
    if (w0 == w1) return;  // written by that workgroup
    for (int w = w0 + grp; w <= w1; w += kGroups) {
      const int64_t slot = 2 * (int64_t)w + (part_begin(w, total, n) >= t0 ? 0 : 1);
      const float2 ml = p.part_ml[slot * pairs + j];
      const f32x4 x = *reinterpret_cast<const f32x4 *>(p.part_o + (slot * pairs + j) * D + e);
      const float mn = fmaxf(M, ml.x), a = fast_exp2(M - mn), b = fast_exp2(ml.x - mn);
      M = mn;
      L = L * a + ml.y * b;
      o = o * a + x * b;
    }
  }
  s_o[grp][threadIdx.x % L4] = o;
  if (e == 0) {
    s_m[grp] = M;
    s_l[grp] = L;
  }
  __syncthreads();
  if (grp) return;
  for (int i = 1; i < kGroups; ++i) {
    const float mn = fmaxf(M, s_m[i]), a = fast_exp2(M - mn), b = fast_exp2(s_m[i] - mn);
    M = mn;
    L = L * a + s_l[i] * b;
    o = o * a + s_o[i][threadIdx.x] * b;
  }
  o *= L == 0.f ? 0.f : 1.f / L;
  if constexpr (BF16) {
    ushort4 y = {f32_to_bf16(o[0]), f32_to_bf16(o[1]), f32_to_bf16(o[2]), f32_to_bf16(o[3])};
    *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) = y;
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(p.o_out) + gp * D + e) = o;
  }
  if (e == 0 && p.lse_out) p.lse_out[gp] = L == 0.f ? kNegInf : (M + __log2f(L)) * kLn2;
}

template <int D, int MT, int NS>
void launch_thin(const MxAttnParams &p, const MxAttnShape &sh, hipStream_t s) {
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  const int grid = p.n_workers ? p.n_workers : n_sb * p.mx.n_kv_heads;
  const size_t lds = p.n_workers ? (size_t)(n_sb + 1) * 4 : 0;
  attn_mx_kernel<D, MT, NS><<<grid, kThreads, lds, s>>>(p);
}

template <int D>
void launch_dim(const MxAttnParams &p, const MxAttnShape &sh, bool bf16, hipStream_t s) {
  const bool wide = sh.pairs > 16;
  if (bf16)
    wide ? launch_thin<D, 2, 1>(p, sh, s) : launch_thin<D, 1, 1>(p, sh, s);
  else
    wide ? launch_thin<D, 2, 3>(p, sh, s) : launch_thin<D, 1, 3>(p, sh, s);
}

}  // namespace

MxAttnShape mx_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16) {
  MxAttnShape L{};
  const int64_t pairs = (int64_t)rows_per_seq * (n_q_heads / n_kv_heads);
  L.pairs = pairs <= 16 ? 16 : 32;
  L.blocks_per_seq = (int32_t)((pairs + L.pairs - 1) / L.pairs);
  const int64_t n_sb = (int64_t)n_seqs * L.blocks_per_seq, blocks = n_sb * n_kv_heads;
  const int64_t steps = ((int64_t)n_ctx + kStep - 1) / kStep;
  // Workgroups share the steps out evenly while their parts can be listed and
  // there are steps to share; otherwise one workgroup takes a block.
  if (steps > 8 && n_sb <= kMaxSeqBlocks && blocks * steps < INT32_MAX)
    L.n_workers = (int32_t)std::min<int64_t>(768, std::max<int64_t>(1, blocks * steps / kMinSteps));
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
  if (L.n_workers) {
    const size_t slots = 2 * (size_t)L.n_workers * L.pairs;
    L.prefix = take((size_t)(n_sb + 1) * 4);
    L.ml = take(slots * 8);
    L.o = take(slots * head_dim * 4);
  }
  L.total = off;
  return L;
}

hipError_t launch_attn_mx(const MxAttnParams &p, const MxAttnShape &sh, int head_dim, bool bf16, hipStream_t s) {
  {
    ProfScope ps("attn_mx", s);
    head_dim == 128 ? launch_dim<128>(p, sh, bf16, s) : launch_dim<64>(p, sh, bf16, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.n_workers) return e;
  ProfScope ps("attn_mx_merge", s);
  const int64_t gp = (int64_t)p.n_seqs * p.mx.rows_per_seq * p.n_q_heads;
  if (head_dim == 128)
    bf16 ? attn_mx_merge_kernel<128, true><<<gp, 256, 0, s>>>(p, sh.pairs)
         : attn_mx_merge_kernel<128, false><<<gp, 256, 0, s>>>(p, sh.pairs);
  else
    bf16 ? attn_mx_merge_kernel<64, true><<<gp, 256, 0, s>>>(p, sh.pairs)
         : attn_mx_merge_kernel<64, false><<<gp, 256, 0, s>>>(p, sh.pairs);
  return hipGetLastError();
}

}  // namespace conduit
