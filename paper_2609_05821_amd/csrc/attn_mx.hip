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
// fp32 queries and probabilities are three exact bf16 parts each.  With bf16 tensors
// the probabilities enter the product as two bf16 parts, up to 2^-17 of each off: the
// output is the 32-bit result but for its own rounding (up to 2^-8), beside which
// one part (up to 2^-8 of each probability) showed.  The sum that they are divided
// by is of the fp32 probabilities.
//
// The work of a call is the list of all key steps of all (sequence, row block,
// KV head) blocks.  Workgroups take equal contiguous parts of it, whatever the
// sequences' lengths; a block that ends up in more than one part is merged by
// a second launch.  Every workgroup derives the list from the positions itself.
//
// Measured: 62 sequences of up to 32,768 tokens (28 heads over 4, head_dim 128, 562
// MB in all) 112.5 us and 6.0 us to merge, 5.1 TB/s, about the rate of a large copy (with
// one part of the probabilities 110.8 us); one of 65,536 tokens 20 us, of 2,048 11 us
// (two launches and four dependent loads deep: positions, page, codes, the merge).
#include "attn_steps.h"

namespace conduit {
namespace {

constexpr int many_lds(int D) { return 4 * kTileKeys * (D + 16) * 2 + kWaves * 4; }

// Sequence blocks whose list workgroups hold in LDS beside what else they have there:
// with many pairs as many as leave two workgroups a CU.  (Heads of 128, a list that
// leaves one, and a workgroup per block instead: 2,060 sequences of 1,024 to 4,096 keys with 5
// rows, 28 heads over 4, 2,286 and 1,632 us; 60,000 rows of 7 heads over their 60,000 keys 10.4 and
// 9.2 ms.)
constexpr int max_seq_blocks(int D, bool many) {
  const int fit = (160 * 1024 / 2 - many_lds(D)) / 4 - 1;
  return many && fit < 4096 ? fit : 4096;
}

__device__ __forceinline__ bf16x8 unpack8(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Values stay finite whatever the pool holds (appends write no byte above this
// one): a key that a row does not see has probability 0 there, and 0 times a NaN
// or an infinity would reach its output.
__device__ __forceinline__ float value_scale(int byte) { return scale_of(min(byte, kMxScaleMax)); }

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
__device__ __forceinline__ void load_step(const MxCache &c, int64_t page, int h, int key0, int lane, Step<D> &st) {
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

// Waves a SIMD holds (workgroups of 4 waves a CU holds) of each variant, by its
// registers.
constexpr int waves_per_simd(int D, int MT, int NS) {
  return D == 128 ? (MT == 1 && NS == 1 ? 3 : 2) : (MT == 1 ? (NS == 1 ? 4 : 3) : NS == 1 ? 3 : 2);
}
// Pairs of a block with few pairs: 32 read the cache once for twice as many, but
// fp32 rows of 128 dims would leave registers for one wave per SIMD only (1,500
// rows over 16k tokens: 32 pairs 1,094 us, 16 pairs 804 us).
constexpr int few_pairs(int D, int64_t pairs, bool bf16) { return pairs <= 16 || (D == 128 && !bf16) ? 16 : 32; }

// MT: groups of 16 pairs of a block.  NS: exact bf16 parts of queries (1: bf16
// tensors, 3: fp32).  W: waves of a workgroup, 4, or 8 for a
// workgroup per block on up to 256 blocks (64 sequences of 2,048 keys: 4 waves 20
// us, 8 waves 16 us; 256 of 512, which leave the CUs several blocks each: 16 and 24 us).
template <int D, int MT, int NS, int W>
__global__ __launch_bounds__(64 * W, waves_per_simd(D, MT, NS)) void attn_mx_kernel(MxAttnParams p) {
  constexpr int kWaves = W, kStep = W * kWaveKeys;
  constexpr int kPairs = 16 * MT;
  constexpr int NP = NS == 1 ? 2 : 3;  // bf16 parts of probabilities
  constexpr int C = D / 32;            // MFMA steps over the dims
  constexpr int DT = D / 16;           // 16-dim tiles of O^T
  constexpr int VP = D + 16;           // value row pitch: 8 rows of a transposing read cover the 64 banks once
  constexpr int kTile = kWaveKeys * VP * 2;  // bytes of a wave's value tile
  constexpr int OP = D + 4;            // pitch of the output rows exchanged at the end (they reuse the tile)
  static_assert(16 * OP * 4 <= kTile, "output rows fit the tile");
  __shared__ __attribute__((aligned(16))) uint8_t s_tile[kWaves][kTile];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ int s_sum[kWaves];
  extern __shared__ int s_prefix[];    // plan_part's list

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int hkv = p.mx.n_kv_heads, r = p.mx.rows_per_seq, G = p.group;
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  u16 *tile = reinterpret_cast<u16 *>(s_tile[wave]);
  float *tile_o = reinterpret_cast<float *>(s_tile[wave]);

  // This workgroup's part [t, t_end) of the step list, or block blockIdx.x.
  const bool shared = W == 4 && p.n_workers;
  Part part{0, 1, 0, 0, 0, 0};
  if (shared && !plan_part(p, kPairs, kStep, s_sum, s_prefix, part)) return;
  const int part0 = part.t;

  while (part.t < part.t_end) {
    const Segment sg = shared ? segment_at(p, n_sb, s_prefix, part)
                                   : Segment{(int)blockIdx.x / hkv, (int)blockIdx.x % hkv, 0, INT32_MAX, 0, 0};
    const int sb = sg.sb, h = sg.h, first = sg.first;
    int last = sg.last;
    const int seq = sb / p.blocks_per_seq, rb = sb - seq * p.blocks_per_seq;
    const int n_pairs = min(kPairs, r * G - rb * kPairs);
    const int64_t row_base = (int64_t)seq * r;

    // The wave's first step is on its way before anything else is (positions past
    // the rows' last key are masked, those past the cache are not loaded).
    const SeqPages pages = seq_pages(p.mx, seq);
    auto index = [&](int key) __attribute__((always_inline)) { return min(key, p.mx.n_ctx - 1) >> p.mx.shift; };
    auto load = [&](int key, int entry, Step<D> &st) __attribute__((always_inline)) {
      const int at = min(key, (p.mx.n_ctx - 1) & ~(kWaveKeys - 1));
      load_step<D>(p.mx, page_number(p.mx, pages, index(at), entry), h, at, lane, st);
    };
    Step<D> st[2];
    int key0 = first * kStep + wave * kWaveKeys;
    int entry = page_entry(pages, index(key0));
    {
      const int next = page_entry(pages, index(key0 + kStep));
      load(key0, entry, st[0]);
      entry = next;  // of the next step to load
    }

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
            split_parts<NS, true>(x, q[mt][c]);
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
#pragma unroll
      for (int i = 0; i < Step<D>::kVL; ++i) {
        u16 *dst = tile + (i * (64 / LPK) + lane / LPK) * VP + (lane % LPK) * 32;
        const float s = value_scale(st.vs[i]);
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
      Parts<NP> pr[MT];
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
        split_parts<NP>(x, pr[mt]);
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
          for (int x = 0; x < NP; ++x)
            o[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, pr[mt].v[x], o[mt][dt], 0, 0, 0);
      }
      wave_lds_fence();
    };

    // Two register sets take turns: a step is loaded while the one before it is used
    // (two steps ahead gain nothing), its page looked up one step earlier still.
    {
      const int end = min(most, last * kStep);  // (last * kStep < n_ctx + kStep <= 2^30 + kStep)
      auto turn = [&](Step<D> &now, Step<D> &next) __attribute__((always_inline)) {
        if (key0 + kStep < end) load(key0 + kStep, entry, next);
        entry = page_entry(pages, index(key0 + 2 * kStep));
        use(now, key0);
        key0 += kStep;
      };
      while (key0 < end) {
        turn(st[0], st[1]);
        if (key0 >= end) break;
        turn(st[1], st[0]);
      }
    }

    // The waves' results, 16 pairs at a time.
    const bool whole = !shared || (first == 0 && last == sg.steps);
    const int slot = 2 * blockIdx.x + (part.t == part0 ? 0 : 1);
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
      if (j < 16 && 16 * mt + j < n_pairs) {
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
    if (!shared) break;
    part.t += last - first;
  }
}

// Many pairs per KV head (the selected rows of a refresh): bound by the matrix
// products and the vector work between them.  The waves of a workgroup take 32
// pairs each and go over the same keys, 64 at a time.  Keys are unpacked by every
// wave for itself straight into operands, values once per workgroup into LDS, two
// tiles ahead.  (1,638 rows of 28 heads over 17,024 keys: 306 us with the 14 that the
// merge takes, 653 TFLOP/s of the two products' and half as much again for the second
// part of the probabilities; matrix cores busy 44% of the cycles, 8.6 vector
// instructions a product.  With one part 246 us; there keys through LDS as well,
// unpacked once for 8 waves, took 5% more, every product and its vector work in a fixed
// slot nothing more or less, both together 13% more.)  Products are
// v_mfma_f32_32x32x16_bf16: beside it a wave issues vector instructions for free, beside
// 16x16x32 it does not (16 of the former with 64 fma between them 543 cycles, 32 of the
// latter, the same products, 659).
//   S^T: lane (key, h) holds half h of the key's dims, codes and scales in one piece
//   each; a pair's column is in two lanes, 16 keys each.
//   O^T: the probabilities are operands as they lie; the values' rows are stored
//   interleaved (v_interleaved_key) so that the transposing reads hit every bank once.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_mx_many_kernel(MxAttnParams p) {
  constexpr int kPairs = kManyPairs;
  constexpr int C = D / 16, DT = D / 32;
  constexpr int VP = D + 16;
  constexpr int LPK = D / 32;                        // lanes of a key's values
  constexpr int VK = kTileKeys / kWaves;             // keys whose values a wave unpacks
  __shared__ __attribute__((aligned(16))) u16 s_v[4][kTileKeys * VP];
  __shared__ int s_sum[kWaves];
  extern __shared__ int s_prefix[];
  static_assert(sizeof(s_v) + sizeof(s_sum) == many_lds(D), "what max_seq_blocks counts on");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int hkv = p.mx.n_kv_heads, r = p.mx.rows_per_seq, G = p.group;
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  Part part{0, 1, 0, 0, 0, 0};
  if (p.n_workers && !plan_part(p, kPairs, kTileKeys, s_sum, s_prefix, part)) return;
  const int part0 = part.t;
  const MxCache &c = p.mx;
  const int v_lane = v_operand_lane_offset_il<VP>(lane);

  while (part.t < part.t_end) {
    const Segment sg = p.n_workers ? segment_at(p, n_sb, s_prefix, part)
                                   : Segment{(int)blockIdx.x / hkv, (int)blockIdx.x % hkv, 0, INT32_MAX, 0, 0};
    const int seq = sg.sb / p.blocks_per_seq, rb = sg.sb - seq * p.blocks_per_seq, h = sg.h;
    const int block0 = rb * kPairs, n_pairs = min(kPairs, r * G - block0);
    const int64_t row_base = (int64_t)seq * r;

    // The lane's pair: its query and how many keys it sees (a lane without one sees
    // all, so that nothing is masked for it).
    const int j = 32 * wave + col, pair = block0 + j;
    bf16x8 q[C];
    int seen = INT32_MAX, most = 0;
#pragma unroll
    for (int x = 0; x < C; ++x) q[x] = bf16x8{};
    if (j < n_pairs) {
      const int row = pair / G;
      seen = most = keys_seen(p.pos[row_base + row], c.n_ctx);
      const u16 *at = static_cast<const u16 *>(p.q) +
                      ((row_base + row) * p.n_q_heads + h * G + pair % G) * D + hh * (D / 2);
#pragma unroll
      for (int x = 0; x < C; ++x) q[x] = as_bf16x8(ld16(at + 8 * x));
    }
    most = __builtin_amdgcn_readfirstlane(wave_max_i(most));
    const int least = __builtin_amdgcn_readfirstlane(wave_min_i(seen));
    __syncthreads();
    if (lane == 0) s_sum[wave] = most;
    __syncthreads();
    int block_most = 0;
    for (int w = 0; w < kWaves; ++w) block_most = max(block_most, s_sum[w]);
    block_most = __builtin_amdgcn_readfirstlane(block_most);
    const int last = min(sg.last, (block_most + kTileKeys - 1) / kTileKeys);

    f32x16 o[DT];
    float m = kMInit, l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x16{};

    // 32 keys in registers (this wave's copy), and its share of a tile's values.
    struct Keys {
      uint32_t k[C];
      uint32_t ks;   // the scale bytes of the lane's dims
    };
    struct Values {
      u32x4 v;
      int vs;
    };
    // Where a tile begins in the code pools and in the scale pools.
    struct Place {
      int64_t codes, scales;
    };
    const int64_t head = (int64_t)h << c.shift;
    auto place = [&](int tile, int page) __attribute__((always_inline)) {
      const int64_t slot = head + ((min(tile, last - 1) * kTileKeys) & ((1 << c.shift) - 1));
      return Place{page * c.code_stride + slot * (D / 2), page * c.scale_stride + slot * (D / kMxBlock)};
    };
    const uint32_t k_lane = col * (D / 2) + hh * (D / 4), ks_lane = col * (D / kMxBlock) + hh * (D / 2 / kMxBlock);
    // (at head_dim 64 half of the lanes hold the wave's 16 keys)
    const uint32_t v_lane4 = min(lane, VK * LPK - 1);
    auto load_keys = [&](const Place &at, int half, Keys &x) __attribute__((always_inline)) {
      const uint8_t *k = c.k + at.codes + half * (32 * (D / 2));
      const uint8_t *ks = c.k_scale + at.scales + half * (32 * (D / kMxBlock));
#pragma unroll
      for (int i = 0; i < C / 4; ++i) {
        const u32x4 y = ld16(k + k_lane + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x.k[4 * i + e] = y[e];
      }
      if constexpr (D == 128)
        x.ks = *reinterpret_cast<const uint16_t *>(ks + ks_lane);
      else
        x.ks = ks[ks_lane];
    };
    auto load_values = [&](const Place &at, Values &x) __attribute__((always_inline)) {
      const uint8_t *v = c.v + at.codes + wave * (VK * (D / 2));
      const uint8_t *vs = c.v_scale + at.scales + wave * (VK * (D / kMxBlock));
      x.v = ld16(v + v_lane4 * 16);
      x.vs = vs[v_lane4];
    };
    // A wave's 16 keys of a tile's values into LDS (of a tile past the last one: the
    // last one's, into a buffer that is not read).
    const int k16 = lane / LPK;
    const uint32_t put_lane =
        (wave * VK + 8 * ((k16 >> 2) & 1) + 2 * (k16 & 3) + ((k16 >> 3) & 1)) * VP + (lane % LPK) * 32;
    auto put_values = [&](int tile, Values &x) __attribute__((always_inline)) {
      const float sc = value_scale(x.vs);
      u16 *dst = s_v[tile & 3] + put_lane;
      if (VK * LPK == 64 || lane < VK * LPK) {
#pragma unroll
        for (int i = 0; i < 4; ++i) st16(dst + 8 * i, __builtin_bit_cast(u32x4, unpack8(x.v[i], sc)));
      }
    };
    const SeqPages pages = seq_pages(c, seq);
    auto index = [&](int tile) __attribute__((always_inline)) { return min(tile, last - 1) * kTileKeys >> c.shift; };
    auto page_of = [&](int tile, int entry) __attribute__((always_inline)) {
      return page_number(c, pages, index(tile), entry);
    };
    auto key_operand = [&](const Keys &x, int d) __attribute__((always_inline)) {
      return unpack8(x.k[d], scale_of(d < 4 ? x.ks & 0xff : x.ks >> 8));
    };
    auto largest = [&](const f32x16 &s) __attribute__((always_inline)) {
      float t[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) t[i] = fmaxf(fmaxf(s[3 * i], s[3 * i + 1]), s[3 * i + 2]);
      return fmaxf(fmaxf(fmaxf(t[0], t[1]), t[2]), fmaxf(fmaxf(t[3], t[4]), s[15])) * p.scale_log2;  // (scale > 0)
    };
    // S^T of 32 keys and the lane's largest (in the log2 domain).
    struct Scores {
      f32x16 s;
      float top;
    };
    auto products = [&](const Keys &x) __attribute__((always_inline)) {
      f32x16 s{};
#pragma unroll
      for (int d = 0; d < C; ++d) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand(x, d), q[d], s, 0, 0, 0);
      return s;
    };
    // The keys from key0 on that the row does not see.
    auto mask = [&](int key0, Scores &x) __attribute__((always_inline)) {
      if (key0 + 32 <= least) return;
      const int limit = seen - key0 - 4 * hh;
#pragma unroll
      for (int i = 0; i < 16; ++i) x.s[i] = (i & 3) + 8 * (i >> 2) < limit ? x.s[i] : kNegInf;
      x.top = largest(x.s);
    };
    // Softmax and O^T products of 32 keys whose S^T is in x, and the S^T products of
    // the next 32 (nx), in one block of code without branches, so that matrix and
    // vector work of one wave overlap; `extra` joins them.
    auto half_step = [&](int tile, int half, Scores &x, const Keys &nx, auto &&extra) __attribute__((always_inline)) {
      if (__any(x.top > m + kSlack)) {
        const float mn = fmaxf(m, half_max(x.top)), a = fast_exp2(m - mn);
        m = mn;
        l *= a;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= a;
      }
      const u16 *at = s_v[tile & 3] + 32 * half * VP + v_lane;
      bf16x8 v0[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) v0[dt] = v_operand_il<VP>(at + 32 * dt);
      const f32x16 sn = products(nx);
      Parts<2> pr[2];  // of 16 keys each
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float e[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          e[y] = fast_exp2(__builtin_fmaf(x.s[8 * i + y], p.scale_log2, -m));
          sum[y & 1] += e[y];
        }
        split_parts<2>(e, pr[i]);
      }
      l += sum[0] + sum[1];
      auto add = [&](int dt, const bf16x8 &v, const Parts<2> &w) __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < 2; ++y) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w.v[y], o[dt], 0, 0, 0);
      };
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) add(dt, v0[dt], pr[0]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) add(dt, v_operand_il<VP>(at + 16 * VP + 32 * dt), pr[1]);
      x.s = sn;
      x.top = largest(sn);
      extra();
    };
    // A tile: S^T of its first half is in x, its second half's keys are in b, the
    // next tile's in c0 and d (loaded two half steps before their use).  Values go
    // two tiles ahead into LDS, so that the waves meet every second tile only.
    Place at1, at2;  // the next two tiles
    int entry3 = 0;  // the table entry of the one after
    auto tile_step = [&](int tile, Scores &x, Keys &a, Keys &b, Keys &c0, Keys &d) __attribute__((always_inline)) {
      Values v;
      load_values(at2, v);
      load_keys(at1, 1, d);
      const int entry4 = page_entry(pages, index(tile + 4));
      const bool active = tile * kTileKeys < most;
      if (active) {
        half_step(tile, 0, x, b, [] {});
        mask(tile * kTileKeys + 32, x);
      }
      load_keys(at2, 0, a);
      at1 = at2;
      at2 = place(tile + 3, page_of(tile + 3, entry3));
      entry3 = entry4;
      if (active) {
        half_step(tile, 1, x, c0, [&] { put_values(tile + 2, v); });
        mask(tile * kTileKeys + 64, x);
      } else {
        put_values(tile + 2, v);
      }
    };

    if (sg.first < last) {
      Keys k0, k1, k2, k3;
      Scores x;
      {
        int entry[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) entry[i] = page_entry(pages, index(sg.first + i));
        entry3 = page_entry(pages, index(sg.first + 3));
        const Place at0 = place(sg.first, page_of(sg.first, entry[0]));
        at1 = place(sg.first + 1, page_of(sg.first + 1, entry[1]));
        at2 = place(sg.first + 2, page_of(sg.first + 2, entry[2]));
        Values v, v1;
        load_values(at0, v);
        load_values(at1, v1);
        load_keys(at0, 0, k0);
        load_keys(at0, 1, k1);
        load_keys(at1, 0, k2);
        put_values(sg.first, v);
        put_values(sg.first + 1, v1);
        x.s = products(k0);
        x.top = largest(x.s);
        mask(sg.first * kTileKeys, x);
      }
      __syncthreads();
      for (int tile = sg.first; tile < last; tile += 2) {
        tile_step(tile, x, k0, k1, k2, k3);
        if (tile + 1 < last) tile_step(tile + 1, x, k2, k3, k0, k1);
        __syncthreads();
      }
    }

    const bool whole = !p.n_workers || (sg.first == 0 && sg.last == sg.steps);
    const int slot = 2 * blockIdx.x + (part.t == part0 ? 0 : 1);
    l += __shfl_xor(l, 32, 64);
    if (j < n_pairs) {
      const int64_t gp = (row_base + pair / G) * p.n_q_heads + h * G + pair % G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 32 * dt + 8 * i + 4 * hh;
          const f32x4 y = {o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
          if (whole)
            *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) =
                make_ushort4(f32_to_bf16(y[0] * inv), f32_to_bf16(y[1] * inv), f32_to_bf16(y[2] * inv),
                             f32_to_bf16(y[3] * inv));
          else
            *reinterpret_cast<f32x4 *>(p.part_o + ((int64_t)slot * kPairs + j) * D + e) = y;
        }
      if (hh == 0) {
        if (!whole)
          p.part_ml[(int64_t)slot * kPairs + j] = make_float2(m, l);
        else if (p.lse_out)
          p.lse_out[gp] = l == 0.f ? kNegInf : (m + __log2f(l)) * kLn2;
      }
    }
    if (!p.n_workers) break;
    part.t += sg.last - sg.first;
  }
}

template <int D, int W>
void launch_few(const MxAttnParams &p, bool wide, bool bf16, int grid, size_t lds, hipStream_t s) {
  if (bf16)
    wide ? attn_mx_kernel<D, 2, 1, W><<<grid, 64 * W, lds, s>>>(p)
         : attn_mx_kernel<D, 1, 1, W><<<grid, 64 * W, lds, s>>>(p);
  else if (!wide)
    attn_mx_kernel<D, 1, 3, W><<<grid, 64 * W, lds, s>>>(p);
  else if constexpr (few_pairs(D, 32, false) == 32)
    attn_mx_kernel<D, 2, 3, W><<<grid, 64 * W, lds, s>>>(p);
}

template <int D>
void launch_dim(const MxAttnParams &p, const MxAttnShape &sh, bool bf16, hipStream_t s) {
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  const int grid = p.n_workers ? p.n_workers : n_sb * p.mx.n_kv_heads;
  const size_t lds = p.n_workers && n_sb > kLaneBlocks ? (size_t)(n_sb + 1) * 4 : 0;
  if (sh.pairs > 32)
    attn_mx_many_kernel<D><<<grid, kThreads, lds, s>>>(p);
  else if (p.n_workers || grid > 256)
    launch_few<D, 4>(p, sh.pairs > 16, bf16, grid, lds, s);
  else
    launch_few<D, 8>(p, sh.pairs > 16, bf16, grid, lds, s);
}

}  // namespace

MxAttnShape mx_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16) {
  MxAttnShape L{};
  const int64_t pairs = (int64_t)rows_per_seq * (n_q_heads / n_kv_heads);
  const bool many = bf16 && pairs > 32;
  L.pairs = many ? kManyPairs : few_pairs(head_dim, pairs, bf16);
  L.blocks_per_seq = (int32_t)((pairs + L.pairs - 1) / L.pairs);
  const int64_t n_sb = (int64_t)n_seqs * L.blocks_per_seq, blocks = n_sb * n_kv_heads;
  const int64_t steps = ((int64_t)n_ctx + kStep - 1) / kStep;
  const int64_t resident =
      256 * (many ? 2 : waves_per_simd(head_dim, L.pairs > 16 ? 2 : 1, bf16 ? 1 : 3));
  // Workgroups share the steps out evenly, for a second launch that merges, from
  // this many steps of a block on (and while the parts' list fits LDS): fewer are
  // done sooner by a workgroup per block, and the more blocks there are the less
  // there is to even out.  One sequence of 4 KV heads: 1,024 keys 9 us by block,
  // 11 us shared; 2,200 keys 14 and 11 us.  64 sequences of up to 2,048: 15 and 20
  // us.  256 of up to 4,096: 75 and 84 us, of up to 8,192: 144 and 140 us.
  const int64_t from = many || blocks < 256 ? 8 : blocks < 1024 ? 16 : 32;
  // (The merge has up to L.pairs workgroups of 256 threads a block, fewer than 2^32.)
  if (steps > from && n_sb <= max_seq_blocks(head_dim, many) && 2 * blocks * steps < INT32_MAX &&
      blocks * L.pairs < 1 << 24)
    L.n_workers = (int32_t)std::min<int64_t>(resident, std::max<int64_t>(1, blocks * steps / kMinSteps));
  lay_out_workspace(L, n_sb, head_dim);
  return L;
}

hipError_t launch_attn_mx(const MxAttnParams &p, const MxAttnShape &sh, int head_dim, bool bf16, hipStream_t s) {
  {
    ProfScope ps("attn_mx", s);
    head_dim == 128 ? launch_dim<128>(p, sh, bf16, s) : launch_dim<64>(p, sh, bf16, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.n_workers) return e;
  return launch_attn_merge(p, sh, "attn_mx_merge", head_dim, bf16, s);
}

}  // namespace conduit
