// Causal attention over the 8-bit KV cache, gfx950.
//
//   o_i = sum_t p_it v_t / sum_t p_it,  p_it = exp(scale q_i k_t),  t = 0 .. pos_i
// with keys and values code * 2^(s - 127), exact in bf16 (4 significant bits).  A call has
// pairs (row, head): those of a sequence that share a KV head share its keys.  The work is
// the list of all key steps of all (sequence, block of pairs, KV head); workgroups take equal
// contiguous parts of it, and a second launch merges blocks that were cut (attn_steps.h).
//
// Few pairs (attn_byte_kernel): bound by reading the cache once, 2 (D + 1 / 16) bytes a key
// and head.  Every wave has 32-key steps of its own in registers, in 16-byte loads that are
// contiguous over the wave, the next step's in flight while this one's are used, and no
// barrier before the end of its range.
//   S^T = K Q^T  v_mfma_f32_16x16x32_bf16, 16 keys x 16 pairs: lane (key, g) has a quarter of
//                the key's dims, decoded by v_cvt_scalef32_pk_bf16_fp8 with the block's
//                scale; the queries are held in the same order of dims.
//   softmax      online, in the log2 domain; a lane has one pair's column, so the running
//                maximum and sum need no exchange between lanes unless the maximum rises by
//                more than kSlack.
//   O^T += V^T P^T  values decoded to bf16 in the wave's own LDS tile and read back with
//                transposing reads; the probabilities are the other operand as they lie.
// bf16 tensors: probabilities enter as two bf16 parts (2^-17 of each off; one part, 2^-8, would
// show beside the output's one rounding); fp32: queries and probabilities as three exact parts.
// The sum they are divided by is of the fp32 probabilities.
// Measured (bf16, D = 128): 62 sequences of up to 32,768 tokens, 28 heads over 4, 1.06 GB: 190 us
// and 5 to merge, 5.5 TB/s (a copy of 4 GiB: 4.5); one of 131,072, 32 heads over 8, 268 MB: 51 and 5;
// 8 of up to 8,211 with 5 rows, 76 MB: 22 and 4, which is mostly the chain of loads a
// workgroup begins with (positions, page, codes) for 4 steps of its own.
//
// Many pairs (attn_byte_many_kernel): bound by the matrix products.  See there.
#include <type_traits>

#include "attn_steps.h"

namespace conduit {
namespace {

// Sequence blocks whose list workgroups hold in LDS.
constexpr int kMaxSeqBlocks = 4096;

// 8 codes as exact bf16 operands, times the block's scale.
__device__ __forceinline__ bf16x8 unpack8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// NaN codes become 0, four at a time: a value that a row does not see has probability 0,
// and 0 times a NaN would reach its output.  (Appends write no NaN among values.)
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
  const uint32_t nan = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // the top bit of bytes that hold one
  return w & ~((nan - (nan >> 7)) | nan);
}

// One 32-key step of a wave in registers.
template <int D>
struct Step {
  static constexpr int kKL = D / 64;      // 16-byte key loads of a lane per 16 keys
  static constexpr int kVL = D / 32;      // 16-byte value loads of a lane
  u32x4 k[2][kKL];
  u32x4 v[kVL];
  int ks, vs;                             // scale bytes of both halves
};

template <int D>
__device__ __forceinline__ void load_step(const MxCache &c, int64_t page, int h, int key0, int lane, Step<D> &st) {
  const int64_t slot = ((int64_t)h << c.shift) + (key0 & ((1 << c.shift) - 1));
  const uint8_t *k = c.k + page * c.code_stride + slot * D;
  const uint8_t *v = c.v + page * c.code_stride + slot * D;
  const int64_t scale = page * c.scale_stride + slot / kByteBlock;
  const int key = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < Step<D>::kKL; ++i) st.k[j][i] = ld16(k + (16 * j + key) * D + 64 * i + 16 * g);
#pragma unroll
  for (int i = 0; i < Step<D>::kVL; ++i) st.v[i] = ld16(v + i * 1024 + lane * 16);
  // (the same in every lane: hidden from the compiler, which would make it a scalar load
  // and wait for it at once)
  int zero = 0;
  asm("" : "+v"(zero));
  st.ks = *reinterpret_cast<const uint16_t *>(c.k_scale + scale + zero);
  st.vs = *reinterpret_cast<const uint16_t *>(c.v_scale + scale + zero);
}

// Waves a SIMD holds (workgroups of 4 waves a CU holds) of each variant, by its
// registers.
constexpr int waves_per_simd(int D, int MT, int NS) {
  return D == 128 ? 2 : (MT == 1 ? (NS == 1 ? 4 : 3) : NS == 1 ? 3 : 2);
}
// Pairs of a block with few pairs: 32 read the cache once for twice as many, but
// fp32 rows of 128 dims would leave registers for one wave per SIMD only (28 heads over 4, 32 and 16
// pairs: 200 rows over 4,096 tokens 70 and 57 us, 64 sequences of 4,096 with 8 rows 156 and 122).
constexpr int few_pairs(int D, int64_t pairs, bool bf16) { return pairs <= 16 || (D == 128 && !bf16) ? 16 : 32; }

// MT: groups of 16 pairs of a block.  NS: exact bf16 parts of queries (1: bf16
// tensors, 3: fp32).  W: waves of a workgroup, 4, or 8 for a
// workgroup per block on up to 256 blocks (64 sequences of up to 2,048 keys, 4 KV heads: 4 waves 26
// us, 8 waves 20; 256 of up to 512, which leave the CUs several blocks each: 21 and 29).
template <int D, int MT, int NS, int W>
__global__ __launch_bounds__(64 * W, waves_per_simd(D, MT, NS)) void attn_byte_kernel(MxAttnParams p) {
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
        const int64_t at = ((row_base + row) * p.n_q_heads + h * G + pair % G) * D + 16 * g;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int e = 64 * (c >> 1) + 8 * (c & 1);
          if constexpr (NS == 1) {
            q[mt][c].v[0] = as_bf16x8(ld16(static_cast<const u16 *>(p.q) + at + e));
          } else {
            const float *src = static_cast<const float *>(p.q) + at + e;
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
      // values: a lane's 16 bytes are 16 dims of one key
      constexpr int LPK = D / 16;  // lanes of a key
      if (key0 + kWaveKeys > least) {
#pragma unroll
        for (int i = 0; i < Step<D>::kVL; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) st.v[i][x] = without_nan(st.v[i][x]);
      }
#pragma unroll
      for (int i = 0; i < Step<D>::kVL; ++i) {
        u16 *dst = tile + (i * (64 / LPK) + lane / LPK) * VP + (lane % LPK) * 16;
        const float s = byte_scale(i < Step<D>::kVL / 2 ? st.vs & 0xff : st.vs >> 8);
#pragma unroll
        for (int x = 0; x < 2; ++x)
          st16(dst + 8 * x, __builtin_bit_cast(u32x4, unpack8(st.v[i][2 * x], st.v[i][2 * x + 1], s)));
      }
      // S^T of the two 16-key halves
      f32x4 s[MT][2];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s[mt][0] = s[mt][1] = f32x4{};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float sc = byte_scale(j ? st.ks >> 8 : st.ks & 0xff);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const bf16x8 kop = unpack8(st.k[j][c >> 1][2 * (c & 1)], st.k[j][c >> 1][2 * (c & 1) + 1], sc);
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

    // Two register sets take turns: a step is loaded while the one before it is used,
    // its page looked up one step earlier still.
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

// Many pairs per KV head (the rows of a refresh, a text's rows over an encoder's states): keys
// and values are decoded once for 256 pairs, 32 a wave, into a ring of four tiles of 64 keys in LDS.
//   S^T = K Q^T     v_mfma_f32_32x32x16_bf16, keys as bf16 with their scale.
//   O^T += V^T W^T  v_mfma_f32_32x32x16_f16: values as their bare codes (exact in fp16), and the
//                   block's scale goes into the weight, as part of the exponent that the
//                   softmax computes anyway:  w = 2^(x + log2 f - M + kHead)  for the score x
//                   (log2 units) and the factor f of its value block, over the running maximum M
//                   of x + log2 f.  A weight is rounded once, by up to 2^-11 of it, where one
//                   bf16 part would lose 2^-8 and two would double the second product; weights
//                   below fp16's normal numbers are off by 2^-25, 2^-36 of the largest.
//   l += 2^(x - m)  the sum, in fp32 over a running maximum m of its own: two exponents a
//                   16-key block then share the exponential, e = 2^(x - at), at = M - kHead - log2 f, and
//                   what a block adds to l is put right by 2^(at - m) once.  Where a block's factor is
//                   so small that e would leave fp32 (at > m + kFar) at is m + kFar: weights of such
//                   a block, below 2^(kManySlack - kFar), are 0 in fp16 either way.
// Both maxima move when a step exceeds them by more than kManySlack: weights stay below
// 2^(kHead + kManySlack) = 2^15, and sums lose nothing.  That M and m stand for the same score to a fraction of a
// weight's rounding needs them to be small: scores beyond kNear are counted from the largest one (`base`).
//
// A step of 32 keys is 2 C slots of one product each, with a share of the vector work of the
// softmax (of the scores computed one step before), an operand read from LDS for C slots
// later, and in turn a tile's loads, decoding and LDS writes.  sched_barrier and the
// empty statements keep each slot's work in it; the compiler otherwise gathers the exponentials and
// the products apart.
//
// What bounds it: the product of 32 x 32 x 16 takes 13.8 ns a SIMD on zeros and 21 on random
// numbers (1.6 PFLOP/s: the chip lowers its clock), 27.6 with the vector work that a slot needs here. A
// tile takes 1.93 to 2.06 us at D = 128, by the card and its clock (64 keys, 256 pairs a CU: 1.04 to 1.11 PFLOP/s over the
// chip), and 1.35 to 1.39 at D = 64.  Where it took 2.06, 64 pairs a wave on one wave a SIMD took as long (2.03
// to 2.06; 1.50 at D = 64), and so did slots that lag the waves behind one another (2.06 to 2.10); keys and values
// decoded by every wave for itself took 620 us for 1,638 rows over 17,024 keys where this takes 224.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
constexpr int kManyWaves = 8;
constexpr int kManyThreads = 64 * kManyWaves;
constexpr int kBytePairs = 32 * kManyWaves;          // pairs of a block
// What beginning a block costs, in tiles: its first tiles and queries, and the rows of the part
// that it leaves for the merge.  With 3, 6, 8 and 12 tiles: 1,638 rows over 17,024 keys, 28 heads over 4, 252 244 245 248
// us; 4,000 over 8,000, 8 heads over 4, 100 97 99 101; 1,000 over 9,000, 16 over 8, 72 73 73 72; 4 sequences of 333 rows to
// all of up to 4,100 states, 32 over 8, 107 105 106 109; 7 of 200 to 6,000, 16 over 4, 77 73 75 76; 16 of 100 to
// 2,500, 32 over 4, 76 74 77 82; 3 of 150 to 20,000, 20 over 4, and 2 of 900 to 5,000, 8 over 8, within 1%.
constexpr int kManyPad = 6;
constexpr int kRing = 4;                             // tiles in LDS
constexpr float kHead = 11.f, kManySlack = 4.f;      // weights stay below 2^(kHead + kManySlack)
constexpr float kFar = 89.f;
// Running maxima up to which scores are taken as they are: M_head and at, which have a scale's exponent of up to 119
// added, are then off by 2^-14 at most, 2^-14.5 of a weight.  (At 2^24 they had been off by 2: beside blocks of other
// scales a weight came to 4 times what it was, from 2^26 on some were infinite.)
constexpr float kNear = 1024.f;

__device__ __forceinline__ u32x4 half8(uint32_t lo, uint32_t hi) {
  const f16x2 r[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true)};
  return __builtin_bit_cast(u32x4, r);
}

template <int D>
__global__ __launch_bounds__(kManyThreads, 2) void attn_byte_many_kernel(MxAttnParams p) {
  constexpr int kPairs = kBytePairs;
  constexpr int C = D / 16, DT = D / 32;
  static_assert(C == 2 * DT, "as many products for scores as for outputs");
  constexpr int KP = D + 8, VP = D + 16;
  constexpr int LPK = D / 16;                          // 16-byte chunks of a key's codes
  constexpr int kChunks = kTileKeys * LPK;             // of a tile, one a thread
  __shared__ __attribute__((aligned(16))) u16 s_k[kRing][kTileKeys * KP];
  __shared__ __attribute__((aligned(16))) u16 s_v[kRing][kTileKeys * VP];
  __shared__ int s_sum[kManyWaves], s_least[kManyWaves];
  extern __shared__ int s_prefix[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int hkv = p.mx.n_kv_heads, r = p.mx.rows_per_seq, G = p.group;
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  Part part{0, 1, 0, 0, 0, 0};
  if (p.n_workers && !plan_part<kManyWaves, 8, kManyPad, true>(p, kPairs, kTileKeys, s_sum, s_prefix, part)) return;
  const int part0 = part.t;
  const MxCache &c = p.mx;
  const int v_lane = v_operand_lane_offset_il<VP>(lane);
  const int k_lane = col * KP + 8 * hh;

  while (part.t < part.t_end) {
    const Segment sg = p.n_workers ? segment_at<kManyPad>(p, n_sb, s_prefix, part)
                                   : Segment{(int)blockIdx.x / hkv, (int)blockIdx.x % hkv, 0, INT32_MAX, 0, 0};
    part.t += sg.listed;
    if (p.n_workers && sg.first == sg.last) continue;
    const int seq = sg.sb / p.blocks_per_seq, rb = sg.sb - seq * p.blocks_per_seq, h = sg.h;
    const int block0 = rb * kPairs, n_pairs = min(kPairs, r * G - block0);
    const int64_t row_base = (int64_t)seq * r;

    // A thread's chunk of a tile's codes in registers, on its way into LDS.
    struct Raw {
      u32x4 k, v;
      int ks;
      uint32_t vs;  // the value scales of the tile's four blocks
    };
    const SeqPages pages = seq_pages(c, seq);
    const int64_t head = (int64_t)h << c.shift;
    const int limit = min(sg.last, (c.n_ctx + kTileKeys - 1) / kTileKeys);  // no tile from here on is read
    auto index = [&](int tile) __attribute__((always_inline)) { return min(tile, limit - 1) * kTileKeys >> c.shift; };
    // Where a tile begins: in the code pools and in the scale pools.
    struct Place {
      int64_t codes, scales;
    };
    auto place = [&](int tile, int entry) __attribute__((always_inline)) {
      const int64_t page = page_number(c, pages, index(tile), entry);
      const int64_t slot = head + ((min(tile, limit - 1) * kTileKeys) & ((1 << c.shift) - 1));
      return Place{page * c.code_stride + slot * D, page * c.scale_stride + slot / kByteBlock};
    };
    // (at head_dim 64 half of the threads)
    const uint32_t chunk = kChunks == kManyThreads ? tid : min(tid, kChunks - 1);
    const uint32_t lane_codes = chunk * 16, lane_scale = chunk / LPK / kByteBlock;
    auto load_keys = [&](const Place &at, Raw &x) __attribute__((always_inline)) {
      x.k = ld16(c.k + at.codes + lane_codes);
      x.ks = (c.k_scale + at.scales)[lane_scale];
    };
    auto load_values = [&](const Place &at, Raw &x) __attribute__((always_inline)) {
      x.v = ld16(c.v + at.codes + lane_codes);
      int zero = 0;
      asm("" : "+v"(zero));
      x.vs = *reinterpret_cast<const uint32_t *>(c.v_scale + at.scales + zero);
    };
    // Page entries first, queries and positions behind them: tiles are asked for as soon as
    // the entries are there, and the rest arrives meanwhile.
    int entry[3], entry3;
#pragma unroll
    for (int i = 0; i < 3; ++i) entry[i] = page_entry(pages, index(sg.first + i));
    entry3 = page_entry(pages, index(sg.first + 3));

    // The lane's pair: its query and how many keys it sees (one that is not there sees all).
    const int j0 = 32 * wave + col, pair = block0 + j0;
    bf16x8 q[C];
    int pos = 0;
#pragma unroll
    for (int x = 0; x < C; ++x) q[x] = bf16x8{};
    if (j0 < n_pairs) {
      const int row = pair / G;
      pos = p.pos[row_base + row];
      const u16 *at =
          static_cast<const u16 *>(p.q) + ((row_base + row) * p.n_q_heads + h * G + pair % G) * D + 8 * hh;
#pragma unroll
      for (int x = 0; x < C; ++x) q[x] = as_bf16x8(ld16(at + 16 * x));
    }
    __builtin_amdgcn_sched_barrier(0);

    Raw raw0, raw;
    const Place at0 = place(sg.first, entry[0]), at1 = place(sg.first + 1, entry[1]);
    const Place at2 = place(sg.first + 2, entry[2]);
    load_keys(at0, raw0);
    load_values(at0, raw0);
    load_keys(at1, raw);
    load_values(at1, raw);
    __builtin_amdgcn_sched_barrier(0);
    const int seen = j0 < n_pairs ? keys_seen(pos, c.n_ctx) : INT32_MAX;
    int most = j0 < n_pairs ? seen : 0;
    most = __builtin_amdgcn_readfirstlane(wave_max_i(most));
    const int least = __builtin_amdgcn_readfirstlane(wave_min_i(seen));
    __syncthreads();
    if (lane == 0) {
      s_sum[wave] = most;
      s_least[wave] = least;
    }
    __syncthreads();
    int block_most = 0, block_least = INT32_MAX;
    for (int w = 0; w < kManyWaves; ++w) {
      block_most = max(block_most, s_sum[w]);
      block_least = min(block_least, s_least[w]);
    }
    block_most = __builtin_amdgcn_readfirstlane(block_most);
    block_least = __builtin_amdgcn_readfirstlane(block_least);
    const int last = min(sg.last, (block_most + kTileKeys - 1) / kTileKeys);

    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x16{};
    // The running maximum of the pair's scores x, that of x + log2 of the value scale, and what
    // follows from them.
    float m, M, m_high, M_high, m_far, M_head, l = 0.f;
    auto set_maxima = [&](float x, float y) __attribute__((always_inline)) {
      m = x;
      M = y;
      m_high = x + kManySlack;
      M_high = y + kManySlack;
      m_far = x + kFar;
      M_head = y - kHead;
    };
    set_maxima(kMInit, kMInit);

    const int put_key = chunk / LPK, put_dim = chunk % LPK * 16;
    const int k_put = put_key * KP + put_dim;
    const int v_put =
        ((put_key & ~15) + 8 * ((put_key >> 2) & 1) + 2 * (put_key & 3) + ((put_key >> 3) & 1)) * VP + put_dim;
    const bool puts = kChunks == kManyThreads || tid < kChunks;
    auto put_keys = [&](int tile, const Raw &x) __attribute__((always_inline)) {
      u16 *dst = s_k[tile & (kRing - 1)] + k_put;
      if (puts) {
        st16(dst, __builtin_bit_cast(u32x4, unpack8(x.k[0], x.k[1], byte_scale(x.ks))));
        st16(dst + 8, __builtin_bit_cast(u32x4, unpack8(x.k[2], x.k[3], byte_scale(x.ks))));
      }
    };
    auto put_values = [&](int tile, const Raw &x) __attribute__((always_inline)) {
      u16 *dst = s_v[tile & (kRing - 1)] + v_put;
      if (puts) {
        st16(dst, half8(x.v[0], x.v[1]));
        st16(dst + 8, half8(x.v[2], x.v[3]));
      }
    };
    auto clean = [&](int tile, Raw &x) __attribute__((always_inline)) {
      if ((tile + 1) * kTileKeys > block_least) {
#pragma unroll
        for (int y = 0; y < 4; ++y) x.v[y] = without_nan(x.v[y]);
      }
    };

    // Scores of 32 keys, and for their softmax: whether the maxima rise in some lane, and the
    // exponents that the two blocks' weights are over.
    struct Scores {
      f32x16 s;
      float top[2], at[2];
      uint64_t rises;
    };
    auto top_of = [&](Scores &x, int b) __attribute__((always_inline)) {
      float t = kNegInf;
#pragma unroll
      for (int i = 0; i < 8; ++i) t = fmaxf(t, x.s[8 * b + i]);
      x.top[b] = t;
    };
    // (scale > 0)
    auto largest = [&](const Scores &x, const float (&sv)[2], float &mx, float &my) __attribute__((always_inline)) {
      mx = fmaxf(x.top[0], x.top[1]) * p.scale_log2;
      my = fmaxf(__builtin_fmaf(x.top[0], p.scale_log2, sv[0]), __builtin_fmaf(x.top[1], p.scale_log2, sv[1]));
    };
    auto compare = [&](Scores &x, const float (&sv)[2]) __attribute__((always_inline)) {
      float mx, my;
      largest(x, sv, mx, my);
      x.rises = __builtin_amdgcn_ballot_w64(mx > m_high) | __builtin_amdgcn_ballot_w64(my > M_high);
    };
    auto exponents = [&](Scores &x, const float (&sv)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) x.at[b] = fminf(M_head - sv[b], m_far);
    };
    // Where a lane's scores are counted from, 0 until a maximum of some lane leaves [-kNear, kNear].  From then on
    // every step is put over it, and it follows the largest score, so that maxima stay small numbers.
    float base = 0.f;
    int look_from = least;  // (first key that some row does not see, or below 0: look at every step)
    auto put_over_base = [&](Scores &x, const float (&sv)[2]) __attribute__((always_inline)) {
      const float top = half_max(fmaxf(x.top[0], x.top[1])), by = (top - base) * p.scale_log2;
      if (by > m_high) {  // (no key yet: top is -inf)
        set_maxima(m - by, M - by);
        base = top;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) x.s[i] -= base;
      x.top[0] -= base;
      x.top[1] -= base;
      compare(x, sv);
      exponents(x, sv);
    };
    // Keys that a row does not see, and maxima that rise: sums and outputs follow.
    auto settle = [&](Scores &x, int key0, const float (&sv)[2]) __attribute__((always_inline)) {
      if (key0 + 32 > look_from) {
        const int limit = seen - key0 - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i) x.s[i] = (i & 3) + 8 * (i >> 2) < limit ? x.s[i] : kNegInf;
        top_of(x, 0);
        top_of(x, 1);
        compare(x, sv);
        if (look_from < 0) x.rises = ~0ull;
      }
      if (__builtin_expect(x.rises != 0, 0)) {  // (one condition a step: with look_from in it 1,638 rows took 1% longer)
        float mx, my;
        if (look_from >= 0) {
          largest(x, sv, mx, my);
          const float mn = fmaxf(m, half_max(mx));
          if (__any(fabsf(mn) > kNear && mn > kMInit)) look_from = INT32_MIN;
        }
        if (look_from < 0) put_over_base(x, sv);
        largest(x, sv, mx, my);
        const float mn = fmaxf(m, half_max(mx)), Mn = fmaxf(M, half_max(my));
        l *= fast_exp2(m - mn);
        const float a = fast_exp2(M - Mn);
        set_maxima(mn, Mn);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= a;
        exponents(x, sv);
      }
    };
    auto scale_of_step = [&](uint32_t vs, int half, float (&sv)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        sv[b] = (float)(min(max((int)(vs >> (16 * half + 8 * b) & 0xff), kByteScaleMin), kByteScaleMax) - 127);
    };

    if (sg.first < last) {
      uint32_t vs0, vs1, vs2;  // value scales of this tile and the next two
      clean(sg.first, raw0);
      put_keys(sg.first, raw0);
      put_values(sg.first, raw0);
      vs0 = __builtin_amdgcn_readfirstlane(raw0.vs);
      clean(sg.first + 1, raw);
      put_keys(sg.first + 1, raw);
      put_values(sg.first + 1, raw);
      vs1 = __builtin_amdgcn_readfirstlane(raw.vs);
      load_keys(at2, raw);
      load_values(at2, raw);
      __syncthreads();
      u32x4 ring[C];  // operands: a step's keys, then its values
      auto key_operand = [&](int step, int x) __attribute__((always_inline)) {
        return ld16(s_k[(step >> 1) & (kRing - 1)] + 32 * (step & 1) * KP + k_lane + 16 * x);
      };
      auto value_operand = [&](int step, int x) __attribute__((always_inline)) {
        return __builtin_bit_cast(u32x4, v_operand_il<VP>(s_v[(step >> 1) & (kRing - 1)] + 32 * (step & 1) * VP +
                                                          v_lane + 16 * (x / DT) * VP + 32 * (x % DT)));
      };
      Scores xa, xb;
      float sv0[2], sv1[2];  // value scales (log2) of this step's blocks and of the next one's
      const int step0 = 2 * sg.first;
      xa.s = f32x16{};
#pragma unroll
      for (int x = 0; x < C; ++x)
        xa.s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(key_operand(step0, x)), q[x], xa.s, 0, 0, 0);
#pragma unroll
      for (int x = 0; x < C; ++x) ring[x] = key_operand(step0 + 1, x);
      scale_of_step(vs0, 0, sv0);
      top_of(xa, 0);
      top_of(xa, 1);
      compare(xa, sv0);
      exponents(xa, sv0);
      settle(xa, 32 * step0, sv0);
      // One step: the softmax of its scores x beside the products of the next scores y, then the
      // outputs' products beside what follows from y.  Slots hold one product and its share of the
      // vector work each: what a slot computes stays there (the empty statements).
      auto step = [&](int s, Scores &x, Scores &y, const float (&svn)[2], auto &&extra) __attribute__((always_inline)) {
        constexpr int kPer = 16 / C;
        float back[2], sum[2] = {0.f, 0.f}, e[16];
        f16x8 pr[2];
        auto finish = [&](int i) __attribute__((always_inline)) {
          sum[i >> 3] = (i & 7) ? sum[i >> 3] + e[i] : e[i];
          asm volatile("" ::"v"(sum[i >> 3]));
          if (i & 1) {
            const f16x2 w = {(_Float16)e[i - 1], (_Float16)e[i]};
            const uint32_t u = __builtin_bit_cast(uint32_t, w);
            asm volatile("" ::"v"(u));
            u32x4 z = __builtin_bit_cast(u32x4, pr[i >> 3]);
            z[(i & 7) >> 1] = u;
            pr[i >> 3] = __builtin_bit_cast(f16x8, z);
          }
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < C; ++j) {
          y.s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ring[j]), q[j], j == 0 ? f32x16{} : y.s, 0, 0, 0);
          ring[j] = value_operand(s, j);
#pragma unroll
          for (int i = kPer * j; i < kPer * (j + 1); ++i) {
            e[i] = fast_exp2(__builtin_fmaf(x.s[i], p.scale_log2, -x.at[i >> 3]));
            asm volatile("" ::"v"(e[i]));
            if (i > 0) finish(i - 1);
          }
          if (j == 1 || j == 2) {
            back[j - 1] = fast_exp2(x.at[j - 1] - m);
            asm volatile("" ::"v"(back[j - 1]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
          if (j == 0) finish(15);
          o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, ring[j]), pr[j / DT], o[j % DT],
                                                             0, 0, 0);
          ring[j] = key_operand(s + 2, j);
          if (j == 0) {
            l = __builtin_fmaf(sum[1], back[1], __builtin_fmaf(sum[0], back[0], l));
            asm volatile("" ::"v"(l));
          }
          extra(j);
          if (j == C - 3 || j == C - 2) {
            top_of(y, j - (C - 3));
            asm volatile("" ::"v"(y.top[j - (C - 3)]));
          }
          if (j == C - 1) {
            compare(y, svn);
            exponents(y, svn);
            asm volatile("" ::"v"(y.at[0]), "v"(y.at[1]), "s"(y.rises));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        settle(y, 32 * s + 32, svn);
      };
      // A wave without pairs, or past its rows' last key, has no products left: it goes on with its share
      // of the tiles (64 sequences of 4,096 keys with 96 pairs: 133 us with its masked products, 96 without).
      const int own = min(last, (most + kTileKeys - 1) / kTileKeys);
      int tile = sg.first;
      for (; tile < own; ++tile) {
        clean(tile + 2, raw);
        scale_of_step(vs0, 1, sv1);
        // Registers are loaded anew once they are in LDS: a tile ahead of their use.
        Place at3;
        step(2 * tile, xa, xb, sv1, [&](int j) __attribute__((always_inline)) {
          if (j == 0) put_keys(tile + 2, raw);
          if (j == 1) at3 = place(tile + 3, entry3);
          if (j == 2) load_keys(at3, raw);
        });
        scale_of_step(vs1, 0, sv0);
        step(2 * tile + 1, xb, xa, sv0, [&](int j) __attribute__((always_inline)) {
          if (j == 0) {
            put_values(tile + 2, raw);
            vs2 = __builtin_amdgcn_readfirstlane(raw.vs);
          }
          if (j == 1) load_values(at3, raw);
          if (j == 2) entry3 = page_entry(pages, index(tile + 4));
        });
        vs0 = vs1;
        vs1 = vs2;
        __syncthreads();
      }
      for (; tile < last; ++tile) {
        clean(tile + 2, raw);
        put_keys(tile + 2, raw);
        put_values(tile + 2, raw);
        const Place at3 = place(tile + 3, entry3);
        load_keys(at3, raw);
        load_values(at3, raw);
        entry3 = page_entry(pages, index(tile + 4));
        __syncthreads();
      }
    }

    const bool whole = !p.n_workers || (sg.first == 0 && sg.last == sg.steps);
    const int slot = 2 * blockIdx.x + (part.t - sg.listed == part0 ? 0 : 1);
    int row_at = j0;  // (hidden: addresses made of it before the first segment would cost registers throughout)
    asm volatile("" : "+v"(row_at));
    l += __shfl_xor(l, 32, 64);
    if (j0 < n_pairs) {
      const float from0 = __builtin_fmaf(base, p.scale_log2, m);  // the maximum, counted from 0
      const int64_t gp = (row_base + pair / G) * p.n_q_heads + h * G + pair % G;
      // What a weight of 1 stands for, in two equal factors: with the smallest value scales 2^-128.
      const float unit = fast_exp2(0.5f * (M - m - kHead)), inv = l == 0.f ? 0.f : unit / l;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 32 * dt + 8 * i + 4 * hh;
          const f32x4 y = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]} * unit;
          if (whole)
            *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) =
                make_ushort4(f32_to_bf16(y[0] * inv), f32_to_bf16(y[1] * inv), f32_to_bf16(y[2] * inv),
                             f32_to_bf16(y[3] * inv));
          else
            *reinterpret_cast<f32x4 *>(p.part_o + ((int64_t)slot * kPairs + row_at) * D + e) = y * unit;
        }
      if (hh == 0) {
        if (!whole)
          p.part_ml[(int64_t)slot * kPairs + row_at] = make_float2(from0, l);
        else if (p.lse_out)
          p.lse_out[gp] = l == 0.f ? kNegInf : (from0 + __log2f(l)) * kLn2;
      }
    }
    if (!p.n_workers) break;
  }
}

template <int D, int W>
void launch_few(const MxAttnParams &p, bool wide, bool bf16, int grid, size_t lds, hipStream_t s) {
  if (bf16)
    wide ? attn_byte_kernel<D, 2, 1, W><<<grid, 64 * W, lds, s>>>(p)
         : attn_byte_kernel<D, 1, 1, W><<<grid, 64 * W, lds, s>>>(p);
  else if (!wide)
    attn_byte_kernel<D, 1, 3, W><<<grid, 64 * W, lds, s>>>(p);
  else if constexpr (few_pairs(D, 32, false) == 32)
    attn_byte_kernel<D, 2, 3, W><<<grid, 64 * W, lds, s>>>(p);
}

template <int D>
void launch_dim(const MxAttnParams &p, const MxAttnShape &sh, bool bf16, hipStream_t s) {
  const int n_sb = p.n_seqs * p.blocks_per_seq;
  const int grid = p.n_workers ? p.n_workers : n_sb * p.mx.n_kv_heads;
  const bool many = sh.pairs == kBytePairs;
  const size_t lds = p.n_workers && (many || n_sb > kLaneBlocks) ? (size_t)(n_sb + 1) * 4 : 0;
  if (many)
    attn_byte_many_kernel<D><<<grid, kManyThreads, lds, s>>>(p);
  else if (p.n_workers || grid > 256)
    launch_few<D, 4>(p, sh.pairs > 16, bf16, grid, lds, s);
  else
    launch_few<D, 8>(p, sh.pairs > 16, bf16, grid, lds, s);
}

}  // namespace

// Whether a block takes kBytePairs pairs.  Such a block reads and decodes its keys once, but takes
// 10 us for its first tile and its end, and is at work on one CU alone; blocks of 32 pairs read the cache
// again for every 32, and spread over the chip.  4 KV heads, blocks of 32 and of 256 pairs, in us, D = 128 (every
// row to the last key):
//   sequences x keys     64 pairs     128         256         512
//   1 x 8,192            16   18      21   22     26   31     35   34
//   1 x 16,384           21   20      25   26     32   32     48   40
//   1 x 65,536           31   33      45   38     74   55    132   86
//   8 x 2,048                                     23   38     38   43
//   8 x 4,096            25   25      36   31     38   46     67   59
//   64 x 4,096           81   90     140  104    271  161    516  314
//   256 x 512            59   62     102   72    195  109    404  220
// and D = 64: 64 x 4,096 keys with 128 pairs 91 and 86, 256 pairs 151 and 116; 256 x 512 with 96 pairs
// 44 and 53, 256 pairs 107 and 76.  So blocks of 256 pairs for calls whose blocks of 32 have 2^18 keys in all, unless
// those give every CU one, two or three to do by itself, of up to 2^20 keys on all CUs together: 256 blocks of 1,024 keys
// take 16 us and in blocks of 256 pairs 38 (D = 64: 11 and 29), of 4,096 38 and 46 (26 and 41), 320 of
// 2,048 37 and 39, of 3,000 52 and 45, 512 of 2,048 38 and 43 (26 and 38), 1,024 of 1,024 43 and 39 (27 and 30).
// With sequences of all lengths up to these, 0.4 to 1.1 of the time of blocks of 256 pairs.
// Of fewer than 256 blocks the two are within 1.2 of one another from 2^18 to 2^19 keys in all, blocks of 32 the faster
// ones with heads of 128 (1 x 8,192 keys with 256 pairs 26 and 31).
inline bool many_pairs(int64_t n_seqs, int64_t n_kv_heads, int64_t n_ctx, int head_dim, int64_t pairs, bool bf16) {
  // (fewer than 2^24 blocks, of up to 2^31 keys)
  const int64_t blocks = n_seqs * n_kv_heads * ((pairs + 31) / 32), of_a_cu = (blocks + 255) / 256;
  const bool fills = blocks >= 256 && blocks < 1024 && of_a_cu * 256 * n_ctx <= 1 << 20;
  return bf16 && pairs > (head_dim == 128 ? 64 : 128) && blocks * n_ctx >= 1 << 18 && !fills;
}

MxAttnShape byte_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16) {
  MxAttnShape L{};
  const int64_t pairs = (int64_t)rows_per_seq * (n_q_heads / n_kv_heads);
  const bool many = many_pairs(n_seqs, n_kv_heads, n_ctx, head_dim, pairs, bf16);
  L.pairs = many ? kBytePairs : few_pairs(head_dim, pairs, bf16);
  L.blocks_per_seq = (int32_t)((pairs + L.pairs - 1) / L.pairs);
  const int64_t n_sb = (int64_t)n_seqs * L.blocks_per_seq, blocks = n_sb * n_kv_heads;
  const int64_t steps = ((int64_t)n_ctx + kStep - 1) / kStep;
  const int64_t resident =
      256 * (many ? 1 : waves_per_simd(head_dim, L.pairs > 16 ? 2 : 1, bf16 ? 1 : 3));
  // Workgroups share the steps out evenly, for a second launch that merges, from
  // this many steps of a block on (and while the parts' list fits LDS): fewer are
  // done sooner by a workgroup per block, and the more blocks there are the less
  // there is to even out.  4 KV heads, by block and shared: one sequence of 512 keys 8 and 11
  // us, of 1,024 11 and 11, of 2,200 18 and 11; 64 of up to 2,048 20 and 23, of 4,096 34 and 39,
  // of 32,768 (shared) 195; 80 of up to 6,000 70 and 58; 256 of up to 4,096 126 and 134, of
  // 8,192 230 and 219.  Blocks of 256 pairs: 192 of 2,048 keys 71 and 86, 64 of 2,048 67
  // and 53, 256 of 4,096 (as even as can be) 143 and 153.
  const int64_t from = blocks < 256 ? 8 : many && blocks < 1024 ? 16 : 32;
  // (The merge has up to L.pairs workgroups of 256 threads a block, fewer than 2^32.)
  if (steps > from && n_sb <= kMaxSeqBlocks && 2 * blocks * (steps + kManyPad) < INT32_MAX &&
      blocks * L.pairs < 1 << 24)
    L.n_workers = (int32_t)std::min<int64_t>(resident, std::max<int64_t>(1, blocks * steps / kMinSteps));
  lay_out_workspace(L, n_sb, head_dim);
  return L;
}

hipError_t launch_attn_byte(const MxAttnParams &p, const MxAttnShape &sh, int head_dim, bool bf16, hipStream_t s) {
  {
    ProfScope ps("attn_byte", s);
    head_dim == 128 ? launch_dim<128>(p, sh, bf16, s) : launch_dim<64>(p, sh, bf16, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.n_workers) return e;
  return launch_attn_merge(p, sh, "attn_byte_merge", head_dim, bf16, s, sh.pairs == kBytePairs ? kManyPad : 0);
}

}  // namespace conduit
