// Causal attention over the 8-bit KV cache, gfx950.
//
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
// fp32 rows of 128 dims would leave registers for one wave per SIMD only (1,500
// rows over 16k tokens: 32 pairs 1,094 us, 16 pairs 804 us).
constexpr int few_pairs(int D, int64_t pairs, bool bf16) { return pairs <= 16 || (D == 128 && !bf16) ? 16 : 32; }

// MT: groups of 16 pairs of a block.  NS: exact bf16 parts of queries (1: bf16
// tensors, 3: fp32).  W: waves of a workgroup, 4, or 8 for a
// workgroup per block on up to 256 blocks (64 sequences of 2,048 keys: 4 waves 20
// us, 8 waves 16 us; 256 of 512, which leave the CUs several blocks each: 16 and 24 us).
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
                                   : Segment{(int)blockIdx.x / hkv, (int)blockIdx.x % hkv, 0, INT32_MAX, 0};
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
  const size_t lds = p.n_workers && n_sb > kLaneBlocks ? (size_t)(n_sb + 1) * 4 : 0;
  if (p.n_workers || grid > 256)
    launch_few<D, 4>(p, sh.pairs > 16, bf16, grid, lds, s);
  else
    launch_few<D, 8>(p, sh.pairs > 16, bf16, grid, lds, s);
}

}  // namespace

MxAttnShape byte_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16) {
  MxAttnShape L{};
  const int64_t pairs = (int64_t)rows_per_seq * (n_q_heads / n_kv_heads);
  L.pairs = few_pairs(head_dim, pairs, bf16);
  L.blocks_per_seq = (int32_t)((pairs + L.pairs - 1) / L.pairs);
  const int64_t n_sb = (int64_t)n_seqs * L.blocks_per_seq, blocks = n_sb * n_kv_heads;
  const int64_t steps = ((int64_t)n_ctx + kStep - 1) / kStep;
  const int64_t resident =
      256 * waves_per_simd(head_dim, L.pairs > 16 ? 2 : 1, bf16 ? 1 : 3);
  // Workgroups share the steps out evenly, for a second launch that merges, from
  // this many steps of a block on (and while the parts' list fits LDS): fewer are
  // done sooner by a workgroup per block, and the more blocks there are the less
  // there is to even out.  One sequence of 4 KV heads: 1,024 keys 9 us by block,
  // 11 us shared; 2,200 keys 14 and 11 us.  64 sequences of up to 2,048: 15 and 20
  // us.  256 of up to 4,096: 75 and 84 us, of up to 8,192: 144 and 140 us.
  const int64_t from = blocks < 256 ? 8 : blocks < 1024 ? 16 : 32;
  // (The merge has up to L.pairs workgroups of 256 threads a block, fewer than 2^32.)
  if (steps > from && n_sb <= kMaxSeqBlocks && 2 * blocks * steps < INT32_MAX &&
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
  return launch_attn_merge(p, sh, "attn_byte_merge", head_dim, bf16, s);
}

}  // namespace conduit
