// What attention over the 4-bit and the 8-bit cache shares (attn_mx.hip,
// attn_byte.hip): how the key steps of a call are listed and shared out over
// workgroups, how pages are looked up, exact bf16 parts of fp32 numbers, and the
// launch that joins blocks which were cut.
#pragma once

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

// Many pairs per KV head: keys of a tile, pairs of a block, and LDS of a workgroup.
constexpr int kTileKeys = 64;
constexpr int kManyPairs = 32 * kWaves;

template <int NS>
struct Parts {
  bf16x8 v[NS];
};

// x as the sum of NS bf16 parts, each the nearest to what those before it leave
// (half a step is up to 2^-8 of a value): three are exact, two up to 2^-17 of x off.
// WIDE: the first part is cut off instead (16 of 24 bits are left, which two parts hold),
// because the largest x would round up to an infinity.
template <int NS, bool WIDE = false>
__device__ __forceinline__ void split_parts(const float (&x)[8], Parts<NS> &out) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      __bf16 b = static_cast<__bf16>(r[j]);
      if (WIDE && s == 0) {
        const u16 top = (u16)(__builtin_bit_cast(uint32_t, r[j]) >> 16);
        b = __builtin_bit_cast(__bf16, top);
      }
      out.v[s][j] = b;
      if (s + 1 < NS) r[j] -= (float)b;
    }
}

__device__ __forceinline__ float scale_of(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

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

// Steps of `step` keys of sequence block sb for one KV head (positions loaded
// BATCH at a time).
template <int BATCH>
__device__ __forceinline__ int block_steps(const MxAttnParams &p, int sb, int pairs, int step) {
  const int s = sb / p.blocks_per_seq, rb = sb - s * p.blocks_per_seq, r = p.mx.rows_per_seq;
  const int lo = rb * pairs / p.group, hi = min((rb * pairs + pairs - 1) / p.group, r - 1);
  const int32_t *pos = p.pos + (int64_t)s * r;
  int top = -1;
  for (int i = lo; i <= hi; i += BATCH) {
    int x[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) x[j] = pos[min(i + j, hi)];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) top = max(top, x[j]);
  }
  return (keys_seen(top, p.mx.n_ctx) + step - 1) / step;
}

// The most keys that a row of each sequence block sees, found by the whole workgroup: a row a
// thread, kept per block in LDS (at most 4,096 blocks of 256 rows).  A thread that reads all
// rows of a block of its own waits for them in turn: with this and attn_merge_many_kernel 256
// blocks of 256 rows over 256 keys took 33 us where they had taken 62.
template <int W>
__device__ __forceinline__ void block_tops(const MxAttnParams &p, int pairs, int *s_top) {
  constexpr int kThreads = 64 * W, kBatch = 8;
  const int tid = threadIdx.x, n_sb = p.n_seqs * p.blocks_per_seq, r = p.mx.rows_per_seq, rows = p.n_seqs * r;
  for (int i = tid; i < n_sb; i += kThreads) s_top[i] = 0;
  __syncthreads();
  for (int row0 = tid; row0 < rows; row0 += kBatch * kThreads) {
    int x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) x[j] = p.pos[min(row0 + j * kThreads, rows - 1)];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int row = row0 + j * kThreads;
      if (row >= rows) break;
      const int s = row / r, i = (row - s * r) * p.group, seen = keys_seen(x[j], p.mx.n_ctx);
      for (int b = i / pairs; b <= (i + p.group - 1) / pairs; ++b) atomicMax(s_top + s * p.blocks_per_seq + b, seen);
    }
  }
  __syncthreads();
}

// Workgroups that share `total` steps: no fewer than kMinSteps each.
constexpr int kMinSteps = 2;
__device__ __forceinline__ int workers(int n_workers, int total) { return min(n_workers, max(1, total / kMinSteps)); }
__device__ __forceinline__ int part_begin(int w, int total, int n) { return (int)((int64_t)w * total / n); }

// The list of key steps of the whole call (sequence block by sequence block and
// there KV head by KV head) and what of it is this workgroup's; workgroup 0 keeps
// the list for the merge.  With up to 64 sequence blocks every wave makes the list
// for itself, a block a lane; with more the workgroup makes it in LDS.
//
// Equal parts may begin in one block and end in the next, and what ends and
// begins there costs a workgroup as much as three steps.  Where parts of up to
// kOver steps more than equal ones can be cut block by block for the workgroups at
// hand, they are (`cut`: their length).  8 sequences of up to 8,192 keys with 5 rows
// 26.0 -> 23.3 us, one of 4,096 with 200 rows 39.5 -> 36.1.
constexpr int kOver = 2;
constexpr int kLaneBlocks = 64;
struct Part {
  int t, t_end;              // places in the list: steps, or with cut parts
  int cut;
  int before, after, steps;  // up to kLaneBlocks: the lane's block in the list, and its steps per head
};
//
// W: waves of the workgroup.  BATCH: see block_steps.  PAD: steps that a block is listed with
// before its own, for what beginning it costs a workgroup (merge: the same).  With blocks of
// many pairs, whose first products wait for queries, pages and a tile in LDS, a workgroup
// that had ten short blocks ended long after one that had half of a long one.
// ROWS: positions read by the whole workgroup (block_tops), for which s_prefix has its n_sb + 1
// entries with few sequence blocks too.
template <int W = kWaves, int BATCH = 8, int PAD = 0, bool ROWS = false>
__device__ __forceinline__ bool plan_part(const MxAttnParams &p, int pairs, int step, int *s_sum, int *s_prefix,
                                          Part &part) {
  constexpr int kWaves = W, kThreads = 64 * W;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_sb = p.n_seqs * p.blocks_per_seq, hkv = p.mx.n_kv_heads, w = blockIdx.x;
  int total = 0;
  if constexpr (ROWS) block_tops<W>(p, pairs, s_prefix);
  auto steps_of = [&](int sb) __attribute__((always_inline)) {
    if constexpr (ROWS) return (s_prefix[sb] + step - 1) / step;
    else return block_steps<BATCH>(p, sb, pairs, step);
  };
  if (n_sb <= kLaneBlocks) {
    part.steps = lane < n_sb ? steps_of(lane) : 0;
    int own = part.steps * hkv;
    int steps = 0;  // of the call, without PAD
    if (PAD) steps = __builtin_amdgcn_readlane((int)wave_inclusive_sum((uint32_t)own), 63);
    if (PAD && own) own += PAD * hkv;
    part.after = (int)wave_inclusive_sum((uint32_t)own);
    part.before = part.after - own;
    total = __builtin_amdgcn_readlane(part.after, 63);
    if (!PAD) steps = total;
    if (w == 0 && wave == 0) {
      if (lane < n_sb) p.prefix[lane] = part.before;
      if (lane == 0) p.prefix[n_sb] = total;
    }
    const int n = workers(p.n_workers, steps), equal = max(1, (steps + n - 1) / n);
    for (int x = equal; x <= equal + kOver; ++x) {
      own = (part.steps + x - 1) / x * hkv;
      const int incl = (int)wave_inclusive_sum((uint32_t)own), all = __builtin_amdgcn_readlane(incl, 63);
      if (all <= p.n_workers) {
        part.cut = x;
        part.after = incl;
        part.before = incl - own;
        part.t = w;
        part.t_end = min(w + 1, all);
        break;
      }
    }
    if (w == 0 && wave == 0) {
      if (lane == 0) *p.cut = part.cut;
      if (lane < n_sb) p.parts[lane] = part.before;
    }
    if (part.cut) return part.t < part.t_end;
  } else {
    for (int b0 = 0; b0 < n_sb; b0 += kThreads) {
      const int sb = b0 + tid;
      int own = sb < n_sb ? steps_of(sb) * hkv : 0;
      if (PAD && own) own += PAD * hkv;
      const int incl = (int)wave_inclusive_sum((uint32_t)own);
      __syncthreads();
      if (lane == 63) s_sum[wave] = incl;
      __syncthreads();
      int before = total;
      for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += s_sum[i];
        total += s_sum[i];
      }
      if (sb < n_sb) s_prefix[sb] = before + incl - own;
    }
    if (tid == 0) s_prefix[n_sb] = total;
    __syncthreads();
    if (w == 0) {
      for (int i = tid; i <= n_sb; i += kThreads) p.prefix[i] = s_prefix[i];
      if (tid == 0) *p.cut = 0;
    }
  }
  const int n = workers(p.n_workers, total);
  if (w >= n) return false;
  part.t = __builtin_amdgcn_readfirstlane(part_begin(w, total, n));
  part.t_end = __builtin_amdgcn_readfirstlane(part_begin(w + 1, total, n));
  return true;
}

// What of a part lies in one (sequence block, KV head): its steps [first, last)
// of `steps` (none where the part ends within PAD), and how far that goes in the list.
struct Segment {
  int sb, h, first, last, steps, listed;
};
template <int PAD = 0>
__device__ __forceinline__ Segment segment_at(const MxAttnParams &p, int n_sb, const int *s_prefix, const Part &part) {
  int sb, begin, steps;
  if (n_sb <= kLaneBlocks) {
    sb = (int)__builtin_popcountll(__ballot(part.after <= part.t));
    begin = __builtin_amdgcn_readlane(part.before, sb);
    steps = __builtin_amdgcn_readlane(part.steps, sb);
  } else {
    int lo = 0, hi = n_sb - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_prefix[mid + 1] > part.t) hi = mid;
      else lo = mid + 1;
    }
    sb = __builtin_amdgcn_readfirstlane(lo);
    begin = __builtin_amdgcn_readfirstlane(s_prefix[lo]);
    steps = __builtin_amdgcn_readfirstlane((s_prefix[lo + 1] - begin) / p.mx.n_kv_heads) - PAD;
  }
  if (PAD && !part.cut) {
    const int h = (part.t - begin) / (steps + PAD), from = part.t - begin - h * (steps + PAD);
    const int to = min(steps + PAD, from + part.t_end - part.t);
    return {sb, h, max(from - PAD, 0), max(to - PAD, 0), steps, to - from};
  }
  const int per_head = part.cut ? (steps + part.cut - 1) / part.cut : steps, at = part.t - begin;
  const int h = at / per_head, rest = at - h * per_head;
  const int first = part.cut ? rest * part.cut : rest;
  const int last = min(steps, first + (part.cut ? part.cut : part.t_end - part.t));
  return {sb, h, first, last, steps, part.cut ? 1 : last - first};
}

// Pages of one sequence, looked up in two parts: the block-table entry is loaded
// well before it is made a page number.  (A load whose address is the same in
// every lane would be made scalar, and waited for, at once: the lane's offset is
// hidden from the compiler.  That wait, for every load in flight, was 1 us a tile.)
struct SeqPages {
  __amdgpu_buffer_rsrc_t table;
  int first;     // page of token 0 without a table
  bool listed;
};
__device__ __forceinline__ SeqPages seq_pages(const MxCache &c, int seq) {
  const int64_t first = (int64_t)seq * c.table_stride;
  SeqPages r;
  r.listed = c.table != nullptr;
  r.first = (int)first;
  // (2^24 pages hold 2^30 tokens; a read past the end returns 0)
  r.table = buffer_rsrc(r.listed ? c.table + first : nullptr, r.listed ? min(c.table_stride, 1 << 24) * 4 : 0);
  return r;
}
__device__ __forceinline__ int page_entry(const SeqPages &s, int i) {
  int off = i * 4;
  asm("" : "+v"(off));
  return __builtin_amdgcn_raw_buffer_load_b32(s.table, off, 0, 0);
}
__device__ __forceinline__ int page_number(const MxCache &c, const SeqPages &s, int i, int entry) {
  const int page = s.listed ? __builtin_amdgcn_readfirstlane(entry) : s.first + i;
  return min(max(page, 0), c.n_pages - 1);
}

// The workgroups w0 .. w1 that worked on a KV head of a block (none: w1 < w0), and where the first's part lies.
struct MergeParts {
  int w0, w1, first;
};
__device__ __forceinline__ MergeParts merge_parts(const MxAttnParams &p, int sb, int h, int pad) {
  const int hkv = p.mx.n_kv_heads;
  const int base = p.prefix[sb], next = p.prefix[sb + 1], total = p.prefix[p.n_seqs * p.blocks_per_seq];
  const int cut = *p.cut;
  const int n = workers(p.n_workers, total), steps = (next - base) / hkv;  // (with `pad`)
  if (steps <= 0) return {0, -1, 0};
  if (cut) {
    const int parts = (steps - pad + cut - 1) / cut, w0 = p.parts[sb] + h * parts;
    return {w0, w0 + parts - 1, 2 * w0};
  }
  // The workgroup that holds step x is the last whose part begins at or
  // before it (doubles: exact below 2^53, quotients far from rounding up).
  const int t0 = base + h * steps, t1 = t0 + steps;
  int w0 = (int)(((double)(t0 + 1) * n - 1) / total), w1 = (int)(((double)t1 * n - 1) / total);
  int first = 2 * w0 + (part_begin(w0, total, n) >= t0 ? 0 : 1);
  while (pad && part_begin(w0 + 1, total, n) - t0 <= pad) first = 2 * ++w0;  // (has no step of its own)
  return {w0, w1, first};
}

// Merge of the blocks that more than one workgroup worked on, and the outputs
// of blocks without keys.  A workgroup takes PW pairs of a block, a group of D / 4
// lanes each; with PW = 1 all groups share the parts of one pair.
template <int D, bool BF16, int PW>
__global__ __launch_bounds__(256) void attn_merge_kernel(MxAttnParams p, int pairs, int pad) {
  constexpr int L4 = D / 4;          // lanes of a part
  constexpr int kGroups = 256 / L4, kShare = kGroups / PW;
  // Parts a group has on their way at a time: where a workgroup shares one pair's,
  // there may be a hundred (one sequence of 65,536 keys, both launches: one at a
  // time 23.8 us, four 19.9).
  constexpr int kBatch = PW == 1 ? 4 : 1;
  __shared__ float s_m[kGroups], s_l[kGroups];
  __shared__ f32x4 s_o[kShare > 1 ? kGroups : 1][L4];
  const int chunks = (min(pairs, p.mx.rows_per_seq * p.group) + PW - 1) / PW, hkv = p.mx.n_kv_heads;
  const int sb = blockIdx.x / (chunks * hkv), rest = blockIdx.x - sb * (chunks * hkv);
  const int h = rest / chunks, chunk = rest - h * chunks;
  const int seq = sb / p.blocks_per_seq, rb = sb - seq * p.blocks_per_seq;
  const int grp = threadIdx.x / L4, share = grp / PW, e = (threadIdx.x % L4) * 4;
  const int j = chunk * PW + grp % PW, pair = rb * pairs + j;
  const bool out = pair < p.mx.rows_per_seq * p.group;
  if (rb * pairs + chunk * PW >= p.mx.rows_per_seq * p.group) return;
  const auto [w0, w1, first] = merge_parts(p, sb, h, pad);
  if (w0 == w1) return;  // written by that workgroup
  float M = kMInit, L = 0.f;
  f32x4 o{};
  if (out)
    for (int w = w0 + share; w <= w1; w += kBatch * kShare) {
      float2 ml[kBatch];
      f32x4 x[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int wi = w + i * kShare;
        ml[i] = make_float2(kMInit, 0.f);
        x[i] = f32x4{};
        if (wi <= w1) {
          const int64_t slot = wi == w0 ? first : 2 * wi;
          ml[i] = p.part_ml[slot * pairs + j];
          x[i] = *reinterpret_cast<const f32x4 *>(p.part_o + (slot * pairs + j) * D + e);
        }
      }
      float mn = M;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) mn = fmaxf(mn, ml[i].x);
      const float a = fast_exp2(M - mn);
      M = mn;
      L *= a;
      o *= a;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const float b = fast_exp2(ml[i].x - mn);
        L += ml[i].y * b;
        o += x[i] * b;
      }
    }
  if constexpr (kShare > 1) {
    s_o[grp][threadIdx.x % L4] = o;
    if (e == 0) {
      s_m[grp] = M;
      s_l[grp] = L;
    }
    __syncthreads();
    if (share) return;
    for (int i = PW + grp; i < kGroups; i += PW) {
      const float mn = fmaxf(M, s_m[i]), a = fast_exp2(M - mn), b = fast_exp2(s_m[i] - mn);
      M = mn;
      L = L * a + s_l[i] * b;
      o = o * a + s_o[i][threadIdx.x % L4] * b;
    }
  }
  if (!out) return;
  o *= L == 0.f ? 0.f : 1.f / L;
  const int64_t gp = ((int64_t)seq * p.mx.rows_per_seq + pair / p.group) * p.n_q_heads + h * p.group + pair % p.group;
  if constexpr (BF16) {
    *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) =
        make_ushort4(f32_to_bf16(o[0]), f32_to_bf16(o[1]), f32_to_bf16(o[2]), f32_to_bf16(o[3]));
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(p.o_out) + gp * D + e) = o;
  }
  if (e == 0 && p.lse_out) p.lse_out[gp] = L == 0.f ? kNegInf : (M + __log2f(L)) * kLn2;
}

// The same for blocks of many pairs, which few workgroups share: PW pairs at a time of kMergePairs
// of a block, whose parts are all on their way at once (8 pairs a workgroup, most of whose
// time goes to finding out whose parts it merges: 15 us of 1,638 rows and 8 KV heads, so 13).
constexpr int kMergePairs = 32;
template <int D, int PW>
__global__ __launch_bounds__(256) void attn_merge_many_kernel(MxAttnParams p, int pairs, int pad) {
  constexpr int L4 = D / 4, kTurns = kMergePairs / PW;
  static_assert(PW * L4 == 256, "a group of lanes a pair");
  const int n_pairs = p.mx.rows_per_seq * p.group, hkv = p.mx.n_kv_heads;
  const int chunks = (min(pairs, n_pairs) + kMergePairs - 1) / kMergePairs;
  const int sb = blockIdx.x / (chunks * hkv), rest = blockIdx.x - sb * (chunks * hkv);
  const int h = rest / chunks, j0 = (rest - h * chunks) * kMergePairs + threadIdx.x / L4;
  const int seq = sb / p.blocks_per_seq, rb = sb - seq * p.blocks_per_seq;
  const int e = (threadIdx.x % L4) * 4;
  if (rb * pairs + (rest - h * chunks) * kMergePairs >= n_pairs) return;
  const MergeParts w = merge_parts(p, sb, h, pad);
  if (w.w0 == w.w1) return;  // written by that workgroup
  float M[kTurns], L[kTurns];
  f32x4 o[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    M[i] = kMInit;
    L[i] = 0.f;
    o[i] = f32x4{};
  }
  for (int x = w.w0; x <= w.w1; ++x) {
    const int64_t slot = (x == w.w0 ? w.first : 2 * (int64_t)x) * pairs + j0;
    float2 ml[kTurns];
    f32x4 y[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      ml[i] = p.part_ml[slot + i * PW];
      y[i] = *reinterpret_cast<const f32x4 *>(p.part_o + (slot + i * PW) * D + e);
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const float mn = fmaxf(M[i], ml[i].x), a = fast_exp2(M[i] - mn), b = fast_exp2(ml[i].x - mn);
      M[i] = mn;
      L[i] = L[i] * a + ml[i].y * b;
      o[i] = o[i] * a + y[i] * b;
    }
  }
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int pair = rb * pairs + j0 + i * PW;
    if (pair >= n_pairs) break;
    o[i] *= L[i] == 0.f ? 0.f : 1.f / L[i];
    const int64_t gp = ((int64_t)seq * p.mx.rows_per_seq + pair / p.group) * p.n_q_heads + h * p.group + pair % p.group;
    *reinterpret_cast<ushort4 *>(static_cast<u16 *>(p.o_out) + gp * D + e) =
        make_ushort4(f32_to_bf16(o[i][0]), f32_to_bf16(o[i][1]), f32_to_bf16(o[i][2]), f32_to_bf16(o[i][3]));
    if (e == 0 && p.lse_out) p.lse_out[gp] = L[i] == 0.f ? kNegInf : (M[i] + __log2f(L[i])) * kLn2;
  }
}

template <int D, int PW>
void launch_merge(const MxAttnParams &p, const MxAttnShape &sh, int pad, int blocks, bool few, bool bf16,
                  hipStream_t s) {
  const int pairs = std::min(sh.pairs, p.mx.rows_per_seq * p.group);  // of the largest block
  const int grid = blocks * (few ? pairs : (pairs + PW - 1) / PW);
  if (few)
    bf16 ? attn_merge_kernel<D, true, 1><<<grid, 256, 0, s>>>(p, sh.pairs, pad)
         : attn_merge_kernel<D, false, 1><<<grid, 256, 0, s>>>(p, sh.pairs, pad);
  else
    attn_merge_kernel<D, true, PW><<<grid, 256, 0, s>>>(p, sh.pairs, pad);
}

// Workspace of a call whose workgroups share the steps.
inline void lay_out_workspace(MxAttnShape &L, int64_t n_sb, int head_dim) {
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
  if (L.n_workers) {
    const size_t slots = 2 * (size_t)L.n_workers * L.pairs;
    L.prefix = take((size_t)(n_sb + 1) * 4);
    L.parts = take((size_t)(kLaneBlocks + 1) * 4);
    L.ml = take(slots * 8);
    L.o = take(slots * head_dim * 4);
  }
  L.total = off;
}

// The launch that merges, where workgroups share the steps.  Few pairs: many parts of
// each, shared out over a workgroup; many pairs: a few parts of each, one group of lanes.
inline hipError_t launch_attn_merge(const MxAttnParams &p, const MxAttnShape &sh, const char *name, int head_dim,
                                    bool bf16, hipStream_t s, int pad = 0) {
  ProfScope ps(name, s);
  const int blocks = p.n_seqs * p.blocks_per_seq * p.mx.n_kv_heads;
  const bool few = sh.pairs <= 32 || p.n_workers > 4 * blocks;
  if (pad && !few) {
    const int grid = blocks * ((std::min(sh.pairs, p.mx.rows_per_seq * p.group) + kMergePairs - 1) / kMergePairs);
    head_dim == 128 ? attn_merge_many_kernel<128, 8><<<grid, 256, 0, s>>>(p, sh.pairs, pad)
                    : attn_merge_many_kernel<64, 16><<<grid, 256, 0, s>>>(p, sh.pairs, pad);
    return hipGetLastError();
  }
  if (head_dim == 128)
    launch_merge<128, 8>(p, sh, pad, blocks, few, bf16, s);
  else
    launch_merge<64, 16>(p, sh, pad, blocks, few, bf16, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace conduit
