// Internal declarations of rotary positions, growing caches and the 4-bit and
// 8-bit caches (rotary.hip, append_byte.hip, attn_mx.hip, attn_byte.hip and the host
// layer).
#pragma once

#include "common.h"

namespace conduit {

// Rotary frequencies, passed by value in kernel arguments.
constexpr int kMaxRotHalf = 128;
struct RopeTable {
  int32_t half;                 // rot_dim / 2; 0: nothing turns
  int32_t n_axes;               // up to 4
  int32_t adjacent;             // pairs (2f, 2f + 1) instead of (f, f + half)
  int32_t inverse;
  const int32_t *pos;           // [axes][n]
  int64_t pos_stride;
  float inv_freq[kMaxRotHalf];
  uint8_t axis[kMaxRotHalf];
};

// The 4-bit cache (conduit_kv_mx) or the 8-bit one (conduit_kv_byte): they differ in
// the bytes of a token's codes and in what shares a scale.
struct MxCache {
  uint8_t *k, *v;
  uint8_t *k_scale, *v_scale;
  int64_t code_stride, scale_stride;  // bytes between pages
  const int32_t *table;               // nullable: page s * table_stride + i
  int32_t table_stride;
  int32_t shift;                      // log2 of the page size
  int32_t n_pages;
  int32_t n_ctx;
  int32_t n_kv_heads;
  int32_t rows_per_seq;               // rows of the call that a sequence has
};

// Page of token t of sequence s, clamped into the pool.
__device__ __forceinline__ int mx_page(const MxCache &c, int s, int t) {
  const int64_t i = (int64_t)s * c.table_stride + (t >> c.shift);
  const int64_t page = c.table ? c.table[i] : i;
  return (int)min(max(page, (int64_t)0), (int64_t)c.n_pages - 1);
}

constexpr int kMxBlock = 32;      // dims that share a scale
constexpr int kMxScaleMin = 2;    // smallest and largest scale byte written
constexpr int kMxScaleMax = 252;
constexpr int kMxScaleNan = 255;

constexpr int kByteBlock = 16;      // tokens of the 8-bit cache that share a scale
constexpr int kByteScaleMin = 10;   // smallest and largest scale byte written
constexpr int kByteScaleMax = 246;

// The factor of a scale byte of the 8-bit cache.  Bytes that no append writes are
// read as the nearest that one does.
__device__ __forceinline__ float byte_scale(int byte) {
  return __builtin_bit_cast(float, (uint32_t)min(max(byte, kByteScaleMin), kByteScaleMax) << 23);
}

// Orders this wave's LDS writes before its reads (and the other way round) for
// the compiler; the hardware keeps a wave's LDS accesses in order.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What a launch of the row kernel does with its rows.
enum RowMode {
  kRowTurn = 0,      // queries only (conduit_rotary)
  kRowAppend = 1,    // and keys and values into a cache of 16 or 32 bits
  kRowAppendMx = 2,  // and keys and values into a 4-bit cache
  kRowLoadMx = 3,    // rows of a 4-bit cache into a cache of 16 or 32 bits
  kRowLoadByte = 4     // rows of an 8-bit cache into a cache of 16 or 32 bits
};

struct RowParams {
  int32_t n;
  int32_t n_q_heads;            // 0 without queries
  int32_t n_kv_heads;           // 0 for kRowTurn
  int32_t head_dim;
  const void *q;
  void *q_out;
  int64_t q_stride, q_out_stride;       // elements
  const void *k_new, *v_new;            // kRowAppend, kRowAppendMx
  int64_t k_new_stride, v_new_stride;
  const int32_t *pos;                   // place in the cache (loads: in kv)
  const int32_t *src_pos;               // kRowLoadMx, kRowLoadByte: place in mx
  void *k, *v;                          // kRowAppend, loads: the cache
  int64_t k_stride, v_stride;
  KvPages pages;
  int32_t n_ctx;
  MxCache mx;                           // kRowAppendMx, kRowLoadMx, kRowLoadByte
  void *k_out, *v_out;                  // kRowAppendMx, nullable: the rows as held
  RopeTable rope;
};
hipError_t launch_rows(const RowParams &p, RowMode mode, bool bf16, hipStream_t s);

// New rows into an 8-bit cache (RowParams without kv; rope may turn).
struct ByteAppendParams {
  RowParams rows;               // n, heads, new rows, positions, mx, k_out, v_out, rope
  const int32_t *n_held;        // nullable [n / rows.mx.rows_per_seq]: tokens held before
};
hipError_t launch_append_byte(const ByteAppendParams &p, bool bf16, hipStream_t s);

// Attention over a 4-bit or an 8-bit cache.
struct MxAttnParams {
  MxCache mx;
  int32_t n_seqs;
  int32_t n_q_heads;
  int32_t group;
  int32_t blocks_per_seq;       // pair blocks of a sequence and KV head
  int32_t n_workers;            // workgroups that share the key steps evenly; 0: one per block
  const void *q;                // [n][n_q_heads][D]
  const int32_t *pos;           // [n]
  float scale_log2;             // logit scale * log2(e)
  void *o_out;                  // [n][n_q_heads][D]
  float *lse_out;               // nullable
  int32_t *prefix;              // [seq blocks + 1]: key steps before each
  int32_t *cut;                 // length of parts that end with their block, or 0
  int32_t *parts;               // [up to 64 seq blocks]: such parts before each
  float2 *part_ml;              // [2 * n_workers][pairs per block] running maximum, denominator
  float *part_o;                // [2 * n_workers][pairs per block][D] unnormalised output
};

// How a call is cut up (shared by the workspace query and the launch).
struct MxAttnShape {
  int32_t pairs;                // (row, head) pairs of a block
  int32_t blocks_per_seq;
  int32_t n_workers;
  size_t prefix, parts, ml, o, total;  // workspace offsets
};
MxAttnShape mx_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16);
hipError_t launch_attn_mx(const MxAttnParams &p, const MxAttnShape &shape, int head_dim, bool bf16, hipStream_t s);
MxAttnShape byte_attn_shape(int32_t n_seqs, int32_t rows_per_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_ctx,
                          int32_t head_dim, bool bf16);
hipError_t launch_attn_byte(const MxAttnParams &p, const MxAttnShape &shape, int head_dim, bool bf16, hipStream_t s);

}  // namespace conduit
