// Attention of many query rows over the same keys: what the kernels of rows_*.hip and their entry points share.
//
// A launch works on SEGMENTS: a set of query rows and the keys that all of them attend to.  chunkkv_cross_attention has a segment per
// sequence, over keys that lie one behind the other; chunkkv_shared_decode_attention one per prefix, whose rows are the query heads of
// all sequences that share it, and one per sequence, over the pages of its own.  Row r of a segment and kv-head is query head r % g of
// its token (or sequence) r / g.
#pragma once
#include <float.h>

#include "paged.h"

namespace ckv {

constexpr int kRowsTile = 64;            // keys that a workgroup holds at a time
constexpr int kRowsNarrow = 32;          // query rows of half a workgroup, where a segment has no more
constexpr int kRowsWide = 128;           // of a workgroup; or twice as many
// Narrow tiles of a workgroup: as many as their slots fit into 128 KB of LDS.
__host__ __device__ constexpr int rows_pairs(int dtype, int head_dim) { return dtype == CHUNKKV_F32 && head_dim == 128 ? 1 : 2; }
constexpr int kCrossSegments = 32;       // segments of a launch: their table travels as kernel arguments
constexpr int kSharedSegments = 72;

// A segment of a launch.  Together in 32 bytes: a workgroup reads them with one load.
struct RowsSegment {
  int32_t rows;                          // query rows of a kv-head
  int32_t most;                          // keys, at most
  int32_t row0;                          // tokens (sequences) before: where its queries are, and of lse
  int32_t splits;                        // ranges that its keys are cut into
  int32_t tiles;                         // workgroups that share a range of a kv-head
  int32_t part;                          // number of its first partial row; -1: its workgroups write the outputs
  int32_t pad[2];
};

// x / d for 0 <= x < 2^31 and 0 < d <= 1024: the product is off by 1 at most, and too large then.
struct Divisor {
  uint32_t d, magic;                     // ceil(2^32 / d), 2^32 - 1 for 1
};
inline Divisor divisor(int d) { return {(uint32_t)d, d == 1 ? 0xFFFFFFFFu : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d)}; }
__device__ __forceinline__ int divided(int x, const Divisor &by) {
  if (by.d == 1) return x;
  const uint32_t q = __umulhi((uint32_t)x, by.magic);
  return (int)(q * by.d > (uint32_t)x ? q - 1 : q);
}

template <int N>
struct RowsArgs {
  static constexpr int kSegments = N;
  PageGeom geom;                         // pages: strides in bytes; keys in a row: tok and head alone
  const int32_t *prefix_table;           // pages: table of the segments below `prefixes`, [prefix][prefix_pitch]
  const int32_t *kv_len, *prefix_len;    // device lengths [segment][Hkv], or null: `most`
  const uint8_t *mask;                   // [segment][mask_pitch], or null
  const void *q, *k, *v;
  void *out;
  float *lse;
  float4 *part_ml;                       // (reference before the scale, sum of the weights as multiplied, sum before their rounding, -) of every partial row
  float *part_o;                         // [d] of every partial row
  int64_t q_tok, q_head, out_tok, out_head;        // bytes
  Divisor heads, group;                  // kv-heads; query heads of one
  int32_t mask_pitch;
  int32_t segments, prefixes;            // of the launch
  int32_t prefix_pitch;
  int32_t tile;                          // query rows of a workgroup: kRowsWide, or twice as many; kRowsNarrow where no segment has more
  int32_t prefix0, seq0;                 // number of its first prefix, of its first sequence
  float scale, scale_log2e;              // as PagedDecodeArgs has them
  static constexpr int kFirst = (N + 15) / 16 * 16 + 1;   // looked through by sixteens
  int32_t first[kFirst];                 // number of the first workgroup of every segment, INT32_MAX past the last one's end
  RowsSegment segment[N];
};
struct CrossArgs {
  RowsArgs<kCrossSegments> r;
  int64_t q_base[kCrossSegments], kv_base[kCrossSegments], out_base[kCrossSegments];   // bytes
};
struct SharedArgs {
  RowsArgs<kSharedSegments> r;
};

// Keys of each of `splits` ranges of n keys: whole tiles, from the length that the device knows.
__host__ __device__ inline int rows_range(int n, int splits) { return ((n + splits - 1) / splits + kRowsTile - 1) / kRowsTile * kRowsTile; }

// Joins partial rows: outputs of `tokens` tokens (sequences), each from the ranges of its own segment and, with a prefix, of that.
constexpr int kJoinSegments = 64;
struct JoinSegment {
  int32_t part, splits, rows;            // its partial rows: [split][kv-head][rows]
  int32_t token0;                        // its first token: where lse is
  int32_t prefix_part, prefix_splits, prefix_rows, prefix_row0;   // those of its prefix, and its first row in them; splits 0: none
  int64_t out_base;                      // bytes
};
struct JoinArgs {
  const float4 *part_ml;
  const float *part_o;
  void *out;
  float *lse;
  int64_t out_tok, out_head;             // bytes
  Divisor heads, group;
  int32_t segments, tokens;
  float scale, scale_log2e;
  int32_t first[kJoinSegments];          // first token of a segment, from the launch's first one on; INT32_MAX past the last one
  JoinSegment segment[kJoinSegments];
};

int launch_cross_bf16(int head_dim, const CrossArgs &a, hipStream_t s);
int launch_cross_f16(int head_dim, const CrossArgs &a, hipStream_t s);
int launch_cross_f32(int head_dim, const CrossArgs &a, hipStream_t s);
int launch_shared_bf16(int head_dim, const SharedArgs &a, hipStream_t s);
int launch_shared_f16(int head_dim, const SharedArgs &a, hipStream_t s);
int launch_shared_f32(int head_dim, const SharedArgs &a, hipStream_t s);
int launch_join(int dtype, int head_dim, const JoinArgs &a, hipStream_t s);

struct RotateRows {
  const void *in;
  void *out;
  int64_t in_seq, in_head, in_tok, out_seq, out_head, out_tok;   // bytes
  int32_t heads;                         // 0: none
  int32_t front_only;                    // 1: in place, elements past rotary are where they belong
};
struct RotateArgs {
  RotateRows q, k;
  const int32_t *positions;              // [sequence][token]
  const float *inv_freq;
  int32_t n_tokens, rotary, parts;       // parts: wavefronts that share a token's rows
  int64_t tokens;                        // of all sequences
  float magnitude;
};
int launch_rotate(int dtype, int head_dim, bool interleaved, const RotateArgs &a, hipStream_t s);

}  // namespace ckv
