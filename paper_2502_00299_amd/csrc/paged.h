// Caches in pages: what the kernels of paged_*.hip and their entry points share.
#pragma once
#include <float.h>

#include "internal.h"

namespace ckv {

// Sequences per launch: their tables travel as kernel arguments, which cost the host 0.25 us per KB and launch.
constexpr int kPagedBatch = 64;
constexpr int kPagedMaxTokens = 1 << 24;
constexpr int kPagedMaxGroup = 256;     // query heads per kv-head
constexpr int64_t kPagedStreamBytes = 128 << 20;   // what a call writes is streamed from here on: half of the memory-side cache

// A pool of pages, strides in bytes.  Slots are addressed by blocks of 16: a page is a whole number of them, so a block
// never crosses pages, whatever the page size is.
struct PageGeom {
  int64_t page, head, tok;
  const int32_t *table;                 // [batch_total][pitch]
  int32_t pitch, n_pages;
  uint32_t blocks, magic;               // 16-row blocks of a page; ceil(2^32 / blocks), not used for one
};

// Page of block `blk` of a sequence.  Exact: blk < 2^20 and blocks <= 256, so blk times the magic number's excess stays below 2^32.
__device__ __forceinline__ uint32_t page_of_block(const PageGeom &g, uint32_t blk) {
  return g.blocks == 1 ? blk : __umulhi(blk, g.magic);
}
// Byte offset in a pool of the first row of block `blk` of kv-head h, whose page's table entry is `page`; -1 where that is not there.
__device__ __forceinline__ int64_t block_offset(const PageGeom &g, int32_t page, int h, uint32_t blk) {
  const int64_t at = (int64_t)page * g.page + (int64_t)h * g.head + (int64_t)((blk - page_of_block(g, blk) * g.blocks) * 16) * g.tok;
  return page >= 0 && page < g.n_pages ? at : -1;
}
__device__ __forceinline__ int64_t block_offset(const PageGeom &g, const int32_t *row, int h, uint32_t blk) {
  return block_offset(g, row[page_of_block(g, blk)], h, blk);
}
// The same for one slot.
__device__ __forceinline__ int64_t slot_offset(const PageGeom &g, const int32_t *row, int h, int slot) {
  const int64_t at = block_offset(g, row, h, (uint32_t)slot >> 4);
  return at < 0 ? -1 : at + (int64_t)(slot & 15) * g.tok;
}

// Sequence of entry x of a grid that counts the entries (ranges, tokens) of all sequences of a launch; first[i]: number of
// the first entry of sequence i, INT32_MAX past the last one.  Two levels, so that at most 18 scalars are compared.
#define CKV_PAGED_SEQUENCE(ARGS, x, nb) paged_sequence<offsetof(ARGS, first)>(x, nb)
template <size_t FIRST>
__device__ __forceinline__ int paged_sequence(int x, int nb) {
  int lo = 0;
  if (nb > 16) {
#pragma unroll
    for (int i = 16; i < kPagedBatch; i += 16) lo += x >= kernarg_at<int32_t>(FIRST, i) ? 16 : 0;
  }
  int b = lo;
#pragma unroll
  for (int i = 1; i < 16; ++i) b += x >= kernarg_at<int32_t>(FIRST, lo + i) ? 1 : 0;
  return b;
}

struct PagedAppendArgs {
  PageGeom geom;
  const void *q, *k, *v;
  void *q_out, *k_pages, *v_pages;
  const void *q_norm, *k_norm;
  const float *inv_freq;
  const int32_t *positions, *kv_len;
  int32_t *kv_len_out, *token_pos;
  float *token_weight;
  int64_t q_tok, k_tok, v_tok;          // bytes
  int32_t tokens, token0;               // of the launch; number of its first token
  int32_t batch0, batch, n_q_heads, n_kv_heads, slot_pitch;
  int32_t rotary, interleaved, parts;   // parts: wavefronts that share a token's rows
  int32_t write_len;                    // 1: the last new token of a sequence writes its length
  float eps;
  int32_t first[kPagedBatch + 16], max_tokens[kPagedBatch];
};

struct PagedLenArgs {                   // kv_len_out = min(kv_len + n_new, max_tokens)
  const int32_t *kv_len;
  int32_t *kv_len_out;
  int32_t batch0, batch, n_kv_heads;
  int32_t n_new[kPagedBatch], max_tokens[kPagedBatch];
};

struct PagedCompactArgs {
  PageGeom geom;
  const void *k[kMaxLayersPerLaunch], *v[kMaxLayersPerLaunch];
  void *k_pages[kMaxLayersPerLaunch], *v_pages[kMaxLayersPerLaunch];
  const float *importance[kMaxLayersPerLaunch];   // of the layer's group, or null
  SeqTable seq;
  const int32_t *sel_chunk, *sel_len, *sel_count;
  int32_t *kv_len, *token_pos;
  float *token_weight;
  int64_t kv_stride_head, kv_stride_tok;          // elements
  int64_t imp_pitch;
  int32_t layer0, reuse, batch0, batch_total, n_kv_heads, window, chunk, elem_bytes, sel_cap, slot_pitch, whole_chunks;
  int32_t entries;                                // selection entries of a workgroup
  int32_t stream;                                 // 1: streaming stores
};

struct PagedDecodeArgs {
  PageGeom geom;
  const void *q, *k, *v;
  float *out, *lse, *weight;
  const int32_t *kv_len;
  float2 *part_ml;                      // (reference before the scale, sum) of every range and query head: [range][Hq]
  float *part_o;                        // [range][Hq][d]
  float *scores;                        // products q . k, before the scale: first_row * Hq numbers of the sequences before, then [Hq][rows_b]
  int32_t batch0, batch, n_q_heads, n_kv_heads, group, slot_pitch;
  int32_t heads;                        // query heads of a kv-head that a workgroup serves: 4, 8 or 16
  float scale, scale_log2e;             // between FLT_MIN and what is finite in both units
  int32_t direct;                       // 1: every head is one range, the range kernel writes the outputs
  int32_t alone;                        // its wavefronts if it adds up the weights as well, and no launch follows; 0
  int32_t first[kPagedBatch + 16];      // number of the first key range of every sequence
  int32_t first_row[kPagedBatch];       // rows of the sequences before, each rounded up to 32
  int32_t max_tokens[kPagedBatch];
};
// Reference of a softmax that has seen no slot: below all scores, which are finite.  References are kept and compared before
// the scale, everywhere: scaled, this one is minus infinity from a scale of 0.715 on, and the factor between two that are is no number.
constexpr float kPagedLowest = -FLT_MAX;
constexpr int kPagedMinRange = 128, kPagedMaxRange = 1024;   // rows of a key range
// Rows of a head that a workgroup of so many wavefronts takes as a whole, its scores beside the ring in LDS.
__host__ __device__ constexpr int alone_rows(int waves) { return waves == 8 ? 960 : 512; }
// Rows of every range of a head with n slots that `splits` ranges share.  From the length that the device knows, so that
// all ranges have work when max_tokens is far above it.
__host__ __device__ inline int paged_range_rows(int n, int splits) {
  const int r = ((n + splits - 1) / splits + 31) & ~31;
  return r < kPagedMinRange ? kPagedMinRange : r;
}

// Slots of (sequence, kv-head), as the device knows them.
__device__ __forceinline__ int paged_length(const PagedDecodeArgs &a, int bl, int h) {
  const int most = CKV_ARG(PagedDecodeArgs, max_tokens, bl);
  if (a.kv_len == nullptr) return most;
  const int n = a.kv_len[(int64_t)(a.batch0 + bl) * a.n_kv_heads + h];
  return n < 0 ? 0 : (n > most ? most : n);
}
// One key range of a head: rows r0 .. r0 + len - 1 (len <= 0: none), and this lane's table entry, that of the range's block `lane`.
// The entry is read together with the length, for the range as it is where the head is as long as it can be; only a head whose
// ranges turn out shorter reads it again.
struct PagedRange {
  int r0, len;
  int32_t page;
};
__device__ __forceinline__ PagedRange paged_range(const PagedDecodeArgs &a, int bl, int h, int split, int splits, int lane) {
  const int most = CKV_ARG(PagedDecodeArgs, max_tokens, bl), full = paged_range_rows(most, splits);
  const int32_t *row = a.geom.table + (int64_t)(a.batch0 + bl) * a.geom.pitch;
  auto entry = [&](int first_row, int rows) __attribute__((always_inline)) {
    return 16 * lane < rows && first_row + 16 * lane < most ? row[page_of_block(a.geom, (uint32_t)(first_row / 16 + lane))] : -1;
  };
  PagedRange r;
  r.page = entry(split * full, full);
  int n = most;
  if (a.kv_len != nullptr) {
    n = a.kv_len[(int64_t)(a.batch0 + bl) * a.n_kv_heads + h];
    n = n < 0 ? 0 : (n > most ? most : n);
  }
  const int rps = paged_range_rows(n, splits);
  r.r0 = split * rps;
  r.len = r.r0 + rps < n ? rps : n - r.r0;
  if (rps != full) r.page = entry(r.r0, rps);
  return r;
}
// Number of key ranges that the launch has for a sequence.
__device__ __forceinline__ int paged_splits(int bl) {
  return CKV_ARG(PagedDecodeArgs, first, bl + 1) - CKV_ARG(PagedDecodeArgs, first, bl);
}
__device__ __forceinline__ float *head_scores(const PagedDecodeArgs &a, int bl, int hq) {
  const int64_t rows = (CKV_ARG(PagedDecodeArgs, max_tokens, bl) + 31) & ~31;
  return a.scores + (int64_t)CKV_ARG(PagedDecodeArgs, first_row, bl) * a.n_q_heads + (int64_t)hq * rows;
}
// Natural log of sum_s exp(scale x(s)), M before the scale: rounded once at its own size, and finite where the logits are.
__device__ __forceinline__ float log_sum_exp(const PagedDecodeArgs &a, float M, float L) {
  return L > 0.f ? __builtin_fmaf(M, a.scale, __builtin_log2f(L) * 0.6931471805599453f) : -__builtin_inff();
}
// Element e of the state (M, L, o) that this workgroup's key range leaves of query head hq of sequence b; M before the scale.
template <int HD>
__device__ __forceinline__ void store_range(const PagedDecodeArgs &a, int b, int hq, int e, float M, float L, float o) {
  const int64_t slot = (int64_t)blockIdx.x * a.n_q_heads + hq;
  if (e == 0) a.part_ml[slot] = make_float2(M, L);
  if (a.direct) {
    const int64_t head = (int64_t)b * a.n_q_heads + hq;
    a.out[head * HD + e] = L > 0.f ? o / L : 0.f;
    if (a.lse != nullptr && e == 0) a.lse[head] = log_sum_exp(a, M, L);
  } else {
    a.part_o[slot * HD + e] = o;
  }
}

// What becomes of the scores: nothing, to the workspace for the launch behind, added up as weights by a workgroup that has a whole head.
enum Scores { kDropped, kStored, kAdded };
// A head's softmax weights are 2^(c (x - M)) / L, x before the scale: M and 1 / L are kept apart, as their sum in log2 units loses log2 L
// beside an M of 2^24.
struct HeadNorm {
  float ref, inv;                       // M, 1 / L; 0 if no slot is there
};
// (the reciprocal instruction is off by a step of fp32 at most; a division costs 0.16 us of 13.75 with 16 heads of 13171 slots)
__device__ __forceinline__ HeadNorm head_norm(float M, float L) { return {M, L > 0.f ? __builtin_amdgcn_rcpf(L) : 0.f}; }
// token_weight[s] += sum_i 2^(c (x_i(s) - M_i)) / L_i, heads in order; x: [heads][alone_rows] in LDS.
template <int NW>
__device__ __forceinline__ void add_weights(const PagedDecodeArgs &a, int b, int h, int len, const float *x, const HeadNorm *norm) {
  float *weight = a.weight + ((int64_t)b * a.n_kv_heads + h) * a.slot_pitch;
  for (int r = threadIdx.x; r < len; r += NW * 64) {
    float sum = 0.f;
    for (int j = 0; j < a.group; ++j) sum += __builtin_amdgcn_exp2f((x[j * alone_rows(NW) + r] - norm[j].ref) * a.scale_log2e) * norm[j].inv;
    weight[r] += sum;
  }
}

constexpr int kEvictLdsKeys = 32768;    // slots of a head whose keys are ranked in LDS
struct PagedEvictArgs {
  PageGeom geom;
  void *k_pages[kMaxLayersPerLaunch], *v_pages[kMaxLayersPerLaunch];
  int32_t *kv_len, *token_pos;          // [layer][batch_total][Hkv]..., from the launch's first layer on
  float *token_weight;
  int32_t *lists;                       // [layer][batch_total][Hkv][1 + 2 * pitch]: number of moves, free slots, as many that move into them
  uint32_t *keys;                       // [layer][batch_total][Hkv][key_pitch]: keys of heads that are too long for LDS
  int32_t pitch, key_pitch;
  int32_t apart;                        // 1: the moves are a launch of their own
  int32_t stream;                       // 1: with streaming stores
  int32_t batch0, batch_total, n_kv_heads, slot_pitch, recent;
  int32_t row_shift;                    // log2 of the 16-byte segments of a row
  int32_t budget[kPagedBatch], max_tokens[kPagedBatch];
};

// ---- host side, shared by the entry points
bool fine_scale(float x);
int check_pages(const chunkkv_pages *p, bool slots = true);   // slots: the call has arrays of slots, and their pitch counts
PageGeom geometry(const chunkkv_pages *p, const int32_t *table);
int launch_paged_append(int dtype, int head_dim, const PagedAppendArgs &a, hipStream_t s);
int launch_paged_len(const PagedLenArgs &a, hipStream_t s);
int launch_paged_compact(int row_bytes, const PagedCompactArgs &a, int n_layers, int batch, hipStream_t s);
int launch_paged_decode(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s);
int launch_paged_mfma(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s);   // 16-bit rows
int launch_paged_f32(int head_dim, const PagedDecodeArgs &a, hipStream_t s);
int launch_paged_evict(const PagedEvictArgs &a, int n_layers, int batch, int max_tokens, hipStream_t s);
bool paged_moves_apart(const PagedEvictArgs &a);   // are there moves enough for a launch of their own
int launch_paged_move(const PagedEvictArgs &a, int n_layers, int batch, hipStream_t s);

}  // namespace ckv
