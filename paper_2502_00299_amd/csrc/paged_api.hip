// Host side of the calls over pages: argument checks, workspace plans and launches.
#include <math.h>
#include <string.h>

#include "paged.h"

namespace ckv {

// Finite and not below zero, by its bits: the build lets the compiler assume that nothing is NaN.
bool fine_scale(float x) {
  uint32_t u;
  memcpy(&u, &x, sizeof(u));
  return u < 0x7F800000u || u == 0x80000000u;
}

int check_pages(const chunkkv_pages *p, bool slots) {
  if (!p || !p->max_tokens) return CHUNKKV_ERR_NULL;
  if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->table_pitch < 1 || (slots && p->slot_pitch < 1)) return CHUNKKV_ERR_SHAPE;
  if (p->n_q_heads % p->n_kv_heads != 0) return CHUNKKV_ERR_SHAPE;
  if (!fine_scale(p->softmax_scale)) return CHUNKKV_ERR_SHAPE;
  if (p->dtype != CHUNKKV_F32 && p->dtype != CHUNKKV_BF16 && p->dtype != CHUNKKV_F16) return CHUNKKV_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return CHUNKKV_ERR_UNSUPPORTED;
  if (p->n_q_heads / p->n_kv_heads > kPagedMaxGroup || p->n_kv_heads > 1023) return CHUNKKV_ERR_UNSUPPORTED;   // grids have 65535 rows
  if (p->page_tokens < 16 || p->page_tokens > 4096 || p->page_tokens % 16 != 0) return CHUNKKV_ERR_UNSUPPORTED;
  const int esz = elem_bytes(p->dtype);
  if (p->stride_tok < p->head_dim || p->stride_head < 0 || p->stride_page < 0) return CHUNKKV_ERR_SHAPE;
  if (p->stride_tok > (1 << 22) / esz) return CHUNKKV_ERR_UNSUPPORTED;   // 16 rows are reached by 32-bit offsets
  if ((p->stride_tok * esz) % 16 || (p->stride_head * esz) % 16 || (p->stride_page * esz) % 16) return CHUNKKV_ERR_SHAPE;
  for (int b = 0; b < p->batch; ++b) {
    const int64_t n = p->max_tokens[b];
    if (n < 0) return CHUNKKV_ERR_SHAPE;
    if (n > kPagedMaxTokens) return CHUNKKV_ERR_UNSUPPORTED;
    if ((slots && n > p->slot_pitch) || n > (int64_t)p->table_pitch * p->page_tokens) return CHUNKKV_ERR_SHAPE;
  }
  return CHUNKKV_OK;
}

PageGeom geometry(const chunkkv_pages *p, const int32_t *table) {
  const int64_t esz = elem_bytes(p->dtype);
  PageGeom g;
  g.page = p->stride_page * esz; g.head = p->stride_head * esz; g.tok = p->stride_tok * esz;
  g.table = table; g.pitch = p->table_pitch; g.n_pages = p->n_pages;
  g.blocks = (uint32_t)p->page_tokens / 16;
  g.magic = (uint32_t)((((uint64_t)1 << 32) + g.blocks - 1) / g.blocks);
  return g;
}

namespace {

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// ---- attention: key ranges and workspace -------------------------------------------------------------------------
struct PagedPlan {
  size_t off_ml, off_o, off_scores, total;
};
int range_count(int tokens, int rows) { return tokens > rows ? ceil_div(tokens, rows) : 1; }
// Rows of a key range for the sequences [b0, b0 + nb) of a launch: the fewest (a multiple of 32, 128 at least) that give a whole
// number of workgroups per CU, as few as ranges of up to kPagedMaxRange rows allow.  Few ranges mean few starts, ends and partial
// results, and with one and a half workgroups per CU half of the CUs wait.  us of a call, so and otherwise (bf16, 8 kv-heads of 4
// heads): 13171 slots, 256 workgroups of 416 rows 15.8, 824 of 128 22.0; 30000, 240 of 1024 25.4, 320 of 768 30.2, 472 of 512 25.8;
// 60000, 472 of 1024 43.9, 944 of 512 46.6; fp32, 20000 slots of 8 heads, 216 of 768 30.3, 320 of 512 37.0.
// Without weights to add up, heads whose K rows take up to 128 KB are one range and nothing has to be joined: us in a graph, so and in
// ranges of 128, 8 heads of 300 slots 7.3 / 8.4, of 512 8.1 / 8.5, d = 64 6.5 / 7.5, fp32 of 200 9.6 / 9.8, of 300 10.9 / 9.9.
constexpr int kPagedShortBytes = 128 << 10;
int short_rows(const chunkkv_pages *p) { return kPagedShortBytes / (p->head_dim * elem_bytes(p->dtype)); }
// With weights, heads as short (where they fill half of the CUs, longer ones too) are one workgroup that needs no launch behind it.
// Four wavefronts, of which two workgroups fit a CU, or eight for the longer heads, where they are few.  us in a graph, ranges and a launch
// behind / eight / four: 8 heads of 128 slots 9.5 / 6.8 / 6.3, of 256 9.5 / 7.7 / 7.3, of 300 9.7 / 8.4 / 8.9, of 512 9.6 / 9.2 / 9.6, of 800 9.8 / 11.6 / -;
// 64 of 300 10.5 / 9.2 / 9.1, of 512 11.2 / 11.3 / 10.6; 128 of 900 18.0 / 16.9 / -; 256 of 300 14.8 / 11.2 / 10.9, of 960 28.8 / 23.8 / -; 512 of 40
// 12.6 / 13.3 / 8.2, of 500 30.7 / 28.3 / 24.4, of 900 49.2 / 45.4 / -; fp32, 8 of 200 11.2 / 10.5 / 10.9, of 300 11.3 / 11.6 / 12.7, 512 of 500 51.6 / 47.3 / 44.2.
constexpr int kPagedAloneHeads = 128, kPagedFourHeads = 64, kPagedFourRows = 256, kCUs = 256;
int paged_alone(const chunkkv_pages *p, int nb, int most, bool weights) {   // -> wavefronts, 0: no
  const int64_t heads = (int64_t)nb * p->n_kv_heads;
  if (!weights || p->n_q_heads / p->n_kv_heads > 8 || most > alone_rows(8) || (heads < kPagedAloneHeads && most > short_rows(p))) return 0;
  return most <= kPagedFourRows || (heads >= kPagedFourHeads && most <= alone_rows(4)) ? 4 : 8;
}
// Query heads of one kv-head that a workgroup serves.  16-bit rows: 4 or 8; 5 to 7 are one padded batch of 8, not two passes over
// K and V: 5 heads of each of 4 kv-heads 131072 slots 47.5 us, in two passes 85.9, 13171 slots 11.6 and 12.2, 848 slots 8.5 and 8.4.  More than
// 8: one batch of 16 from 20 MB of K and V on, where reading them again is what costs; below, more workgroups are faster.  us of 16
// and of 8 at a time: 16 heads of each of 8 kv-heads 60000 slots 46.3 / 84.0, 16 sequences of 3000 40.5 / 67.6, 13171 slots 17.2 / 17.2, 900 slots 10.4 / 9.4; 12 of
// 4 60000 slots 26.7 / 43.2; 9 of one 60000 slots (31 MB) 15.7 / 17.3, 13171 (7 MB) 11.4 / 11.5; 16 of 2 13171 slots (13 MB) 12.7 / 12.2.  fp32: 16.
constexpr int64_t kPagedWideBytes = 20 << 20;
int heads_at_once(const chunkkv_pages *p, int b0, int nb) {
  const int g = p->n_q_heads / p->n_kv_heads;
  if (p->dtype == CHUNKKV_F32) return 16;
  if (g <= 8) return g > 4 ? 8 : 4;
  int64_t rows = 0;
  for (int b = b0; b < b0 + nb; ++b) rows += p->max_tokens[b];
  return 2 * rows * p->n_kv_heads * p->head_dim * elem_bytes(p->dtype) >= kPagedWideBytes ? 16 : 8;
}
int range_rows(const chunkkv_pages *p, int b0, int nb, bool weights) {
  const int g = p->n_q_heads / p->n_kv_heads, G = heads_at_once(p, b0, nb);
  const int64_t per_range = (int64_t)p->n_kv_heads * ((g + G - 1) / G);   // workgroups
  int64_t rows = 0;
  int most = 1;
  for (int b = b0; b < b0 + nb; ++b) {
    rows += p->max_tokens[b];
    most = p->max_tokens[b] > most ? p->max_tokens[b] : most;
  }
  if (paged_alone(p, nb, most, weights) || (!weights && most <= short_rows(p))) return kPagedMaxRange;
  const int64_t round = kCUs, rounds = (rows * per_range + round * kPagedMaxRange - 1) / (round * kPagedMaxRange);
  int lo = kPagedMinRange / 32, hi = kPagedMaxRange / 32;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    int64_t n = 0;
    for (int b = b0; b < b0 + nb; ++b) n += range_count(p->max_tokens[b], 32 * mid);
    if (n * per_range <= rounds * round) hi = mid;
    else lo = mid + 1;
  }
  return 32 * lo;
}

// The launches of a call follow one another on the stream and share the workspace.
void paged_plan(const chunkkv_pages *p, bool weights, PagedPlan *pl) {
  int64_t ranges = 0, rows = 0;
  for (int b0 = 0; b0 < p->batch; b0 += kPagedBatch) {
    const int nb = p->batch - b0 < kPagedBatch ? p->batch - b0 : kPagedBatch, r = range_rows(p, b0, nb, weights);
    int64_t n = 0, m = 0;
    for (int b = b0; b < b0 + nb; ++b) {
      n += range_count(p->max_tokens[b], r);
      m += (p->max_tokens[b] + 31) & ~31;
    }
    ranges = n > ranges ? n : ranges;
    rows = m > rows ? m : rows;
  }
  const size_t places = (size_t)ranges * p->n_q_heads;
  pl->off_ml = 0;
  pl->off_o = align256(places * sizeof(float2));
  pl->off_scores = pl->off_o + align256(places * p->head_dim * sizeof(float));
  pl->total = pl->off_scores + (weights ? align256((size_t)rows * p->n_q_heads * sizeof(float)) : 0);
}

// ---- eviction: room for the lists --------------------------------------------------------------------------------
int check_evict(const chunkkv_pages *p, int32_t n_layers, const int32_t *budget) {
  const int rc = check_pages(p);
  if (rc) return rc;
  if (!budget) return CHUNKKV_ERR_NULL;
  if (n_layers < 1) return CHUNKKV_ERR_SHAPE;
  for (int b = 0; b < p->batch; ++b)
    if (budget[b] < 0) return CHUNKKV_ERR_SHAPE;
  return CHUNKKV_OK;
}
// Most slots that a head of sequence b can move, and that any head can.
int most_moves(const chunkkv_pages *p, const int32_t *budget, int b) {
  const int over = p->max_tokens[b] - budget[b], m = over < budget[b] ? over : budget[b];
  return m > 0 ? m : 0;
}
int list_pitch(const chunkkv_pages *p, const int32_t *budget) {
  int most = 0;
  for (int b = 0; b < p->batch; ++b) most = most_moves(p, budget, b) > most ? most_moves(p, budget, b) : most;
  return most;
}

// Keys per head that the workspace has room for: of the sequences that are too long for LDS and can be over their budget.
int key_pitch(const chunkkv_pages *p, const int32_t *budget) {
  int most = 0;
  for (int b = 0; b < p->batch; ++b)
    if (p->max_tokens[b] > budget[b] && p->max_tokens[b] > most) most = p->max_tokens[b];
  return most > kEvictLdsKeys ? most : 0;
}
struct EvictPlan {
  size_t off_keys, total;
};
EvictPlan evict_plan(const chunkkv_pages *p, int32_t n_layers, const int32_t *budget) {
  const size_t heads = (size_t)n_layers * p->batch * p->n_kv_heads;
  EvictPlan pl;
  pl.off_keys = align256(heads * (2 * (size_t)list_pitch(p, budget) + 1) * sizeof(int32_t));
  pl.total = pl.off_keys + align256(heads * (size_t)key_pitch(p, budget) * sizeof(uint32_t));
  return pl;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

int chunkkv_paged_compact(const chunkkv_problem *prob, const chunkkv_pages *pages, int32_t n_layers, int32_t reuse,
                          const void *const *k, const void *const *v, const int32_t *sel_chunk, const int32_t *sel_len,
                          const int32_t *sel_count, const float *const *token_importance, const int32_t *page_table,
                          void *const *k_pages, void *const *v_pages, int32_t *kv_len, int32_t *token_pos,
                          float *token_weight, void *stream) {
  int rc = check_problem(prob, false);
  if (rc) return rc;
  if ((rc = check_pages(pages))) return rc;
  if (prob->batch != pages->batch || prob->n_q_heads != pages->n_q_heads || prob->n_kv_heads != pages->n_kv_heads || prob->head_dim != pages->head_dim || prob->dtype != pages->dtype)
    return CHUNKKV_ERR_SHAPE;
  for (int b = 0; b < prob->batch; ++b)
    if ((int64_t)prob->n_keep[b] + prob->window > pages->max_tokens[b]) return CHUNKKV_ERR_SHAPE;
  if (n_layers < 1 || reuse < 1) return CHUNKKV_ERR_SHAPE;
  if (!k || !v || !sel_chunk || !sel_len || !sel_count || !page_table || !k_pages || !v_pages || !kv_len) return CHUNKKV_ERR_NULL;
  for (int l = 0; l < n_layers; ++l) {
    if (!k[l] || !v[l] || !k_pages[l] || !v_pages[l]) return CHUNKKV_ERR_NULL;
    if (token_importance && !token_importance[l / reuse]) return CHUNKKV_ERR_NULL;
    if (misaligned(k[l]) || misaligned(v[l]) || misaligned(k_pages[l]) || misaligned(v_pages[l])) return CHUNKKV_ERR_SHAPE;
  }
  hipStream_t s = (hipStream_t)stream;
  int64_t kept = 0;
  for (int b = 0; b < prob->batch; ++b) kept += prob->n_keep[b] + prob->window;
  const int64_t written = 2 * kept * n_layers * prob->n_kv_heads * prob->head_dim * elem_bytes(prob->dtype);
  for (int l0 = 0; l0 < n_layers; l0 += kMaxLayersPerLaunch) {
    const int nl = n_layers - l0 < kMaxLayersPerLaunch ? n_layers - l0 : kMaxLayersPerLaunch;
    for (int b0 = 0; b0 < prob->batch; b0 += kMaxBatchPerLaunch) {
      const int nb = prob->batch - b0 < kMaxBatchPerLaunch ? prob->batch - b0 : kMaxBatchPerLaunch;
      PagedCompactArgs a;
      memset(&a, 0, sizeof(a));
      a.geom = geometry(pages, page_table);
      for (int i = 0; i < nl; ++i) {
        a.k[i] = k[l0 + i]; a.v[i] = v[l0 + i]; a.k_pages[i] = k_pages[l0 + i]; a.v_pages[i] = v_pages[l0 + i];
        a.importance[i] = token_importance ? token_importance[(l0 + i) / reuse] : nullptr;
      }
      for (int i = 0; i < nb; ++i) {
        a.seq.seqlen[i] = prob->seqlen[b0 + i];
        a.seq.n_keep[i] = prob->n_keep[b0 + i];
        a.seq.kv_base[i] = prob->kv_base[b0 + i];
      }
      a.sel_chunk = sel_chunk; a.sel_len = sel_len; a.sel_count = sel_count; a.sel_cap = prob->sel_cap;
      const int64_t heads0 = (int64_t)l0 * prob->batch * prob->n_kv_heads;
      a.kv_len = kv_len + heads0;
      a.token_pos = token_pos ? token_pos + heads0 * pages->slot_pitch : nullptr;
      a.token_weight = token_weight ? token_weight + heads0 * pages->slot_pitch : nullptr;
      a.kv_stride_head = prob->kv_stride_head; a.kv_stride_tok = prob->kv_stride_tok;
      a.imp_pitch = (int64_t)prob->score_cap * prob->chunk;
      a.layer0 = l0; a.reuse = reuse; a.batch0 = b0; a.batch_total = prob->batch; a.n_kv_heads = prob->n_kv_heads;
      // rows that span less than 2 GiB are fewer than 2^24: larger chunks are one, and sums with their size would pass 32 bits
      a.window = prob->window; a.chunk = prob->chunk < kPagedMaxTokens ? prob->chunk : kPagedMaxTokens; a.elem_bytes = elem_bytes(prob->dtype); a.slot_pitch = pages->slot_pitch;
      a.whole_chunks = (prob->flags & CHUNKKV_FLAG_WHOLE_CHUNKS) ? 1 : 0;
      a.stream = written > kPagedStreamBytes;
      Timed t(kCompact, s);
      if ((rc = launch_paged_compact(prob->head_dim * elem_bytes(prob->dtype), a, nl, nb, s))) return rc;
    }
  }
  return CHUNKKV_OK;
}

int chunkkv_paged_append(const chunkkv_pages *pages, const int32_t *n_new, const void *q, int64_t q_stride_tok,
                         const void *k, int64_t k_stride_tok, const void *v, int64_t v_stride_tok,
                         const int32_t *positions, const void *q_norm, const void *k_norm, float eps,
                         const float *inv_freq, int32_t rotary_dim, int32_t interleaved, void *q_out,
                         const int32_t *page_table, void *k_pages, void *v_pages, const int32_t *kv_len,
                         int32_t *kv_len_out, int32_t *token_pos, float *token_weight, void *stream) {
  int rc = check_pages(pages);
  if (rc) return rc;
  if (!n_new || !page_table || !k_pages || !v_pages || !kv_len || !kv_len_out || (rotary_dim > 0 && !inv_freq)) return CHUNKKV_ERR_NULL;
  int64_t total = 0;
  bool none = false, many = false;
  for (int b = 0; b < pages->batch; ++b) {
    if (n_new[b] < 0) return CHUNKKV_ERR_SHAPE;
    total += n_new[b];
    none |= n_new[b] == 0;
    many |= n_new[b] > 1;
  }
  if (total > 0) {   // arrays of no tokens may be anything
    if (!k || !v || !positions || (q != nullptr) != (q_out != nullptr) || (q_norm && !q)) return CHUNKKV_ERR_NULL;
  }
  if (rotary_dim < 0 || rotary_dim > pages->head_dim || (inv_freq && rotary_dim == 0) || !fine_scale(eps)) return CHUNKKV_ERR_SHAPE;
  if (rotary_dim % 16 != 0) return CHUNKKV_ERR_UNSUPPORTED;
  const int esz = elem_bytes(pages->dtype), d = pages->head_dim;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(q_norm) || misaligned(k_norm) || misaligned(q_out) || misaligned(k_pages) || misaligned(v_pages))
    return CHUNKKV_ERR_SHAPE;
  if ((total > 0) && ((q && q_stride_tok < (int64_t)pages->n_q_heads * d) || k_stride_tok < (int64_t)pages->n_kv_heads * d || v_stride_tok < (int64_t)pages->n_kv_heads * d)) return CHUNKKV_ERR_SHAPE;
  if ((q && (q_stride_tok * esz) % 16) || (k_stride_tok * esz) % 16 || (v_stride_tok * esz) % 16) return CHUNKKV_ERR_SHAPE;
  if (total > kPagedMaxTokens) return CHUNKKV_ERR_UNSUPPORTED;
  // Who writes the lengths: the append kernel where every sequence has a token in it and nobody reads a length that it
  // has written (one token each), or they go to another array; otherwise a kernel of their own.
  const bool in_place = kv_len_out == kv_len;
  const bool with_tokens = in_place ? !many : !none;
  hipStream_t s = (hipStream_t)stream;
  int64_t token0 = 0;
  for (int b0 = 0; b0 < pages->batch; b0 += kPagedBatch) {
    const int nb = pages->batch - b0 < kPagedBatch ? pages->batch - b0 : kPagedBatch;
    PagedAppendArgs a;
    memset(&a, 0, sizeof(a));
    a.geom = geometry(pages, page_table);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_pages = k_pages; a.v_pages = v_pages;
    a.q_norm = q_norm; a.k_norm = k_norm; a.eps = eps; a.inv_freq = inv_freq; a.rotary = rotary_dim; a.interleaved = interleaved != 0;
    a.positions = positions; a.kv_len = kv_len; a.kv_len_out = kv_len_out; a.token_pos = token_pos; a.token_weight = token_weight;
    a.q_tok = q_stride_tok * esz; a.k_tok = k_stride_tok * esz; a.v_tok = v_stride_tok * esz;
    a.token0 = (int32_t)token0; a.batch0 = b0; a.batch = nb; a.n_q_heads = pages->n_q_heads; a.n_kv_heads = pages->n_kv_heads;
    a.slot_pitch = pages->slot_pitch; a.write_len = with_tokens;
    for (int i = 0; i < kPagedBatch + 16; ++i) a.first[i] = INT32_MAX;
    for (int i = 0; i < nb; ++i) {
      a.first[i] = a.tokens;
      a.max_tokens[i] = pages->max_tokens[b0 + i];
      a.tokens += n_new[b0 + i];
    }
    if (a.tokens > 0) {
      Timed t(kCompact, s);
      if ((rc = launch_paged_append(pages->dtype, d, a, s))) return rc;
    }
    token0 += a.tokens;
    if (with_tokens) continue;
    PagedLenArgs f;
    f.kv_len = kv_len; f.kv_len_out = kv_len_out; f.batch0 = b0; f.batch = nb; f.n_kv_heads = pages->n_kv_heads;
    for (int i = 0; i < nb; ++i) { f.n_new[i] = n_new[b0 + i]; f.max_tokens[i] = pages->max_tokens[b0 + i]; }
    Timed t(kCompact, s);
    if ((rc = launch_paged_len(f, s))) return rc;
  }
  return CHUNKKV_OK;
}

size_t chunkkv_paged_decode_workspace_bytes(const chunkkv_pages *pages, int32_t with_weights) {
  if (check_pages(pages)) return 0;
  PagedPlan pl;
  paged_plan(pages, with_weights != 0, &pl);
  return pl.total;
}

int chunkkv_paged_decode_attention(const chunkkv_pages *pages, const int32_t *page_table, const int32_t *kv_len,
                                   const void *q, const void *k_pages, const void *v_pages, float *out, float *lse,
                                   float *token_weight, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_pages(pages);
  if (rc) return rc;
  if (!page_table || !q || !k_pages || !v_pages || !out) return CHUNKKV_ERR_NULL;
  if (misaligned(q) || misaligned(k_pages) || misaligned(v_pages)) return CHUNKKV_ERR_SHAPE;
  PagedPlan pl;
  paged_plan(pages, token_weight != nullptr, &pl);
  if (!workspace || workspace_bytes < pl.total || misaligned(workspace)) return CHUNKKV_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const float scale = pages->softmax_scale > 0.f ? pages->softmax_scale : 1.0f / sqrtf((float)pages->head_dim);
  for (int b0 = 0; b0 < pages->batch; b0 += kPagedBatch) {
    const int nb = pages->batch - b0 < kPagedBatch ? pages->batch - b0 : kPagedBatch;
    PagedDecodeArgs a;
    memset(&a, 0, sizeof(a));
    a.geom = geometry(pages, page_table);
    a.q = q; a.k = k_pages; a.v = v_pages; a.out = out; a.lse = lse; a.weight = token_weight; a.kv_len = kv_len;
    a.part_ml = (float2 *)((char *)workspace + pl.off_ml);
    a.part_o = (float *)((char *)workspace + pl.off_o);
    a.scores = (float *)((char *)workspace + pl.off_scores);
    a.batch0 = b0; a.batch = nb; a.n_q_heads = pages->n_q_heads; a.n_kv_heads = pages->n_kv_heads;
    a.group = pages->n_q_heads / pages->n_kv_heads; a.slot_pitch = pages->slot_pitch; a.heads = heads_at_once(pages, b0, nb);
    // A scale that vanishes in fp32 gives all slots the same weight; kept above zero, which minus infinity cannot be multiplied by.  One
    // that is finite and not so times log2 e tells apart what any as large does: the largest scores have all the weight.
    a.scale = scale > FLT_MIN ? scale : FLT_MIN;
    a.scale_log2e = a.scale < FLT_MAX / 1.4426952f ? a.scale * 1.4426950408889634f : FLT_MAX;
    const int r = range_rows(pages, b0, nb, token_weight != nullptr);
    for (int i = 0; i < kPagedBatch + 16; ++i) a.first[i] = INT32_MAX;
    int ranges = 0, rows = 0;
    a.direct = 1;
    for (int i = 0; i < nb; ++i) {
      const int n = pages->max_tokens[b0 + i], c = range_count(n, r);
      a.first[i] = ranges; a.first_row[i] = rows; a.max_tokens[i] = n;
      ranges += c;
      rows += (n + 31) & ~31;
      if (c > 1) a.direct = 0;
    }
    a.first[nb] = ranges;
    int most = 1;
    for (int i = 0; i < nb; ++i) most = a.max_tokens[i] > most ? a.max_tokens[i] : most;
    a.alone = paged_alone(pages, nb, most, token_weight != nullptr);
    Timed t(kDecode, s);
    if ((rc = launch_paged_decode(pages->dtype, pages->head_dim, a, s))) return rc;
  }
  return CHUNKKV_OK;
}

size_t chunkkv_paged_evict_workspace_bytes(const chunkkv_pages *pages, int32_t n_layers, const int32_t *budget) {
  if (check_evict(pages, n_layers, budget)) return 0;
  return evict_plan(pages, n_layers, budget).total;
}

int chunkkv_paged_evict(const chunkkv_pages *pages, int32_t n_layers, const int32_t *budget, int32_t recent,
                        const int32_t *page_table, void *const *k_pages, void *const *v_pages, int32_t *kv_len,
                        int32_t *token_pos, float *token_weight, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_evict(pages, n_layers, budget);
  if (rc) return rc;
  if (recent < 0) return CHUNKKV_ERR_SHAPE;
  for (int b = 0; b < pages->batch; ++b)
    if (recent > budget[b]) return CHUNKKV_ERR_SHAPE;
  if (!page_table || !k_pages || !v_pages || !kv_len || !token_pos || !token_weight) return CHUNKKV_ERR_NULL;
  for (int l = 0; l < n_layers; ++l) {
    if (!k_pages[l] || !v_pages[l]) return CHUNKKV_ERR_NULL;
    if (misaligned(k_pages[l]) || misaligned(v_pages[l])) return CHUNKKV_ERR_SHAPE;
  }
  const EvictPlan pl = evict_plan(pages, n_layers, budget);
  if (!workspace || workspace_bytes < pl.total || misaligned(workspace)) return CHUNKKV_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const int pitch = list_pitch(pages, budget);
  int64_t movable = 0;   // slots, at most
  for (int b = 0; b < pages->batch; ++b) movable += most_moves(pages, budget, b);
  const int64_t written = 2 * movable * n_layers * pages->n_kv_heads * pages->head_dim * elem_bytes(pages->dtype);
  for (int l0 = 0; l0 < n_layers; l0 += kMaxLayersPerLaunch) {
    const int nl = n_layers - l0 < kMaxLayersPerLaunch ? n_layers - l0 : kMaxLayersPerLaunch;
    const int64_t heads0 = (int64_t)l0 * pages->batch * pages->n_kv_heads;
    for (int b0 = 0; b0 < pages->batch; b0 += kPagedBatch) {
      const int nb = pages->batch - b0 < kPagedBatch ? pages->batch - b0 : kPagedBatch;
      PagedEvictArgs a;
      memset(&a, 0, sizeof(a));
      a.geom = geometry(pages, page_table);
      for (int i = 0; i < nl; ++i) { a.k_pages[i] = k_pages[l0 + i]; a.v_pages[i] = v_pages[l0 + i]; }
      a.kv_len = kv_len + heads0;
      a.token_pos = token_pos + heads0 * pages->slot_pitch;
      a.token_weight = token_weight + heads0 * pages->slot_pitch;
      a.lists = (int32_t *)workspace + heads0 * (2 * (int64_t)pitch + 1);
      a.key_pitch = key_pitch(pages, budget);
      a.keys = (uint32_t *)((char *)workspace + pl.off_keys) + heads0 * a.key_pitch;
      a.pitch = pitch; a.batch0 = b0; a.batch_total = pages->batch; a.n_kv_heads = pages->n_kv_heads; a.slot_pitch = pages->slot_pitch;
      a.recent = recent; a.row_shift = 31 - __builtin_clz(pages->head_dim * elem_bytes(pages->dtype) / 16);
      a.stream = written > kPagedStreamBytes;
      int most = 0;
      for (int i = 0; i < nb; ++i) {
        const int n = pages->max_tokens[b0 + i];
        a.budget[i] = budget[b0 + i]; a.max_tokens[i] = n;
        if (n > budget[b0 + i] && n > most) most = n;
      }
      if (most == 0) continue;   // nobody can be over the budget
      { Timed t(kTopk, s); rc = launch_paged_evict(a, nl, nb, most, s); }
      if (rc) return rc;
      if (paged_moves_apart(a)) { Timed t(kCompact, s); rc = launch_paged_move(a, nl, nb, s); }
      if (rc) return rc;
    }
  }
  return CHUNKKV_OK;
}

}  // extern "C"
