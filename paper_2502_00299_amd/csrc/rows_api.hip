// Host side of the calls for caches that many queries read: argument checks, workspace plans and launches.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <memory>
#include <new>

#include "rows.h"

namespace ckv {
namespace {

constexpr int64_t kMostElements = (int64_t)1 << 56;   // strides and bases: what no memory has
constexpr int kMaxQueryRows = 1 << 30;   // of a sequence (or prefix) and kv-head
constexpr int kLaunchPrefixes = kSharedSegments - kJoinSegments;   // prefixes of a launch: the others of its segments are sequences
constexpr int kRotateMaxHeads = 1 << 16;
// Of a launch: a grid has less than 2^32 threads, 512 of a workgroup here, and up to 32 of a row of the join.
constexpr int64_t kMostBlocks = ((int64_t)1 << 23) - 1, kMostPartials = ((int64_t)1 << 27) - 1;

// Do rows of d elements that are written overlap?  Axes by stride, each behind all of the ones before; bounds checked before: no product overflows.
struct Axis {
  int64_t stride, n;
};
template <int N>
bool overlap(Axis (&axis)[N], int64_t d) {
  std::sort(axis, axis + N, [](const Axis &x, const Axis &y) { return x.stride < y.stride; });
  __int128 end = d;
  for (const Axis &x : axis) {
    if (x.n <= 1) continue;
    if (x.stride < end) return true;
    end += (__int128)x.stride * (x.n - 1);
  }
  return false;
}

// Rows of two axes at bases of their own, one lattice for each of n sequences: count[0] rows on the small axis, count[1] on the large one, both 0 or
// neither.  overlap() has passed for the largest counts, so a lattice's rows do not overlap each other; do those of two?
struct Lattice {
  int64_t base, count[2];
};
struct Lattices {
  int64_t small, large, d;               // strides; elements of a row

  // Ends of x: of its rows on the small axis, of all.
  __int128 end(const Lattice &x, bool all) const { return (__int128)x.base + (x.count[0] - 1) * (__int128)small + (all ? (x.count[1] - 1) * (__int128)large : 0) + d; }
  // Is there a pair of rows less than d apart?  Steps i of the large axis and j of the small one lie between a row of x and one of y: only few i leave
  // the rest within reach of the small axis, and of the j the two nearest to it.
  bool meet(const Lattice &x, const Lattice &y) const {
    const __int128 apart = (__int128)y.base - x.base;     // apart + i large + j small = 0, nearly
    const int64_t j0 = -(x.count[0] - 1), j1 = y.count[0] - 1, i0 = -(x.count[1] - 1), i1 = y.count[1] - 1;
    auto floor_div = [](__int128 a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
    auto near = [&](__int128 rest) {                      // some j: |rest + j small| < d
      __int128 j = small > 0 ? floor_div(-rest, small) : 0;
      for (int e = 0; e < 2; ++e, ++j) {
        const __int128 k = j < j0 ? j0 : (j > j1 ? j1 : j), gap = rest + k * small;
        if (gap < d && gap > -d) return true;
      }
      return false;
    };
    if (large == 0) return near(apart);
    // -apart - j small within d of i large, for j in [j0, j1]
    __int128 lo = floor_div(-apart - j1 * (__int128)small - d, large), hi = floor_div(-apart - j0 * (__int128)small + d, large) + 1;
    lo = lo < i0 ? i0 : lo;
    hi = hi > i1 ? i1 : hi;
    for (__int128 i = lo; i <= hi; ++i)
      if (near(apart + i * large)) return true;
    return false;
  }
};
// One behind the other in the order of nth, as they mostly are: each whole, or (sequences between the rows of one another's large axis) within one step of it.
template <typename F>
bool lattices_in_line(int n, F &&nth, const Lattices &l) {
  __int128 whole = 0, step = 0;
  int64_t lowest = -1;
  bool apart = true, beside = true;
  for (int i = 0; i < n && (apart || beside); ++i) {
    const Lattice x = nth(i);
    if (x.count[0] == 0) continue;
    apart &= x.base >= whole;
    beside &= x.base >= step;
    whole = l.end(x, true);
    step = l.end(x, false);
    if (lowest < 0) lowest = x.base;
  }
  return apart || (beside && step - lowest <= l.large);
}
template <typename F>
bool lattices_meet(int n, F &&nth, const Lattices &l) {
  if (lattices_in_line(n, nth, l)) return false;
  const std::unique_ptr<int32_t[]> order(new (std::nothrow) int32_t[n]);   // by base; without memory every pair is looked at
  auto sorted = [&](int i) { return nth(order ? order[i] : i); };
  if (order) {
    for (int i = 0; i < n; ++i) order[i] = i;
    std::sort(order.get(), order.get() + n, [&](int x, int y) { return nth(x).base < nth(y).base; });
    if (lattices_in_line(n, sorted, l)) return false;
  }
  for (int i = 0; i < n; ++i) {
    const Lattice x = sorted(i);
    for (int j = i + 1; x.count[0] > 0 && j < n; ++j) {
      const Lattice y = sorted(j);
      if (order && l.end(x, true) <= y.base) break;
      if (y.count[0] > 0 && l.meet(x, y)) return true;
    }
  }
  return false;
}

// ---- key ranges ---------------------------------------------------------------------------------------------------
// Segments of a call, as the plan sees them.
struct Shape {
  int rows, most;
};
constexpr int kKeptPlans = 16;   // of a call's first launches, between its size and its launches; those of later ones are made again
struct RowsPlan {
  int tile, pairs;       // rows of a wide workgroup, kRowsNarrow: there is none; narrow tiles of a workgroup
  int range[2];          // keys of a range of a wide segment, of a narrow one; a multiple of kRowsTile
};
int ranges_of(const Shape &x, const RowsPlan &pl) {
  const int range = pl.range[x.rows <= kRowsNarrow];
  return x.rows == 0 ? 0 : (x.most > range ? (x.most + range - 1) / range : 1);
}
int tiles_of(const Shape &x, const RowsPlan &pl) { return x.rows <= kRowsNarrow ? 1 : (x.rows + pl.tile - 1) / pl.tile; }
int64_t blocks_of(const Shape &x, const RowsPlan &pl, int n_kv_heads) {
  const int64_t n = (int64_t)ranges_of(x, pl) * n_kv_heads;
  return x.rows <= kRowsNarrow ? (n + pl.pairs - 1) / pl.pairs : n * tiles_of(x, pl);
}

// Narrow segments alone: ranges that are a workgroup for each CU together, kLeastRange at least; a segment of up to kShortKeys has no launch
// behind it where it need not.  Fewer and longer ones leave CUs idle, more of them cost more starts and partial rows.  Eight tokens of 32 heads on
// 8 over 13171 keys, bf16, d = 128: 16.4 us with ranges of 512, 18.4 with 256, 24.9 with 128; eight sequences of one token over 16384 keys each:
// 95.5 with 4096, 98.5 with 1024, 107.6 with 8192; eight of up to 64 keys behind 848: 12.6 with 128, 14.9 with 1024.  One token over 512 (768)
// keys in one launch, d = 128: 8.8 (10.7) us, in two 10.8 (10.7); d = 64: 7.7 (8.9) and 10.8 (10.6).
//
// Otherwise the ranges and the tile whose last workgroup ends first, by an estimate in microseconds: a workgroup costs kStart, kRow for each of
// its rows where ranges are joined (written and read again), and its keys, by type and kind.  The launch ends when the longest workgroups have
// gone through in rounds, when all CUs have done their share, or when all keys have come from memory, whichever is last.  61 tokens of 32 heads
// on 8 over 13171 keys, bf16, d = 128: 33 to 35 us as estimated (128 rows, ranges of 832), 36.7 with 256 rows and ranges of 448, 42.3 with 256 and
// 832, 44.2 with 128 and 640; 64 sequences behind 131072 keys: 194 (256 rows, 4096), 200 (128, 8192), 230 (256, 8192).  Other sizes that were
// swept lie within 4 % of their best.
//
// A plan is that of one launch: a call's launches run one behind the other.  128 sequences of one token, one kv-head and 16384 keys, bf16, d = 128: 365 us
// with ranges for the sum of all, 202 so; 64 prefixes of 8192 slots with 16 sequences of 32 heads on 8 each 937 and 650; 300 sequences behind 5000
// slots 122 and 127 (143 without `of_many`, which tries ranges for the wide segments alone too).
constexpr int kLeastRange = 128, kShortKeys = 768, kCUs = 256;
constexpr float kStart = 5.f, kJoin = 3.5f, kRow = 0.05f, kBytes = 5.5e6f;
constexpr float kKey[2][2][3] = {   // [fp32][d = 128][256 rows, 128, narrow]
    {{0.020f, 0.012f, 0.008f}, {0.030f, 0.018f, 0.016f}}, {{0.13f, 0.066f, 0.018f}, {0.25f, 0.13f, 0.034f}}};
int whole_tiles(float keys) { return keys < (float)kPagedMaxTokens ? ((int)keys + kRowsTile - 1) / kRowsTile * kRowsTile : kPagedMaxTokens; }
template <typename F>
RowsPlan plan_rows(int n, F &&shape, int n_kv_heads, int dtype, int head_dim, bool always_joined, bool of_many) {
  float keys = 0.f, wide_keys[2] = {0.f, 0.f};   // of all segments; of wide ones times their workgroups, 256 rows and 128
  int most = 1, rows_most = 0;
  for (int i = 0; i < n; ++i) {
    const Shape x = shape(i);
    if (x.rows == 0) continue;
    most = x.most > most ? x.most : most;
    rows_most = x.rows > rows_most ? x.rows : rows_most;
    keys += (float)x.most;
    if (x.rows > kRowsNarrow)
      for (int k = 0; k < 2; ++k) wide_keys[k] += (float)x.most * (float)((x.rows + (256 >> k) - 1) / (256 >> k));
  }
  const int whole = (most + kRowsTile - 1) / kRowsTile * kRowsTile, pairs = rows_pairs(dtype, head_dim);
  RowsPlan best = {kRowsNarrow, 1, {whole, whole}};
  if (rows_most <= kRowsNarrow) {
    if (!always_joined && most <= kShortKeys) return best;
    int range = whole_tiles(keys * n_kv_heads / kCUs);
    for (int again = 0; again < 2; ++again) {   // ends of segments are workgroups too
      if (range < kLeastRange) range = kLeastRange;
      int64_t blocks = 0, segments = 0;
      best.range[1] = range;
      for (int i = 0; i < n; ++i) {
        blocks += ranges_of(shape(i), best);
        segments += shape(i).rows > 0;
      }
      blocks *= n_kv_heads;
      segments *= n_kv_heads;
      if (blocks <= kCUs || 2 * segments > kCUs) break;
      range = whole_tiles((float)range * (float)(blocks - segments) / (float)(kCUs - segments));
    }
    return best;
  }
  float least = FLT_MAX;
  const float memory = 2.f * keys * n_kv_heads * head_dim * elem_bytes(dtype) / kBytes + kStart;
  const float *rate = kKey[dtype == CHUNKKV_F32][head_dim == 128];
  for (int k = 0; k < 2; ++k) {
    const float tile = 1.f / (float)(kRowsWide << (1 - k));
    // tries ranges of so many keys; -> workgroups, of all segments or of the wide ones
    auto attempt = [&](int range, bool all = true) {
      RowsPlan pl = {kRowsWide << (1 - k), pairs, {range, whole_tiles((float)range * rate[k] / rate[2])}};
      const float per[2] = {1.f / (float)pl.range[0], 1.f / (float)pl.range[1]};
      float total = 0.f, blocks = 0.f, wide = 0.f, full = 0.f, longest[2] = {0.f, 0.f};
      bool joined = always_joined;
      for (int i = 0; i < n; ++i) {
        const Shape x = shape(i);
        if (x.rows == 0) continue;
        const bool narrow = x.rows <= kRowsNarrow, cut = x.most > pl.range[narrow];
        const int rows = x.rows < pl.tile ? x.rows : pl.tile;
        const float count = (cut ? ceilf((float)x.most * per[narrow]) : 1.f) * (narrow ? 1.f / (float)pairs : ceilf((float)x.rows * tile));
        const float cost = (float)(cut ? pl.range[narrow] : x.most) * rate[narrow ? 2 : k] + kStart + (cut ? (float)rows * kRow : 0.f);
        total += count * cost;
        blocks += count;
        wide += narrow ? 0.f : count;
        longest[narrow] = cost > longest[narrow] ? cost : longest[narrow];
        full += !narrow && 2 * x.most > pl.range[0] ? count : 0.f;
        joined |= cut;
      }
      blocks *= (float)n_kv_heads;
      const float rounds = ceilf(full * (float)n_kv_heads / kCUs), even = total * (float)n_kv_heads / kCUs;
      float end = rounds * longest[0] + (blocks > rounds * kCUs ? longest[1] : 0.f);   // narrow ones behind the wide
      end = end > even ? end : even;
      end = (end > memory ? end : memory) + (joined ? kJoin : 0.f);
      if (end < least) {
        least = end;
        best = pl;
      }
      return all ? blocks : wide * (float)n_kv_heads;
    };
    attempt(whole);
    // half a workgroup to a CU, one, two or three; the last for segments of unlike length (three of 41 to 418 fp32 tokens: 227 us, 266 without)
    for (int share : {kCUs / 2, kCUs, 2 * kCUs, 3 * kCUs}) {
      int range = whole_tiles(wide_keys[k] * n_kv_heads / (float)share);
      for (int again = 0; again < 3 && range < whole; ++again) {
        if (range < kLeastRange) range = kLeastRange;
        const float blocks = attempt(range);
        if (blocks <= (float)share) break;
        range = whole_tiles((float)range * blocks / (float)share);   // ends of segments are more workgroups than that
      }
    }
    // a launch of a call that has others: so many workgroups of its wide segments, beside which narrow ones may be most of the launch
    for (int share : {kCUs / 2, kCUs, 2 * kCUs}) {
      int range = whole_tiles(wide_keys[k] * n_kv_heads / (float)share);
      for (int again = 0; of_many && again < 3 && range < whole; ++again) {
        if (range < kLeastRange) range = kLeastRange;
        const float blocks = attempt(range, false);
        if (blocks <= (float)share) break;
        range = whole_tiles((float)range * blocks / (float)share);
      }
    }
  }
  return best;
}

void set_scale(float given, int head_dim, float *scale, float *scale_log2e) {   // as chunkkv_paged_decode_attention has them
  const float x = given > 0.f ? given : 1.0f / sqrtf((float)head_dim);
  *scale = x > FLT_MIN ? x : FLT_MIN;
  *scale_log2e = *scale < FLT_MAX / 1.4426952f ? *scale * 1.4426950408889634f : FLT_MAX;
}

size_t partial_bytes(int64_t rows, int head_dim, size_t *off_o) {
  *off_o = align256((size_t)rows * sizeof(float4));
  return *off_o + align256((size_t)rows * head_dim * sizeof(float));
}

// ---- cross attention ------------------------------------------------------------------------------------------------
int check_cross(const chunkkv_cross *c) {
  if (!c || !c->q_len || !c->seqlen || !c->q_base || !c->kv_base || !c->out_base) return CHUNKKV_ERR_NULL;
  if (c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads != 0 || !fine_scale(c->softmax_scale) || c->mask_pitch < 0) return CHUNKKV_ERR_SHAPE;
  if (c->dtype != CHUNKKV_F32 && c->dtype != CHUNKKV_BF16 && c->dtype != CHUNKKV_F16) return CHUNKKV_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return CHUNKKV_ERR_UNSUPPORTED;
  const int g = c->n_q_heads / c->n_kv_heads, esz = elem_bytes(c->dtype);
  if (g > kPagedMaxGroup || c->n_kv_heads > 1023) return CHUNKKV_ERR_UNSUPPORTED;
  if (c->kv_stride_tok < c->head_dim || c->kv_stride_head < 0 || c->q_stride_head < 0 || c->q_stride_tok < 0 || c->out_stride_head < 0 || c->out_stride_tok < 0) return CHUNKKV_ERR_SHAPE;
  if (c->kv_stride_tok > (1 << 22) / esz) return CHUNKKV_ERR_UNSUPPORTED;   // 16 rows are reached by 32-bit offsets
  const int64_t strides[] = {c->kv_stride_tok, c->kv_stride_head, c->q_stride_tok, c->q_stride_head, c->out_stride_tok, c->out_stride_head};
  for (int64_t x : strides) {
    if (x > kMostElements) return CHUNKKV_ERR_UNSUPPORTED;
    if ((x * esz) % 16) return CHUNKKV_ERR_SHAPE;
  }
  int64_t tokens = 0, most = 0;
  for (int b = 0; b < c->batch; ++b) {
    if (c->q_len[b] < 0 || c->seqlen[b] < 0 || c->q_base[b] < 0 || c->kv_base[b] < 0 || c->out_base[b] < 0) return CHUNKKV_ERR_SHAPE;
    if (c->q_base[b] > kMostElements || c->kv_base[b] > kMostElements || c->out_base[b] > kMostElements) return CHUNKKV_ERR_UNSUPPORTED;
    if ((c->q_base[b] * esz) % 16 || (c->kv_base[b] * esz) % 16 || (c->out_base[b] * esz) % 16) return CHUNKKV_ERR_SHAPE;
    if (c->seqlen[b] > kPagedMaxTokens || (int64_t)c->q_len[b] * g > kMaxQueryRows) return CHUNKKV_ERR_UNSUPPORTED;
    tokens += c->q_len[b];
    most = c->q_len[b] > most ? c->q_len[b] : most;
  }
  if (tokens > kMaxQueryRows) return CHUNKKV_ERR_UNSUPPORTED;
  Axis axis[2] = {{c->out_stride_head, c->n_q_heads}, {c->out_stride_tok, most}};
  return most > 0 && overlap(axis, c->head_dim) ? CHUNKKV_ERR_SHAPE : CHUNKKV_OK;
}

// Outputs of two sequences in one place: whichever workgroup came last would have written them.
bool cross_outputs_meet(const chunkkv_cross *c) {
  int64_t most = 0;
  for (int b = 0; b < c->batch; ++b) most = c->q_len[b] > most ? c->q_len[b] : most;
  const bool heads_small = most <= 1 || (c->n_q_heads > 1 && c->out_stride_head < c->out_stride_tok);
  // the stride of an axis of one entry can be anything
  const int64_t head = c->n_q_heads > 1 ? c->out_stride_head : 0, tok = most > 1 ? c->out_stride_tok : 0;
  const Lattices l = {heads_small ? head : tok, heads_small ? tok : head, c->head_dim};
  return lattices_meet(c->batch, [&](int b) {
    const int64_t n = c->q_len[b], heads = n > 0 ? c->n_q_heads : 0;
    return heads_small ? Lattice{c->out_base[b], {heads, n}} : Lattice{c->out_base[b], {n, heads}};
  }, l);
}

// The launches of a call follow one another on the stream and share the workspace; each is planned for the whole card.
struct CrossPlan {
  RowsPlan kept[kKeptPlans];
  int64_t partials;
  size_t off_o, total;
};
Shape cross_shape(const chunkkv_cross *c, int b) { return {c->q_len[b] * (c->n_q_heads / c->n_kv_heads), c->seqlen[b]}; }
int cross_count(const chunkkv_cross *c, int b0) { return c->batch - b0 < kCrossSegments ? c->batch - b0 : kCrossSegments; }
RowsPlan cross_launch_plan(const chunkkv_cross *c, int b0) {   // of the sequences from b0 on
  return plan_rows(cross_count(c, b0), [&](int i) { return cross_shape(c, b0 + i); }, c->n_kv_heads, c->dtype, c->head_dim, false, c->batch > kCrossSegments);
}
int cross_plan(const chunkkv_cross *c, CrossPlan *pl) {
  pl->partials = 0;
  for (int b0 = 0; b0 < c->batch; b0 += kCrossSegments) {
    const RowsPlan plan = cross_launch_plan(c, b0);
    if (b0 / kCrossSegments < kKeptPlans) pl->kept[b0 / kCrossSegments] = plan;
    int64_t rows = 0, items = 0;
    for (int i = 0; i < cross_count(c, b0); ++i) {
      const Shape x = cross_shape(c, b0 + i);
      const int splits = ranges_of(x, plan);
      if (splits > 1) rows += (int64_t)splits * c->n_kv_heads * x.rows;
      items += blocks_of(x, plan, c->n_kv_heads);
    }
    if (rows > kMostPartials || items > kMostBlocks) return CHUNKKV_ERR_UNSUPPORTED;
    pl->partials = rows > pl->partials ? rows : pl->partials;
  }
  pl->total = partial_bytes(pl->partials, c->head_dim, &pl->off_o);
  return CHUNKKV_OK;
}

// ---- attention behind shared prefixes -------------------------------------------------------------------------------
int check_shared(const chunkkv_pages *w, const chunkkv_pages *p, const int32_t *n_sharing) {
  int rc = check_pages(w, false);
  if (rc) return rc;
  if ((rc = check_pages(p, false))) return rc;
  if (!n_sharing) return CHUNKKV_ERR_NULL;
  if (w->n_q_heads != p->n_q_heads || w->n_kv_heads != p->n_kv_heads || w->head_dim != p->head_dim || w->dtype != p->dtype || w->page_tokens != p->page_tokens ||
      w->n_pages != p->n_pages || w->table_pitch < 1 || w->stride_page != p->stride_page || w->stride_head != p->stride_head || w->stride_tok != p->stride_tok ||
      w->softmax_scale != p->softmax_scale)
    return CHUNKKV_ERR_SHAPE;
  int64_t total = 0;
  for (int i = 0; i < w->batch; ++i) {
    if (n_sharing[i] < 0) return CHUNKKV_ERR_SHAPE;
    total += n_sharing[i];
  }
  if (total != p->batch) return CHUNKKV_ERR_SHAPE;
  return (int64_t)p->batch * (p->n_q_heads / p->n_kv_heads) > kMaxQueryRows ? CHUNKKV_ERR_UNSUPPORTED : CHUNKKV_OK;
}

// Launch l has up to kLaunchPrefixes prefixes and kJoinSegments sequences of a call, and is planned for the whole card.
struct SharedPlan {
  RowsPlan kept[kKeptPlans];
  int64_t partials, prefix_partials;
  size_t off_o, total;
};
struct SharedCall {
  const chunkkv_pages *w, *p;
  const int32_t *n_sharing;

  // Prefix i, sequence b; one without keys has no rows.
  Shape prefix(int i) const { return {w->max_tokens[i] > 0 ? n_sharing[i] * (p->n_q_heads / p->n_kv_heads) : 0, w->max_tokens[i]}; }
  Shape sequence(int b) const { return {p->max_tokens[b] > 0 ? p->n_q_heads / p->n_kv_heads : 0, p->max_tokens[b]}; }
  static int part(int n, int each, int l) { return (int64_t)l * each >= n ? 0 : (n - l * each < each ? n - l * each : each); }
  int prefixes(int l) const { return part(w->batch, kLaunchPrefixes, l); }
  int sequences(int l) const { return part(p->batch, kJoinSegments, l); }
  // Segment i of launch l, which has np prefixes: those, then its sequences.
  Shape segment(int l, int np, int i) const { return i < np ? prefix(l * kLaunchPrefixes + i) : sequence(l * kJoinSegments + i - np); }
  RowsPlan plan(int l) const {
    const int np = prefixes(l), g = p->n_q_heads / p->n_kv_heads;
    const int i0 = np > 0 ? l * kLaunchPrefixes : 0, b0 = sequences(l) > 0 ? l * kJoinSegments : 0;
    const int32_t *whole = w->max_tokens + i0, *sharing = n_sharing + i0, *own = p->max_tokens + b0;
    auto shape = [&](int i) {   // as segment()
      const int most = i < np ? whole[i] : own[i - np];
      return Shape{most > 0 ? (i < np ? sharing[i] * g : g) : 0, most};
    };
    return plan_rows(np + sequences(l), shape, p->n_kv_heads, p->dtype, p->head_dim, true, prefixes(1) + sequences(1) > 0);
  }
};
int shared_plan(const SharedCall &c, SharedPlan *pl) {
  int64_t rows[2] = {0, 0}, items = 0;   // partial rows of prefixes, of sequences
  for (int l = 0; c.prefixes(l) + c.sequences(l) > 0; ++l) {
    const RowsPlan plan = c.plan(l);
    if (l < kKeptPlans) pl->kept[l] = plan;
    const int np = c.prefixes(l), n = np + c.sequences(l);
    for (int i = 0; i < n; ++i) {
      const Shape x = c.segment(l, np, i);
      rows[i >= np] += (int64_t)ranges_of(x, plan) * c.p->n_kv_heads * x.rows;
      items += blocks_of(x, plan, c.p->n_kv_heads);
    }
  }
  pl->prefix_partials = rows[0];
  pl->partials = rows[0] + rows[1];
  if (pl->partials > kMostPartials || items > kMostBlocks) return CHUNKKV_ERR_UNSUPPORTED;
  pl->total = partial_bytes(pl->partials, c.p->head_dim, &pl->off_o);
  return CHUNKKV_OK;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t chunkkv_cross_workspace_bytes(const chunkkv_cross *cross) {
  CrossPlan pl;
  if (check_cross(cross) || cross_plan(cross, &pl)) return 0;
  return pl.total > 256 ? pl.total : 256;   // 0 is an invalid problem
}

int chunkkv_cross_attention(const chunkkv_cross *c, const int32_t *kv_len, const uint8_t *kv_mask, const void *q, const void *k, const void *v,
                            void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_cross(c);
  if (rc) return rc;
  CrossPlan pl;
  if ((rc = cross_plan(c, &pl))) return rc;
  if (pl.partials > 0 && (!workspace || workspace_bytes < pl.total || misaligned(workspace))) return CHUNKKV_ERR_WORKSPACE;
  if (cross_outputs_meet(c)) return CHUNKKV_ERR_SHAPE;
  int64_t tokens = 0;
  int longest = 0;
  for (int b = 0; b < c->batch; ++b) {
    tokens += c->q_len[b];
    longest = c->seqlen[b] > longest ? c->seqlen[b] : longest;
  }
  if (tokens > 0 && (!q || !out || (longest > 0 && (!k || !v)))) return CHUNKKV_ERR_NULL;   // arrays of no tokens may be anything
  if (kv_mask && c->mask_pitch < longest) return CHUNKKV_ERR_SHAPE;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out)) return CHUNKKV_ERR_SHAPE;
  if (tokens == 0) return CHUNKKV_OK;
  hipStream_t s = (hipStream_t)stream;
  const int esz = elem_bytes(c->dtype), g = c->n_q_heads / c->n_kv_heads;
  int token0 = 0;
  for (int b0 = 0; b0 < c->batch; b0 += kCrossSegments) {
    const int nb = cross_count(c, b0);
    const RowsPlan plan = b0 / kCrossSegments < kKeptPlans ? pl.kept[b0 / kCrossSegments] : cross_launch_plan(c, b0);
    CrossArgs a;
    JoinArgs j;
    memset(&a, 0, sizeof(a));
    memset(&j, 0, sizeof(j));
    auto &r = a.r;
    r.geom.head = c->kv_stride_head * esz; r.geom.tok = c->kv_stride_tok * esz;
    r.kv_len = kv_len; r.mask = kv_mask; r.mask_pitch = c->mask_pitch;
    r.q = q; r.k = k; r.v = v; r.out = out; r.lse = lse;
    r.part_ml = (float4 *)workspace; r.part_o = (float *)((char *)workspace + pl.off_o);
    r.q_tok = c->q_stride_tok * esz; r.q_head = c->q_stride_head * esz; r.out_tok = c->out_stride_tok * esz; r.out_head = c->out_stride_head * esz;
    r.heads = divisor(c->n_kv_heads); r.group = divisor(g); r.segments = nb; r.seq0 = b0; r.tile = plan.tile;
    set_scale(c->softmax_scale, c->head_dim, &r.scale, &r.scale_log2e);
    for (int &x : r.first) x = INT32_MAX;
    j.part_ml = r.part_ml; j.part_o = r.part_o; j.out = out; j.lse = lse; j.out_tok = r.out_tok; j.out_head = r.out_head;
    j.heads = divisor(c->n_kv_heads); j.group = divisor(g); j.scale = r.scale; j.scale_log2e = r.scale_log2e;
    for (int i = 0; i < kJoinSegments; ++i) j.first[i] = INT32_MAX;
    int items = 0, parts = 0;
    for (int i = 0; i < nb; ++i) {
      const int b = b0 + i;
      const Shape x = cross_shape(c, b);
      const int splits = ranges_of(x, plan);
      RowsSegment &seg = r.segment[i];
      r.first[i] = items;
      seg.rows = x.rows; seg.most = x.most; seg.row0 = token0; seg.splits = splits; seg.tiles = tiles_of(x, plan); seg.part = -1;
      a.q_base[i] = c->q_base[b] * esz; a.kv_base[i] = c->kv_base[b] * esz; a.out_base[i] = c->out_base[b] * esz;
      if (splits > 1 && x.rows > 0) {
        seg.part = parts;
        const int n = j.segments++;
        j.first[n] = j.tokens;
        j.segment[n] = {parts, splits, x.rows, token0, 0, 0, 0, 0, a.out_base[i]};
        j.tokens += c->q_len[b];
        parts += splits * c->n_kv_heads * x.rows;
      }
      items += (int)blocks_of(x, plan, c->n_kv_heads);
      token0 += c->q_len[b];
    }
    r.first[nb] = items;
    if (items == 0) continue;
    Timed t(kDecode, s);
    rc = c->dtype == CHUNKKV_BF16 ? launch_cross_bf16(c->head_dim, a, s) : (c->dtype == CHUNKKV_F16 ? launch_cross_f16(c->head_dim, a, s) : launch_cross_f32(c->head_dim, a, s));
    if (rc) return rc;
    if (j.segments > 0 && (rc = launch_join(c->dtype, c->head_dim, j, s))) return rc;
  }
  return CHUNKKV_OK;
}

size_t chunkkv_shared_decode_workspace_bytes(const chunkkv_pages *prefix, const chunkkv_pages *pages, const int32_t *n_sharing) {
  SharedPlan pl;
  if (check_shared(prefix, pages, n_sharing) || shared_plan({prefix, pages, n_sharing}, &pl)) return 0;
  return pl.total > 256 ? pl.total : 256;
}

int chunkkv_shared_decode_attention(const chunkkv_pages *prefix, const chunkkv_pages *pages, const int32_t *n_sharing, const int32_t *prefix_table,
                                    const int32_t *prefix_len, const int32_t *page_table, const int32_t *kv_len, const void *q, const void *k_pages,
                                    const void *v_pages, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_shared(prefix, pages, n_sharing);
  if (rc) return rc;
  if (!prefix_table || !page_table || !q || !k_pages || !v_pages || !out) return CHUNKKV_ERR_NULL;
  if (misaligned(q) || misaligned(k_pages) || misaligned(v_pages) || misaligned(out)) return CHUNKKV_ERR_SHAPE;
  const SharedCall c = {prefix, pages, n_sharing};
  SharedPlan pl;
  if ((rc = shared_plan(c, &pl))) return rc;
  if (pl.partials > 0 && (!workspace || workspace_bytes < pl.total || misaligned(workspace))) return CHUNKKV_ERR_WORKSPACE;
  auto plan_of = [&](int l) { return l < kKeptPlans ? pl.kept[l] : c.plan(l); };
  hipStream_t s = (hipStream_t)stream;
  const int d = pages->head_dim, esz = elem_bytes(pages->dtype), g = pages->n_q_heads / pages->n_kv_heads, hkv = pages->n_kv_heads;
  float4 *part_ml = (float4 *)workspace;
  float *part_o = (float *)((char *)workspace + pl.off_o);
  float scale, scale_log2e;
  set_scale(pages->softmax_scale, d, &scale, &scale_log2e);
  // Partial rows: those of the prefixes, then those of the sequences.
  int parts[2] = {0, (int)pl.prefix_partials}, before = 0;   // before: sequences of the prefixes before
  for (int l = 0; c.prefixes(l) + c.sequences(l) > 0; ++l) {
    const int np = c.prefixes(l), nb = c.sequences(l), i0 = np > 0 ? l * kLaunchPrefixes : 0, b0 = nb > 0 ? l * kJoinSegments : 0;
    const RowsPlan plan = plan_of(l);
    SharedArgs a;
    memset(&a, 0, sizeof(a));
    auto &r = a.r;
    r.geom = geometry(pages, page_table);
    r.prefix_table = prefix_table; r.prefix_pitch = prefix->table_pitch;
    r.kv_len = kv_len; r.prefix_len = prefix_len;
    r.q = q; r.k = k_pages; r.v = v_pages; r.lse = lse;   // lse: whether there is one; the join writes it, and the outputs
    r.part_ml = part_ml; r.part_o = part_o;
    r.q_tok = (int64_t)pages->n_q_heads * d * esz; r.q_head = (int64_t)d * esz;
    r.heads = divisor(hkv); r.group = divisor(g); r.segments = np + nb; r.prefixes = np; r.prefix0 = i0; r.seq0 = b0; r.tile = plan.tile;
    r.scale = scale; r.scale_log2e = scale_log2e;
    for (int &x : r.first) x = INT32_MAX;
    int items = 0;
    for (int i = 0; i < np + nb; ++i) {
      const bool own = i >= np;
      const Shape x = c.segment(l, np, i);
      const int splits = ranges_of(x, plan);
      RowsSegment &seg = r.segment[i];
      r.first[i] = items;
      seg.rows = x.rows; seg.most = x.most; seg.row0 = own ? b0 + i - np : before; seg.splits = splits; seg.tiles = tiles_of(x, plan); seg.part = parts[own];
      if (!own) before += n_sharing[i0 + i];
      items += (int)blocks_of(x, plan, hkv);
      parts[own] += splits * hkv * x.rows;
    }
    r.first[np + nb] = items;
    if (items == 0) continue;
    Timed t(kDecode, s);
    rc = pages->dtype == CHUNKKV_BF16 ? launch_shared_bf16(d, a, s) : (pages->dtype == CHUNKKV_F16 ? launch_shared_f16(d, a, s) : launch_shared_f32(d, a, s));
    if (rc) return rc;
  }
  // every sequence's own ranges and those of its prefix, in the order in which their rows were numbered: each by the plan of its launch
  int i = 0, nth = 0, prefix_part = 0, own_part = (int)pl.prefix_partials;
  RowsPlan of_prefix = plan_of(0);
  for (int l = 0; c.sequences(l) > 0; ++l) {
    const int nb = c.sequences(l), b0 = l * kJoinSegments;
    const RowsPlan plan = plan_of(l);
    JoinArgs j;
    memset(&j, 0, sizeof(j));
    j.part_ml = part_ml; j.part_o = part_o; j.out = out; j.lse = lse; j.out_tok = (int64_t)pages->n_q_heads * d * esz; j.out_head = (int64_t)d * esz;
    j.heads = divisor(hkv); j.group = divisor(g); j.scale = scale; j.scale_log2e = scale_log2e; j.segments = j.tokens = nb;
    for (int n = 0; n < kJoinSegments; ++n) j.first[n] = n < nb ? n : INT32_MAX;
    for (int n = 0; n < nb; ++n, ++nth) {
      while (nth == n_sharing[i]) {
        const Shape x = c.prefix(i);
        prefix_part += ranges_of(x, of_prefix) * hkv * x.rows;
        ++i;
        nth = 0;
        if (i % kLaunchPrefixes == 0) of_prefix = plan_of(i / kLaunchPrefixes);
      }
      const Shape whole = c.prefix(i), own = c.sequence(b0 + n);
      j.segment[n] = {own_part, ranges_of(own, plan), own.rows, b0 + n, prefix_part, ranges_of(whole, of_prefix), whole.rows, nth * g, (b0 + n) * j.out_tok};
      own_part += j.segment[n].splits * hkv * own.rows;
    }
    Timed t(kDecode, s);
    if ((rc = launch_join(pages->dtype, d, j, s))) return rc;
  }
  return CHUNKKV_OK;
}

// ---- rotation ---------------------------------------------------------------------------------------------------------
int chunkkv_rotary_frequencies(int32_t rotary_dim, double base, double factor, double slow, double fast, double trained_tokens, float *inv_freq) {
  if (!inv_freq) return CHUNKKV_ERR_NULL;
  // (a NaN fails none of the opposite comparisons in this build: looked at by its bits)
  const double given[] = {base, factor, slow, fast, trained_tokens};
  for (double x : given) {
    uint64_t u;
    memcpy(&u, &x, sizeof(u));
    if ((u & 0x7FF0000000000000ull) == 0x7FF0000000000000ull) return CHUNKKV_ERR_SHAPE;
  }
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || base <= 1.0 || factor < 1.0 || slow < 0.0 || fast < slow || trained_tokens < 0.0) return CHUNKKV_ERR_SHAPE;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const double f = pow(base, -2.0 * i / rotary_dim), turns = trained_tokens * f / 6.283185307179586;
    const double stay = trained_tokens == 0.0 ? 0.0 : (turns >= fast ? 1.0 : (turns <= slow ? 0.0 : (turns - slow) / (fast - slow)));
    inv_freq[i] = (float)(f * stay + f / factor * (1.0 - stay));
  }
  return CHUNKKV_OK;
}

int chunkkv_rotate(int32_t dtype, int32_t head_dim, int32_t n_seq, int32_t n_tokens, const chunkkv_rows *q, const chunkkv_rows *k, const int32_t *positions,
                   const float *inv_freq, int32_t rotary_dim, int32_t interleaved, float magnitude, void *stream) {
  if (dtype != CHUNKKV_F32 && dtype != CHUNKKV_BF16 && dtype != CHUNKKV_F16) return CHUNKKV_ERR_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return CHUNKKV_ERR_UNSUPPORTED;
  if (n_seq < 0 || n_tokens < 0 || rotary_dim < 1 || rotary_dim > head_dim || !fine_scale(magnitude)) return CHUNKKV_ERR_SHAPE;
  if (rotary_dim % 16 != 0) return CHUNKKV_ERR_UNSUPPORTED;
  const int esz = elem_bytes(dtype);
  RotateArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = (int64_t)n_seq * n_tokens;
  const chunkkv_rows *given[2] = {q, k};
  RotateRows *rows[2] = {&a.q, &a.k};
  int64_t heads = 0;
  for (int i = 0; i < 2; ++i) {
    const chunkkv_rows *x = given[i];
    if (!x) continue;
    if (x->n_heads < 1) return CHUNKKV_ERR_SHAPE;
    if (x->n_heads > kRotateMaxHeads) return CHUNKKV_ERR_UNSUPPORTED;
    if (a.tokens > 0 && (!x->in || !x->out)) return CHUNKKV_ERR_NULL;
    if (misaligned(x->in) || misaligned(x->out)) return CHUNKKV_ERR_SHAPE;
    const int64_t in[3] = {x->in_stride_seq, x->in_stride_head, x->in_stride_tok}, out[3] = {x->out_stride_seq, x->out_stride_head, x->out_stride_tok};
    for (int e = 0; e < 3; ++e) {
      if (in[e] > kMostElements || out[e] > kMostElements) return CHUNKKV_ERR_UNSUPPORTED;
      if (in[e] < 0 || out[e] < 0 || (in[e] * esz) % 16 || (out[e] * esz) % 16) return CHUNKKV_ERR_SHAPE;
      // in place, a row has to be where it was
      const int n = e == 0 ? n_seq : (e == 1 ? x->n_heads : n_tokens);
      if (x->in == x->out && n > 1 && in[e] != out[e]) return CHUNKKV_ERR_SHAPE;
    }
    *rows[i] = {x->in, x->out, in[0] * esz, in[1] * esz, in[2] * esz, out[0] * esz, out[1] * esz, out[2] * esz, x->n_heads, x->in == x->out};
    heads += x->n_heads;
  }
  if (heads == 0 || (a.tokens > 0 && !positions) || !inv_freq) return CHUNKKV_ERR_NULL;
  if (a.tokens > kPagedMaxTokens) return CHUNKKV_ERR_UNSUPPORTED;
  if (a.tokens == 0) return CHUNKKV_OK;
  for (const chunkkv_rows *x : given) {
    if (!x) continue;
    Axis axis[3] = {{x->out_stride_seq, n_seq}, {x->out_stride_head, x->n_heads}, {x->out_stride_tok, n_tokens}};
    if (overlap(axis, head_dim)) return CHUNKKV_ERR_SHAPE;
  }
  a.positions = positions; a.inv_freq = inv_freq; a.n_tokens = n_tokens; a.rotary = rotary_dim;
  a.magnitude = magnitude == 0.f ? 1.f : magnitude;
  hipStream_t s = (hipStream_t)stream;
  Timed t(kCompact, s);
  return launch_rotate(dtype, head_dim, interleaved != 0, a, s);
}

}  // extern "C"
