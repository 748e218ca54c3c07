// Attention of many query rows over the same keys: the kernel.
//
//   out_r = sum_s softmax_s(scale * q_r . k_s) v_s
//
// A workgroup of eight wavefronts has a tile of a segment's query rows (rows.h) and a range of its keys.  Three ways:
//   256 rows   every wavefront has 32 rows and all keys, which come in tiles of 64 through a ring in LDS that all share: the most products to
//              a byte of LDS;
//   128 rows   two wavefronts have the same 32 rows, each half of the keys; their states are merged in the end.  Half as many partial
//              rows where there are few rows, but every key is read twice as often;
//   32 rows    what a decoding step has: either half of the workgroup has a tile and range of its own, and each of its four wavefronts 32 keys
//              at a time, every fourth, through LDS slots of its own, without a barrier; four states are merged in the end.
// The plan in rows_api.hip chooses.  Keys go from memory into LDS without passing registers, three tiles (one, for fp32 and d = 128) ahead of
// their use; a barrier to a tile is all that wavefronts wait for.
//
// Measured (MI355X).  Wide, 16 bits: bound by issue, not by one unit: the matrix cores are busy for half of the cycles, exponentials, sums and
// roundings take most of the rest, at the clock that this power allows: 4096 tokens over 16384 keys, 32 heads on 8, d = 128, bf16: 955 to 1005 us
// by the card, 1150 to 1095 TFLOP/s, where a matrix product of 8192^3 reaches 1175 to 1200.  Wide fp32: by its products, 129 of 152 TFLOP/s a tile; short calls also by starts and
// partial rows.  Narrow: by memory, eight tokens over 16384 keys each (537 MB) 95 us, 5.6 TB/s; a few hundred keys by latency, 7 us.
// Tried and slower: scores of the next block beside the weights of this one in one stream of instructions (3 to 8 %), half of the wavefronts half
// a block behind the others (4 %).  Wave priorities change nothing.
//
//   scores   S[key][row] = K Q^T by 32x32 products, keys the M dimension: a lane holds 16 keys of row lane % 32, so a row's
//            statistics need no exchange but one between the two halves of a wavefront, at the end.
//   output   O^T[dim][row] = V^T P^T: the order in which keys are summed is free, so the weights are the B operand where the scores left
//            them, and V^T comes out of LDS in that order, by transposing reads (16 bits) or as rows (fp32).
//
// Weights of 16-bit types.  32 rows, which are bound by memory and latency: a weight is two numbers of the type, it rounded and what that leaves, both multiplied
// (2^-16 of it in bf16, 2^-22 in fp16), so outputs are as good as their own rounding; normalised by the sum of the weights.  One number instead: eight tokens over
// up to 2048 masked keys 13.7 us rather than 14.1, others the same within 1 %, with errors of 1.94e-3 rather than 1.67e-3 of the outputs, which is
// their rounding alone.  More rows, which are bound by issue and products: rounded to the type once, to nearest (1.95e-3 to 2.14e-3), as the second product would cost as much
// as the scores; normalised by the sum of the rounded ones, so they add up to one; the log-sum-exp takes the sum before.  fp16 weights are held 2^9 times as large, so
// that the smallest normal one is 2^-23 of the reference.  Scores, references, sums and outputs are fp32.
// The reference of the online softmax is lazy: weights are taken from the one there is, and only where 32 of them add up to kOver is the maximum
// looked for and the reference moved.  Looking at it before every block instead: 1044 us rather than 988 for 4096 tokens over 16384 keys of a
// head dimension of 128 with 32 query heads on 8, 198 rather than 189 for 64 sequences behind a prefix of 131072.
#pragma once
#include "decode_mfma.h"
#include "rows.h"

namespace ckv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <int DT>
__device__ __forceinline__ f32x16 mma32(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
  if constexpr (DT == CHUNKKV_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two numbers rounded to a 16-bit type, and the sum of such a pair and x.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (DT == CHUNKKV_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
}
template <int DT>
__device__ __forceinline__ float add2(uint32_t pair, float x) {
  if constexpr (DT == CHUNKKV_BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), x, false);
  else return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), __builtin_bit_cast(f16x2, 0x3C003C00u), x, false);
}
// Number i of such a pair.
template <int DT>
__device__ __forceinline__ float part(uint32_t pair, int i) {
  if constexpr (DT == CHUNKKV_BF16) return __uint_as_float(i == 0 ? pair << 16 : pair & 0xFFFF0000u);
  else return (float)__builtin_bit_cast(f16x2, pair)[i];
}

// Four numbers as four elements of a row.
template <int DT>
__device__ __forceinline__ void store4(char *to, const f32x4 &x) {
  if constexpr (DT == CHUNKKV_F32) *(f32x4 *)to = x;
  else *(uint2 *)to = make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]));
}

// Transposing reads of the V operands of 32 keys: v[ks][i] for keys 16 ks .. and dims 32 i .. at a[i]; keys 0..3 of a lane's half and, 8 rows on,
// its next four.  One assembly block with its own wait, as read_v4.
template <int ROW>
__device__ __forceinline__ void read_vt(const uint32_t (&a)[2], u32x4 (&v)[2][2]) {
  uint64_t x[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%10\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%11\n\tds_read_b64_tr_b16 %5, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:%11\n\tds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(a[0]), "v"(a[1]), "n"(8 * ROW), "n"(16 * ROW), "n"(24 * ROW)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i / 2][i % 2] = u32x4{(uint32_t)x[2 * i], (uint32_t)(x[2 * i] >> 32), (uint32_t)x[2 * i + 1], (uint32_t)(x[2 * i + 1] >> 32)};
}
template <int ROW>
__device__ __forceinline__ void read_vt(const uint32_t (&a)[4], u32x4 (&v)[2][4]) {
  uint64_t x[16];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:%20\n\t"
      "ds_read_b64_tr_b16 %2, %17\n\tds_read_b64_tr_b16 %3, %17 offset:%20\n\t"
      "ds_read_b64_tr_b16 %4, %18\n\tds_read_b64_tr_b16 %5, %18 offset:%20\n\t"
      "ds_read_b64_tr_b16 %6, %19\n\tds_read_b64_tr_b16 %7, %19 offset:%20\n\t"
      "ds_read_b64_tr_b16 %8, %16 offset:%21\n\tds_read_b64_tr_b16 %9, %16 offset:%22\n\t"
      "ds_read_b64_tr_b16 %10, %17 offset:%21\n\tds_read_b64_tr_b16 %11, %17 offset:%22\n\t"
      "ds_read_b64_tr_b16 %12, %18 offset:%21\n\tds_read_b64_tr_b16 %13, %18 offset:%22\n\t"
      "ds_read_b64_tr_b16 %14, %19 offset:%21\n\tds_read_b64_tr_b16 %15, %19 offset:%22\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]), "=&v"(x[9]), "=&v"(x[10]),
        "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(8 * ROW), "n"(16 * ROW), "n"(24 * ROW)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = u32x4{(uint32_t)x[2 * i], (uint32_t)(x[2 * i] >> 32), (uint32_t)x[2 * i + 1], (uint32_t)(x[2 * i + 1] >> 32)};
}

// Number of the segment of workgroup x.
template <int N>
__device__ __forceinline__ int rows_segment(int x, int n) {
  constexpr size_t FIRST = offsetof(RowsArgs<N>, first);
  int lo = 0;
  if (n > 16) {
#pragma unroll
    for (int i = 16; i < N; i += 16) lo += x >= kernarg_at<int32_t>(FIRST, i) ? 16 : 0;
  }
  int s = lo;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += x >= kernarg_at<int32_t>(FIRST, lo + i) ? 1 : 0;
  return s;
}
__device__ __forceinline__ RowsSegment rows_segment_at(size_t offset) {
  auto at = [&](int i) { return kernarg_at<int32_t>(offset, i); };
  return {at(0), at(1), at(2), at(3), at(4), at(5), {0, 0}};
}

// What a workgroup, or half of one, works on.
struct RowsWork {
  int h, rows, row0, split, part;           // row0: first row of the tile
  int r0, len;                              // keys r0 .. r0 + len - 1
  const int32_t *table;                     // pages: of the segment
  int32_t page;                             // pages: entry of block `lane` of the range
  const char *k, *v;                        // keys in a row: of (segment, kv-head), key r0
  const uint8_t *mask;                      // of key r0, or null
  const char *q;                            // of the segment's first token
  char *out;                                // keys in a row: of the segment's first token
  float *lse;                               // and of that, or null
};

template <bool PAGED>
using RowsArgsOf = std::conditional_t<PAGED, SharedArgs, CrossArgs>;

// Item `x` of segment s, `seg`, whose rows are `tile` to a workgroup (or half of one).
template <bool PAGED, bool MASK>
__device__ __forceinline__ RowsWork rows_work(const RowsArgsOf<PAGED> &a, const RowsSegment &seg, int s, int x, int tile, int lane) {
  const auto &r = a.r;
  RowsWork w;
  w.rows = seg.rows;
  w.part = seg.part;
  // kv-heads are the fastest index: workgroups go to the eight XCDs in turn, so those that read the same keys meet in one or two L2s
  const int y = divided(x, r.heads);
  w.h = x - y * (int)r.heads.d;
  w.split = seg.tiles == 1 ? y : y / seg.tiles;
  w.row0 = (y - w.split * seg.tiles) * tile;
  const int most = seg.most, tok0 = seg.row0, splits = seg.splits;
  const int32_t *lengths = r.kv_len;
  int64_t seq = r.seq0 + s;
  w.table = nullptr;
  if constexpr (PAGED) {
    if (s < r.prefixes) {
      seq = r.prefix0 + s;
      w.table = r.prefix_table + seq * r.prefix_pitch;
      lengths = r.prefix_len;
    } else {
      seq -= r.prefixes;
      w.table = r.geom.table + seq * r.geom.pitch;
    }
  }
  // The table's entries are read beside the length, for the range as it is where the segment is as long as it can be; only one whose
  // ranges turn out shorter reads them again.
  const int full = rows_range(most, splits);
  auto entry = [&](int first, int end) __attribute__((always_inline)) {
    const int key = first + 16 * lane;
    return key < end ? w.table[page_of_block(r.geom, (uint32_t)key >> 4)] : -1;
  };
  if constexpr (PAGED) w.page = entry(w.split * full, most < (w.split + 1) * full ? most : (w.split + 1) * full);
  int n = most, range = full;
  if (lengths != nullptr) {
    n = lengths[seq * (int)r.heads.d + w.h];
    n = n < 0 ? 0 : (n > most ? most : n);
    range = rows_range(n, splits);
  }
  w.r0 = w.split * range;
  w.len = n - w.r0 < range ? n - w.r0 : range;
  if constexpr (PAGED) {
    if (range != full) w.page = entry(w.r0, w.r0 + w.len);
  }
  w.q = (const char *)r.q;
  w.out = nullptr;
  w.k = (const char *)r.k;
  w.v = (const char *)r.v;
  w.mask = nullptr;
  w.lse = nullptr;
  if constexpr (PAGED) {
    w.q += tok0 * r.q_tok;
  } else {
    w.q += kernarg_at<int64_t>(offsetof(CrossArgs, q_base), s);
    w.out = (char *)r.out + kernarg_at<int64_t>(offsetof(CrossArgs, out_base), s);
    if (r.lse != nullptr) w.lse = r.lse + (int64_t)tok0 * (int)(r.heads.d * r.group.d);
    const int64_t at = kernarg_at<int64_t>(offsetof(CrossArgs, kv_base), s) + w.h * r.geom.head + w.r0 * r.geom.tok;
    w.k += at;
    w.v += at;
    if constexpr (MASK) w.mask = r.mask + seq * r.mask_pitch + w.r0;
  }
  return w;
}

template <int DT, int HD>
struct RowsShape {
  static constexpr int kEsz = DT == CHUNKKV_F32 ? 4 : 2, kRow = HD * kEsz, kSegs = kRow / 16;   // bytes and 16-byte segments of a row
  static constexpr int kRpl = 1024 / kRow;           // rows that one 1 KB load fills
  static constexpr int kTile = kRowsTile * kRow;     // bytes of a tile of K or V
  static constexpr int kStages = DT == CHUNKKV_F32 && HD == 128 ? 2 : 4;   // tiles of K and V in the ring
  static constexpr int kLds = kStages * 2 * kTile;
  static constexpr int kQ = DT == CHUNKKV_F32 ? HD / 8 : HD / 16, kD = HD / 32;    // 16-byte reads of a key by a lane, 32-dim output tiles
  static constexpr int kAhead = kQ < 8 ? kQ : 8;     // of which so many are in flight
  // Two workgroups to a CU where 128 registers do, a block of 32 keys at a time: one's weights run beside the other's products.  512 (1024) query
  // tokens of 16 heads over 8 x 1654 keys, fp16: 44 (87) us with one, which takes both blocks of a tile at a time, 46 (79) with two; under a
  // mask with holes 63 (113) and 58 (89).
  static constexpr bool kTwo = DT != CHUNKKV_F32 && HD == 64;
  static constexpr int kNarrow = rows_pairs(DT, HD);   // narrow tiles of a workgroup
  static_assert(kLds >= kNarrow * 4 * 2 * 32 * kRow, "slots of the wavefronts");
  static_assert(kLds >= 8 * 32 * HD * 4 && 2 * 32 * kRow >= 32 * HD * 4, "states of the wavefronts");
  // 16-byte segments lie at position segment ^ swizzle(row), so that neither the fragment reads nor the transposing ones meet in a bank
  static __device__ __forceinline__ int kswz(int i) { return kSegs == 8 ? (i >> 1) & 7 : i & 15; }
  static __device__ __forceinline__ int vswz(int i) { return DT == CHUNKKV_F32 ? 0 : (kSegs == 16 ? 4 * (i & 3) : 4 * ((i >> 1) & 1)); }
};

// A wavefront's 32 query rows and what they have seen: row n = lane % 32 in both halves of the wavefront.
template <int DT, int HD, bool LSE, bool FINE = false>
struct Rows {
  using S = RowsShape<DT, HD>;
  // FINE: weights of 16-bit types are two numbers, kParts.  kWhole: they are multiplied as they are, so there is one sum of them.
  static constexpr bool kWhole = DT == CHUNKKV_F32 || FINE;
  static constexpr int kParts = DT != CHUNKKV_F32 && FINE ? 2 : 1;
  // fp16 weights are held 2^kOff times as large.  A row's reference moves to its maximum when that is kRise above it in log2 units; kOver: more
  // than the weights of 32 keys add up to where it is not, and no less than what a weight may be.
  static constexpr float kOff = DT == CHUNKKV_F16 ? 9.f : 0.f, kRise = DT == CHUNKKV_F16 ? 1.f : 3.f, kOver = DT == CHUNKKV_F16 ? 65536.f : 512.f;
  static_assert(kOver > 32.f * (DT == CHUNKKV_F16 ? 1024.f : 8.f), "sums");
  u32x4 qf[S::kQ];
  f32x16 acc[S::kD];
  float m, l, le, c1;
  float ref;                             // kOff - m c1
  uint64_t rough;                        // not 0: that there is no such reference yet, or one too large to be rounded

  __device__ __forceinline__ void load(const char *from, int half, float scale_log2e) {
#pragma unroll
    for (int i = 0; i < S::kQ; ++i) qf[i] = *(const u32x4 *)(from + (2 * i + half) * 16);
    m = kPagedLowest;
    l = le = ref = 0.f;
    c1 = scale_log2e;
    rough = 1;
#pragma unroll
    for (int i = 0; i < S::kD; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  }
  // The rows are there from here on: said behind the first loads of keys, or the compiler waits for those too in front of the loop.
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int i = 0; i < S::kQ; ++i) asm volatile("" : "+v"(qf[i]));
  }
  __device__ __forceinline__ void product(const u32x4 &kf, int i, f32x16 &sc) const {
    if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[i][e]), sc, 0, 0, 0);
    } else {
      sc = mma32<DT>(kf, qf[i], sc);
    }
  }
  // `bits`: keys of a 32-key block that count, the same for all lanes.  The condition of an element is two scalar instructions, one bit
  // for either half of the wavefront.
  static __device__ __forceinline__ void leave_out(f32x16 &sc, uint32_t bits) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = 8 * (e / 4) + e % 4;
      const uint64_t lanes = (uint32_t)((int32_t)(bits << (31 - key)) >> 31) | (uint64_t)(uint32_t)((int32_t)(bits << (27 - key)) >> 31) << 32;
      sc[e] = __builtin_amdgcn_inverse_ballot_w64(lanes) ? sc[e] : -__builtin_inff();
      if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // or all conditions are made first, more than there are registers for
    }
  }
  // Is a row's reference outgrown by the scores of NKB blocks?  mx: their maximum.
  template <int NKB>
  __device__ __forceinline__ bool rises(const f32x16 (&sc)[NKB], float &mx) const {
    mx = sc[0][0];
#pragma unroll
    for (int b = 0; b < NKB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[b][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));  // of the other half's keys
    return (mx - m) * c1 > kRise || m == kPagedLowest;
  }
  __device__ __forceinline__ void move(bool rise, float mx) {
    const float m_new = rise ? fmaxf(mx, kPagedLowest) : m, f = __builtin_amdgcn_exp2f((m - m_new) * c1);
    m = m_new;
    l *= f;
    if constexpr (LSE && !kWhole) le *= f;
#pragma unroll
    for (int i = 0; i < S::kD; ++i) acc[i] *= f;
  }
  // Weights of NKB blocks: p, and for 16-bit types pk, pairs rounded, and behind them what that leaves; their sums.
  template <int NKB, typename F>
  static __device__ __forceinline__ void weights(F &&exponent, float (&p)[NKB][16], uint32_t (&pk)[NKB][8 * kParts], float &sum, float &exact) {
    constexpr int NS = LSE ? 2 : 4;      // sums in parallel, as registers allow
    float s4[NS], e4[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) s4[i] = e4[i] = 0.f;
#pragma unroll
    for (int b = 0; b < NKB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) p[b][e] = __builtin_amdgcn_exp2f(exponent(b, e));
#pragma unroll
    for (int b = 0; b < NKB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (DT == CHUNKKV_F32) {
          s4[e % NS] += p[b][2 * e] + p[b][2 * e + 1];
        } else if constexpr (FINE) {
          const float x = p[b][2 * e], y = p[b][2 * e + 1];
          pk[b][e] = pack2<DT>(x, y);
          pk[b][8 + e] = pack2<DT>(x - part<DT>(pk[b][e], 0), y - part<DT>(pk[b][e], 1));
          s4[e % NS] += x + y;
        } else {
          pk[b][e] = pack2<DT>(p[b][2 * e], p[b][2 * e + 1]);
          s4[e % NS] = add2<DT>(pk[b][e], s4[e % NS]);
          if constexpr (LSE) e4[e % NS] += p[b][2 * e] + p[b][2 * e + 1];
        }
      }
    sum = s4[0] + s4[1];
    exact = e4[0] + e4[1];
    if constexpr (NS == 4) sum += s4[2] + s4[3];
  }
  // The weights, after the references have moved; the sums take them in.
  template <int NKB>
  __device__ __forceinline__ void weigh(const f32x16 (&sc)[NKB], float (&p)[NKB][16], uint32_t (&pk)[NKB][8 * kParts]) {
    float sum, exact, mx;
    const bool rise = rises<NKB>(sc, mx);
    if (__builtin_amdgcn_ballot_w64(rise) != 0) move(rise, mx);
    weights<NKB>([&](int b, int e) __attribute__((always_inline)) { return __builtin_fmaf(sc[b][e] - m, c1, kOff); }, p, pk, sum, exact);
    l += sum;
    if constexpr (LSE && !kWhole) le += exact;
  }
  // The same where references seldom move: from the ones there are, without a look at the maximum, and again only if that was too low.
  template <int NKB>
  __device__ __forceinline__ void weigh_on(const f32x16 (&sc)[NKB], float (&p)[NKB][16], uint32_t (&pk)[NKB][8 * kParts]) {
    float sum, exact, mx;
    weights<NKB>([&](int b, int e) __attribute__((always_inline)) { return __builtin_fmaf(sc[b][e], c1, ref); }, p, pk, sum, exact);
    if ((__builtin_amdgcn_ballot_w64(sum >= kOver) | rough) != 0) {
      const bool rise = rises<NKB>(sc, mx);
      move(rise, mx);
      weights<NKB>([&](int b, int e) __attribute__((always_inline)) { return __builtin_fmaf(sc[b][e] - m, c1, kOff); }, p, pk, sum, exact);
      ref = kOff - m * c1;
      // taken in log2 units, a reference is off by 2^-24 of it: below 2^14 no more than the scores themselves
      rough = __builtin_amdgcn_ballot_w64(fabsf(m * c1) >= 0x1p14f);
    }
    l += sum;
    if constexpr (LSE && !kWhole) le += exact;
  }
  // Values of 32 keys at `at` in LDS, this lane's place among them at vat[].  16 bits: read ahead of their use.  `bits`: keys that count.
  struct Values {
    u32x4 v[2][S::kD];
  };
  static __device__ __forceinline__ void read_values(uint32_t at, const uint32_t (&vat)[S::kD], Values &x) {
    if constexpr (DT != CHUNKKV_F32) {
      uint32_t from[S::kD];
#pragma unroll
      for (int i = 0; i < S::kD; ++i) from[i] = at + vat[i];
      read_vt<S::kRow>(from, x.v);
    }
  }
  __device__ __forceinline__ void values(const char *smem, uint32_t at, const uint32_t (&vat)[S::kD], const Values &x, const float (&p)[16], const uint32_t (&pk)[8 * kParts], uint32_t bits) {
    if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if ((bits >> (8 * (e / 4)) & 0xFF) == 0) continue;   // keys of these four steps: none counts
        const char *from = smem + at + vat[0] + (8 * (e / 4) + e % 4) * S::kRow;
        float vf[S::kD];
        if constexpr (S::kD == 4) {
          const f32x4 y = *(const f32x4 *)from;
#pragma unroll
          for (int i = 0; i < 4; ++i) vf[i] = y[i];
        } else {
          const f32x2 y = *(const f32x2 *)from;
          vf[0] = y[0];
          vf[1] = y[1];
        }
#pragma unroll
        for (int i = 0; i < S::kD; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[i], p[e], acc[i], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
          const u32x4 pf = {pk[8 * j + 4 * ks], pk[8 * j + 4 * ks + 1], pk[8 * j + 4 * ks + 2], pk[8 * j + 4 * ks + 3]};
#pragma unroll
          for (int i = 0; i < S::kD; ++i) acc[i] = mma32<DT>(x.v[ks][i], pf, acc[i]);
        }
      }
    }
  }
  // Halves of a row together; fp16 weights back to their size.
  __device__ __forceinline__ void close() {
    l += __shfl_xor(l, 32);
    if constexpr (LSE && !kWhole) le += __shfl_xor(le, 32);
    if constexpr (kWhole) le = l;
    if constexpr (kOff != 0.f) {
      l *= 0x1p-9f;
      le *= 0x1p-9f;
#pragma unroll
      for (int i = 0; i < S::kD; ++i) acc[i] *= 0x1p-9f;
    }
  }
  // State of wavefront `wave` into LDS: [wavefront][32 rows][HD], 16-byte pieces at piece ^ row; behind them [wavefront][32] of (m, l, le).
  // Dims of acc[i][e]: 16 bits 32 i + 8 (e / 4) + 4 half + e % 4, fp32 kD (8 (e / 4) + 4 half + e % 4) + i.
  static __device__ __forceinline__ uint32_t piece(int wave, int row, int dim) {
    return (uint32_t)((wave * 32 + row) * HD + (((dim / 4) ^ (row & (HD / 4 - 1))) * 4) + dim % 4);
  }
  __device__ __forceinline__ void put(float *o, float4 *ml, int wave, int n, int half) const {
    if (half == 0) ml[wave * 32 + n] = make_float4(m, l, le, 0.f);
#pragma unroll
    for (int e = 0; e < 16; e += DT == CHUNKKV_F32 ? 1 : 4) {
      if constexpr (DT == CHUNKKV_F32 && S::kD == 4) {
        *(f32x4 *)(o + piece(wave, n, 4 * (2 * (e / 4 * 4) + 4 * half + e % 4))) = f32x4{acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
      } else if constexpr (DT == CHUNKKV_F32) {
        *(f32x2 *)(o + piece(wave, n, 2 * (2 * (e / 4 * 4) + 4 * half + e % 4))) = f32x2{acc[0][e], acc[1][e]};
      } else {
#pragma unroll
        for (int i = 0; i < S::kD; ++i) *(f32x4 *)(o + piece(wave, n, 32 * i + 2 * e + 4 * half)) = f32x4{acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]};
      }
    }
  }
};

// States of wavefronts in LDS, W of them of the same 32 rows, to outputs or, behind shared prefixes always, partial rows; eight threads to a row.
template <int DT, int HD, bool PAGED, bool LSE, int W, typename R>
__device__ __forceinline__ void rows_finish(const R &r, const RowsWork &w, const float *o, const float4 *ml, int rows, int t, int threads) {
  const int heads = (int)(r.heads.d * r.group.d), first = t % 8 * 4;   // every eighth 16-byte piece of a row
  for (int i = t / 8; i < rows; i += threads / 8) {
    const int row = w.row0 + i, wave = i / 32 * W, n = i % 32;
    float f[W], M = kPagedLowest, l = 0.f, le = 0.f;
    float4 s[W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      s[k] = ml[(wave + k) * 32 + n];
      M = fmaxf(M, s[k].x);
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
      f[k] = W == 1 ? 1.f : __builtin_amdgcn_exp2f((s[k].x - M) * r.scale_log2e);
      l += s[k].y * f[k];
      le += s[k].z * f[k];
    }
    f32x4 x[HD / 32];
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < W; ++k) x[j] += *(const f32x4 *)(o + Rows<DT, HD, LSE>::piece(wave + k, n, first + 32 * j)) * f[k];
    }
    if (!PAGED && w.part < 0) {
      const int token = divided(row, r.group), head = w.h * (int)r.group.d + (row - token * (int)r.group.d);
      const float inv = l > 0.f ? 1.f / l : 0.f;
      char *to = w.out + token * r.out_tok + head * r.out_head + first * RowsShape<DT, HD>::kEsz;
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) store4<DT>(to + 32 * j * RowsShape<DT, HD>::kEsz, x[j] * inv);
      if (LSE && w.lse != nullptr && first == 0)
        w.lse[(int64_t)token * heads + head] = le > 0.f ? __builtin_fmaf(M, r.scale, __builtin_log2f(le) * 0.6931471805599453f) : -__builtin_inff();
    } else {
      const int64_t p = w.part + ((int64_t)w.split * (int)r.heads.d + w.h) * w.rows + row;
      if (first == 0) r.part_ml[p] = make_float4(M, l, le, 0.f);
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) *(f32x4 *)(r.part_o + p * HD + first + 32 * j) = x[j];
    }
  }
}

// The keys of a range: which there are, and loads of 16-row blocks of theirs.  They are looked up by windows of 64 blocks, a block to a
// lane, one window ahead: a load then takes its block's place out of those registers.
template <int DT, int HD, bool PAGED, bool MASK>
struct RowsKeys {
  using S = RowsShape<DT, HD>;
  const RowsArgsOf<PAGED> &a;
  const RowsWork &w;
  int lane;
  uint32_t tok;
  uint32_t live = 0, at_lo = 0, at_hi = 0, span = 0;   // of this lane's block: keys that count; where it is in the pools; bytes to the end of its last
                                                       // key, 0: none that counts
  uint64_t full = 0;                     // blocks of the window all of whose keys count
  int32_t page_next = -1;                // pages: entry of the next window's block
  u32x4 mask_next = {0, 0, 0, 0};        // bytes of the mask, of the next window's block
  __device__ __forceinline__ RowsKeys(const RowsArgsOf<PAGED> &a_, const RowsWork &w_, int lane_) : a(a_), w(w_), lane(lane_), tok((uint32_t)a_.r.geom.tok) {
    if constexpr (PAGED) page_next = w.page;
    fetch_mask(0);
  }
  __device__ __forceinline__ void fetch_mask(int window) {
    if constexpr (MASK) {
      const int key = 16 * (64 * window + lane), left = w.len - key;
      const uint8_t *from = w.mask + key;
      mask_next = u32x4{0, 0, 0, 0};
      if (left >= 16) {
        __builtin_memcpy(&mask_next, from, 16);
      } else if (left > 0) {
#pragma unroll
        for (int i = 0; i < 15; ++i)
          if (i < left) mask_next[i / 4] |= (uint32_t)from[i] << (8 * (i % 4));
      }
    }
  }
  // Before the first look at block 64 `window`.
  __device__ __forceinline__ void open(int window) {
    const int blk = 64 * window + lane, left = w.len - 16 * blk;
    live = left >= 16 ? 0xFFFFu : (left > 0 ? (1u << left) - 1 : 0u);
    int64_t at = (int64_t)(16 * blk) * tok;
    if constexpr (PAGED) {
      at = block_offset(a.r.geom, page_next, w.h, (uint32_t)(w.r0 / 16 + blk));
      if (at < 0) live = 0;
      page_next = left > 1024 ? w.table[page_of_block(a.r.geom, (uint32_t)(w.r0 / 16 + blk + 64))] : -1;
    }
    if constexpr (MASK) {
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // a bit for every byte that is not zero
        uint32_t y = mask_next[i];
        y |= y >> 4;
        y |= y >> 2;
        y |= y >> 1;
        bits |= (((y & 0x01010101u) * 0x01020408u) >> 24) << (4 * i);
      }
      live &= bits;
      fetch_mask(window + 1);
    }
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    span = live == 0 ? 0u : ((left < 16 ? (uint32_t)left : 16u) - 1) * tok + S::kRow;
    full = __builtin_amdgcn_ballot_w64(live == 0xFFFFu);
  }
  // Keys key0 .. key0 + 16 N - 1 that count, one bit each.
  template <int N>
  __device__ __forceinline__ uint64_t alive(int key0) const {
    const int blk = key0 / 16 & 63;
    constexpr uint32_t kAll = (1u << N) - 1;
    if (((uint32_t)(full >> blk) & kAll) == kAll) return N == 4 ? ~0ull : (1ull << (16 * N % 64)) - 1;
    uint64_t bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bits |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)live, blk + i) << (16 * i);
    return bits;
  }
  // Where the block of key key0 is, a multiple of 16 in the open window, and its span.
  struct Place {
    uint64_t at;
    uint32_t span;
  };
  __device__ __forceinline__ Place place(int key0) const {
    const int blk = key0 / 16 & 63;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)at_lo, blk), hi = (uint32_t)__builtin_amdgcn_readlane((int)at_hi, blk);
    return {(uint64_t)hi << 32 | lo, (uint32_t)__builtin_amdgcn_readlane((int)span, blk)};
  }
  // N loads from a block, at this lane's offsets in it; rows past its span, all of one without, arrive as zeros.
  template <int N>
  static __device__ __forceinline__ void load(const char *base, const Place &p, const uint32_t *off, char *to) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(base + p.at), 0, (int)p.span, 0x00020000);
#pragma unroll
    for (int j = 0; j < N; ++j) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(to + j * 1024), 16, off[j], 0, 0, 0);
  }
  // The same of values: rows that the mask leaves out are asked for behind every span.  They are multiplied by weights of zero, whatever
  // bits there are, so they have to arrive as zeros.  `bits`: which rows of these loads count.
  template <int N>
  __device__ __forceinline__ void load_values(const char *base, const Place &p, const uint32_t (&off)[N], char *to, uint32_t bits) const {
    uint32_t at[N];
#pragma unroll
    for (int j = 0; j < N; ++j) at[j] = !MASK || bits >> (S::kRpl * j + lane / S::kSegs) & 1 ? off[j] : 0x80000000u;
    load<N>(base, p, at, to);
  }
};

// This lane's places in a block of 32 keys in LDS.  K: key n, segment 2 i + half is at kat ^ 32 i.  V, 16 bits: keys 4 half + (lane % 16) / 4 of
// 16, dims 32 i + 16 (lane / 16 % 2) + 4 (lane % 4) ..; fp32: key 4 half of eight, dims kD n ..
template <int DT, int HD>
__device__ __forceinline__ void rows_places(int lane, uint32_t lds0, uint32_t &kat, uint32_t (&vat)[HD / 32]) {
  using S = RowsShape<DT, HD>;
  const int n = lane & 31, half = lane >> 5;
  kat = (uint32_t)(n * S::kRow + ((half ^ S::kswz(n)) * 16));
#pragma unroll
  for (int i = 0; i < S::kD; ++i) {
    if constexpr (DT == CHUNKKV_F32) {
      vat[i] = (uint32_t)(4 * half * S::kRow + n * S::kD * 4);
    } else {
      const int p = lane & 15, key = 4 * half + p / 4, seg = 4 * i + 2 * (lane >> 4 & 1) + (p % 4) / 2;
      vat[i] = lds0 + (uint32_t)(key * S::kRow + ((seg ^ S::vswz(key)) * 16) + (p & 1) * 8);
    }
  }
}

// Query row `row` of a tile; for one that is not there, one that is.
template <typename R>
__device__ __forceinline__ const char *rows_query(const R &r, const RowsWork &w, int row) {
  const int i = row < w.rows ? row : (w.rows > 0 ? w.rows - 1 : 0), token = divided(i, r.group);
  return w.q + token * r.q_tok + (w.h * (int)r.group.d + (i - token * (int)r.group.d)) * r.q_head;
}

// A barrier that waits for LDS, not for the loads that are on their way.
__device__ __forceinline__ void rows_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 256 rows (WK = 1) or 128 (WK = 2: wavefronts that share rows).
template <int DT, int HD, bool PAGED, bool MASK, bool LSE, int WK>
__device__ __forceinline__ void rows_wide(const RowsArgsOf<PAGED> &a, const RowsWork &w, char *smem, int wave, int lane) {
  using S = RowsShape<DT, HD>;
  const auto &r = a.r;
  constexpr int NL = 8 / S::kRpl, NST = S::kStages;   // loads of a wavefront's eight rows of a tile
  // Wavefronts that share rows have halves of a tile's keys, or every other tile: half as many barriers, with one step rather than three
  // tiles on their way, which d = 64 has more of the gain than the loss of.  23 sequences behind prefixes of 20995, 4096 and 10460 keys, fp16: 20.4 ->
  // 19.1 us, 4096 rows over 2048 keys 77.9 -> 73.5; with d = 128 28.1 -> 29.0.
  constexpr int PAIR = WK == 2 && HD == 64 ? 2 : 1;    // tiles to a barrier
  constexpr int NKB = 2 * PAIR / WK;       // 32-key blocks that a wavefront has of them
  constexpr int NB = S::kTwo || DT == CHUNKKV_F32 ? 1 : NKB;    // of which so many at a time
  const int n = lane & 31, half = lane >> 5, wk = WK == 2 ? wave & 1 : 0, wr = wave / WK;
  const bool idle = w.row0 + 32 * wr >= w.rows;      // this wavefront's rows are not there: it loads and waits with the others
  RowsKeys<DT, HD, PAGED, MASK> keys(a, w, lane);
  uint32_t koff[NL], voff[NL];           // of a lane in this wavefront's rows of a tile, 8 wave ..: half of a block
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int i = S::kRpl * j + lane / S::kSegs, pos = lane % S::kSegs, in_block = 8 * (wave & 1) + i;
    koff[j] = (uint32_t)in_block * keys.tok + (uint32_t)((pos ^ S::kswz(in_block)) * 16);
    voff[j] = (uint32_t)in_block * keys.tok + (uint32_t)((pos ^ S::vswz(in_block)) * 16);
  }
  const int tiles = w.len > 0 ? (w.len + kRowsTile - 1) / kRowsTile : 0;
  uint64_t alive[NST - PAIR];            // keys that count, of the tiles in flight
  auto issue = [&](int t, int stage) __attribute__((always_inline)) {   // tiles past the last one too: the number of loads in flight is known at every wait
    if ((t & 15) == 0) keys.open(t / 16);
    const uint64_t bits = keys.template alive<4>(kRowsTile * t);
    char *to = smem + stage * 2 * S::kTile + wave * 8 * S::kRow;
    const int key0 = kRowsTile * t + 16 * (wave / 2);
    const auto place = keys.place(key0);
    keys.template load<NL>(w.k, place, koff, to);
    keys.template load_values<NL>(w.v, place, voff, to + S::kTile, (uint32_t)(bits >> (8 * wave)));
    return bits;
  };
  uint32_t kat, vat[S::kD];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  rows_places<DT, HD>(lane, lds0, kat, vat);
  Rows<DT, HD, LSE> x;
  x.load(rows_query(r, w, w.row0 + 32 * wr + n), half, r.scale_log2e);
#pragma unroll
  for (int t = 0; t < NST - PAIR; ++t) alive[t] = issue(t, t);
  x.settle();
  for (int t = 0; t < tiles; t += PAIR) {
    const int stage = (PAIR == 2 ? t + wk : t) % NST, first = PAIR == 2 ? 0 : 32 * wk;   // first: key of the tile
    const uint32_t base = (uint32_t)stage * 2 * S::kTile + (uint32_t)(first * S::kRow);
    __builtin_amdgcn_s_waitcnt(vm_imm((NST - 2 * PAIR) * 2 * NL));
    const uint64_t now = PAIR == 2 && wk == 1 ? alive[1] : alive[0];
    rows_barrier();
#pragma unroll
    for (int i = 0; i < NST - 2 * PAIR; ++i) alive[i] = alive[i + PAIR];
#pragma unroll
    for (int i = NST - PAIR; i < NST; ++i) alive[i - PAIR] = issue(t + i, (t + i) % NST);
    if (now == 0 || idle) continue;
#pragma unroll
    for (int b0 = 0; b0 < NKB; b0 += NB) {
      // fp32, whose products take the time, has none with keys that do not count: 600 tokens over one key 27 -> 17 us (d = 64: 17 -> 11), over 4000
      // keys 1 % slower
      if (DT == CHUNKKV_F32 && (uint32_t)(now >> (32 * b0 + first)) == 0) continue;
      const uint32_t at0 = base + (uint32_t)(b0 * 32 * S::kRow);
      f32x16 sc[NB];
      u32x4 kf[S::kAhead];
      auto read_k = [&](int j) __attribute__((always_inline)) {   // read j of these blocks, one after the other
        if (j < NB * S::kQ) kf[j % S::kAhead] = *(const u32x4 *)(smem + at0 + ((kat ^ (uint32_t)(32 * (j % S::kQ))) + (uint32_t)(j / S::kQ * 32 * S::kRow)));
      };
#pragma unroll
      for (int j = 0; j < S::kAhead; ++j) read_k(j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
        for (int i = 0; i < S::kQ; ++i) {
          x.product(kf[i % S::kAhead], i, sc[b]);
          read_k(b * S::kQ + i + S::kAhead);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      typename Rows<DT, HD, LSE>::Values vf;
      x.read_values(at0 + (uint32_t)S::kTile, vat, vf);   // while the products run
      if (now != ~0ull) {
#pragma unroll
        for (int b = 0; b < NB; ++b) x.leave_out(sc[b], (uint32_t)(now >> (32 * (b0 + b) + first)));
      }
      float p[NB][16];
      uint32_t pk[NB][8];
      x.template weigh_on<NB>(sc, p, pk);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const uint32_t at = at0 + (uint32_t)(S::kTile + b * 32 * S::kRow);
        if (b > 0) x.read_values(at, vat, vf);
        x.values(smem, at, vat, vf, p[b], pk[b], (uint32_t)(now >> (32 * (b0 + b) + first)));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(vm_imm(0));   // the empty loads write into LDS too
  x.close();
  __syncthreads();                         // the tiles are read
  if (!idle) x.put((float *)smem, (float4 *)(smem + S::kLds), wave, n, half);
  __syncthreads();
  const int left = w.rows - w.row0, most = 256 / WK;
  rows_finish<DT, HD, PAGED, LSE, WK>(r, w, (const float *)smem, (const float4 *)(smem + S::kLds), left < most ? left : most, wave * 64 + lane, 512);
}

// 32 rows, by four wavefronts.
template <int DT, int HD, bool PAGED, bool MASK, bool LSE>
__device__ __forceinline__ void rows_narrow(const RowsArgsOf<PAGED> &a, const RowsWork &w, char *smem, float4 *ml, int wave, int lane) {
  using S = RowsShape<DT, HD>;
  const auto &r = a.r;
  constexpr int NL = 16 / S::kRpl, SLOT = 32 * S::kRow;   // loads of a block; a slot has two
  const int n = lane & 31, half = lane >> 5;
  RowsKeys<DT, HD, PAGED, MASK> keys(a, w, lane);
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int i = S::kRpl * j + lane / S::kSegs, pos = lane % S::kSegs;
    koff[j] = (uint32_t)i * keys.tok + (uint32_t)((pos ^ S::kswz(i)) * 16);
    voff[j] = (uint32_t)i * keys.tok + (uint32_t)((pos ^ S::vswz(i)) * 16);
  }
  char *kslot = smem + wave * 2 * SLOT, *vslot = kslot + SLOT;
  auto key_of = [&](int s) { return 32 * (wave + 4 * s); };
  const int steps_all = w.len > 0 ? (w.len + 31) / 32 : 0, steps = (steps_all - wave + 3) / 4;
  auto look = [&](int s) __attribute__((always_inline)) {   // keys of step s that count
    if ((s & 7) == 0) keys.open(s / 8);
    return (uint32_t)keys.template alive<2>(key_of(s));
  };
  typename RowsKeys<DT, HD, PAGED, MASK>::Place place[2];
  auto issue_k = [&](int s) __attribute__((always_inline)) {   // V of a step has K's places
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      place[t] = keys.place(key_of(s) + 16 * t);
      keys.template load<NL>(w.k, place[t], koff, kslot + t * NL * 1024);
    }
  };
  auto issue_v = [&](uint32_t bits) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) keys.template load_values<NL>(w.v, place[t], voff, vslot + t * NL * 1024, bits >> (16 * t));
  };
  uint32_t kat, vat[S::kD];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  rows_places<DT, HD>(lane, lds0, kat, vat);
  const uint32_t kbase = (uint32_t)(wave * 2 * SLOT);
  using X = Rows<DT, HD, LSE, true>;
  X x;
  x.load(rows_query(r, w, n), half, r.scale_log2e);
  uint32_t bits = look(0);
  issue_k(0);
  issue_v(bits);
  x.settle();
  for (int s = 0; s < steps; ++s) {
    const uint32_t now = bits;
    __builtin_amdgcn_s_waitcnt(vm_imm(2 * NL));
    u32x4 kf[S::kAhead];
    f32x16 sc[1];
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
#pragma unroll
    for (int i0 = 0; i0 < S::kQ; i0 += S::kAhead) {
#pragma unroll
      for (int i = 0; i < S::kAhead; ++i) kf[i] = *(const u32x4 *)(smem + kbase + (kat ^ (uint32_t)(32 * (i0 + i))));
      if (i0 + S::kAhead == S::kQ) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // the fragments are in registers: the K slot is free
        bits = look(s + 1);
        issue_k(s + 1);
      }
#pragma unroll
      for (int i = 0; i < S::kAhead; ++i) x.product(kf[i], i0 + i, sc[0]);
    }
    if (now != 0) {
      if (now != ~0u) x.leave_out(sc[0], now);
      float p[1][16];
      uint32_t pk[1][8 * X::kParts];
      x.template weigh<1>(sc, p, pk);
      __builtin_amdgcn_s_waitcnt(vm_imm(2 * NL));
      typename X::Values vf;
      x.read_values(kbase + SLOT, vat, vf);
      x.values(smem, kbase + SLOT, vat, vf, p[0], pk[0], now);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vm_imm(2 * NL) & 0xC07F);   // V of this step is there and read
    issue_v(bits);
  }
  __builtin_amdgcn_s_waitcnt(vm_imm(0));
  x.close();
  __syncthreads();                         // the other wavefronts' slots are read
  if (n < w.rows) x.put((float *)smem, ml, wave, n, half);
  __syncthreads();
  rows_finish<DT, HD, PAGED, LSE, 4>(r, w, (const float *)smem, ml, w.rows, wave * 64 + lane, 256);
}

// Segment of this workgroup, and its number in it.
template <typename R>
__device__ __forceinline__ RowsSegment rows_find(const R &r, int &s, int &x) {
  constexpr int N = R::kSegments;
  s = rows_segment<N>(blockIdx.x, r.segments);
  x = blockIdx.x - kernarg_at<int32_t>(offsetof(RowsArgs<N>, first), s);
  return rows_segment_at(offsetof(RowsArgs<N>, segment) + s * sizeof(RowsSegment));
}

constexpr int kRowsThreads = 512;
template <int DT, int HD, bool PAGED, bool MASK, bool LSE>
__global__ __launch_bounds__(kRowsThreads, (RowsShape<DT, HD>::kTwo ? 4 : 2)) void rows_kernel(RowsArgsOf<PAGED> a) {
  using S = RowsShape<DT, HD>;
  __shared__ __align__(16) char smem[S::kLds + 8 * 32 * sizeof(float4)];
  const auto &r = a.r;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  int s, x;
  const RowsSegment seg = rows_find(r, s, x);
  if (seg.rows <= kRowsNarrow) {
    const int hf = wave / 4, items = seg.splits * (int)r.heads.d, item = S::kNarrow * x + hf;
    if (hf >= S::kNarrow) return;
    const bool none = item >= items;     // an odd number: the other half waits with it, over no keys
    RowsWork w = rows_work<PAGED, MASK>(a, seg, s, none ? items - 1 : item, kRowsNarrow, lane);
    if (none) w.len = w.rows = 0;
    rows_narrow<DT, HD, PAGED, MASK, LSE>(a, w, smem + hf * 4 * 2 * 32 * S::kRow, (float4 *)(smem + S::kLds) + hf * 4 * 32, wave & 3, lane);
  } else {
    const RowsWork w = rows_work<PAGED, MASK>(a, seg, s, x, r.tile, lane);
    if (r.tile == 2 * kRowsWide) rows_wide<DT, HD, PAGED, MASK, LSE, 1>(a, w, smem, wave, lane);
    else rows_wide<DT, HD, PAGED, MASK, LSE, 2>(a, w, smem, wave, lane);
  }
}

// Where no segment has more than 32 rows: half a workgroup each.  Less code to fetch and no other half to wait for, which is what short
// ranges consist of.
template <int DT, int HD, bool PAGED, bool MASK, bool LSE>
__global__ __launch_bounds__(kThreads, DT == CHUNKKV_F32 && HD == 128 ? 1 : 2) void rows_narrow_kernel(RowsArgsOf<PAGED> a) {
  using S = RowsShape<DT, HD>;
  __shared__ __align__(16) char smem[4 * 2 * 32 * S::kRow + 4 * 32 * sizeof(float4)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  int s, x;
  const RowsSegment seg = rows_find(a.r, s, x);
  const RowsWork w = rows_work<PAGED, MASK>(a, seg, s, x, kRowsNarrow, lane);
  rows_narrow<DT, HD, PAGED, MASK, LSE>(a, w, smem, (float4 *)(smem + 4 * 2 * 32 * S::kRow), wave, lane);
}

template <int DT, int HD, bool PAGED, bool MASK, bool LSE>
int launch_rows_of(const RowsArgsOf<PAGED> &a, hipStream_t s) {
  const dim3 grid((uint32_t)a.r.first[a.r.segments]);
  if (a.r.tile == kRowsNarrow) hipLaunchKernelGGL((rows_narrow_kernel<DT, HD, PAGED, MASK, LSE>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((rows_kernel<DT, HD, PAGED, MASK, LSE>), grid, dim3(kRowsThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}
template <int DT, int HD, bool PAGED, bool MASK>
int launch_rows(const RowsArgsOf<PAGED> &a, hipStream_t s) {
  return a.r.lse != nullptr ? launch_rows_of<DT, HD, PAGED, MASK, true>(a, s) : launch_rows_of<DT, HD, PAGED, MASK, false>(a, s);
}
template <int DT, int HD>
int launch_rows_cross(const CrossArgs &a, hipStream_t s) {
  return a.r.mask != nullptr ? launch_rows<DT, HD, false, true>(a, s) : launch_rows<DT, HD, false, false>(a, s);
}

}  // namespace ckv
