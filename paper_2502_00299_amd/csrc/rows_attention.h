// Attention of many query rows over the same keys: the kernel.
//
//   out_r = sum_s softmax_s(scale * q_r . k_s) v_s
//
// A workgroup of four wavefronts has a tile of a segment's query rows (rows.h) and a range of its keys, which it walks in tiles of 64
// that all its wavefronts share through LDS.  128 rows: every wavefront has 32 of them and all keys.  64 rows, where a segment has no
// more: two wavefronts have the first 32, each half of a tile's keys, two the others; their states are merged in the end.
//
//   scores   S[key][row] = K Q^T by 32x32 products, keys the M dimension: a lane holds 16 keys of row lane % 32, so a row's
//            statistics need no exchange but one between the two halves of a wavefront, at the end.
//   output   O^T[dim][row] = V^T P^T: the order in which keys are summed is free, so the weights are the B operand where the scores left
//            them, and V^T comes out of LDS in that order, by transposing reads (16 bits) or as rows (fp32).
//
// Weights of 16-bit types are rounded to that type once, to nearest: the output has that type, and what the rounding of a weight leaves
// in it is as much as its own does (2^-8 of the weight's part in bf16).  They are normalised by the sum of the rounded ones, so they add up
// to one; the log-sum-exp takes the sum before.  fp16 weights are held 2^10 times as large, so that the smallest normal one is 2^-24 of the
// reference.  Scores, references, sums and outputs are fp32.
// The reference of the online softmax is lazy: it moves when the weights of a row and tile add up to more than kOver.
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

// Transposing reads of the V operands of 16 keys: dims 32 i .. of the i-th address, keys 0..3 and, 8 rows on, 4..7 of a lane's half.
// One assembly block with its own wait, as read_v4.
template <int OFF, int STEP>
__device__ __forceinline__ void read_vt(uint32_t a0, uint32_t a1, u32x4 (&v)[2]) {
  uint64_t x[4];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
      "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
      : "v"(a0), "v"(a1), "n"(OFF), "n"(OFF + STEP)
      : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i) v[i] = u32x4{(uint32_t)x[2 * i], (uint32_t)(x[2 * i] >> 32), (uint32_t)x[2 * i + 1], (uint32_t)(x[2 * i + 1] >> 32)};
}
template <int OFF, int STEP>
__device__ __forceinline__ void read_vt(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, u32x4 (&v)[4]) {
  uint64_t x[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
      "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
      "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF), "n"(OFF + STEP)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = u32x4{(uint32_t)x[2 * i], (uint32_t)(x[2 * i] >> 32), (uint32_t)x[2 * i + 1], (uint32_t)(x[2 * i + 1] >> 32)};
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
#define CKV_ROWS(FIELD, I) kernarg_at<int32_t>(offsetof(std::remove_cv_t<std::remove_reference_t<decltype(r)>>, FIELD), (I))

// What a workgroup works on; the same for all its threads.
struct RowsWork {
  int h, rows, row0, split, splits, part;   // row0: first row of the tile
  int r0, len;                              // keys r0 .. r0 + len - 1
  const int32_t *table;                     // pages: of the segment
  const char *k, *v;                        // keys in a row: of (segment, kv-head), key r0
  const uint8_t *mask;                      // of key r0, or null
  const char *q;                            // of the segment's first token
  char *out;
  float *lse;
};

template <bool PAGED>
using RowsArgsOf = std::conditional_t<PAGED, SharedArgs, CrossArgs>;

template <bool PAGED, bool MASK>
__device__ __forceinline__ RowsWork rows_work(const RowsArgsOf<PAGED> &a) {
  const auto &r = a.r;
  RowsWork w;
  int x = blockIdx.x;
  const int s = rows_segment<std::remove_reference_t<decltype(r)>::kSegments>(x, r.segments), first = CKV_ROWS(first, s);
  const int items = CKV_ROWS(first, s + 1) - first;
  x -= first;
  w.rows = CKV_ROWS(rows, s);
  w.part = CKV_ROWS(part, s);
  // kv-heads are the fastest index: workgroups go to the eight XCDs in turn, so those that read the same keys meet in one or two L2s
  const int tiles = rows_tiles(w.rows), y = x / r.n_kv_heads;
  w.h = x - y * r.n_kv_heads;
  w.split = y / tiles;
  w.row0 = (y - w.split * tiles) * rows_tile(w.rows);
  w.splits = items / (tiles * r.n_kv_heads);
  const int most = CKV_ROWS(most, s), tok0 = CKV_ROWS(row0, s);
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
  int n = most;
  if (lengths != nullptr) {
    n = lengths[seq * r.n_kv_heads + w.h];
    n = n < 0 ? 0 : (n > most ? most : n);
  }
  const int range = rows_range(n, w.splits);
  w.r0 = w.split * range;
  w.len = n - w.r0 < range ? n - w.r0 : range;
  w.q = (const char *)r.q;
  w.out = (char *)r.out;
  w.k = (const char *)r.k;
  w.v = (const char *)r.v;
  w.mask = nullptr;
  w.lse = r.lse != nullptr ? r.lse + (int64_t)tok0 * r.n_kv_heads * r.group : nullptr;
  if constexpr (PAGED) {
    w.q += tok0 * r.q_tok;
    w.out += tok0 * r.out_tok;
  } else {
    w.q += kernarg_at<int64_t>(offsetof(CrossArgs, q_base), s);
    w.out += kernarg_at<int64_t>(offsetof(CrossArgs, out_base), s);
    const int64_t at = kernarg_at<int64_t>(offsetof(CrossArgs, kv_base), s) + w.h * r.geom.head + w.r0 * r.geom.tok;
    w.k += at;
    w.v += at;
    if constexpr (MASK) w.mask = r.mask + seq * r.mask_pitch + w.r0;
  }
  return w;
}

// WK: wavefronts that share the keys of a tile, 1 or 2
template <int DT, int HD, bool PAGED, bool MASK, bool LSE, int WK>
__device__ __forceinline__ void rows_body(const RowsArgsOf<PAGED> &a, const RowsWork &w, char *smem) {
  const auto &r = a.r;
  constexpr int ESZ = DT == CHUNKKV_F32 ? 4 : 2, ROWB = HD * ESZ, SEGS = ROWB / 16;   // bytes and 16-byte segments of a row
  constexpr int RPL = 1024 / ROWB, NLD = 16 / RPL;   // rows that one 1 KB load fills; loads of a wavefront's 16 rows
  constexpr int TILE = kRowsTile * ROWB;
  constexpr int NKS = DT == CHUNKKV_F32 ? HD / 8 : HD / 16, NDT = HD / 32;             // 16-byte reads of a key by a lane, 32-dim output tiles
  constexpr int NKB = 2 / WK;                        // 32-key blocks of a tile that a wavefront has
  constexpr float kOff = DT == CHUNKKV_F16 ? 10.f : 0.f, kOver = DT == CHUNKKV_F16 ? 32768.f : (DT == CHUNKKV_BF16 ? 256.f : 16.f);
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = WK == 2 ? wave & 1 : 0, wr = wave / WK;
  const int row = w.row0 + 32 * wr + n, g = r.group;
  const int token = row / g, head = w.h * g + (row - token * g);
  const bool idle = w.row0 + 32 * wr >= w.rows;      // this wavefront's rows are not there: it loads and waits with the others

  u32x4 qf[NKS];
#pragma unroll
  for (int i = 0; i < NKS; ++i) qf[i] = u32x4{0, 0, 0, 0};
  if (row < w.rows) {
    const char *from = w.q + token * r.q_tok + head * r.q_head;
#pragma unroll
    for (int i = 0; i < NKS; ++i) qf[i] = *(const u32x4 *)(from + (2 * i + half) * 16);
  }

  // Loads: this wavefront's rows of a tile are 16 wave ..; lane l of load j lands at row RPL j + l / SEGS, position l % SEGS and
  // fetches segment position ^ swizzle(row), so that neither the fragment reads nor the transposing ones meet in a bank.
  const uint32_t tok = (uint32_t)r.geom.tok;
  auto kswz = [](int i) { return SEGS == 8 ? (i >> 1) & 7 : i & 15; };
  auto vswz = [](int i) { return DT == CHUNKKV_F32 ? 0 : (SEGS == 16 ? 4 * (i & 3) : 4 * ((i >> 1) & 1)); };
  uint32_t koff[NLD], voff[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int i = RPL * j + lane / SEGS, pos = lane % SEGS;
    koff[j] = (uint32_t)i * tok + (uint32_t)((pos ^ kswz(i)) * 16);
    voff[j] = (uint32_t)i * tok + (uint32_t)((pos ^ vswz(i)) * 16);
  }
  const int tiles = w.len > 0 ? (w.len + kRowsTile - 1) / kRowsTile : 0;
  // pages: entry of block `lane` of the current window of 64 blocks, and of the next one
  int32_t page = -1, page_next = -1;
  uint64_t present = ~0ull;
  auto entry = [&](int window) __attribute__((always_inline)) {
    const int blk = 64 * window + lane;
    return 16 * blk < w.len ? w.table[page_of_block(r.geom, (uint32_t)(w.r0 / 16 + blk))] : -1;
  };
  // Keys of tile t that are there: one bit each.
  uint8_t byte = 0;                                  // of key `lane` of the tile after the next one
  auto load_mask = [&](int t) __attribute__((always_inline)) {
    if constexpr (MASK) {
      const int key = kRowsTile * t + lane;
      byte = key < w.len ? w.mask[key] : 0;
    }
  };
  auto alive_of = [&](int t) __attribute__((always_inline)) {
    const int left = w.len - kRowsTile * t;
    uint64_t m = left >= 64 ? ~0ull : (left > 0 ? (1ull << left) - 1 : 0ull);
    if constexpr (MASK) m = __builtin_amdgcn_ballot_w64(byte != 0);
    if constexpr (PAGED) {
      const uint32_t four = (uint32_t)(present >> (4 * (t & 15))) & 15u;
      if (four != 15u)
        for (int i = 0; i < 4; ++i)
          if ((four >> i & 1) == 0) m &= ~(0xFFFFull << (16 * i));
    }
    return m;
  };
  auto next_window = [&](int t) __attribute__((always_inline)) {   // before the first look at tile t
    if constexpr (PAGED) {
      if ((t & 15) == 0) {
        page = page_next;
        page_next = entry(t / 16 + 1);
        present = __builtin_amdgcn_ballot_w64(page >= 0 && page < r.geom.n_pages);
      }
    }
  };
  auto issue = [&](int t, int buf) __attribute__((always_inline)) {
    const int key0 = kRowsTile * t + 16 * wave, left = w.len - key0, rows = left < 16 ? left : 16;
    int64_t at = 0;
    bool there = rows > 0;
    if constexpr (PAGED) {
      const int blk = 4 * (t & 15) + wave;
      at = block_offset(r.geom, __builtin_amdgcn_readlane(page, blk), w.h, (uint32_t)(w.r0 / 16 + key0 / 16));
      there = there && at >= 0;
      at = there ? at : 0;
    } else {
      at = there ? key0 * r.geom.tok : 0;
    }
    const int span = there ? (int)((uint32_t)(rows - 1) * tok) + ROWB : 0;
    char *to = smem + buf * 2 * TILE + wave * 16 * ROWB;
    const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc((void *)(w.k + at), 0, span, 0x00020000);
    const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc((void *)(w.v + at), 0, span, 0x00020000);
#pragma unroll
    for (int j = 0; j < NLD; ++j) __builtin_amdgcn_raw_ptr_buffer_load_lds(krs, (__attribute__((address_space(3))) void *)(to + j * 1024), 16, koff[j], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < NLD; ++j) __builtin_amdgcn_raw_ptr_buffer_load_lds(vrs, (__attribute__((address_space(3))) void *)(to + TILE + j * 1024), 16, voff[j], 0, 0, 0);
  };

  // LDS addresses of this lane.  K: key n of a block, segment 2 i + half.  V, 16 bits: keys 4 half + (lane % 16) / 4 of 16, dims 32 i +
  // 16 (lane / 16 % 2) + 4 (lane % 4) ..; fp32: key 4 half of eight, dims NDT n ..
  const uint32_t kat = (uint32_t)((32 * wk + n) * ROWB + ((half ^ kswz(n)) * 16));
  uint32_t vat[NDT];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
#pragma unroll
  for (int i = 0; i < NDT; ++i) {
    if constexpr (DT == CHUNKKV_F32) {
      vat[i] = (uint32_t)(TILE + (32 * wk + 4 * half) * ROWB + n * NDT * 4);
    } else {
      const int p = lane & 15, key = 4 * half + p / 4, seg = 4 * i + 2 * (lane >> 4 & 1) + (p % 4) / 2;
      vat[i] = lds0 + (uint32_t)(TILE + (32 * wk + key) * ROWB + ((seg ^ vswz(key)) * 16) + (p & 1) * 8);
    }
  }

  const float c1 = r.scale_log2e;
  float m = kPagedLowest, mc = 0.f, l = 0.f, le = 0.f;
  // Are the references in log2 units below 2^14: their rounding, 2^-24 of them, is then no more than the scores' own, and the difference to
  // them one operation with the scale.
  bool plain = false;
  f32x16 acc[NDT];
#pragma unroll
  for (int i = 0; i < NDT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;

  if constexpr (PAGED) page_next = entry(0);
  next_window(0);
  load_mask(0);
  uint64_t alive = tiles > 0 ? alive_of(0) : 0;
  load_mask(1);
  if (alive != 0) issue(0, 0);
  for (int t = 0; t < tiles; ++t) {
    const uint32_t buf = (uint32_t)(t & 1) * 2 * TILE;
    __builtin_amdgcn_s_waitcnt(vm_imm(0));
    if constexpr (MASK) {
      // values of masked keys are multiplied by weights of zero, whatever bits they are: each wavefront clears those it has loaded
      const int left = w.len - kRowsTile * t - 16 * wave;
      const uint32_t dead = ~(uint32_t)(alive >> (16 * wave)) & (left >= 16 ? 0xFFFFu : (left > 0 ? (1u << left) - 1 : 0u));
      if (dead != 0 && alive != 0) {
#pragma unroll
        for (int j = 0; j < NLD; ++j)
          if (dead >> (RPL * j + lane / SEGS) & 1) *(u32x4 *)(smem + buf + TILE + wave * 16 * ROWB + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      }
    }
    __syncthreads();
    const uint64_t now = alive;
    if (t + 1 < tiles) {
      next_window(t + 1);
      alive = alive_of(t + 1);
      if (alive != 0) issue(t + 1, (t + 1) & 1);
      load_mask(t + 2);
    }
    if (now == 0 || idle) continue;

    f32x16 sc[NKB];
#pragma unroll
    for (int b = 0; b < NKB; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
      for (int i = 0; i < NKS; ++i) {
        const u32x4 kf = *(const u32x4 *)(smem + buf + ((kat ^ (uint32_t)(32 * i)) + (uint32_t)(b * 32 * ROWB)));
        if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[i][e]), sc[b], 0, 0, 0);
        } else {
          sc[b] = mma32<DT>(kf, qf[i], sc[b]);
        }
      }
    }
    if (now != ~0ull) {
#pragma unroll
      for (int b = 0; b < NKB; ++b) {
        const uint32_t bits = (uint32_t)(now >> (32 * (b + wk))) >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[b][e] = bits >> (8 * (e / 4) + e % 4) & 1 ? sc[b][e] : -__builtin_inff();
      }
    }
    // weights of the tile and their sums
    float p[NKB][16], sum, exact;
    uint32_t pk[NKB][8];
    auto weights = [&]() __attribute__((always_inline)) {
      if (plain) {
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) p[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][e], c1, kOff - mc));
      } else {
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) p[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][e] - m, c1, kOff));
      }
      float s4[4] = {0.f, 0.f, 0.f, 0.f}, e4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < NKB; ++b)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (DT == CHUNKKV_F32) {
            s4[e % 4] += p[b][2 * e] + p[b][2 * e + 1];
          } else {
            pk[b][e] = pack2<DT>(p[b][2 * e], p[b][2 * e + 1]);
            s4[e % 4] = add2<DT>(pk[b][e], s4[e % 4]);
            if constexpr (LSE) e4[e % 4] += p[b][2 * e] + p[b][2 * e + 1];
          }
        }
      sum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
      exact = (e4[0] + e4[1]) + (e4[2] + e4[3]);
    };
    weights();
    if (__builtin_amdgcn_ballot_w64(sum >= kOver) != 0) {
      // move the references of the rows that outgrew them, in both halves
      float mx = sc[0][0];
#pragma unroll
      for (int b = 0; b < NKB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[b][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float over = fmaxf(sum, __shfl_xor(sum, 32));
      const float m_new = over >= kOver ? mx : m;
      const float f = __builtin_amdgcn_exp2f((m - m_new) * c1);
      m = m_new;
      mc = m * c1;
      plain = __builtin_amdgcn_ballot_w64(fabsf(mc) >= 0x1p14f) == 0;
      l *= f;
      if constexpr (LSE) le *= f;
#pragma unroll
      for (int i = 0; i < NDT; ++i) acc[i] *= f;
      weights();
    }
    l += sum;
    if constexpr (LSE) le += exact;
#pragma unroll
    for (int b = 0; b < NKB; ++b) {
      if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const char *from = smem + buf + vat[0] + (b * 32 + 8 * (e / 4) + e % 4) * ROWB;
          float vf[NDT];
          if constexpr (NDT == 4) {
            const f32x4 x = *(const f32x4 *)from;
#pragma unroll
            for (int i = 0; i < 4; ++i) vf[i] = x[i];
          } else {
            const f32x2 x = *(const f32x2 *)from;
            vf[0] = x[0];
            vf[1] = x[1];
          }
#pragma unroll
          for (int i = 0; i < NDT; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[i], p[b][e], acc[i], 0, 0, 0);
        }
      } else {
        auto half_block = [&](auto at) __attribute__((always_inline)) {
          constexpr int ks = decltype(at)::value;
          u32x4 vf[NDT];
          constexpr int OFF = ks * 16 * ROWB;
          const uint32_t base = buf + (uint32_t)(b * 32 * ROWB);
          if constexpr (NDT == 4) read_vt<OFF, 8 * ROWB>(base + vat[0], base + vat[1], base + vat[2], base + vat[3], vf);
          else read_vt<OFF, 8 * ROWB>(base + vat[0], base + vat[1], vf);
          const u32x4 pf = {pk[b][4 * ks], pk[b][4 * ks + 1], pk[b][4 * ks + 2], pk[b][4 * ks + 3]};
#pragma unroll
          for (int i = 0; i < NDT; ++i) acc[i] = mma32<DT>(vf[i], pf, acc[i]);
        };
        half_block(std::integral_constant<int, 0>{});
        half_block(std::integral_constant<int, 1>{});
      }
    }
  }

  // ---- halves of a row, then the wavefronts that share rows
  l += __shfl_xor(l, 32);
  if constexpr (LSE) le += __shfl_xor(le, 32);
  if constexpr (DT == CHUNKKV_F32) le = l;
  if constexpr (kOff != 0.f) {
    l *= 0x1p-10f;
    le *= 0x1p-10f;
#pragma unroll
    for (int i = 0; i < NDT; ++i) acc[i] *= 0x1p-10f;
  }
  if constexpr (WK == 2) {
    __syncthreads();                     // the tiles are read
    float *state = (float *)smem + wr * (16 * NDT + 3) * 64 + lane;
    if (wk == 1) {
      state[0] = m;
      state[64] = l;
      state[128] = le;
#pragma unroll
      for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) state[(3 + 16 * i + e) * 64] = acc[i][e];
    }
    __syncthreads();
    if (wk == 1) return;
    const float m1 = state[0], M = fmaxf(m, m1), f0 = __builtin_amdgcn_exp2f((m - M) * c1), f1 = __builtin_amdgcn_exp2f((m1 - M) * c1);
    m = M;
    l = l * f0 + state[64] * f1;
    le = le * f0 + state[128] * f1;
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] = acc[i][e] * f0 + state[(3 + 16 * i + e) * 64] * f1;
  }
  if (row >= w.rows) return;
  // dims of acc[i][e]: 16 bits 32 i + 8 (e / 4) + 4 half + e % 4, fp32 NDT (8 (e / 4) + 4 half + e % 4) + i
  if (w.part < 0) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    char *to = w.out + token * r.out_tok + head * r.out_head;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NDT; ++i) *(float *)(to + (NDT * (2 * e + 4 * half + j) + i) * 4) = acc[i][e + j] * inv;
      } else {
#pragma unroll
        for (int i = 0; i < NDT; ++i)
          *(uint2 *)(to + (32 * i + 2 * e + 4 * half) * 2) = make_uint2(pack2<DT>(acc[i][e] * inv, acc[i][e + 1] * inv), pack2<DT>(acc[i][e + 2] * inv, acc[i][e + 3] * inv));
      }
    }
    if (LSE && w.lse != nullptr && half == 0)
      w.lse[(int64_t)token * r.n_kv_heads * g + head] = le > 0.f ? __builtin_fmaf(m, r.scale, __builtin_log2f(le) * 0.6931471805599453f) : -__builtin_inff();
  } else {
    const int64_t at = w.part + ((int64_t)w.split * r.n_kv_heads + w.h) * w.rows + row;
    if (half == 0) r.part_ml[at] = make_float4(m, l, le, 0.f);
    float *to = r.part_o + at * HD;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      if constexpr (DT == CHUNKKV_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NDT; ++i) to[NDT * (2 * e + 4 * half + j) + i] = acc[i][e + j];
      } else {
#pragma unroll
        for (int i = 0; i < NDT; ++i) *(f32x4 *)(to + 32 * i + 2 * e + 4 * half) = f32x4{acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]};
      }
    }
  }
}

template <int DT, int HD, bool PAGED, bool MASK, bool LSE>
__global__ __launch_bounds__(kThreads, DT == CHUNKKV_F32 && HD == 128 ? 1 : 2) void rows_kernel(RowsArgsOf<PAGED> a) {
  __shared__ __align__(16) char smem[4 * kRowsTile * HD * (DT == CHUNKKV_F32 ? 4 : 2)];
  const RowsWork w = rows_work<PAGED, MASK>(a);
  if (w.rows > kRowsNarrow) rows_body<DT, HD, PAGED, MASK, LSE, 1>(a, w, smem);
  else rows_body<DT, HD, PAGED, MASK, LSE, 2>(a, w, smem);
}

template <int DT, int HD, bool PAGED, bool MASK>
int launch_rows(const RowsArgsOf<PAGED> &a, hipStream_t s) {
  const dim3 grid((uint32_t)a.r.first[a.r.segments]);
  if (a.r.lse != nullptr) hipLaunchKernelGGL((rows_kernel<DT, HD, PAGED, MASK, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((rows_kernel<DT, HD, PAGED, MASK, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}
template <int DT, int HD>
int launch_rows_cross(const CrossArgs &a, hipStream_t s) {
  return a.r.mask != nullptr ? launch_rows<DT, HD, false, true>(a, s) : launch_rows<DT, HD, false, false>(a, s);
}

}  // namespace ckv
