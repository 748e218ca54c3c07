// Attention of one new token over pages of 16-bit rows, on the matrix cores: the range kernel.
//
// Bound by HBM bandwidth for long caches: every K and V row is read once.  Layout of the two contractions, weights as
// sums of 16-bit parts and the lazy reference of the online softmax are those of decode_mfma.hip, which says why; what
// differs is where rows come from and what else is kept.
// (16 heads fill the columns: each part is a product of its own, three for bf16 and four for fp16.)
//
// Rows: a step of 32 slots is two blocks of 16, and a block never crosses pages.  Lane i of every wavefront looks up block
// i of its range (a range has at most 64), one load of 64 table entries; a step then takes two blocks' addresses out
// of those registers by readlane, and each block has a buffer descriptor of its own, which covers exactly the rows that hold
// tokens: slots past the last one, and blocks whose page is not there, read as zeros without touching memory.
// A wavefront has one slot for K and one for V, each refilled as soon as it is read.  A second pair is slower, as it takes the place
// of other workgroups: 131072 slots 95.8 us, 89.0 so (d = 64: 47.2, 46.4), 13171 slots 16.1 and 14.7.
// Weights: kStored keeps the scores (fp32, before the scale) for the launch that adds up what every slot received.  They go
// out by a buffer store whose idle columns lie out of range, so every step has one and the waits can count them together with
// the loads (both leave the counter in the order they were issued).  17 MB of them beside 537 MB of K and V cost 10 us.
// kAdded keeps them in LDS: a head that is one range knows its log-sum-exps in the end and adds its own weights, and nothing
// follows.  It has four wavefronts or eight (paged_alone says when); eight for ranges that are joined are slower, with as many rows in
// flight: 13171 slots 16.2 us, four 15.2.
// Grid: x = key range of any sequence, y = (batch of G query heads, kv-head).
#include "decode_mfma.h"
#include "paged.h"

namespace ckv {

// A step's eight weights (of keys 4 q + i and 16 + 4 q + i) as B operands: part `part` of each, as decode_mfma.hip explains.
template <bool BF, int G, int NSET>
__device__ __forceinline__ void weight_parts(const float (&p)[8], int part, u32x4 (&pf)[NSET]) {
#pragma unroll
  for (int i2 = 0; i2 < 4; ++i2) {
    if constexpr (BF) {
      float x[2][NSET];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float p0 = p[2 * i2 + e];
        const float p1 = p0 - __uint_as_float(__float_as_uint(p0) & 0xFFFF0000u);
        const float p2 = p1 - __uint_as_float(__float_as_uint(p1) & 0xFFFF0000u);
        if constexpr (G == 4) x[e][0] = part == 0 ? p0 : (part == 1 ? p1 : p2);
        else if constexpr (G == 8) { x[e][0] = part == 0 ? p0 : p1; x[e][1] = p2; }
        else { x[e][0] = p0; x[e][1] = p1; x[e][2] = p2; }
      }
#pragma unroll
      for (int st = 0; st < NSET; ++st)   // upper halves: the truncation
        pf[st][i2] = __builtin_amdgcn_perm(__float_as_uint(x[1][st]), __float_as_uint(x[0][st]), 0x07060302u);
    } else {
      const float a0 = p[2 * i2] * 32768.f, b0 = p[2 * i2 + 1] * 32768.f;   // exact
      const fp16x2 h0 = __builtin_amdgcn_cvt_pkrtz(a0, b0);
      const float a1 = (a0 - (float)h0[0]) * 2048.f, b1 = (b0 - (float)h0[1]) * 2048.f;   // what is left of a number below 2^16 is below 2^5
      const fp16x2 h1 = __builtin_amdgcn_cvt_pkrtz(a1, b1);
      const float a2 = (a1 - (float)h1[0]) * 2048.f, b2 = (b1 - (float)h1[1]) * 2048.f;
      const fp16x2 h2 = __builtin_amdgcn_cvt_pkrtz(a2, b2);
      const float a3 = (a2 - (float)h2[0]) * 2048.f, b3 = (b2 - (float)h2[1]) * 2048.f;
      const fp16x2 h3 = __builtin_amdgcn_cvt_pkrtz(a3, b3);
      const uint32_t w0 = __builtin_bit_cast(uint32_t, h0), w1 = __builtin_bit_cast(uint32_t, h1), w2 = __builtin_bit_cast(uint32_t, h2), w3 = __builtin_bit_cast(uint32_t, h3);
      if constexpr (G == 4) pf[0][i2] = part < 2 ? (part == 0 ? w0 : w1) : (part == 2 ? w2 : w3);
      else if constexpr (G == 8) { pf[0][i2] = part == 0 ? w0 : w1; pf[1][i2] = part == 0 ? w2 : w3; }
      else { pf[0][i2] = w0; pf[1][i2] = w1; pf[2][i2] = w2; pf[3][i2] = w3; }
    }
  }
}

// Parts of a head, added up: lanes n < G hold the output of head n afterwards.
template <bool BF, int G, int NSET, int NMT>
__device__ __forceinline__ void join_parts(f32x4 (&acc)[NSET][NMT]) {
  constexpr float kS0 = BF ? 1.f : 0x1p-15f, kS1 = BF ? 1.f : 0x1p-26f, kS2 = BF ? 1.f : 0x1p-37f, kS3 = BF ? 0.f : 0x1p-48f;
#pragma unroll
  for (int mt = 0; mt < NMT; ++mt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = acc[0][mt][i];
      if constexpr (G == 4) {
        const float rest = BF ? row_shl<8>(x) : row_shl<8>(x) * kS2 + row_shl<12>(x) * kS3;
        acc[0][mt][i] = x * kS0 + (row_shl<4>(x) * kS1 + rest);
      } else if constexpr (G == 16) {
        float rest = acc[2][mt][i] * kS2;
        if constexpr (!BF) rest += acc[3][mt][i] * kS3;
        acc[0][mt][i] = x * kS0 + (acc[1][mt][i] * kS1 + rest);
      } else {
        const float y = acc[1][mt][i], rest = BF ? y : y * kS2 + row_shl<8>(y) * kS3;
        acc[0][mt][i] = x * kS0 + (row_shl<8>(x) * kS1 + rest);
      }
    }
}

// DT: bf16 or fp16, HD: head dim, G: 4, 8 or 16 query heads per workgroup, NW: wavefronts
template <int DT, int HD, int G, int NW, int W>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void paged_mfma_kernel(PagedDecodeArgs a) {
  constexpr int ROWB = HD * 2, SEGS = ROWB / 16;   // bytes and 16-byte segments of a row
  constexpr int RPL = 1024 / ROWB;                 // rows that one 1 KB load fills
  constexpr int NLB = 16 / RPL, NLD = 2 * NLB;     // loads of a block, of a slot
  constexpr int SLOT = kStepKeys * ROWB;
  constexpr int NKS = HD / 32, NMT = HD / 16;      // products of a 16-key score tile, 16-dim output tiles
  constexpr bool BF = DT == CHUNKKV_BF16;
  constexpr int NSET = G == 4 ? 1 : (G == 8 ? 2 : (BF ? 3 : 4));   // products per output tile
  constexpr int RING = NW * 2 * SLOT;
  static_assert(RING >= NW * G * (HD + 2) * 4 + G * 8, "the states of the wavefronts take the ring's place");
  __shared__ __align__(16) char smem[RING + (W == kAdded ? G * alone_rows(NW) * 4 : 0)];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q = lane >> 4;
  int h = blockIdx.y, j0 = 0;
  if (gridDim.y != (uint32_t)a.n_kv_heads) {   // more than one batch of heads per kv-head
    h = blockIdx.y % a.n_kv_heads;
    j0 = blockIdx.y / a.n_kv_heads * G;
  }
  const int g = a.group;
  const int bl = CKV_PAGED_SEQUENCE(PagedDecodeArgs, (int)blockIdx.x, a.batch), b = a.batch0 + bl;
  const int split = blockIdx.x - CKV_ARG(PagedDecodeArgs, first, bl), splits = paged_splits(bl);
  // query operand: column n holds head n % G (heads the kv-head does not have read as zero); before the lookups, whose wait
  // is theirs too
  const int head = n % G, part = n / G;
  u32x4 qf[NKS];
  {
    const char *qrow = (const char *)a.q + ((int64_t)b * a.n_q_heads + (int64_t)h * g + j0) * ROWB;
    const __amdgpu_buffer_rsrc_t qrs = __builtin_amdgcn_make_buffer_rsrc((void *)qrow, 0, (g - j0) * ROWB, 0x00020000);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(qrs, head * ROWB + (4 * ks + q) * 16, 0, 0));
  }
  // block `lane` of the range: its place in the pools, and the bytes from its first row to the end of its last one that
  // holds a token (0: no such row, or no page)
  const PagedRange range = paged_range(a, bl, h, split, splits, lane);
  const int r0 = range.r0, len = range.len;
  if (len <= 0 && split > 0) return;                   // the join knows how many ranges hold rows
  int64_t block_at = 0;
  uint32_t block_span = 0;
  const uint32_t tok = (uint32_t)a.geom.tok;
  if (16 * lane < len) {
    const int64_t at = block_offset(a.geom, range.page, h, (uint32_t)(r0 / 16 + lane));
    const int rows = len - 16 * lane < 16 ? len - 16 * lane : 16;
    if (at >= 0) {
      block_at = at;
      block_span = (uint32_t)(rows - 1) * tok + ROWB;
    }
  }
  __builtin_amdgcn_s_waitcnt(vm_imm(0));   // said here, or the compiler waits for the whole ring in front of the loop
  const int nstep_all = len > 0 ? (len + kStepKeys - 1) / kStepKeys : 0;
  const int nstep = (nstep_all - wave + NW - 1) / NW;  // steps wave, wave + NW, ... are this wavefront's

  // Load j of a block fills rows RPL j ..; lane l lands at row RPL j + l / SEGS, position l % SEGS and fetches segment
  // position ^ swizzle(row).  K: 16 rows of one segment per fragment read; V: 8 rows of two segments per transposing read.
  auto kswz = [](int row) { return SEGS == 16 ? (row & 15) : ((row >> 1) & 7); };
  auto vswz = [](int row) { return SEGS == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  uint32_t koff[NLB], voff[NLB];
#pragma unroll
  for (int j = 0; j < NLB; ++j) {
    const int row = RPL * j + lane / SEGS, pos = lane % SEGS;
    koff[j] = (uint32_t)row * tok + (uint32_t)((pos ^ kswz(row)) * 16);
    voff[j] = (uint32_t)row * tok + (uint32_t)((pos ^ vswz(row)) * 16);
  }
  const uint32_t ks_ = (uint32_t)(wave * 2 * SLOT), vs_ = ks_ + SLOT;   // this wavefront's slots
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  // Steps past the last one are issued too, through empty descriptors (their blocks have no rows): the number of loads in
  // flight is known at every wait.
  auto issue = [&](const void *base, const uint32_t *off, int step, uint32_t slot) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int blk = 2 * (wave + step * NW) + t, at = blk & 63;
      const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)block_at, at), hi = (uint32_t)__builtin_amdgcn_readlane((int)(block_at >> 32), at);
      const int in_range = __builtin_amdgcn_readlane((int)block_span, at), span = blk < 64 ? in_range : 0;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)base + (int64_t)(((uint64_t)hi << 32) | lo)), 0, span, 0x00020000);
#pragma unroll
      for (int j = 0; j < NLB; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(smem + slot + (t * NLB + j) * 1024), 16, off[j], 0, 0, 2);
    }
  };

  // LDS addresses: K fragment of row 16 t + n, segment 4 ks + q; V piece of keys 16 t + 4 q + (n / 4), dims 16 mt + 4 (n % 4)
  uint32_t kaddr[NKS], vaddr[NMT];
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) kaddr[ks] = (uint32_t)(n * ROWB + (((4 * ks + q) ^ kswz(n)) * 16));
  {
    const int row = 4 * q + n / 4;
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt) vaddr[mt] = lds0 + (uint32_t)(row * ROWB + (((2 * mt + (n % 4) / 2) ^ vswz(row)) * 16) + (n & 1) * 8);
  }
  static_assert(SEGS == 16 || SEGS == 8, "rows 16 apart share the swizzle");

  // where this lane's scores go: slots 4 q .. of a step's first block from the columns of the first part, of its second block from
  // those of the second, which hold the same products (16 heads have no second: two stores); out of range for the other columns
  const uint32_t spitch = W == kStored ? ((uint32_t)CKV_ARG(PagedDecodeArgs, max_tokens, bl) + 31u) & ~31u : 0u;
  const int sheads = g - j0 < G ? g - j0 : G;
  const __amdgpu_buffer_rsrc_t srs = __builtin_amdgcn_make_buffer_rsrc(W == kStored ? (void *)head_scores(a, bl, h * g + j0) : nullptr, 0, (int)((uint32_t)sheads * spitch * 4u), 0x00020000);
  const bool scored = head < sheads && part < 2;
  const uint32_t soff = ((uint32_t)head * spitch + (uint32_t)(r0 + 16 * part + 4 * q)) * 4u;
  float *lscores = (float *)(smem + RING);   // [G][alone_rows(NW)]
  auto keep = [&](int key, const f32x4 &x) __attribute__((always_inline)) {
    if constexpr (W == kAdded) {
      if (scored) *(f32x4 *)(lscores + head * alone_rows(NW) + key + 16 * part + 4 * q) = x;
      return;
    }
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), srs, scored ? (int)(soff + (uint32_t)key * 4u) : -1, 0, 0);
  };
  // Accesses behind the slot that is waited for: the loads of the other one and, from the second step on, the stores of a step.
  constexpr int kStores = G == 16 ? 2 : 1, kBehind = NLD + (W == kStored ? kStores : 0);
  static_assert(kBehind < 64, "vmcnt");
  auto wait = [&](int s) __attribute__((always_inline)) {
    if (W == kStored && s == 0) __builtin_amdgcn_s_waitcnt(vm_imm(NLD));
    else __builtin_amdgcn_s_waitcnt(vm_imm(kBehind));
  };

  const float c1 = a.scale_log2e;
  issue(a.k, koff, 0, ks_);
  issue(a.v, voff, 0, vs_);
  float m = kPagedLowest, l = 0.f;   // m before the scale: a difference of scores is exact where it counts, however large they are
  f32x4 acc[NSET][NMT];
#pragma unroll
  for (int s = 0; s < NSET; ++s)
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt) acc[s][mt] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int s = 0; s < nstep; ++s) {
    wait(s);
    u32x4 kf[2][NKS];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) kf[t][ks] = *(const u32x4 *)(smem + (ks_ + kaddr[ks] + (uint32_t)(t * 16 * ROWB)));
    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // two chains, added at the end: half the roundings at full magnitude
      f32x4 even = {0.f, 0.f, 0.f, 0.f}, odd = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NKS; ks += 2) {
        even = mma16<DT>(kf[t][ks], qf[ks], even);
        odd = mma16<DT>(kf[t][ks + 1], qf[ks + 1], odd);
      }
      sc[t] = even + odd;
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // the fragments are in registers: the K slot is free
    issue(a.k, koff, s + 1, ks_);

    const int key0 = (wave + s * NW) * kStepKeys;
    const int span0 = __builtin_amdgcn_readlane((int)block_span, key0 / 16), span1 = __builtin_amdgcn_readlane((int)block_span, key0 / 16 + 1);   // key0 < 1024
    if (key0 + kStepKeys > len || span0 == 0 || span1 == 0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[t][i] = (t == 0 ? span0 : span1) != 0 && key0 + 16 * t + 4 * q + i < len ? sc[t][i] : -__builtin_inff();   // times any scale
    }
    float p[8];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f((sc[i / 4][i % 4] - m) * c1);
    };
    weights();
    float sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    float over = sum;
    if constexpr (!BF) over = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
    constexpr float kOver = BF ? 16.f : 1.96875f;   // fp16: 2^15 times it is the largest 11-bit number below 2^16
    if (__builtin_amdgcn_ballot_w64(over >= kOver) != 0) {
      // move the reference of the head columns that outgrew it (the four lanes of a column together)
      float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      over = fmaxf(over, __shfl_xor(over, 16));
      over = fmaxf(over, __shfl_xor(over, 32));
      const float m_new = over >= kOver ? mx : m;
      const float f = __builtin_amdgcn_exp2f((m - m_new) * c1);
      m = m_new;
      l *= f;
#pragma unroll
      for (int st = 0; st < NSET; ++st)
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) acc[st][mt] *= f;
      weights();
      sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    }
    l += sum;
    u32x4 pf[NSET];
    weight_parts<BF, G, NSET>(p, part, pf);
    wait(s);
#pragma unroll
    for (int m4 = 0; m4 < NMT; m4 += 4) {
      u32x4 vf[4];
      read_v4<16 * ROWB>(vs_ + vaddr[m4], vs_ + vaddr[m4 + 1], vs_ + vaddr[m4 + 2], vs_ + vaddr[m4 + 3], vf);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int st = 0; st < NSET; ++st) acc[st][m4 + i] = mma16<DT>(vf[i], pf[st], acc[st][m4 + i]);
    }
    issue(a.v, voff, s + 1, vs_);
    if constexpr (W != kDropped) {   // last, so that no wait for rows is one for a store of the same step
      __builtin_amdgcn_sched_barrier(0);
      f32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = part == 0 ? sc[0][i] : sc[1][i];
      keep(key0, x);
      if constexpr (G == 16) keep(key0 + 16, sc[1]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // ---- parts of a head -> its output (lanes n < G), lanes of a column -> its sum
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  join_parts<BF, G, NSET>(acc);
  // ---- merge the wavefronts through LDS, in wavefront order; the loads of the empty steps still write zeros into the slots
  __builtin_amdgcn_s_waitcnt(vm_imm(0));
  __syncthreads();
  float *s_m = (float *)smem, *s_l = s_m + NW * G, *s_o = s_l + NW * G;   // [NW][G], [NW][G], [NW][G][HD]
  HeadNorm *s_norm = (HeadNorm *)(s_o + NW * G * HD);                              // [G]
  if (n < G) {
    if (q == 0) { s_m[wave * G + n] = m; s_l[wave * G + n] = l; }
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt) *(f32x4 *)(s_o + (wave * G + n) * HD + 16 * mt + 4 * q) = acc[0][mt];
  }
  __syncthreads();
  for (int t = tid; t < G * HD; t += NW * 64) {
    const int j = t / HD, e = t % HD;
    if (j0 + j >= g) break;
    float M = s_m[j];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w * G + j]);
    float L = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f((s_m[w * G + j] - M) * c1);
      L += s_l[w * G + j] * f;
      o += s_o[(w * G + j) * HD + e] * f;
    }
    store_range<HD>(a, b, h * g + j0 + j, e, M, L, o);
    if (W == kAdded && e == 0) s_norm[j] = head_norm(M, L);
  }
  if constexpr (W == kAdded) {
    __syncthreads();
    add_weights<NW>(a, b, h, len, lscores, s_norm);
  }
}

template <int DT, int HD, int G>
int launch_g(const PagedDecodeArgs &a, hipStream_t s) {
  const dim3 grid(a.first[a.batch], a.n_kv_heads * ((a.group + G - 1) / G));
  auto go = [&](auto kern, int waves) { hipLaunchKernelGGL(kern, grid, dim3(waves * 64), 0, s, a); };
  if constexpr (G <= 8) {   // no more heads than that are alone
    if (a.alone == 8) go(paged_mfma_kernel<DT, HD, G, 8, kAdded>, 8);
    if (a.alone == 4) go(paged_mfma_kernel<DT, HD, G, 4, kAdded>, 4);
    if (a.alone) return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
  }
  if (a.weight != nullptr) go(paged_mfma_kernel<DT, HD, G, 4, kStored>, 4);
  else go(paged_mfma_kernel<DT, HD, G, 4, kDropped>, 4);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}
template <int DT, int HD>
int launch_16(const PagedDecodeArgs &a, hipStream_t s) {
  return a.heads == 4 ? launch_g<DT, HD, 4>(a, s) : (a.heads == 8 ? launch_g<DT, HD, 8>(a, s) : launch_g<DT, HD, 16>(a, s));
}
int launch_paged_mfma(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s) {
  if (dtype == CHUNKKV_BF16) return head_dim == 128 ? launch_16<CHUNKKV_BF16, 128>(a, s) : launch_16<CHUNKKV_BF16, 64>(a, s);
  return head_dim == 128 ? launch_16<CHUNKKV_F16, 128>(a, s) : launch_16<CHUNKKV_F16, 64>(a, s);
}

}  // namespace ckv
