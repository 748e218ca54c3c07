// Attention of one new token over pages of fp32 rows, on the matrix cores: the range kernel.
//
// Bound by HBM bandwidth for long caches, by latency for short ones.  fp32 products (v_mfma_f32_16x16x4) have a sixteenth of the
// 16-bit rate and are still three times what the rows of a kv-head come in at; all 16 columns are query heads, so up to
// 16 of them share one pass over K and V.  (On the vector ALU, four heads at a time: 20000 slots of 8 kv-heads, 8 heads each 60 us.)
//
//   scores   S[key][head] = K Q^T, 16 keys a step.  A lane reads 16 bytes of a key (four k's), which go into four products; k is
//            summed in any order, so the query operand has the same one.  A chain of products per 16-byte read, added up as
//            a tree: 19 roundings in a row for 128 products.  A lane ends with the scores of keys 4q..4q+3 for head lane % 16.
//   output   O^T[dim][head] = V^T P^T, four products per 16 dims: the i-th takes keys i, 4 + i, 8 + i, 12 + i, whose weights lie where
//            the scores left them.  A lane reads 16 bytes of such a key, dims 4n..4n+3 of 64: the e-th float belongs to the
//            tile of dims e, 4 + e, 8 + e, ...
//
// Rows come as in paged_decode_mfma.hip: by loads into LDS slots of the wavefront's own, block by block of a page, without a
// barrier in the loop; K segments are XOR-swizzled by their row, V rows are read whole and need none.  The online softmax has its
// lazy reference, the scores their three ways (Scores).
// Grid: x = key range of any sequence, y = (batch of 16 query heads, kv-head).
#include "decode_mfma.h"
#include "paged.h"

namespace ckv {

// HD: head dim, NW: wavefronts
template <int HD, int NW, int W>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void paged_f32_kernel(PagedDecodeArgs a) {
  constexpr int G = 16, ROWB = HD * 4, SEGS = ROWB / 16;   // bytes and 16-byte segments of a row
  constexpr int RPL = 1024 / ROWB, NLD = 16 / RPL;         // rows that one 1 KB load fills, loads of a slot
  constexpr int SLOT = 16 * ROWB;
  constexpr int NKS = HD / 16, NH = HD / 64;               // 64-byte pieces of a key, 64-dim pieces of the output
  constexpr int RING = NW * 2 * SLOT, AH = 8;        // AH: most heads of a workgroup that adds up weights
  static_assert(RING >= NW * G * (HD + 2) * 4 + G * 8, "the states of the wavefronts take the ring's place");
  __shared__ __align__(16) char smem[RING + (W == kAdded ? AH * alone_rows(NW) * 4 : 0)];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q = lane >> 4;
  int h = blockIdx.y, j0 = 0;
  if (gridDim.y != (uint32_t)a.n_kv_heads) {   // more than one batch of heads per kv-head
    h = blockIdx.y % a.n_kv_heads;
    j0 = blockIdx.y / a.n_kv_heads * G;
  }
  const int g = a.group, heads = g - j0 < G ? g - j0 : G;
  const int bl = CKV_PAGED_SEQUENCE(PagedDecodeArgs, (int)blockIdx.x, a.batch), b = a.batch0 + bl;
  const int split = blockIdx.x - CKV_ARG(PagedDecodeArgs, first, bl), splits = paged_splits(bl);
  // query operand: column n holds head n (heads the kv-head does not have read as zero)
  f32x4 qf[NKS];
  {
    const char *qrow = (const char *)a.q + ((int64_t)b * a.n_q_heads + (int64_t)h * g + j0) * ROWB;
    const __amdgpu_buffer_rsrc_t qrs = __builtin_amdgcn_make_buffer_rsrc((void *)qrow, 0, heads * ROWB, 0x00020000);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(qrs, n * ROWB + (4 * ks + q) * 16, 0, 0));
  }
  // block `lane` of the range, as in paged_decode_mfma.hip
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
  const int nstep_all = len > 0 ? (len + 15) / 16 : 0;
  const int nstep = (nstep_all - wave + NW - 1) / NW;  // blocks wave, wave + NW, ... are this wavefront's

  uint32_t koff[NLD], voff[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int row = RPL * j + lane / SEGS, pos = lane % SEGS;
    koff[j] = (uint32_t)row * tok + (uint32_t)((pos ^ row) * 16);
    voff[j] = (uint32_t)row * tok + (uint32_t)(pos * 16);
  }
  const uint32_t ks_ = (uint32_t)(wave * 2 * SLOT), vs_ = ks_ + SLOT;   // this wavefront's slots
  auto issue = [&](const void *base, const uint32_t *off, int step, uint32_t slot) __attribute__((always_inline)) {
    const int blk = wave + step * NW, at = blk & 63;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)block_at, at), hi = (uint32_t)__builtin_amdgcn_readlane((int)(block_at >> 32), at);
    const int in_range = __builtin_amdgcn_readlane((int)block_span, at), span = blk < 64 ? in_range : 0;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)base + (int64_t)(((uint64_t)hi << 32) | lo)), 0, span, 0x00020000);
#pragma unroll
    for (int j = 0; j < NLD; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(smem + slot + j * 1024), 16, off[j], 0, 0, 2);
  };
  uint32_t kaddr[NKS];
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) kaddr[ks] = (uint32_t)(n * ROWB + (((4 * ks + q) ^ n) * 16));
  const uint32_t vaddr = (uint32_t)(4 * q * ROWB + n * 16);

  const uint32_t spitch = W == kStored ? ((uint32_t)CKV_ARG(PagedDecodeArgs, max_tokens, bl) + 31u) & ~31u : 0u;
  const __amdgpu_buffer_rsrc_t srs = __builtin_amdgcn_make_buffer_rsrc(W == kStored ? (void *)head_scores(a, bl, h * g + j0) : nullptr, 0, (int)((uint32_t)heads * spitch * 4u), 0x00020000);
  const bool scored = n < heads;
  const uint32_t soff = ((uint32_t)n * spitch + (uint32_t)(r0 + 4 * q)) * 4u;
  float *lscores = (float *)(smem + RING);   // [AH][alone_rows(NW)]
  // Accesses behind the slot that is waited for: the loads of the other one and, from the second step on, a store.
  constexpr int kBehind = NLD + (W == kStored ? 1 : 0);
  static_assert(kBehind < 64, "vmcnt");
  auto wait = [&](int s) __attribute__((always_inline)) {
    if (W == kStored && s == 0) __builtin_amdgcn_s_waitcnt(vm_imm(NLD));
    else __builtin_amdgcn_s_waitcnt(vm_imm(kBehind));
  };

  const float c1 = a.scale_log2e;
  issue(a.k, koff, 0, ks_);
  issue(a.v, voff, 0, vs_);
  float m = kPagedLowest, l = 0.f;   // m before the scale
  f32x4 acc[NH][4];
#pragma unroll
  for (int t = 0; t < NH; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int s = 0; s < nstep; ++s) {
    wait(s);
    f32x4 kf[NKS], part[NKS];
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) kf[ks] = *(const f32x4 *)(smem + (ks_ + kaddr[ks]));
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) part[ks] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) part[ks] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[ks][e], qf[ks][e], part[ks], 0, 0, 0);
#pragma unroll
    for (int o = NKS / 2; o > 0; o /= 2)
#pragma unroll
      for (int ks = 0; ks < o; ++ks) part[ks] += part[ks + o];
    f32x4 sc = part[0];
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // the fragments are in registers: the K slot is free
    issue(a.k, koff, s + 1, ks_);

    const int key0 = (wave + s * NW) * 16;
    const int span = __builtin_amdgcn_readlane((int)block_span, wave + s * NW);   // below 64
    if (key0 + 16 > len || span == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[i] = span != 0 && key0 + 4 * q + i < len ? sc[i] : -__builtin_inff();   // times any scale
    }
    if constexpr (W == kAdded) {
      if (scored) *(f32x4 *)(lscores + n * alone_rows(NW) + key0 + 4 * q) = sc;
    }
    float p[4];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f((sc[i] - m) * c1);
    };
    weights();
    float sum = (p[0] + p[1]) + (p[2] + p[3]);
    if (__builtin_amdgcn_ballot_w64(sum >= 16.f) != 0) {
      // move the reference of the head columns that outgrew it (the four lanes of a column together)
      float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), over = sum;
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      over = fmaxf(over, __shfl_xor(over, 16));
      over = fmaxf(over, __shfl_xor(over, 32));
      const float m_new = over >= 16.f ? mx : m;
      const float f = __builtin_amdgcn_exp2f((m - m_new) * c1);
      m = m_new;
      l *= f;
#pragma unroll
      for (int t = 0; t < NH; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] *= f;
      weights();
      sum = (p[0] + p[1]) + (p[2] + p[3]);
    }
    l += sum;
    wait(s);
#pragma unroll
    for (int t = 0; t < NH; ++t) {
      f32x4 vf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) vf[i] = *(const f32x4 *)(smem + (vs_ + vaddr + (uint32_t)(i * ROWB + t * 256)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][e], p[i], acc[t][e], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // the V slot is free
    issue(a.v, voff, s + 1, vs_);
    if constexpr (W == kStored) {   // last, so that no wait for rows is one for a store of the same step
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sc), srs, scored ? (int)(soff + (uint32_t)key0 * 4u) : -1, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // ---- merge the wavefronts through LDS, in wavefront order; the loads of the empty steps still write zeros into the slots
  __builtin_amdgcn_s_waitcnt(vm_imm(0));
  __syncthreads();
  float *s_m = (float *)smem, *s_l = s_m + NW * G, *s_o = s_l + NW * G;   // [NW][G], [NW][G], [NW][G][HD]
  HeadNorm *s_norm = (HeadNorm *)(s_o + NW * G * HD);                              // [G]
  if (scored) {
    if (q == 0) { s_m[wave * G + n] = m; s_l[wave * G + n] = l; }
#pragma unroll
    for (int t = 0; t < NH; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(f32x4 *)(s_o + (wave * G + n) * HD + 64 * t + 16 * q + 4 * r) = f32x4{acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
  }
  __syncthreads();
  for (int t = tid; t < heads * HD; t += NW * 64) {
    const int j = t / HD, e = t % HD;
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

template <int HD>
int launch_hd(const PagedDecodeArgs &a, hipStream_t s) {
  const dim3 grid(a.first[a.batch], a.n_kv_heads * ((a.group + 15) / 16));
  auto go = [&](auto kern, int waves) { hipLaunchKernelGGL(kern, grid, dim3(waves * 64), 0, s, a); };
  if (a.alone == 8) go(paged_f32_kernel<HD, 8, kAdded>, 8);
  else if (a.alone == 4) go(paged_f32_kernel<HD, 4, kAdded>, 4);
  else if (a.weight != nullptr) go(paged_f32_kernel<HD, 4, kStored>, 4);
  else go(paged_f32_kernel<HD, 4, kDropped>, 4);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}
int launch_paged_f32(int head_dim, const PagedDecodeArgs &a, hipStream_t s) {
  return head_dim == 128 ? launch_hd<128>(a, s) : launch_hd<64>(a, s);
}

}  // namespace ckv
