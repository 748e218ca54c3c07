// Attention of one new token per sequence over pages, and what every slot received of it.
//
// out_i = sum_s softmax_s(scale * q_i . k_s) v_s over the slots of a kv-head; a head's slots are cut into key ranges, each a
// workgroup that leaves (maximum, sum, weighted values) of its rows, joined afterwards in range order.
// This file holds the range kernel for fp32 pages, on the vector ALU, and the launch behind the ranges; 16-bit pages go to
// paged_decode_mfma.hip.
//
// A row is spread over LPR = d / 4 lanes, 16 bytes each; the lanes of a row reduce their partial dot products with DPP adds,
// each group of LPR lanes runs its own online softmax over the rows it meets, and groups, wavefronts and ranges are merged by
// the (max, sum, weighted output) rule, always in the same order.  The addresses of a range's 16-row blocks are looked up
// once, by one lane each, and kept in LDS.  A wavefront has the rows of its next round on their way while it works on one.
#include "paged.h"

namespace ckv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr float kNegBig = -1.0e30f, kMasked = -3.0e38f;

// HD: head dim, G: query heads of a workgroup, NW: its wavefronts, W: 1 = the scores are kept for the weights
template <int HD, int G, int NW, int W>
__global__ __launch_bounds__(NW * 64) void paged_f32_kernel(PagedDecodeArgs a) {
  constexpr int LPR = HD / 4, RPW = 64 / LPR, U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane / LPR, seg = lane % LPR;
  const int h = blockIdx.y, j0 = blockIdx.z * G;
  const int bl = CKV_PAGED_SEQUENCE(PagedDecodeArgs, (int)blockIdx.x, a.batch), b = a.batch0 + bl;
  const int split = blockIdx.x - CKV_ARG(PagedDecodeArgs, first, bl), splits = paged_splits(bl);
  __shared__ int64_t s_block[kPagedMaxRange / 16];
  f32x4 q[G];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    q[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (j0 + j < a.group) q[j] = *(const f32x4 *)((const float *)a.q + ((int64_t)b * a.n_q_heads + (int64_t)h * a.group + j0 + j) * HD + seg * 4);
  }
  static_assert(kPagedMaxRange / 16 == 64, "a block per lane");
  const PagedRange range = paged_range(a, bl, h, split, splits, lane);
  const int r0 = range.r0, r1 = r0 + range.len;
  if (range.len <= 0 && split > 0) return;   // the join knows how many ranges hold rows
  if (wave == 0 && 16 * lane < range.len) s_block[lane] = block_offset(a.geom, range.page, h, (uint32_t)(r0 / 16 + lane));
  __syncthreads();

  const char *kbase = (const char *)a.k + seg * 16, *vbase = (const char *)a.v + seg * 16;
  float m[G], l[G];
  f32x4 o[G];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    m[j] = kNegBig;
    l[j] = 0.f;
    o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c1 = a.scale_log2e;
  const bool keeps = W != 0 && seg < G && j0 + seg < a.group;
  float *scores = keeps ? head_scores(a, bl, h * a.group + j0 + seg) : nullptr;
  f32x4 kn[U], vn[U];
  auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = base + u * RPW + grp;
      const int64_t at = row < r1 ? s_block[(row - r0) >> 4] : -1;
      kn[u] = vn[u] = f32x4{0.f, 0.f, 0.f, 0.f};   // rows that are not there count as zeros, whatever is in memory
      if (at >= 0) {
        const int64_t off = at + (int64_t)(row & 15) * a.geom.tok;
        kn[u] = __builtin_nontemporal_load((const f32x4 *)(kbase + off));
        vn[u] = __builtin_nontemporal_load((const f32x4 *)(vbase + off));
      }
    }
  };
  const int base0 = r0 + wave * (U * RPW);
  if (base0 < r1) load(base0);
  for (int base = base0; base < r1; base += NW * U * RPW) {
    f32x4 kr[U], vr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { kr[u] = kn[u]; vr[u] = vn[u]; }
    if (base + NW * U * RPW < r1) load(base + NW * U * RPW);
    float s[U][G];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = base + u * RPW + grp;
      const bool there = row < r1 && s_block[(row - r0) >> 4] >= 0;
#pragma unroll
      for (int j = 0; j < G; ++j) {
        float d = kr[u][0] * q[j][0];
#pragma unroll
        for (int e = 1; e < 4; ++e) d = __builtin_fmaf(kr[u][e], q[j][e], d);
        d = row_sum<LPR>(d);
        s[u][j] = there ? d * c1 : kMasked;
      }
      if constexpr (W != 0) {   // lane j of a row keeps the score of head j
        float mine = s[u][0];
#pragma unroll
        for (int j = 1; j < G; ++j) mine = seg == j ? s[u][j] : mine;
        if (keeps && row < r1) scores[row] = mine;
      }
    }
#pragma unroll
    for (int j = 0; j < G; ++j) {
      float smax = s[0][j];
#pragma unroll
      for (int u = 1; u < U; ++u) smax = fmaxf(smax, s[u][j]);
      if (__builtin_amdgcn_ballot_w64(smax > m[j]) != 0) {
        const float m_new = fmaxf(m[j], smax);
        const float f = __builtin_amdgcn_exp2f(m[j] - m_new);
        l[j] *= f;
        o[j] *= f;
        m[j] = m_new;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) s[u][j] = __builtin_amdgcn_exp2f(s[u][j] - m[j]);   // now the weight
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < G; ++j) {
        l[j] += s[u][j];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = __builtin_fmaf(s[u][j], vr[u][e], o[j][e]);
      }
  }
  // the row groups of the wavefront (lanes that hold the same 16 bytes of a row)
#pragma unroll
  for (int x = LPR; x < 64; x *= 2) {
#pragma unroll
    for (int j = 0; j < G; ++j) {
      const float m_o = __shfl_xor(m[j], x), l_o = __shfl_xor(l[j], x);
      const float M = fmaxf(m[j], m_o);
      const float fa = __builtin_amdgcn_exp2f(m[j] - M), fb = __builtin_amdgcn_exp2f(m_o - M);
      l[j] = l[j] * fa + l_o * fb;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = o[j][e] * fa + __shfl_xor(o[j][e], x) * fb;
      m[j] = M;
    }
  }
  // the wavefronts, through LDS: a thread per element folds their states in order
  __shared__ float s_m[NW][G], s_l[NW][G];
  __shared__ f32x4 s_o[NW][G][LPR];
  if (grp == 0) {
#pragma unroll
    for (int j = 0; j < G; ++j) {
      if (seg == 0) { s_m[wave][j] = m[j]; s_l[wave][j] = l[j]; }
      s_o[wave][j][seg] = o[j];
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < G * HD; t += NW * 64) {
    const int j = t / HD, e = t % HD;
    if (j0 + j >= a.group) break;
    float M = s_m[0][j];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][j]);
    float L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][j] - M);
      L += s_l[w][j] * f;
      acc += ((const float *)s_o[w][j])[e] * f;
    }
    store_range<HD>(a, b, h * a.group + j0 + j, e, M, L, acc);
  }
}

// The launch behind the ranges.
//
// Its first `joins` workgroups join a query head each: out = sum_r o_r 2^(m_r - M) / sum_r l_r 2^(m_r - M).  A thread owns four
// columns and every so many-th range, four of them in flight; the groups of ranges are folded through LDS in order.
// With weights (W = 1) the others add token_weight[s] += sum_i 2^(x_i(s) - lse_i) to the slots of one key range of one kv-head,
// heads in order: the scores of the first four heads are on their way while the log-sum-exps are formed from all ranges' pairs.
template <int HD, int W>
__global__ __launch_bounds__(kThreads) void paged_finish_kernel(PagedDecodeArgs a, int joins) {
  constexpr int TPR = HD / 4, NG = kThreads / TPR, UN = 4;
  __shared__ float s_acc[NG][HD + 2];
  __shared__ float s_lse[W != 0 ? kPagedMaxGroup : 1];
  const int t = threadIdx.x;
  if (W == 0 || (int)blockIdx.x < joins) {
    const int bl = blockIdx.x / a.n_q_heads, hq = blockIdx.x % a.n_q_heads, col = t % TPR, grp = t / TPR;
    const int n = paged_length(a, bl, hq / a.group), rps = paged_range_rows(n, paged_splits(bl)), used = n > 0 ? (n + rps - 1) / rps : 1;
    const int64_t slot = (int64_t)CKV_ARG(PagedDecodeArgs, first, bl) * a.n_q_heads + hq;
    const float2 *ml = a.part_ml + slot;
    const float *po = a.part_o + slot * HD + col * 4;
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, m = kNegBig, lsum = 0.f;
    for (int r0 = grp; r0 < used; r0 += UN * NG) {
      float2 p[UN];
      float4 o4[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int64_t r = (int64_t)(r0 + u * NG < used ? r0 + u * NG : r0) * a.n_q_heads;
        p[u] = ml[r];
        o4[u] = *(const float4 *)(po + r * HD);
      }
      float mm = m;
#pragma unroll
      for (int u = 0; u < UN; ++u) mm = fmaxf(mm, p[u].x);
      const float f0 = __builtin_amdgcn_exp2f(m - mm);
      lsum *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const float f = r0 + u * NG < used ? __builtin_amdgcn_exp2f(p[u].x - mm) : 0.f;
        lsum += p[u].y * f;
        acc[0] += o4[u].x * f; acc[1] += o4[u].y * f; acc[2] += o4[u].z * f; acc[3] += o4[u].w * f;
      }
      m = mm;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s_acc[grp][col * 4 + e] = acc[e];
    if (col == 0) { s_acc[grp][HD] = lsum; s_acc[grp][HD + 1] = m; }
    __syncthreads();
    if (t < HD) {
      float M = s_acc[0][HD + 1];
#pragma unroll
      for (int g = 1; g < NG; ++g) M = fmaxf(M, s_acc[g][HD + 1]);
      float v = 0.f, L = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const float f = __builtin_amdgcn_exp2f(s_acc[g][HD + 1] - M);
        v += s_acc[g][t] * f;
        L += s_acc[g][HD] * f;
      }
      const int64_t head = (int64_t)(a.batch0 + bl) * a.n_q_heads + hq;
      a.out[head * HD + t] = L > 0.f ? v / L : 0.f;
      if (a.lse != nullptr && t == 0) a.lse[head] = L > 0.f ? (M + __builtin_log2f(L)) * 0.6931471805599453f : -__builtin_inff();
    }
    return;
  }
  if constexpr (W != 0) {
    const int x = blockIdx.x - joins, h = x % a.n_kv_heads, range = x / a.n_kv_heads, lane = t & 63, wave = t >> 6;
    const int bl = CKV_PAGED_SEQUENCE(PagedDecodeArgs, range, a.batch), b = a.batch0 + bl;
    const int first = CKV_ARG(PagedDecodeArgs, first, bl), split = range - first, splits = paged_splits(bl);
    const int n = paged_length(a, bl, h), rps = paged_range_rows(n, splits), used = n > 0 ? (n + rps - 1) / rps : 1;
    const int r0 = split * rps, len = r0 + rps < n ? rps : n - r0;
    if (len <= 0) return;
    constexpr int NR = kPagedMaxRange / kThreads;   // rows of a thread
    const uint32_t pitch = ((uint32_t)CKV_ARG(PagedDecodeArgs, max_tokens, bl) + 31u) & ~31u;
    const float *scores = head_scores(a, bl, h * a.group) + r0;
    float *weight = a.weight + ((int64_t)b * a.n_kv_heads + h) * a.slot_pitch + r0;
    float sx[4][NR], sum[NR];
    auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          sx[j][i] = kNegBig;
          if (j0 + j < a.group && t + i * kThreads < len) sx[j][i] = scores[(int64_t)(j0 + j) * pitch + t + i * kThreads];
        }
    };
    load(0);
    float old[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      sum[i] = 0.f;
      old[i] = t + i * kThreads < len ? weight[t + i * kThreads] : 0.f;
    }
    for (int j = wave; j < a.group; j += kThreads / 64) {
      float m = kNegBig, l = 0.f;
      for (int r = lane; r < used; r += 64) {
        const float2 p = a.part_ml[(int64_t)(first + r) * a.n_q_heads + h * a.group + j];
        const float mm = fmaxf(m, p.x);
        l = l * __builtin_amdgcn_exp2f(m - mm) + p.y * __builtin_amdgcn_exp2f(p.x - mm);
        m = mm;
      }
      float M = m;
      for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
      l *= __builtin_amdgcn_exp2f(m - M);
      for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
      if (lane == 0) s_lse[j] = l > 0.f ? M + __builtin_log2f(l) : 3.0e38f;   // no slot is there: no weight
    }
    __syncthreads();
    for (int j0 = 0;;) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float lse = j0 + j < a.group ? s_lse[j0 + j] : 3.0e38f;
#pragma unroll
        for (int i = 0; i < NR; ++i) sum[i] += __builtin_amdgcn_exp2f(sx[j][i] - lse);
      }
      j0 += 4;
      if (j0 >= a.group) break;
      load(j0);
    }
#pragma unroll
    for (int i = 0; i < NR; ++i)
      if (t + i * kThreads < len) weight[t + i * kThreads] = old[i] + sum[i];
  }
}

// Query heads of one kv-head that a workgroup serves.  Matrix cores: 4 or 8; 5 to 7 are one padded batch of 8, not two passes over
// K and V.  Vector ALU: 1, 2 or 4 (registers).
int paged_decode_heads(int dtype, int group) {
  if (dtype != CHUNKKV_F32) return group > 4 ? 8 : 4;
  return group > 2 ? 4 : group;
}

// Up to two workgroups a CU, at d = 128, the rows of a range are spread over eight wavefronts, so that most have one or two rounds of
// them to wait for: 300 slots of 8 kv-heads, 4 heads each 12.0 us a call, with four 13.8; at d = 64, where a round is 64 rows, 11187 slots
// of four sequences 20.1, with four 16.6.
template <int HD, int G>
int launch_f32(const PagedDecodeArgs &a, hipStream_t s) {
  const int ranges = a.first[a.batch];
  const dim3 grid(ranges, a.n_kv_heads, (a.group + G - 1) / G);
  const bool wide = HD == 128 && (int64_t)grid.x * grid.y * grid.z <= 512;
  if (a.weight != nullptr) {
    if (wide) hipLaunchKernelGGL((paged_f32_kernel<HD, G, 8, 1>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((paged_f32_kernel<HD, G, 4, 1>), grid, dim3(256), 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((paged_f32_kernel<HD, G, 8, 0>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((paged_f32_kernel<HD, G, 4, 0>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

template <int HD>
int launch_decode_hd(int dtype, const PagedDecodeArgs &a, hipStream_t s) {
  const int G = paged_decode_heads(dtype, a.group), ranges = a.first[a.batch];
  int rc;
  if (dtype != CHUNKKV_F32) rc = launch_paged_mfma(dtype, HD, a, s);
  else rc = G == 1 ? launch_f32<HD, 1>(a, s) : (G == 2 ? launch_f32<HD, 2>(a, s) : launch_f32<HD, 4>(a, s));
  if (rc || a.alone) return rc;
  const int joins = a.direct ? 0 : a.batch * a.n_q_heads;
  if (a.weight != nullptr) hipLaunchKernelGGL((paged_finish_kernel<HD, 1>), dim3(joins + ranges * a.n_kv_heads), dim3(kThreads), 0, s, a, joins);
  else if (joins > 0) hipLaunchKernelGGL((paged_finish_kernel<HD, 0>), dim3(joins), dim3(kThreads), 0, s, a, joins);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_decode(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s) {
  return head_dim == 128 ? launch_decode_hd<128>(dtype, a, s) : launch_decode_hd<64>(dtype, a, s);
}

}  // namespace ckv
