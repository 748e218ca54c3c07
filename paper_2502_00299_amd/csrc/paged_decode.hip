// Attention of one new token per sequence over pages, and what every slot received of it.
//
// out_i = sum_s softmax_s(scale * q_i . k_s) v_s over the slots of a kv-head; a head's slots are cut into key ranges, each a
// workgroup that leaves (maximum, sum, weighted values) of its rows, joined afterwards in range order.  The range kernels are in
// paged_decode_mfma.hip (16-bit pages) and paged_decode_f32.hip; this file holds the launch behind them.
#include "paged.h"

namespace ckv {

// The launch behind the ranges.
//
// Its first `joins` workgroups join a query head each: out = sum_r o_r f_r / sum_r l_r f_r, f_r = 2^(c (m_r - M)), c the scale in log2 units.  A thread owns four
// columns and every so many-th range, four of them in flight; the groups of ranges are folded through LDS in order.
// With weights (W = 1) the others add token_weight[s] += sum_i 2^(c (x_i(s) - M_i)) / L_i to the slots of one key range of one kv-head,
// heads in order: the scores of the first four heads are on their way while M_i and 1 / L_i are formed from all ranges' pairs.
template <int HD, int W>
__global__ __launch_bounds__(kThreads) void paged_finish_kernel(PagedDecodeArgs a, int joins) {
  constexpr int TPR = HD / 4, NG = kThreads / TPR, UN = 4;
  __shared__ float s_acc[NG][HD + 2];
  __shared__ HeadNorm s_norm[W != 0 ? kPagedMaxGroup : 1];
  const int t = threadIdx.x;
  const float c1 = a.scale_log2e;
  if (W == 0 || (int)blockIdx.x < joins) {
    const int bl = blockIdx.x / a.n_q_heads, hq = blockIdx.x % a.n_q_heads, col = t % TPR, grp = t / TPR;
    const int n = paged_length(a, bl, hq / a.group), rps = paged_range_rows(n, paged_splits(bl)), used = n > 0 ? (n + rps - 1) / rps : 1;
    const int64_t slot = (int64_t)CKV_ARG(PagedDecodeArgs, first, bl) * a.n_q_heads + hq;
    const float2 *ml = a.part_ml + slot;
    const float *po = a.part_o + slot * HD + col * 4;
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, m = kPagedLowest, lsum = 0.f;
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
      const float f0 = __builtin_amdgcn_exp2f((m - mm) * c1);
      lsum *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const float f = r0 + u * NG < used ? __builtin_amdgcn_exp2f((p[u].x - mm) * c1) : 0.f;
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
        const float f = __builtin_amdgcn_exp2f((s_acc[g][HD + 1] - M) * c1);
        v += s_acc[g][t] * f;
        L += s_acc[g][HD] * f;
      }
      const int64_t head = (int64_t)(a.batch0 + bl) * a.n_q_heads + hq;
      a.out[head * HD + t] = L > 0.f ? v / L : 0.f;
      if (a.lse != nullptr && t == 0) a.lse[head] = log_sum_exp(a, M, L);
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
          sx[j][i] = -__builtin_inff();
          if (j0 + j < a.group && t + i * kThreads < len) sx[j][i] = __builtin_nontemporal_load(scores + (int64_t)(j0 + j) * pitch + t + i * kThreads);   // for the last time
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
      float m = kPagedLowest, l = 0.f;
      for (int r = lane; r < used; r += 64) {
        const float2 p = a.part_ml[(int64_t)(first + r) * a.n_q_heads + h * a.group + j];
        const float mm = fmaxf(m, p.x);
        l = l * __builtin_amdgcn_exp2f((m - mm) * c1) + p.y * __builtin_amdgcn_exp2f((p.x - mm) * c1);
        m = mm;
      }
      float M = m;
      for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
      l *= __builtin_amdgcn_exp2f((m - M) * c1);
      for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
      if (lane == 0) s_norm[j] = head_norm(M, l);
    }
    __syncthreads();
    for (int j0 = 0;;) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const HeadNorm norm = j0 + j < a.group ? s_norm[j0 + j] : HeadNorm{0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NR; ++i) sum[i] += __builtin_amdgcn_exp2f((sx[j][i] - norm.ref) * c1) * norm.inv;
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

template <int HD>
int launch_finish(const PagedDecodeArgs &a, hipStream_t s) {
  const int joins = a.direct ? 0 : a.batch * a.n_q_heads, ranges = a.first[a.batch];
  if (a.weight != nullptr) hipLaunchKernelGGL((paged_finish_kernel<HD, 1>), dim3(joins + ranges * a.n_kv_heads), dim3(kThreads), 0, s, a, joins);
  else if (joins > 0) hipLaunchKernelGGL((paged_finish_kernel<HD, 0>), dim3(joins), dim3(kThreads), 0, s, a, joins);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_decode(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s) {
  const int rc = dtype == CHUNKKV_F32 ? launch_paged_f32(head_dim, a, s) : launch_paged_mfma(dtype, head_dim, a, s);
  if (rc || a.alone) return rc;
  return head_dim == 128 ? launch_finish<128>(a, s) : launch_finish<64>(a, s);
}

}  // namespace ckv
