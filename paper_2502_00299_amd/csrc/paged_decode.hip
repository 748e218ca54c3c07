// Attention of one new token per sequence over pages, and what every slot received of it.
//
// out_i = sum_s softmax_s(scale * q_i . k_s) v_s over the slots of a kv-head; a head's slots are cut into key ranges, each a
// workgroup that leaves (maximum, sum, weighted values) of its rows, joined afterwards in range order.
// This file holds the vector-ALU range kernel and the join.
//
// A row is spread over LPR = d * element size / 16 lanes, 16 bytes each; the lanes of a row reduce their partial dot
// products with DPP adds, each group of LPR lanes runs its own online softmax over the rows it meets, and groups,
// wavefronts and ranges are merged by the (max, sum, weighted output) rule, always in the same order.  The addresses of a
// range's 16-row blocks are looked up once, by one lane each, and kept in LDS.
#include "paged.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr float kNegBig = -1.0e30f, kMasked = -3.0e38f;

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_amdgcn_update_dpp(0.f, x, CTRL, 0xf, 0xf, false);
}
// Sum over the LPR lanes that share a row; every lane of the group ends with the same bits.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x = dpp_add<0xB1>(x);                            // quad_perm [1,0,3,2]
  x = dpp_add<0x4E>(x);                            // quad_perm [2,3,0,1]
  if constexpr (LPR >= 8) x = dpp_add<0x141>(x);   // row_half_mirror: the other quad of 8 lanes
  if constexpr (LPR >= 16) x = dpp_add<0x140>(x);  // row_mirror: the other half of 16 lanes
  if constexpr (LPR >= 32) x += __shfl_xor(x, 16);
  return x;
}
template <int DT, int EPL>
__device__ __forceinline__ void widen(const u32x4 &r, float (&f)[EPL]) {
  if constexpr (DT == CHUNKKV_F32) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  } else if constexpr (DT == CHUNKKV_BF16) {
    const bf16x8 x = __builtin_bit_cast(bf16x8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)x[i];
  } else {
    const f16x8 x = __builtin_bit_cast(f16x8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)x[i];
  }
}

// DT: chunkkv_dtype, HD: head dim, G: query heads of a workgroup, W: 1 = the scores are kept for the weights
template <int DT, int HD, int G, int W>
__global__ __launch_bounds__(kThreads) void paged_decode_kernel(PagedDecodeArgs a) {
  constexpr int ESZ = DT == CHUNKKV_F32 ? 4 : 2, ROWB = HD * ESZ;
  constexpr int LPR = ROWB / 16, RPW = 64 / LPR, EPL = 16 / ESZ, U = 4, NW = kThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane / LPR, seg = lane % LPR;
  const int h = blockIdx.y, j0 = blockIdx.z * G;
  const int bl = CKV_PAGED_SEQUENCE(PagedDecodeArgs, (int)blockIdx.x, a.batch), b = a.batch0 + bl;
  const int split = blockIdx.x - CKV_ARG(PagedDecodeArgs, first, bl), splits = paged_splits(bl);
  const int n = paged_length(a, bl, h), rps = paged_range_rows(n, splits);
  const int r0 = split * rps, r1 = r0 + rps < n ? r0 + rps : n;
  if (r0 >= n && split > 0) return;   // the join knows how many ranges hold rows

  __shared__ int64_t s_block[kPagedMaxRange / 16];
  for (int i = threadIdx.x; r0 + 16 * i < r1; i += kThreads)
    s_block[i] = block_offset(a.geom, a.geom.table + (int64_t)b * a.geom.pitch, h, (uint32_t)(r0 / 16 + i));
  __syncthreads();

  const char *kbase = (const char *)a.k + seg * 16, *vbase = (const char *)a.v + seg * 16;
  float qf[G][EPL];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    u32x4 r = {0, 0, 0, 0};
    if (j0 + j < a.group) r = *(const u32x4 *)((const char *)a.q + ((int64_t)b * a.n_q_heads + (int64_t)h * a.group + j0 + j) * ROWB + seg * 16);
    widen<DT, EPL>(r, qf[j]);
  }
  float m[G], l[G], o[G][EPL];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    m[j] = kNegBig;
    l[j] = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[j][e] = 0.f;
  }
  const float c1 = a.scale_log2e;
  for (int base = r0 + wave * (U * RPW); base < r1; base += NW * U * RPW) {
    u32x4 kr[U], vr[U];
    bool valid[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = base + u * RPW + grp;
      const int64_t at = row < r1 ? s_block[(row - r0) >> 4] : -1;
      valid[u] = at >= 0;
      kr[u] = vr[u] = u32x4{0, 0, 0, 0};   // rows that are not there count as zeros, whatever is in memory
      if (valid[u]) {
        const int64_t off = at + (int64_t)(row & 15) * a.geom.tok;
        kr[u] = __builtin_nontemporal_load((const u32x4 *)(kbase + off));
        vr[u] = __builtin_nontemporal_load((const u32x4 *)(vbase + off));
      }
    }
    float s[U][G];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float kf[EPL];
      widen<DT, EPL>(kr[u], kf);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        float d = kf[0] * qf[j][0];
#pragma unroll
        for (int e = 1; e < EPL; ++e) d = __builtin_fmaf(kf[e], qf[j][e], d);
        d = row_sum<LPR>(d);
        s[u][j] = valid[u] ? d * c1 : kMasked;
      }
    }
    if constexpr (W != 0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = base + u * RPW + grp;
#pragma unroll
        for (int j = 0; j < G; ++j)
          if (seg == j && row < r1 && j0 + j < a.group) head_scores(a, bl, h * a.group + j0 + j)[row] = s[u][j];
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
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[j][e] *= f;
        m[j] = m_new;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) s[u][j] = __builtin_amdgcn_exp2f(s[u][j] - m[j]);   // now the weight
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float vf[EPL];
      widen<DT, EPL>(vr[u], vf);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        l[j] += s[u][j];
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[j][e] = __builtin_fmaf(s[u][j], vf[e], o[j][e]);
      }
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
      for (int e = 0; e < EPL; ++e) o[j][e] = o[j][e] * fa + __shfl_xor(o[j][e], x) * fb;
      m[j] = M;
    }
  }
  // the wavefronts, through LDS: thread (j, seg) folds their states in order
  __shared__ float s_m[NW][G][LPR], s_l[NW][G][LPR], s_o[NW][G][LPR][EPL];
  if (grp == 0) {
#pragma unroll
    for (int j = 0; j < G; ++j) {
      s_m[wave][j][seg] = m[j];
      s_l[wave][j][seg] = l[j];
#pragma unroll
      for (int e = 0; e < EPL; ++e) s_o[wave][j][seg][e] = o[j][e];
    }
  }
  __syncthreads();
  const int t = threadIdx.x, j = t / LPR, sg = t % LPR;
  if (t >= G * LPR || j0 + j >= a.group) return;
  float M = s_m[0][j][sg];
#pragma unroll
  for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][j][sg]);
  float L = 0.f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = __builtin_amdgcn_exp2f(s_m[w][j][sg] - M);
    L += s_l[w][j][sg] * f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] += s_o[w][j][sg][e] * f;
  }
#pragma unroll
  for (int e = 0; e < EPL; ++e) store_range<HD>(a, b, h * a.group + j0 + j, sg * EPL + e, M, L, acc[e]);
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

template <int HD>
int launch_decode_hd(int dtype, const PagedDecodeArgs &a, hipStream_t s) {
  const int G = paged_decode_heads(dtype, a.group), ranges = a.first[a.batch];
  if (dtype != CHUNKKV_F32) {
    const int rc = launch_paged_mfma(dtype, HD, a, s);
    if (rc) return rc;
  } else {
    const dim3 grid(ranges, a.n_kv_heads, (a.group + G - 1) / G);
    auto go = [&](auto g) {
      constexpr int GG = decltype(g)::value;
      if (a.weight != nullptr) hipLaunchKernelGGL((paged_decode_kernel<CHUNKKV_F32, HD, GG, 1>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((paged_decode_kernel<CHUNKKV_F32, HD, GG, 0>), grid, dim3(kThreads), 0, s, a);
    };
    if (G == 1) go(std::integral_constant<int, 1>{});
    else if (G == 2) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 4>{});
    if (hipGetLastError() != hipSuccess) return CHUNKKV_ERR_LAUNCH;
  }
  const int joins = a.direct ? 0 : a.batch * a.n_q_heads;
  if (a.weight != nullptr) hipLaunchKernelGGL((paged_finish_kernel<HD, 1>), dim3(joins + ranges * a.n_kv_heads), dim3(kThreads), 0, s, a, joins);
  else if (joins > 0) hipLaunchKernelGGL((paged_finish_kernel<HD, 0>), dim3(joins), dim3(kThreads), 0, s, a, joins);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_decode(int dtype, int head_dim, const PagedDecodeArgs &a, hipStream_t s) {
  return head_dim == 128 ? launch_decode_hd<128>(dtype, a, s) : launch_decode_hd<64>(dtype, a, s);
}

}  // namespace ckv
