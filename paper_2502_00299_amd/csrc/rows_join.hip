// Partial rows of attention to their outputs: out = sum_i o_i f_i / sum_i l_i f_i, f_i = 2^(c (m_i - M)), over the ranges of a row's own
// segment and, behind a shared prefix, those of the prefix, in this order.
//
// HD / 4 threads have a row's columns, four each; G groups of them share a row's partials (four of them in flight) and are added up
// through LDS in order.  Bound by latency where there are few rows: a workgroup to a row then; by reading the partial rows otherwise: a
// group to a row.  One token of 32 heads over 13171 keys with either: 15.9 and 20.9 us for the call, 61 tokens (1952 rows): 31.0 and 31.5, 100
// tokens (3200 rows): 43.3 and 41.9.  16 MB of them (1952 rows of 16 ranges, d = 128) take 5.0 us, 35 MB (2048 rows of 33) 8.9.
#include "rotary.h"
#include "rows.h"

namespace ckv {

template <int DT, int HD, int G>
__global__ __launch_bounds__(kThreads) void rows_join_kernel(JoinArgs a) {
  constexpr int TPR = HD / 4, RPB = kThreads / (TPR * G), UN = 4;
  __shared__ f32x4 s_acc[G > 1 ? G : 1][TPR];
  __shared__ float s_m[G], s_l[G], s_e[G];
  const int t = threadIdx.x, col = t % TPR, grp = G > 1 ? t / TPR : 0, hkv = (int)a.heads.d, g = (int)a.group.d, hq_all = hkv * g;
  const int64_t x = (int64_t)blockIdx.x * RPB + (G > 1 ? 0 : t / TPR);
  if (x >= (int64_t)a.tokens * hq_all) return;   // with groups, a whole workgroup
  const int token = (int)(x / hq_all), hq = (int)(x - (int64_t)token * hq_all), h = divided(hq, a.group), j = hq - h * g;
  // segment of the token; the rows of a workgroup may belong to several
  int s = token;
  if (a.segments != a.tokens) {
    s = 0;
    for (int i = 1; i < a.segments; ++i) s += token >= kernarg_at<int32_t>(offsetof(JoinArgs, first), i) ? 1 : 0;
  }
  const size_t place = offsetof(JoinArgs, segment) + s * sizeof(JoinSegment);
  auto number = [&](int i) { return kernarg_at<int32_t>(place, i); };
  const JoinSegment seg = {number(0), number(1), number(2), number(3), number(4), number(5), number(6), number(7), kernarg_at<int64_t>(place + 32, 0)};
  const int nth = a.segments != a.tokens ? token - kernarg_at<int32_t>(offsetof(JoinArgs, first), s) : 0;
  const int own = seg.splits, all = own + seg.prefix_splits;
  const int64_t at = seg.part + (int64_t)h * seg.rows + (int64_t)nth * g + j;
  const int64_t prefix_at = seg.prefix_part + (int64_t)h * seg.prefix_rows + seg.prefix_row0 + (int64_t)nth * g + j;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = kPagedLowest, l = 0.f, le = 0.f;
  const float c1 = a.scale_log2e;
  for (int i0 = grp; i0 < all; i0 += UN * G) {
    float4 ml[UN];
    f32x4 o[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = i0 + u * G < all ? i0 + u * G : i0;
      const int64_t p = i < own ? at + (int64_t)i * hkv * seg.rows : prefix_at + (int64_t)(i - own) * hkv * seg.prefix_rows;
      ml[u] = a.part_ml[p];
      o[u] = *(const f32x4 *)(a.part_o + p * HD + col * 4);
    }
    float mm = m;
#pragma unroll
    for (int u = 0; u < UN; ++u) mm = fmaxf(mm, ml[u].x);
    const float f0 = __builtin_amdgcn_exp2f((m - mm) * c1);
    l *= f0;
    le *= f0;
    acc *= f0;
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const float f = i0 + u * G < all ? __builtin_amdgcn_exp2f((ml[u].x - mm) * c1) : 0.f;
      l += ml[u].y * f;
      le += ml[u].z * f;
      acc += o[u] * f;
    }
    m = mm;
  }
  if constexpr (G > 1) {
    s_acc[grp][col] = acc;
    if (col == 0) { s_m[grp] = m; s_l[grp] = l; s_e[grp] = le; }
    __syncthreads();
    if (grp != 0) return;
    float M = s_m[0];
#pragma unroll
    for (int i = 1; i < G; ++i) M = fmaxf(M, s_m[i]);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    l = le = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const float f = __builtin_amdgcn_exp2f((s_m[i] - M) * c1);
      l += s_l[i] * f;
      le += s_e[i] * f;
      acc += s_acc[i][col] * f;
    }
    m = M;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  char *to = (char *)a.out + seg.out_base + nth * a.out_tok + hq * a.out_head;
  if constexpr (DT == CHUNKKV_F32) {
    *(f32x4 *)(to + col * 16) = acc * inv;
  } else if constexpr (DT == CHUNKKV_BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *(bf16x4 *)(to + col * 8) = __builtin_convertvector(acc * inv, bf16x4);
  } else {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    *(f16x4 *)(to + col * 8) = __builtin_convertvector(acc * inv, f16x4);
  }
  if (a.lse != nullptr && col == 0)
    a.lse[(int64_t)(seg.token0 + nth) * hq_all + hq] = le > 0.f ? __builtin_fmaf(m, a.scale, __builtin_log2f(le) * 0.6931471805599453f) : -__builtin_inff();
}

template <int DT, int HD>
int launch_join_of(const JoinArgs &a, hipStream_t s) {
  constexpr int TPR = HD / 4, G = kThreads / TPR;
  const int64_t rows = (int64_t)a.tokens * (int)(a.heads.d * a.group.d);
  if (rows <= 2048) hipLaunchKernelGGL((rows_join_kernel<DT, HD, G>), dim3((uint32_t)rows), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((rows_join_kernel<DT, HD, 1>), dim3((uint32_t)((rows + G - 1) / G)), dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_join(int dtype, int head_dim, const JoinArgs &a, hipStream_t s) {
  if (head_dim == 128) {
    if (dtype == CHUNKKV_F32) return launch_join_of<CHUNKKV_F32, 128>(a, s);
    return dtype == CHUNKKV_BF16 ? launch_join_of<CHUNKKV_BF16, 128>(a, s) : launch_join_of<CHUNKKV_F16, 128>(a, s);
  }
  if (dtype == CHUNKKV_F32) return launch_join_of<CHUNKKV_F32, 64>(a, s);
  return dtype == CHUNKKV_BF16 ? launch_join_of<CHUNKKV_BF16, 64>(a, s) : launch_join_of<CHUNKKV_F16, 64>(a, s);
}

}  // namespace ckv
