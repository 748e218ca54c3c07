// New tokens of a paged cache: head norm and rotation of queries and keys, keys and values into their slots.
//
// A row (one head of one token) is spread over LPR = d * element size / 16 lanes, 16 bytes each; a wavefront takes 64 / LPR
// rows at a time, a key row together with its value row, so the slot's address is formed once for both and kv_len[b][h]
// has one reader per token.  Per row: sum of squares over the lanes, scale, rotation, one rounding, store.  All rows of a
// token have the same angles, so a wavefront that takes several of them computes sines and cosines once; its lanes hold
// those of their own elements.
// Angles: position * inv_freq / 2 pi in double, reduced to a part of a revolution there (off by 3 * 2^-25 of one at a
// position of 2^31, by 2^-34 at 2^20), sine and cosine of that part in fp32.
// Bound by bytes for a prompt (every row is read and written once), by latency for single tokens.
#include "paged.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int DT, int EPL>
__device__ __forceinline__ void widen(const u32x4 &r, float (&f)[EPL]) {
  if constexpr (DT == CHUNKKV_F32) {
    const f32x4 x = __builtin_bit_cast(f32x4, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = x[i];
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
template <int DT, int EPL>
__device__ __forceinline__ u32x4 narrow(const float (&f)[EPL]) {   // to nearest, ties to even
  if constexpr (DT == CHUNKKV_F32) {
    return __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]});
  } else if constexpr (DT == CHUNKKV_BF16) {
    bf16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)f[i];
    return __builtin_bit_cast(u32x4, x);
  } else {
    f16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (_Float16)f[i];
    return __builtin_bit_cast(u32x4, x);
  }
}

template <int DT, int HD>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int ESZ = DT == CHUNKKV_F32 ? 4 : 2, ROWB = HD * ESZ;
  constexpr int LPR = ROWB / 16, RPW = 64 / LPR, EPL = 16 / ESZ;
  const int lane = threadIdx.x & 63, seg = lane % LPR, grp = lane / LPR;
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x * (kThreads / 64) + (int)(threadIdx.x >> 6));
  const int t = unit / a.parts, part = unit - t * a.parts;
  if (t >= a.tokens) return;
  const int bl = CKV_PAGED_SEQUENCE(PagedAppendArgs, t, a.batch), b = a.batch0 + bl;
  const int nth = t - CKV_ARG(PagedAppendArgs, first, bl);
  const int64_t tok = (int64_t)a.token0 + t;
  const int32_t position = a.positions[tok];
  const int nq = a.q != nullptr ? a.n_q_heads : 0, items = nq + a.n_kv_heads;

  // rotation of this lane's elements seg * EPL ..: element e turns by (cs[e], sn[e]) with its partner's value
  const int x0 = seg * EPL, half = a.rotary / 2;
  const bool turns = x0 < a.rotary;
  float cs[EPL], sn[EPL];
  int partner = lane;
  if (a.rotary > 0) {
    if (!a.interleaved && turns) partner = x0 < half ? lane + half / EPL : lane - half / EPL;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const int i = a.interleaved ? (x0 + e) / 2 : (x0 < half ? x0 + e : x0 - half + e);
      double rev = 0.0;
      if (turns) rev = (double)position * (double)a.inv_freq[i] * 0.15915494309189535;
      rev -= __builtin_rint(rev);
      float s, c;
      sincospif(2.f * (float)rev, &s, &c);
      cs[e] = c;
      // the second of a pair adds what the first subtracts
      sn[e] = (a.interleaved ? (e & 1) != 0 : x0 >= half) ? s : -s;
      if (!turns) { cs[e] = 1.f; sn[e] = 0.f; }
    }
  }
  float wq[EPL], wk[EPL];
  u32x4 raw = {0, 0, 0, 0};
  if (a.q_norm != nullptr) raw = *(const u32x4 *)((const char *)a.q_norm + seg * 16);
  widen<DT, EPL>(raw, wq);
  if (a.k_norm != nullptr) raw = *(const u32x4 *)((const char *)a.k_norm + seg * 16);
  widen<DT, EPL>(raw, wk);

  const int max_tokens = CKV_ARG(PagedAppendArgs, max_tokens, bl);
  for (int i0 = part * RPW; i0 < items; i0 += a.parts * RPW) {
    const int item = i0 + grp;
    if (item >= items) continue;
    const bool is_q = item < nq;
    const int h = item - nq;   // kv-head
    const char *from = is_q ? (const char *)a.q + tok * a.q_tok + (int64_t)item * ROWB : (const char *)a.k + tok * a.k_tok + (int64_t)h * ROWB;
    u32x4 x = *(const u32x4 *)(from + seg * 16), val = {0, 0, 0, 0};
    int64_t at = -1;
    if (!is_q) {
      val = *(const u32x4 *)((const char *)a.v + tok * a.v_tok + (int64_t)h * ROWB + seg * 16);
      const int64_t bh = (int64_t)b * a.n_kv_heads + h;
      int n = a.kv_len[bh];
      n = n < 0 ? 0 : (n > max_tokens ? max_tokens : n);
      const int slot = n + nth;   // below 2^31: both are at most 2^24 more than a count of tokens
      if (slot < max_tokens) {
        at = slot_offset(a.geom, a.geom.table + (int64_t)b * a.geom.pitch, h, slot);
        if (seg == 0) {
          if (a.token_pos != nullptr) a.token_pos[bh * a.slot_pitch + slot] = position;
          if (a.token_weight != nullptr) a.token_weight[bh * a.slot_pitch + slot] = 0.f;
        }
      }
      if (seg == 0 && a.write_len && t + 1 == (bl + 1 < a.batch ? CKV_ARG(PagedAppendArgs, first, bl + 1) : a.tokens))
        a.kv_len_out[bh] = slot + 1 < max_tokens ? slot + 1 : max_tokens;
    }
    const bool norm = is_q ? a.q_norm != nullptr : a.k_norm != nullptr;
    float y[EPL];
    widen<DT, EPL>(x, y);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if (norm) {
      const float inv = 1.0f / sqrtf(ss * (1.0f / HD) + a.eps);
#pragma unroll
      for (int e = 0; e < EPL; ++e) y[e] = y[e] * inv * (is_q ? wq[e] : wk[e]);
    }
    if (a.rotary > 0) {
      float z[EPL];
#pragma unroll
      for (int e = 0; e < EPL; ++e) z[e] = a.interleaved ? y[e ^ 1] : __shfl(y[e], partner);
#pragma unroll
      for (int e = 0; e < EPL; ++e) y[e] = turns ? __builtin_fmaf(y[e], cs[e], z[e] * sn[e]) : y[e];
    }
    if (norm || a.rotary > 0) x = narrow<DT, EPL>(y);   // otherwise the bits that came
    if (is_q) {
      *(u32x4 *)((char *)a.q_out + (tok * a.n_q_heads + item) * ROWB + seg * 16) = x;
    } else if (at >= 0) {
      *(u32x4 *)((char *)a.k_pages + at + seg * 16) = x;
      *(u32x4 *)((char *)a.v_pages + at + seg * 16) = val;
    }
  }
}

__global__ __launch_bounds__(kThreads) void paged_len_kernel(PagedLenArgs a) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.batch * a.n_kv_heads) return;
  const int bl = i / a.n_kv_heads;
  const int64_t bh = (int64_t)a.batch0 * a.n_kv_heads + i;
  const int64_t most = a.max_tokens[bl];
  int64_t n = a.kv_len[bh];
  n = (n < 0 ? 0 : (n > most ? most : n)) + a.n_new[bl];
  a.kv_len_out[bh] = (int32_t)(n < most ? n : most);
}

template <int DT>
int launch_append(int head_dim, const PagedAppendArgs &a, dim3 grid, hipStream_t s) {
  if (head_dim == 128) hipLaunchKernelGGL((paged_append_kernel<DT, 128>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((paged_append_kernel<DT, 64>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_append(int dtype, int head_dim, const PagedAppendArgs &args, hipStream_t s) {
  PagedAppendArgs a = args;
  if (a.tokens == 0) return CHUNKKV_OK;
  const int rows = 64 / (head_dim * elem_bytes(dtype) / 16);
  const int groups = ((a.q != nullptr ? a.n_q_heads : 0) + a.n_kv_heads + rows - 1) / rows;   // loads of a token's rows
  int parts = (int)((4096 + a.tokens - 1) / a.tokens);
  a.parts = parts > groups ? groups : parts;
  const dim3 grid((uint32_t)(((int64_t)a.tokens * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
  if (dtype == CHUNKKV_F32) return launch_append<CHUNKKV_F32>(head_dim, a, grid, s);
  if (dtype == CHUNKKV_BF16) return launch_append<CHUNKKV_BF16>(head_dim, a, grid, s);
  return launch_append<CHUNKKV_F16>(head_dim, a, grid, s);
}

int launch_paged_len(const PagedLenArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(paged_len_kernel, dim3((uint32_t)(((int64_t)a.batch * a.n_kv_heads + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
