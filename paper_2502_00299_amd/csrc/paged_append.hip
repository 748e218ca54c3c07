// New tokens of a paged cache: head norm and rotation of queries and keys, keys and values into their slots.
//
// A row (one head of one token) is spread over LPR = d * element size / 16 lanes, 16 bytes each; a wavefront takes 64 / LPR
// rows at a time, a key row together with its value row, so the slot's address is formed once for both and kv_len[b][h]
// has one reader per token.  Per row: sum of squares over the lanes (DPP), scale, rotation, one rounding, store.
// Bound by HBM for prompts (8192 tokens of 32 + 8 + 8 heads, bf16, 38 us, 5.3 TB/s), by latency for single ones (8 tokens 3.6 us from a graph).
// Angles: position * inv_freq / 2 pi in double, reduced to a part of a revolution there (off by 3 * 2^-25 of one at a
// position of 2^31, by 2^-34 at 2^20).  Sine and cosine in fp32 of that part rounded to fp32, which takes up to 2^-26 of a
// revolution or 1.6 * 2^-24 in radians from it, and the first-order step back over what was taken (0.03 us of a single token's
// 3.0).  All rows of a token have the same angles: a wavefront's row groups form a share of them each and exchange them, once
// for all the rows that it takes.
// The two halves of a pair lie in lanes LPR/2 apart where the whole head turns (one or two DPP moves), further in where a
// part of it does, in one lane where neighbours are pairs.
#include "paged.h"
#include "rotary.h"

namespace ckv {

template <int DT, int HD, int TURN>
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

  // Element e of this lane turns by (cs[e], sn[e]) with its partner's value; the second of a pair adds what the first subtracts.
  const int x0 = seg * EPL, half = a.rotary / 2;
  const bool turns = TURN == kWhole || x0 < a.rotary;
  constexpr int NA = TURN == kNeighbours ? EPL / 2 : EPL;           // angles of a lane
  constexpr int CNT = NA > RPW ? NA / RPW : 1;                      // of which a row group forms so many
  float cs[TURN == kNone ? 1 : NA], sn[TURN == kNone ? 1 : NA];
  if constexpr (TURN != kNone) {
    float c_own[CNT], s_own[CNT];
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
      const int k = (grp * CNT + i) % NA;
      const int f = TURN == kNeighbours ? x0 / 2 + k : (x0 < half ? x0 + k : x0 - half + k);
      double rev = turns ? (double)position * (double)a.inv_freq[f] * 0.15915494309189535 : 0.0;
      rev -= __builtin_rint(rev);
      const float part = (float)rev, rest = (float)(rev - (double)part) * 6.2831853f;   // in radians
      float s, c;
      sincospif(2.f * part, &s, &c);
      s_own[i] = __builtin_fmaf(c, rest, s);
      c_own[i] = __builtin_fmaf(-s, rest, c);
    }
#pragma unroll
    for (int k = 0; k < NA; ++k) {
      const int from = (k / CNT) * LPR + seg;
      cs[k] = __shfl(c_own[k % CNT], from);
      sn[k] = __shfl(s_own[k % CNT], from);
      if (TURN != kNeighbours && x0 < half) sn[k] = -sn[k];
    }
  }
  int partner = lane;
  if (TURN == kFront && turns) partner = x0 < half ? lane + half / EPL : lane - half / EPL;
  float wq[EPL], wk[EPL];
  u32x4 raw = {0, 0, 0, 0};
  if (a.q_norm != nullptr) raw = *(const u32x4 *)((const char *)a.q_norm + seg * 16);
  widen<DT, EPL>(raw, wq);
  if (a.k_norm != nullptr) raw = *(const u32x4 *)((const char *)a.k_norm + seg * 16);
  widen<DT, EPL>(raw, wk);

  const int max_tokens = CKV_ARG(PagedAppendArgs, max_tokens, bl);
  const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
  const bool last = t + 1 == (bl + 1 < a.batch ? CKV_ARG(PagedAppendArgs, first, bl + 1) : a.tokens);
  // rows of the next round are on their way while those of this one are worked on
  u32x4 x_next = {0, 0, 0, 0}, v_next = {0, 0, 0, 0};
  auto load = [&](int item) __attribute__((always_inline)) {
    if (item < items) {
      const char *from = item < nq ? (const char *)a.q + tok * a.q_tok + (int64_t)item * ROWB : (const char *)a.k + tok * a.k_tok + (int64_t)(item - nq) * ROWB;
      x_next = __builtin_nontemporal_load((const u32x4 *)(from + seg * 16));
      if (item >= nq) v_next = __builtin_nontemporal_load((const u32x4 *)((const char *)a.v + tok * a.v_tok + (int64_t)(item - nq) * ROWB + seg * 16));
    }
  };
  load(part * RPW + grp);
  for (int i0 = part * RPW; i0 < items; i0 += a.parts * RPW) {
    const int item = i0 + grp;
    u32x4 x = x_next;
    const u32x4 val = v_next;
    load(item + a.parts * RPW);
    const bool is_q = item < nq, is_kv = item >= nq && item < items;
    const int h = item - nq;   // kv-head
    int64_t at = -1;
    if (is_kv) {
      const int64_t bh = (int64_t)b * a.n_kv_heads + h;
      int n = a.kv_len[bh];
      n = n < 0 ? 0 : (n > max_tokens ? max_tokens : n);
      const int slot = n + nth;   // at most 2^24 and as many new tokens
      if (slot < max_tokens) {
        at = slot_offset(a.geom, table, h, slot);
        if (seg == 0) {
          if (a.token_pos != nullptr) a.token_pos[bh * a.slot_pitch + slot] = position;
          if (a.token_weight != nullptr) a.token_weight[bh * a.slot_pitch + slot] = 0.f;
        }
      }
      if (seg == 0 && a.write_len && last) a.kv_len_out[bh] = slot + 1 < max_tokens ? slot + 1 : max_tokens;
    }
    const bool norm = is_q ? a.q_norm != nullptr : a.k_norm != nullptr;
    float y[EPL];
    widen<DT, EPL>(x, y);
    if (a.q_norm != nullptr || a.k_norm != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
      ss = row_sum<LPR>(ss);
      const float inv = norm ? 1.0f / sqrtf(ss * (1.0f / HD) + a.eps) : 1.0f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float w = is_q ? wq[e] : wk[e];
        y[e] = y[e] * inv * (norm ? w : 1.0f);
      }
    }
    if constexpr (TURN == kNeighbours) {
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        const float p = y[e], q = y[e + 1], c = turns ? cs[e / 2] : 1.f, s = turns ? sn[e / 2] : 0.f;
        y[e] = __builtin_fmaf(p, c, -q * s);
        y[e + 1] = __builtin_fmaf(q, c, p * s);
      }
    } else if constexpr (TURN != kNone) {
      float z[EPL];
#pragma unroll
      for (int e = 0; e < EPL; ++e) z[e] = TURN == kWhole ? other_half<LPR>(y[e]) : __shfl(y[e], partner);
#pragma unroll
      for (int e = 0; e < EPL; ++e) y[e] = turns ? __builtin_fmaf(y[e], cs[e], z[e] * sn[e]) : y[e];
    }
    if (norm || TURN != kNone) x = narrow<DT, EPL>(y);   // otherwise the bits that came
    if (is_q) {
      *(u32x4 *)((char *)a.q_out + (tok * a.n_q_heads + item) * ROWB + seg * 16) = x;
    } else if (is_kv && at >= 0) {
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

template <int DT, int HD>
int launch_append(const PagedAppendArgs &a, dim3 grid, hipStream_t s) {
  if (a.rotary == 0) hipLaunchKernelGGL((paged_append_kernel<DT, HD, kNone>), grid, dim3(kThreads), 0, s, a);
  else if (a.interleaved) hipLaunchKernelGGL((paged_append_kernel<DT, HD, kNeighbours>), grid, dim3(kThreads), 0, s, a);
  else if (a.rotary == HD) hipLaunchKernelGGL((paged_append_kernel<DT, HD, kWhole>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((paged_append_kernel<DT, HD, kFront>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_append(int dtype, int head_dim, const PagedAppendArgs &args, hipStream_t s) {
  PagedAppendArgs a = args;
  const int rows = 64 / (head_dim * elem_bytes(dtype) / 16);
  const int rounds = ((a.q != nullptr ? a.n_q_heads : 0) + a.n_kv_heads + rows - 1) / rows;   // of a token's rows
  // Wavefronts that share a token: so many that there are 4096, or that each has five rounds, whichever is more; then the fewest with
  // as many rounds each.  us by wavefronts, bf16, 10 rounds: 300 tokens 2 6.2, 4 5.5, 10 4.8; 600: 4 6.7, 5 6.3, 8 8.2; 2080: 1 17.2, 2 14.6, 4 16.1;
  // 8192: 1 39.6, 2 38.4, 4 45.1; 40000: 1 194, 2 184, 4 209; fp32, 20 rounds: 600: 4 10.2, 7 9.7, 8 10.9; 8192: 1 92.9, 3 81.5, 4 78.9, 8 86.5;
  // fp16 of d = 64, 2 rounds: 8192: 1 15.7, 2 19.2.
  int parts = (4096 + a.tokens - 1) / a.tokens;
  if (parts < rounds / 5) parts = rounds / 5;
  if (parts > rounds) parts = rounds;
  const int each = (rounds + parts - 1) / parts;
  a.parts = (rounds + each - 1) / each;
  const dim3 grid((uint32_t)(((int64_t)a.tokens * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
  if (head_dim == 128) {
    if (dtype == CHUNKKV_F32) return launch_append<CHUNKKV_F32, 128>(a, grid, s);
    return dtype == CHUNKKV_BF16 ? launch_append<CHUNKKV_BF16, 128>(a, grid, s) : launch_append<CHUNKKV_F16, 128>(a, grid, s);
  }
  if (dtype == CHUNKKV_F32) return launch_append<CHUNKKV_F32, 64>(a, grid, s);
  return dtype == CHUNKKV_BF16 ? launch_append<CHUNKKV_BF16, 64>(a, grid, s) : launch_append<CHUNKKV_F16, 64>(a, grid, s);
}

int launch_paged_len(const PagedLenArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(paged_len_kernel, dim3((uint32_t)(((int64_t)a.batch * a.n_kv_heads + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
