// Rotation of queries and keys by position, from rows anywhere to rows anywhere.
//
// A row (one head of one token) is spread over LPR = d * element size / 16 lanes, 16 bytes each; a wavefront takes 64 / LPR rows of a
// token at a time, query and key rows alike, with the next ones on their way.  Angles and pairs as in rotary.h: all rows of a token
// share its angles, which a wavefront forms once.  Per row: rotation in fp32, one rounding, store.
// Bound by HBM for prompts (32768 tokens of 40 heads, bf16, d = 128: 671 MB read and written in 125 us, 5.4 TB/s), by the chain position, angle, row
// for a few thousand tokens (4503 of 32 heads, 74 MB: 18.4 us), by one launch for a step (3.4 us in a graph, 7.5 with the host's checks).
// Twice (four times) as many wavefronts to a token: 4096 tokens 17.9 -> 18.0 (19.4) us, 9000 half-rotated ones 32.7 -> 32.6 (29.8); two rows ahead
// instead of one: the same.
#include "rotary.h"
#include "rows.h"

namespace ckv {

template <int DT, int HD, int TURN>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
  constexpr int ESZ = DT == CHUNKKV_F32 ? 4 : 2, ROWB = HD * ESZ;
  constexpr int LPR = ROWB / 16, RPW = 64 / LPR, EPL = 16 / ESZ;
  const int lane = threadIdx.x & 63, seg = lane % LPR, grp = lane / LPR;
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t t = a.parts == 1 ? unit : unit / a.parts;
  const int part = (int)(unit - t * a.parts);
  if (t >= a.tokens) return;
  const int64_t seq = a.tokens == a.n_tokens ? 0 : t / a.n_tokens, tok = t - seq * a.n_tokens;
  const int x0 = seg * EPL, items = a.q.heads + a.k.heads;
  const bool turns = TURN == kWhole || x0 < a.rotary;
  constexpr int NA = lane_angles(TURN, EPL);
  float cs[NA], sn[NA];
  form_angles<TURN, LPR, EPL>(a.positions[t], a.inv_freq, a.rotary, lane, cs, sn);
#pragma unroll
  for (int k = 0; k < NA; ++k) {
    cs[k] *= a.magnitude;
    sn[k] *= a.magnitude;
  }
  const int partner = TURN == kFront ? front_partner<EPL>(a.rotary, lane, x0) : lane;
  const char *q_in = (const char *)a.q.in + seq * a.q.in_seq + tok * a.q.in_tok + seg * 16, *k_in = (const char *)a.k.in + seq * a.k.in_seq + tok * a.k.in_tok + seg * 16;
  char *q_out = (char *)a.q.out + seq * a.q.out_seq + tok * a.q.out_tok + seg * 16, *k_out = (char *)a.k.out + seq * a.k.out_seq + tok * a.k.out_tok + seg * 16;
  u32x4 next = {0, 0, 0, 0};
  auto load = [&](int item) __attribute__((always_inline)) {
    if (item < items) next = __builtin_nontemporal_load((const u32x4 *)(item < a.q.heads ? q_in + item * a.q.in_head : k_in + (item - a.q.heads) * a.k.in_head));
  };
  load(part * RPW + grp);
  for (int i0 = part * RPW; i0 < items; i0 += a.parts * RPW) {
    const int item = i0 + grp;
    u32x4 x = next;
    load(item + a.parts * RPW);
    float y[EPL];
    widen<DT, EPL>(x, y);
    turn_row<TURN, LPR, EPL>(y, cs, sn, turns, partner);
    if (turns) x = narrow<DT, EPL>(y);   // otherwise the bits that came
    const bool is_q = item < a.q.heads;
    if (item < items && (turns || !(is_q ? a.q.front_only : a.k.front_only)))
      *(u32x4 *)(is_q ? q_out + item * a.q.out_head : k_out + (item - a.q.heads) * a.k.out_head) = x;
  }
}

template <int DT, int HD>
int launch_turn(const RotateArgs &a, bool interleaved, dim3 grid, hipStream_t s) {
  if (interleaved) hipLaunchKernelGGL((rotate_kernel<DT, HD, kNeighbours>), grid, dim3(kThreads), 0, s, a);
  else if (a.rotary == HD) hipLaunchKernelGGL((rotate_kernel<DT, HD, kWhole>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((rotate_kernel<DT, HD, kFront>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_rotate(int dtype, int head_dim, bool interleaved, const RotateArgs &args, hipStream_t s) {
  RotateArgs a = args;
  const int rows = 64 / (head_dim * (dtype == CHUNKKV_F32 ? 4 : 2) / 16);
  const int rounds = (a.q.heads + a.k.heads + rows - 1) / rows;   // of a token's rows
  // wavefronts that share a token, as paged_append.hip has them
  int parts = (int)((4096 + a.tokens - 1) / a.tokens);
  if (parts < rounds / 5) parts = rounds / 5;
  if (parts > rounds) parts = rounds;
  const int most = (int)((1 << 25) / a.tokens);   // a grid's row has 2^32 threads
  if (parts > most) parts = most;
  const int each = (rounds + parts - 1) / parts;
  a.parts = (rounds + each - 1) / each;
  const dim3 grid((uint32_t)((a.tokens * a.parts + kThreads / 64 - 1) / (kThreads / 64)));
  if (head_dim == 128) {
    if (dtype == CHUNKKV_F32) return launch_turn<CHUNKKV_F32, 128>(a, interleaved, grid, s);
    return dtype == CHUNKKV_BF16 ? launch_turn<CHUNKKV_BF16, 128>(a, interleaved, grid, s) : launch_turn<CHUNKKV_F16, 128>(a, interleaved, grid, s);
  }
  if (dtype == CHUNKKV_F32) return launch_turn<CHUNKKV_F32, 64>(a, interleaved, grid, s);
  return dtype == CHUNKKV_BF16 ? launch_turn<CHUNKKV_BF16, 64>(a, interleaved, grid, s) : launch_turn<CHUNKKV_F16, 64>(a, interleaved, grid, s);
}

}  // namespace ckv
