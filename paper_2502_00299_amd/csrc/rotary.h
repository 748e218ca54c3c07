// Rows in 16 bytes per lane, and pairs of their elements that turn by an angle.
//
// The two halves of a pair lie in lanes LPR/2 apart where the whole head turns (one or two DPP moves), further in where a
// part of it does, in one lane where neighbours are pairs.
#pragma once
#include "internal.h"

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

// Value of the lane LPR / 2 further on in its row.
template <int LPR>
__device__ __forceinline__ float other_half(float x) {
  if constexpr (LPR == 8) {
    const float y = __builtin_amdgcn_update_dpp(0.f, x, 0x141, 0xf, 0xf, false);   // row_half_mirror: 7 - i
    return __builtin_amdgcn_update_dpp(0.f, y, 0x1B, 0xf, 0xf, false);             // quad_perm [3,2,1,0]
  } else if constexpr (LPR == 16) {
    return __builtin_amdgcn_update_dpp(0.f, x, 0x128, 0xf, 0xf, false);            // row_ror:8
  } else {
    return __shfl_xor(x, 16);
  }
}

// How rows turn: not at all (new tokens of a cache alone), whole heads by halves, the front of a head by halves, neighbours.
enum Turn { kNone, kWhole, kFront, kNeighbours };

// Cosine and sine of position * inv_freq, by the steps of paged_append.hip, which says how far off they are.  That kernel keeps a text of its own of these
// steps and of the pairs' below: with this one the compiler joins other products and sums, which moves a last bit here and there of what it has always stored.
struct Turned {
  float cos, sin;
};
__device__ __forceinline__ Turned turned(int32_t position, float inv_freq) {
  double rev = (double)position * (double)inv_freq * 0.15915494309189535;
  rev -= __builtin_rint(rev);
  const float part = (float)rev, rest = (float)(rev - (double)part) * 6.2831853f;   // in radians
  float s, c;
  sincospif(2.f * part, &s, &c);
  return {__builtin_fmaf(-s, rest, c), __builtin_fmaf(c, rest, s)};
}

// Angles that a lane holds, and those of this lane: element e turns by (cs[e], sn[e]) with its partner's value (neighbours: elements 2 e and
// 2 e + 1); the second of a pair adds what the first subtracts.  The 64 / LPR row groups of a wavefront form a share of them each.
__host__ __device__ constexpr int lane_angles(int turn, int epl) { return turn == kNeighbours ? epl / 2 : epl; }
template <int TURN, int LPR, int EPL>
__device__ __forceinline__ void form_angles(int32_t position, const float *inv_freq, int rotary, int lane, float (&cs)[lane_angles(TURN, EPL)], float (&sn)[lane_angles(TURN, EPL)]) {
  constexpr int RPW = 64 / LPR, NA = lane_angles(TURN, EPL);
  constexpr int CNT = NA > RPW ? NA / RPW : 1;                      // angles that a row group forms
  const int seg = lane % LPR, grp = lane / LPR, x0 = seg * EPL, half = rotary / 2;
  const bool turns = TURN == kWhole || x0 < rotary;
  float c_own[CNT], s_own[CNT];
#pragma unroll
  for (int i = 0; i < CNT; ++i) {
    const int k = (grp * CNT + i) % NA;
    const int f = TURN == kNeighbours ? x0 / 2 + k : (x0 < half ? x0 + k : x0 - half + k);
    const Turned own = turned(position, turns ? inv_freq[f] : 0.f);
    s_own[i] = own.sin;
    c_own[i] = own.cos;
  }
#pragma unroll
  for (int k = 0; k < NA; ++k) {
    const int from = (k / CNT) * LPR + seg;
    cs[k] = __shfl(c_own[k % CNT], from);
    sn[k] = __shfl(s_own[k % CNT], from);
    if (TURN != kNeighbours && x0 < half) sn[k] = -sn[k];
  }
}
// Lane that has the other halves of this lane's pairs where the front of a head turns.
template <int EPL>
__device__ __forceinline__ int front_partner(int rotary, int lane, int x0) {
  const int half = rotary / 2;
  return x0 < rotary ? (x0 < half ? lane + half / EPL : lane - half / EPL) : lane;
}
template <int TURN, int LPR, int EPL>
__device__ __forceinline__ void turn_row(float (&y)[EPL], const float (&cs)[lane_angles(TURN, EPL)], const float (&sn)[lane_angles(TURN, EPL)], bool turns, int partner) {
  if constexpr (TURN == kNeighbours) {
#pragma unroll
    for (int e = 0; e < EPL; e += 2) {
      const float p = y[e], q = y[e + 1], c = turns ? cs[e / 2] : 1.f, s = turns ? sn[e / 2] : 0.f;
      y[e] = __builtin_fmaf(p, c, -q * s);
      y[e + 1] = __builtin_fmaf(q, c, p * s);
    }
  } else {
    float z[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) z[e] = TURN == kWhole ? other_half<LPR>(y[e]) : __shfl(y[e], partner);
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = turns ? __builtin_fmaf(y[e], cs[e], z[e] * sn[e]) : y[e];
  }
}

}  // namespace ckv
