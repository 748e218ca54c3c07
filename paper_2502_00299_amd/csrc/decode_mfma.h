// What the matrix-core decode kernels share: products, lane exchanges, transposing reads, waits.
#pragma once
#include "internal.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __fp16 fp16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kStepKeys = 32;
static constexpr float kNegBig = -1.0e30f;

template <int DT>
__device__ __forceinline__ f32x4 mma16(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
  if constexpr (DT == CHUNKKV_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// lane i of a row of 16 gets the value of lane i + N
template <int N>
__device__ __forceinline__ float row_shl(float x) {
  return __builtin_amdgcn_update_dpp(0.f, x, 0x100 + N, 0xf, 0xf, true);
}

// Transposing reads of four 16-dim pieces of V, keys 4 q .. of both 16-key tiles (the second `OFF` bytes further on).
// One assembly block with its own wait: the compiler takes the builtin for a read of everything that is on its way
// into LDS and would wait for all of it.
template <int OFF>
__device__ __forceinline__ void read_v4(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, u32x4 (&v)[4]) {
  uint64_t x[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = u32x4{(uint32_t)x[2 * i], (uint32_t)(x[2 * i] >> 32), (uint32_t)x[2 * i + 1], (uint32_t)(x[2 * i + 1] >> 32)};
}

constexpr int vm_imm(int n) { return (n & 0xF) | ((n >> 4) << 14) | 0x0F70; }

// The integer form of isfinite, kept from the optimizer: the build lets it assume that nothing is NaN.
__device__ __forceinline__ bool finite_bits(float x) {
  uint32_t u = __float_as_uint(x);
  asm("" : "+v"(u));
  return (u & 0x7F800000u) != 0x7F800000u;
}

}  // namespace ckv
