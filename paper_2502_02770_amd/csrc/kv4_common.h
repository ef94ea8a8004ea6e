// K and V rows in 4 bits as operands of matrix instructions: the quarter waves' exchange of code words, codes as bf16 numbers.
#pragma once
#include "tw_common.h"

#ifdef __HIPCC__
typedef __bf16 tw_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 tw_f16x2 __attribute__((ext_vector_type(2)));
typedef float tw_v4f __attribute__((ext_vector_type(4)));

// Sum and maximum over the four quarters of the wave (lanes of the same number in each), for all of them.
__device__ __forceinline__ float tw_quarters_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float tw_quarters_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Word w of quarter j -> word j of quarter w: of a row's codes, read as 16 bytes of group j, word j of every group.
__device__ __forceinline__ void tw_transpose_quarters(uint4& x) {
  const auto a = __builtin_amdgcn_permlane32_swap(x.x, x.z, false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(x.y, x.w, false, false);
  const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  x = make_uint4(c[0], c[1], d[0], d[1]);
}

// (x & mask) | bits in one instruction.  (Written as two operations they stay two, with a literal each; and not as inline assembly, which the
// compiler does not count where a matrix instruction has still to read or write a register.)
__device__ __forceinline__ uint32_t tw_and_or(uint32_t x, uint32_t mask, uint32_t bits) { return (uint32_t)__builtin_amdgcn_bitop3_b32((int)x, (int)mask, (int)bits, 0xEA); }

// The 8 codes of a word as 128 + c in bf16, which holds them exactly; dims in the order 0 2 4 6 1 3 5 7.  A row of q likewise.
__device__ __forceinline__ tw_bf16x8 tw_codes_bf16(uint32_t w) {
  union { uint32_t u[4]; tw_bf16x8 v; } x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.u[i] = tw_and_or(w >> (4 * i), 0x000F000Fu, 0x43004300u);
  return x.v;
}
__device__ __forceinline__ tw_bf16x8 tw_as_bf16(const uint4& x) { union { uint4 u; tw_bf16x8 v; } y; y.u = x; return y.v; }
__device__ __forceinline__ tw_bf16x8 tw_q_like_codes(const uint4& x) {
  return tw_as_bf16(make_uint4(__builtin_amdgcn_perm(x.y, x.x, 0x05040100u), __builtin_amdgcn_perm(x.w, x.z, 0x05040100u),
                               __builtin_amdgcn_perm(x.y, x.x, 0x07060302u), __builtin_amdgcn_perm(x.w, x.z, 0x07060302u)));
}

// The halves of a (scale | zero << 16) word.
__device__ __forceinline__ float tw_half_lo(uint32_t w) { union { uint32_t u; tw_f16x2 h; } x; x.u = w; return (float)x.h.x; }
__device__ __forceinline__ float tw_half_hi(uint32_t w) { union { uint32_t u; tw_f16x2 h; } x; x.u = w; return (float)x.h.y; }
#endif
