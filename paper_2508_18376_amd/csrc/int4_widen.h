// Weights of 4 bits for the 16-bit matrix instructions, exactly, with the scale and the zero point left to the sums.
//
// Eight weights are a word; its 4-bit numbers j and j + 4 lie in its two halves alike, so that one shift and one and-or bring both to the top of a mantissa:
// (1 + q[j] / 16, 1 + q[j + 4] / 16), half an instruction a weight.  The rest is linear:
//   sum of x (q - z) s = 16 s sum of x (1 + q / 16) - (16 + z) s sum of x
// with the sum of x from the same matrix instructions against ones.  The terms are up to some seven times larger than x (q - z) / 16, which costs three bits of
// the sums' 24.  x is brought to the order of the weights' pairs by four byte permutations for eight values.
//
// The two sums can be beyond fp32, or infinity less infinity, where x (q - z) s is not: outputs that come out infinite or NaN are worked out again as the formula has
// them (sum_again).  No other output can be wrong for that reason: an infinity or NaN on the way stays one.
//
// x is the first operand of instructions of 16 x 16 x 32, so that lane 16 q + i has output channel i of sixteen, whose scale and zero point are its own, and rows
// 4 q .. + 3 of the results.
#pragma once
#include "int4_matmul.h"

namespace dsmoe {

typedef __bf16 qbf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 qf16x8 __attribute__((ext_vector_type(8)));
typedef int qi32x4 __attribute__((ext_vector_type(4)));
typedef float qf32x4 __attribute__((ext_vector_type(4)));

template <int TY>
struct Unit {
  static constexpr uint32_t one = TY == kElemBF16 ? 0x3f803f80u : 0x3c003c00u, mask = TY == kElemBF16 ? 0x00780078u : 0x03c003c0u;
  static constexpr int up = TY == kElemBF16 ? 3 : 6;  // where the mantissa's top four bits are
};

template <int TY>
__device__ __forceinline__ void mac4(qf32x4& c, const qi32x4& a, const qi32x4& b) {
  if constexpr (TY == kElemBF16)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(qbf16x8, a), __builtin_bit_cast(qbf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(qf16x8, a), __builtin_bit_cast(qf16x8, b), c, 0, 0, 0);
}

// Unit::one in a vector register: an and-or takes one constant from the scalar ones (left to itself the compiler makes it two instructions with literals).
template <int TY>
__device__ __forceinline__ uint32_t one_of() {
  uint32_t one = Unit<TY>::one;
  asm("" : "+v"(one));
  return one;
}
// eight weights as 1 + q / 16, in pairs (j, j + 4)
template <int TY>
__device__ __forceinline__ qi32x4 widened(uint32_t w, uint32_t one) {
  qi32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int by = 4 * j - Unit<TY>::up;
    v[j] = (int)(((by < 0 ? w << -by : w >> by) & Unit<TY>::mask) | one);
  }
  return v;
}
// eight values of x in the same order
__device__ __forceinline__ qi32x4 paired(const qi32x4& x) {
  return qi32x4{(int)__builtin_amdgcn_perm((uint32_t)x[2], (uint32_t)x[0], 0x05040100u), (int)__builtin_amdgcn_perm((uint32_t)x[2], (uint32_t)x[0], 0x07060302u),
                (int)__builtin_amdgcn_perm((uint32_t)x[3], (uint32_t)x[1], 0x05040100u), (int)__builtin_amdgcn_perm((uint32_t)x[3], (uint32_t)x[1], 0x07060302u)};
}
// a scale from its bits, in the low half of a word unless it is of 32 bits
template <int TY, bool S32>
__device__ __forceinline__ float scale_of(uint32_t bits) {
  if (S32) return __uint_as_float(bits);
  return TY == kElemBF16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
// The sum of x (q - z) s over the values from .. to - 1 of the contraction (from: a multiple of 8), in 64 bits.  (64 rows on 8 groups of 4096 x 14336: 55 us, 3.8 ms if
// all outputs are infinite; that they are finite costs nothing to see.)
template <int TY>
__device__ __forceinline__ float sum_again(const Int4Args& a, int group, int64_t row, int64_t channel, int from, int to) {
  const char* x = a.x + row * a.x_row;
  const uint8_t* w = a.w + group * a.w_group + channel * a.w_row;
  const int64_t s_at = group * a.s_group + channel * a.s_row, z_at = group * a.z_group + channel * a.z_row;
  double sum = 0;
#pragma unroll 1
  for (int k = from; k < to && sum == sum; k += 8) {  // (a NaN stays one)
    const int block = k >> a.shift;
    const double s = int4_scale(a, s_at + block), z = a.zero ? a.zero[z_at + block] : 8;
    uint16_t v[8] = {};
    uint32_t q = 0;
    if (k + 8 <= to) {
      __builtin_memcpy(v, x + 2ll * k, 16);
      __builtin_memcpy(&q, w + (k >> 1), 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k + e < to) {
          v[e] = *(const uint16_t*)(x + 2ll * (k + e));
          q |= (uint32_t)(w[(k + e) >> 1] >> (4 * (e & 1)) & 15) << (4 * e);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < to) sum = fma((double)elem_to_f32((const char*)&v[e], TY), ((double)(q >> (4 * e) & 15) - z) * s, sum);
  }
  return (float)sum;
}
// (16 + z) / 16
__device__ __forceinline__ float zero_of(uint32_t z) { return 1.f + (float)z * (1.f / 16); }

}  // namespace dsmoe
