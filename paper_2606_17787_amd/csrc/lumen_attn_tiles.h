// What the kernels share that take tiles of keys from LDS through the matrix
// units: fragments, the order of a tile's 16-byte chunks, the range of the weights,
// and what infinities and NaN need.
#ifndef LUMEN_ATTN_TILES_H
#define LUMEN_ATTN_TILES_H

#include "lumen_attn_common.h"

namespace lumen_attn_detail {

// 16-bit fragments of the matrix instructions, and their products.
typedef short frag8 __attribute__((ext_vector_type(8)));
typedef short frag4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <bool kBf16>
__device__ __forceinline__ f32x16 mfma(frag8 a, frag8 b, f32x16 c) {
  if constexpr (kBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(
        __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

#define CONSTANT_PTR(T, p) ((const __attribute__((address_space(4))) T *)(p))

// A row's running maximum is moved when a score passes it by this (in log2).
constexpr float kSlack = 8.0f;
// Weights are taken times 2^lift.  bf16: at most 1, so that the sums overflow no
// sooner than those of weights under the true maximum would (a mean of n values
// under 3.4e38 / n never does).  fp16: up to 2^15, and where the maximum is not
// behind, a weight only rounds to a subnormal or 0 when it is under 2^-21 or
// 2^-32 of the largest.
template <bool kBf16>
constexpr float lift() { return kBf16 ? -kSlack : 7.0f; }
constexpr int kMfma = 0x8, kDsRead = 0x100;  // of sched_group_barrier

// The chunks of a tile's row are permuted by row, so that neither the reads of K
// nor the transposing reads of V meet in a bank.
template <int D>
__device__ __forceinline__ int swizzle_k(int row) {
  return D == 128 ? row & 15 : (row >> 1) & 7;
}
template <int D>
__device__ __forceinline__ int swizzle_v(int row) {
  // 0, 4, 10, 14 for the four rows that one transposing read takes
  return D == 128 ? (row & 3) * 4 + ((row & 2) ? 2 : 0) : (row & 3) * 2;
}

template <bool kBf16>
__device__ __forceinline__ bool not_finite16(uint32_t x) {
  constexpr uint32_t kExp = kBf16 ? 0x7f80 : 0x7c00;
  return (x & kExp) == kExp;
}

// Adds a row's infinities and NaN, whatever the weight, where it is seen.
template <int D, bool kBf16>
__device__ __forceinline__ void add_nonfinite(const uint16_t *row, bool seen, f32x16 *o) {
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const frag4 x = *reinterpret_cast<const frag4 *>(row + d * 32 + 8 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint16_t bits = uint16_t(x[j]);
        if (seen && not_finite16<kBf16>(bits)) o[d][4 * i + j] += value<kBf16>(bits);
      }
    }
}

}  // namespace lumen_attn_detail

#endif  // LUMEN_ATTN_TILES_H
