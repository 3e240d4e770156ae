// fewrows.hpp -- weights streamed past a few rows of activations: the products of 16 weight rows
// with 16 activation rows, fragments loaded straight from HBM into registers.
#pragma once
#include "common.hpp"

namespace hmoe {

// acc += A B^T over one step of 64 bytes of K: lane l holds 16 bytes (bf16: 8, fp32: 4 elements) of
// row l % 16 at byte 16 (l / 16) of the step.  Lane l of acc has rows 4 (l / 16) .. + 3 of A against row l % 16 of B.
template <typename T>
__device__ __forceinline__ void step_mfma(i32x4 a, i32x4 b, floatx4& acc) {
  if constexpr (sizeof(T) == 2) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0,
                                                  0, 0);
  } else {
    const floatx4 fa = __builtin_bit_cast(floatx4, a), fb = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], acc, 0, 0, 0);
  }
}

// A value that feeds a bf16 product without losing its low bits: v = hi + lo up to 2^-16 of it, each a
// bf16 operand of its own MFMA.  hi is cut off rather than rounded, so that no finite v becomes
// infinite.  (fp32 data: the value itself.)
template <typename T>
struct Halves {
  static constexpr int N = sizeof(T) == 2 ? 2 : 1;
  T part[N];
  __device__ __forceinline__ explicit Halves(float v) {
    if constexpr (N == 1) {
      part[0] = v;
    } else {
      const float hi = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
      part[0] = from_f32<T>(hi);
      part[1] = from_f32<T>(fabsf(v) == INFINITY ? 0.f : v - hi);
    }
  }
};

}  // namespace hmoe
