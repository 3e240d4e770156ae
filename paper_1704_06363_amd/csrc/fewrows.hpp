// fewrows.hpp -- weights streamed past a few rows of activations: the products of 16 weight rows
// with 16 activation rows, fragments loaded straight from HBM into registers.
#pragma once
#include "lanes.hpp"

namespace hmoe {

template <typename T>
using quad = T __attribute__((ext_vector_type(4)));

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

// body(wv, xv) for the steps s0 <= s < s1 of a reduction over kd elements, with this lane's 16 bytes of the
// rows at w and x.  The loads of U steps go out together: under a bound on K of their own (which the
// compiler does not move loads across) they ran one step at a time.  kd is a multiple of 8: past it, in
// the last step, both operands are zeros.
template <typename T, int U, int MI, int NX, class Body>
__device__ __forceinline__ void stream_steps(const T* const (&w)[MI], const T* const (&x)[NX], int kd, int s0, int s1,
                                             Body body) {
  constexpr int N = 16 / sizeof(T), STEP = 4 * N;
  const int lg = (threadIdx.x & 63) >> 4;
  const int ragged = kd % STEP ? kd / STEP : -1;  // the step with less than STEP elements
  for (int s = s0; s < s1; s += U) {
    i32x4 wv[U][MI], xv[U][NX];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (s + u < s1 ? s + u : s1 - 1) * STEP + lg * N;
      const int in = at < kd ? at : kd - N;
#pragma unroll
      for (int i = 0; i < MI; ++i) wv[u][i] = *reinterpret_cast<const i32x4*>(w[i] + in);
#pragma unroll
      for (int j = 0; j < NX; ++j) xv[u][j] = *reinterpret_cast<const i32x4*>(x[j] + in);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;
      if (s + u == ragged) {
        const bool out = ragged * STEP + lg * N >= kd;
#pragma unroll
        for (int i = 0; i < MI; ++i)
          if (out) wv[u][i] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < NX; ++j)
          if (out) xv[u][j] = i32x4{0, 0, 0, 0};
      }
      body(wv[u], xv[u]);
    }
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

// The slot-th of the groups 0 .. G - 1 that have rows, in ascending order, and its rows of the `total`
// in ascending order, at most HMOE_FEW_ROWS.  A row whose group is outside [0, G) has none.  False if
// there are not that many groups.  Entered by workgroups of THREADS >= 128; G <= 4096.
template <int THREADS>
__device__ __forceinline__ bool few_group(const int32_t* __restrict__ group, int total, int G, int slot, int* s_group,
                                          int* s_rows, int* s_count) {
  __shared__ uint32_t mask[128];
  const int t = threadIdx.x;
  if (t < 128) mask[t] = 0;
  if (t == 0) *s_group = -1;
  __syncthreads();
  for (int q = t; q < total; q += THREADS) {
    const int e = group[q];
    if (e >= 0 && e < G) atomicOr(&mask[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
  if (t < 64) {
    const uint32_t m0 = mask[2 * t], m1 = mask[2 * t + 1];
    const int c = __popc(m0) + __popc(m1);
    int inc = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o, 64);
      if (t >= o) inc += v;
    }
    const int before = inc - c;
    if (slot >= before && slot < inc) {
      uint64_t both = ((uint64_t)m1 << 32) | m0;
      for (int i = slot - before; i > 0; --i) both &= both - 1;
      *s_group = 64 * t + __builtin_ctzll(both);
    }
  }
  __syncthreads();
  const int e = *s_group;
  if (e < 0) return false;
  if (t < 64) {
    int count = 0;
    for (int b = 0; b < total; b += 64) {
      const bool mine = b + t < total && group[b + t] == e;
      const uint64_t hit = __ballot(mine);
      if (mine) s_rows[count + lanes_below(hit)] = b + t;
      count += __popcll(hit);
    }
    if (t == 0) *s_count = count;
  }
  __syncthreads();
  return true;
}

}  // namespace hmoe
