// fewrows.hpp -- weights streamed past a few rows of activations: the products of 16 weight rows
// with 16 activation rows, fragments loaded straight from HBM into registers.
#pragma once
#include "lanes.hpp"

namespace hmoe {

template <typename T>
using quad = T __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int uniform_int(int v) { return __builtin_amdgcn_readfirstlane(v); }

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

// v[f] of lane 4 i + q becomes v[q] of lane 4 i + f, for each of the four dwords.
__device__ __forceinline__ void quad_transpose(i32x4 (&v)[4]) {
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  // every lane takes part in the moves, whichever value it keeps
  const auto pick1 = [&](bool other, int x, int mine) {
    const int o = __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true);
    return other ? o : mine;
  };
  const auto pick2 = [&](bool other, int x, int mine) {
    const int o = __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true);
    return other ? o : mine;
  };
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int a0 = v[0][d], a1 = v[1][d], a2 = v[2][d], a3 = v[3][d];
    const int b0 = pick1(odd, a1, a0), b1 = pick1(!odd, a0, a1);
    const int b2 = pick1(odd, a3, a2), b3 = pick1(!odd, a2, a3);
    v[0][d] = pick2(high, b2, b0);
    v[2][d] = pick2(!high, b0, b2);
    v[1][d] = pick2(high, b3, b1);
    v[3][d] = pick2(!high, b1, b3);
  }
}

// The reduction runs over groups of 256 bytes of K, four MFMA steps.  In load f of a group this lane takes 16
// bytes of row group_row(f) of the tile at byte 16 group_chunk(): four rows of 256 contiguous bytes to a
// load, where adjacent lanes read adjacent bytes.  After quad_transpose register f has row l % 16, chunk
// 4 (l / 16) + f -- an MFMA operand, the lane groups' chunks standing for other places of K than
// usual, the same ones for both operands.  (Loaded as the MFMA holds them, adjacent lanes are in different
// rows and every lane's 16 bytes are a request of their own, 64 cycles of the CU's address unit
// for a load instead of 16: that alone was 52 of the 54 us of 48 rows against 50000 columns of 1024 with 16
// adapters.)
__device__ __forceinline__ int group_row(int f) { return (threadIdx.x & 12) + f; }
__device__ __forceinline__ int group_chunk() { return ((threadIdx.x & 48) >> 2) + (threadIdx.x & 3); }
template <typename T>
__host__ __device__ constexpr int group_size() {  // elements of K
  return 256 / (int)sizeof(T);
}
template <typename T>
__host__ __device__ inline int groups_of(int kd) {
  return (kd + group_size<T>() - 1) / group_size<T>();
}

// body(wv, xv) with the operands of each step of the groups g0 <= g < g1.  wo and xo: byte offsets from the
// tiles' wb, and from xb, of this lane's row of load f (kd elements from there); below 2^32.  The loads of UG groups go out together.  kd is a
// multiple of 8: past it, in the last group, both operands are zeros.
template <typename T, int UG, int MI, int NX, class Row, class Body>
__device__ __forceinline__ void stream_groups_of(const T* const (&wb)[MI], const uint32_t (&wo)[MI][4], Row xrow, int kd,
                                                 int g0, int g1, Body body) {
  constexpr int N = 16 / sizeof(T), GROUP = group_size<T>();
  const int own = group_chunk() * N;
  for (int g = g0; g < g1; g += UG) {
    i32x4 wv[UG][MI][4], xv[UG][NX][4];
#pragma unroll
    for (int u = 0; u < UG; ++u) {
      const int at = (g + u < g1 ? g + u : g1 - 1) * GROUP + own;
      const uint32_t in = (at < kd ? at : 0) * (uint32_t)sizeof(T);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) wv[u][i][f] = *reinterpret_cast<const i32x4*>(reinterpret_cast<const char*>(wb[i]) + (wo[i][f] + in));
#pragma unroll
      for (int j = 0; j < NX; ++j)
#pragma unroll
        for (int f = 0; f < 4; ++f) xv[u][j][f] = *reinterpret_cast<const i32x4*>(xrow(j, f, in));
    }
#pragma unroll
    for (int u = 0; u < UG; ++u) {
      if (g + u >= g1) break;
      if ((g + u + 1) * GROUP > kd) {
        const bool out = (g + u) * GROUP + own >= kd;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
#pragma unroll
          for (int i = 0; i < MI; ++i)
            if (out) wv[u][i][f] = i32x4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < NX; ++j)
            if (out) xv[u][j][f] = i32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int i = 0; i < MI; ++i) quad_transpose(wv[u][i]);
#pragma unroll
      for (int j = 0; j < NX; ++j) quad_transpose(xv[u][j]);
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        i32x4 a[MI], x[NX];
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = wv[u][i][f];
#pragma unroll
        for (int j = 0; j < NX; ++j) x[j] = xv[u][j][f];
        body(a, x);
      }
    }
  }
}

template <typename T, int UG, int MI, int NX, class Body>
__device__ __forceinline__ void stream_groups(const T* const (&wb)[MI], const uint32_t (&wo)[MI][4], const T* xb,
                                              const uint32_t (&xo)[NX][4], int kd, int g0, int g1, Body body) {
  const char* xc = reinterpret_cast<const char*>(xb);
  stream_groups_of<T, UG, MI, NX>(wb, wo, [&](int j, int f, uint32_t at) { return xc + (xo[j][f] + at); }, kd, g0, g1, body);
}
// The same with x's rows anywhere.
template <typename T, int UG, int MI, int NX, class Body>
__device__ __forceinline__ void stream_groups(const T* const (&wb)[MI], const uint32_t (&wo)[MI][4],
                                              const T* const (&xr)[NX][4], int kd, int g0, int g1, Body body) {
  stream_groups_of<T, UG, MI, NX>(
      wb, wo, [&](int j, int f, uint32_t at) { return reinterpret_cast<const char*>(xr[j][f]) + at; }, kd, g0, g1, body);
}

// An fp32 value as M bf16 numbers that add up to it, each an operand of its own MFMA: two are good to 2^-16 of
// the value, the first two of three as well, three hold all of its bits.  All but the last are cut off rather than
// rounded, so that no finite value becomes infinite.  None is 0 unless the value is, because an infinite factor
// would make NaN of it: a value of one number is halved, and a third number without anything to hold is 2^-126, or
// 2^-40 of smaller values, which no sum notices.  (fp32 data: the value itself.)
template <typename T, int M>
struct Parts {
  static constexpr int N = sizeof(T) == 2 ? M : 1;
  T part[N];
  __device__ __forceinline__ explicit Parts(float v) {
    const float half = 0.5f * v, least = copysignf(fminf(fabsf(v) * 0x1p-40f, 0x1p-126f), v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float hi = i + 1 < N ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : v;
      const bool all = hi == v;  // infinities too
      part[i] = from_f32<T>(i == 0 && i + 1 < N && all ? half : hi);
      v = all ? (i == 0 ? half : least) : v - hi;
    }
  }
};
template <typename T>
using Halves = Parts<T, 2>;

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
