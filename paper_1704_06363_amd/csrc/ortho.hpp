// ortho.hpp -- what the kernels of orthogonalised updates share (ortho.hip, ortho_small.hip).
#pragma once
#include "common.hpp"
#include "train_launch.hpp"

namespace hmoe {

typedef _Float16 f16;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kScaleX = 0x1p13f, kScaleA = 0x1p12f, kScaleQ = 0x1p8f;

// The problem as the iterations see it.
struct Ortho {
  int K, rows, cols;
  int r, l;    // r <= l, X [r][l]
  int rp, lp;  // rounded up to 32
  bool tall;   // rows > cols: X is U^T
  int blocks;  // of a matrix's sum of squares
  __host__ __device__ int64_t x_size() const { return (int64_t)rp * 2 * lp; }  // of a matrix, in fp16 numbers
  __host__ __device__ int64_t a_size() const { return (int64_t)r * 2 * rp; }
};
inline Ortho ortho_of(int K, int rows, int cols) {
  Ortho o;
  o.K = K;
  o.rows = rows;
  o.cols = cols;
  o.tall = rows > cols;
  o.r = o.tall ? cols : rows;
  o.l = o.tall ? rows : cols;
  o.rp = (o.r + 31) / 32 * 32;
  o.lp = (o.l + 31) / 32 * 32;
  const int64_t want = cdiv((int64_t)rows * cols, 256 * 32), most = cdiv(8 * (int64_t)device_cus(), K);
  o.blocks = (int)(want < most ? want : most);
  return o;
}
// Four entries of U from `at` on, v as it is after k_ortho_start.
__device__ __forceinline__ floatx4 ortho_u(const OrthoStep& s, int64_t at) {
  if (s.G) {
    if (s.dt == HMOE_BF16) {
      const bf16x4 v = *reinterpret_cast<const bf16x4*>(static_cast<const bf16*>(s.G) + at);
      return floatx4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    }
    return *reinterpret_cast<const floatx4*>(static_cast<const float*>(s.G) + at);
  }
  const floatx4 g = *reinterpret_cast<const floatx4*>(s.g + at);
  if (!s.v) return g;
  const floatx4 v = *reinterpret_cast<const floatx4*>(s.v + at);
  if (!s.nesterov) return v;
  floatx4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = fmaf(s.momentum, v[e], g[e]);
  return u;
}
// The same with v = momentum v + g first.
__device__ __forceinline__ floatx4 ortho_first_u(const OrthoStep& s, int64_t at, floatx4 g, floatx4 v) {
  floatx4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = fmaf(s.momentum, v[e], g[e]);
    u[e] = s.nesterov ? fmaf(s.momentum, v[e], g[e]) : v[e];
  }
  *reinterpret_cast<floatx4*>(s.v + at) = v;
  return u;
}
__device__ __forceinline__ floatx4 ortho_first_u(const OrthoStep& s, int64_t at) {
  if (s.G || !s.v) return ortho_u(s, at);
  return ortho_first_u(s, at, *reinterpret_cast<const floatx4*>(s.g + at), *reinterpret_cast<const floatx4*>(s.v + at));
}

__device__ __forceinline__ void pair_of(float v, f16& hi, f16& lo) {
  hi = (f16)v;
  // of what fp16 holds no more, as an infinity; a lo of NaN beside it would be NaN too
  lo = (f16)(v - (float)hi);
}

// 4 x 4 values of the lanes 4 q .. 4 q + 3 transposed: lane 4 q + s gets element s of each.
__device__ __forceinline__ void quad_transpose(float (&v)[4]) {
  const int s = threadIdx.x & 3;
  // lanes a distance of 1 apart trade their odd and even elements, then those 2 apart halves
  float x[4];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const float give = (s & 1) ? v[2 * p] : v[2 * p + 1];
    const float got = dpp<0xB1>(give);
    x[2 * p] = (s & 1) ? got : v[2 * p];
    x[2 * p + 1] = (s & 1) ? v[2 * p + 1] : got;
  }
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const float give = (s & 2) ? x[p] : x[p + 2];
    const float got = dpp<0x4E>(give);
    v[p] = (s & 2) ? got : x[p];
    v[p + 2] = (s & 2) ? x[p + 2] : got;
  }
}

// Four consecutive entries of the result where the call wants them: in O, or as the step of w and w_lo.
__device__ __forceinline__ void ortho_put4(const OrthoStep& s, int64_t at, const float (&v)[4]) {
  floatx4 w = {v[0], v[1], v[2], v[3]};
  if (!s.G) {
    w = *reinterpret_cast<const floatx4*>(s.w + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = fmaf(-s.rate, v[e], s.keep * w[e]);
    *reinterpret_cast<floatx4*>(s.w + at) = w;
    if (!s.w_lo) return;
  }
  void* out = s.G ? s.O : s.w_lo;
  if (s.dt == HMOE_BF16)
    *reinterpret_cast<bf16x4*>(static_cast<bf16*>(out) + at) = bf16x4{(bf16)w[0], (bf16)w[1], (bf16)w[2], (bf16)w[3]};
  else
    *reinterpret_cast<floatx4*>(static_cast<float*>(out) + at) = w;
}

// ortho_small.hip: matrices with a short side of up to 128 and few columns, whole iterations to a launch.
size_t small_ortho_ws(const Ortho& o);  // 0: not for these sizes
int launch_small_ortho(const OrthoStep& s, const Ortho& o, int steps, const float* coef, Workspace& ws, hipStream_t st);

// k_ortho_start: the momentum and the sums of squares, part[K][o.blocks].
int launch_ortho_start(const OrthoStep& s, const Ortho& o, double* part, hipStream_t st);

}  // namespace hmoe
