// ortho.hip -- Newton-Schulz iterations towards the orthogonal factor of K matrices, alone and as the update of a
// step with momentum:  X = U / |U|,  X <- a X + (b A + c A^2) X,  A = X X^T.
//
// With rows <= cols as they are and rows > cols transposed, X is [r][l], r <= l, and A [r][r].  A step is three
// products on the matrix cores (r^2 l for A and r^3 for A^2, which are symmetric: the tiles on and above the
// diagonal are computed, the others are their mirror images; 2 r^2 l for the last), and so are its bounds.
//
// fp32 matrix instructions run at a sixteenth of the rate of fp16 ones.  Small singular values grow by a
// factor of a in every step, and so does what rounding adds to them: iterates of one 16-bit number (an error of
// 8e-2 after five steps where X has a rank of 3, 1.3e-2 with a floor of noise) are not enough.  Values are
// held as two fp16 numbers, hi + lo, 22 bits, and a product is hi hi + hi lo + lo hi, summed in fp32: three
// instructions, and as exact as fp32 products (measured: 2e-6 after five steps where those give 4e-6).
// fp16 spans little: X is stored times 2^13, A and b A + c A^2 times 2^12, so that entries up to 8 and 16 fit and the
// smallest lo, 2^-25, is 2^-38 of X -- 2^-25 of the mean entry of a matrix of 8192 x 8192.
#include "gemm.hpp"
#include "primitives.hpp"
#include "slices.hpp"
#include "train_launch.hpp"

namespace hmoe {

namespace {

typedef _Float16 f16;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kScaleX = 0x1p13f, kScaleA = 0x1p12f;

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
Ortho ortho_of(int K, int rows, int cols) {
  Ortho o;
  o.K = K;
  o.rows = rows;
  o.cols = cols;
  o.tall = rows > cols;
  o.r = o.tall ? cols : rows;
  o.l = o.tall ? rows : cols;
  o.rp = (o.r + 31) / 32 * 32;
  o.lp = (o.l + 31) / 32 * 32;
  const int64_t want = cdiv((int64_t)rows * cols, 256 * 32), most = cdiv(4 * (int64_t)device_cus(), K);
  o.blocks = (int)(want < most ? want : most);
  return o;
}
struct OrthoSpace {
  f16 *X[2], *A, *B;
  double* part;  // [K][blocks]
};
OrthoSpace ortho_carve(const Ortho& o, Workspace& ws) {
  OrthoSpace s;
  for (int i = 0; i < 2; ++i) s.X[i] = ws.take<f16>((size_t)o.K * o.x_size());
  s.A = ws.take<f16>((size_t)o.K * o.a_size());
  s.B = ws.take<f16>((size_t)o.K * o.a_size());
  s.part = ws.take<double>((size_t)o.K * o.blocks);
  return s;
}

// ------------------------------------------------------------------ the start

// Four entries of U from `at` on.
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

// v = momentum v + g, and the sums of squares of U, in fp64 (entries of 1e-30 and of 1e30 have squares there), of
// blockIdx.x's part of matrix m0 + blockIdx.y.
__global__ void __launch_bounds__(256) k_ortho_start(OrthoStep s, Ortho o, int m0, double* __restrict__ part) {
  __shared__ double sh[4];
  const int m = m0 + blockIdx.y;
  const int64_t size = (int64_t)o.rows * o.cols, base = m * size;
  double sum = 0.0;
  for (int64_t q = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; q < size; q += (int64_t)gridDim.x * 1024) {
    if (!s.G && s.v) {
      const floatx4 g = *reinterpret_cast<const floatx4*>(s.g + base + q);
      floatx4 v = *reinterpret_cast<const floatx4*>(s.v + base + q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(s.momentum, v[e], g[e]);
      *reinterpret_cast<floatx4*>(s.v + base + q) = v;
    }
    const floatx4 u = ortho_u(s, base + q);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = fma((double)u[e], (double)u[e], sum);
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)m * o.blocks + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__device__ __forceinline__ void pair_of(float v, f16& hi, f16& lo) {
  hi = (f16)v;
  // of what fp16 holds no more, as an infinity; a lo of NaN beside it would be NaN too
  lo = (f16)(v - (float)hi);
}

// X = U / |U| in pairs, 64 x 64 entries to a workgroup, zeros where X is padded -- in both buffers: later steps write
// the entries that there are, and columns past l as products with zeros.
__global__ void __launch_bounds__(256) k_ortho_split(OrthoStep s, Ortho o, int m0, const double* __restrict__ part,
                                                     f16* __restrict__ X, f16* __restrict__ X1) {
  __shared__ float t[64][65];
  __shared__ double s_norm;
  const int m = m0 + blockIdx.y, tiles = (o.lp + 63) / 64;
  const int i0 = (int)(blockIdx.x / tiles) * 64, j0 = (int)(blockIdx.x % tiles) * 64;
  if (threadIdx.x < 64) {
    double sum = 0.0;
    for (int b = threadIdx.x; b < o.blocks; b += 64) sum += part[(int64_t)m * o.blocks + b];
    sum = wave_sum(sum);
    if (threadIdx.x == 0) s_norm = sqrt(sum);
  }
  const int64_t base = (int64_t)m * o.rows * o.cols;
  // rows of U, four entries to a thread: of X, or of X^T
  for (int q = threadIdx.x; q < 64 * 16; q += 256) {
    const int a = q / 16, b = q % 16 * 4;
    const int row = (o.tall ? j0 : i0) + a, col = (o.tall ? i0 : j0) + b;
    floatx4 u = {0.f, 0.f, 0.f, 0.f};
    if (row < o.rows && col < o.cols) u = ortho_u(s, base + (int64_t)row * o.cols + col);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (o.tall) t[b + e][a] = u[e]; else t[a][b + e] = u[e];
    }
  }
  __syncthreads();
  const double norm = s_norm;
  f16* Xm = X + m * o.x_size();
  f16* X1m = X1 + m * o.x_size();
  for (int q = threadIdx.x; q < 64 * 8; q += 256) {
    const int i = q / 8, j = q % 8 * 8;
    if (i0 + i >= o.rp || j0 + j >= o.lp) continue;
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = t[i][j + e];
      const float x = norm == 0.0 ? 0.f : (float)((double)u / norm * (double)kScaleX);
      f16 h, l;
      pair_of(x, h, l);
      hi[e] = h;
      lo[e] = l;
    }
    const int64_t at = (int64_t)(i0 + i) * 2 * o.lp + pair_at(j0 + j);
    *reinterpret_cast<f16x8*>(Xm + at) = hi;
    *reinterpret_cast<f16x8*>(Xm + at + kPairLo) = lo;
    if (i0 + i >= o.r) {
      *reinterpret_cast<f16x8*>(X1m + at) = hi;
      *reinterpret_cast<f16x8*>(X1m + at + kPairLo) = lo;
    }
  }
}

// ------------------------------------------------------------------ the products

// Four values from column c (a multiple of 4) of a row of pairs.
__device__ __forceinline__ void put_pairs(f16* row, int c, const float (&v)[4]) {
  f16x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f16 h, l;
    pair_of(v[e], h, l);
    hi[e] = h;
    lo[e] = l;
  }
  *reinterpret_cast<f16x4*>(row + pair_at(c)) = hi;
  *reinterpret_cast<f16x4*>(row + pair_at(c) + kPairLo) = lo;
}
__device__ __forceinline__ void get_pairs(const f16* row, int c, float (&v)[4]) {
  const f16x4 hi = *reinterpret_cast<const f16x4*>(row + pair_at(c));
  const f16x4 lo = *reinterpret_cast<const f16x4*>(row + pair_at(c) + kPairLo);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)hi[e] + (float)lo[e];
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

// Tile `b` of those on and above the diagonal of `nt` x `nt`, column by column.
__device__ __forceinline__ void upper_tile(int b, int& mi, int& ni) {
  int c = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
  while (c * (c + 1) / 2 > b) --c;
  while ((c + 1) * (c + 2) / 2 <= b) ++c;
  ni = c;
  mi = b - c * (c + 1) / 2;
}

// SQUARE: out = b A + c A A^T (A [r][rp]), otherwise out = A = X X^T (X [r][lp]).
template <class C, bool SQUARE>
__global__ void __launch_bounds__(C::THREADS) k_ortho_gram(const f16* __restrict__ in, Ortho o, int m0, float b, float c,
                                                           f16* __restrict__ out) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int m = m0 + blockIdx.y;
  int mi, ni;
  upper_tile(blockIdx.x, mi, ni);
  const int r0 = mi * C::BM, c0 = ni * C::BN, ld = 2 * (SQUARE ? o.rp : o.lp);
  const f16* A = in + m * (SQUARE ? o.a_size() : o.x_size());
  f16* to = out + m * o.a_size();
  const int m_rows = o.r - r0 < C::BM ? o.r - r0 : C::BM, n_cols = o.r - c0 < C::BN ? o.r - c0 : C::BN;
  floatx4 acc[C::MI][C::NJ];
  PipeTile<C, true, true> t;
  const bf16* units = reinterpret_cast<const bf16*>(A);
  t.prime(units + (int64_t)r0 * ld, ld, m_rows, units + (int64_t)c0 * ld, ld, n_cols, ld, smem);
  t.run(smem, acc);
  const Frag<C> f;
  const float scale = SQUARE ? c / kScaleA : kScaleA / (kScaleX * kScaleX);
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) {
      const int row = r0 + f.row(i, 0), col = c0 + f.col(j, 0);
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e] * scale;
      if (row < o.r && col < o.rp) {
        if constexpr (SQUARE) {
          float a[4];
          get_pairs(A + (int64_t)row * ld, col, a);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(b, a[e], v[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = col + e < o.r ? v[e] : 0.f;  // rows past r have no product
        put_pairs(to + (int64_t)row * 2 * o.rp, col, v);
      }
      if (mi == ni) continue;
      quad_transpose(v);  // now of column col + s, rows 4 q .. 4 q + 3 of the 16
      const int tr = col + (f.lr & 3), tc = r0 + f.row(i, 0) - (f.lr & 3);
      if (tr < o.r) put_pairs(to + (int64_t)tr * 2 * o.rp, tc, v);
    }
}

// X' = a X + B X; LAST: the result goes where `s` says.
template <class C, bool LAST>
__global__ void __launch_bounds__(C::THREADS) k_ortho_apply(const f16* __restrict__ B, const f16* __restrict__ X, Ortho o,
                                                            int m0, float a, f16* __restrict__ out, OrthoStep s) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int m = m0 + blockIdx.y;
  const TileCoord tc = tile_plain<C>(o.r, o.lp, o.rp);
  if (!tc.valid) return;
  const f16* Xm = X + m * o.x_size();
  floatx4 acc[C::MI][C::NJ];
  PipeTile<C, true, false> t;
  t.prime(reinterpret_cast<const bf16*>(B + m * o.a_size()) + tc.m0 * 2 * o.rp, 2 * o.rp, tc.m_rows,
          reinterpret_cast<const bf16*>(Xm) + 2 * tc.n0, 2 * o.lp, tc.n_cols, 2 * o.rp, smem);
  t.run(smem, acc);
  const Frag<C> f;
  const int64_t base = (int64_t)m * o.rows * o.cols;
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) {
      const int row = (int)tc.m0 + f.row(i, 0), col = tc.n0 + f.col(j, 0);
      if (row >= o.r || col >= o.lp) continue;
      float v[4];
      get_pairs(Xm + (int64_t)row * 2 * o.lp, col, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(a, v[e], acc[i][j][e] * (1.f / kScaleA));
      if constexpr (!LAST) {
        put_pairs(out + m * o.x_size() + (int64_t)row * 2 * o.lp, col, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= 1.f / kScaleX;
        if (!o.tall) {
          if (col >= o.l) continue;  // l = cols, a multiple of 8
          const int64_t at = base + (int64_t)row * o.cols + col;
          if (s.G) {
            if (s.dt == HMOE_BF16) {
              bf16x4 y;
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = (bf16)v[e];
              *reinterpret_cast<bf16x4*>(static_cast<bf16*>(s.O) + at) = y;
            } else {
              *reinterpret_cast<floatx4*>(static_cast<float*>(s.O) + at) = floatx4{v[0], v[1], v[2], v[3]};
            }
          } else {
            floatx4 w = *reinterpret_cast<const floatx4*>(s.w + at);
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w[e] = fmaf(-s.rate, v[e], s.keep * w[e]);
              y[e] = (bf16)w[e];
            }
            *reinterpret_cast<floatx4*>(s.w + at) = w;
            if (s.w_lo) {
              if (s.dt == HMOE_BF16) *reinterpret_cast<bf16x4*>(static_cast<bf16*>(s.w_lo) + at) = y;
              else *reinterpret_cast<floatx4*>(static_cast<float*>(s.w_lo) + at) = w;
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (col + e >= o.l) continue;
            const int64_t at = base + (int64_t)(col + e) * o.cols + row;
            if (s.G) {
              if (s.dt == HMOE_BF16) static_cast<bf16*>(s.O)[at] = (bf16)v[e];
              else static_cast<float*>(s.O)[at] = v[e];
            } else {
              const float w = fmaf(-s.rate, v[e], s.keep * s.w[at]);
              s.w[at] = w;
              if (s.w_lo) {
                if (s.dt == HMOE_BF16) static_cast<bf16*>(s.w_lo)[at] = (bf16)w;
                else static_cast<float*>(s.w_lo)[at] = w;
              }
            }
          }
        }
      }
    }
}

typedef CfgPair<256, 256, 128, 64, false> PairLarge;
typedef CfgPair<256, 256, 128, 64, true> PairLargeKS;
typedef CfgPair<128, 128, 64, 64, false> PairSmall;
typedef CfgPair<128, 256, 64, 64, true> PairSmallKS;  // the swizzle of a K-strided operand spans 256 columns

template <class C, bool SQUARE>
int ortho_gram(const f16* in, const Ortho& o, float b, float c, f16* out, hipStream_t st) {
  const int64_t nt = cdiv(o.r, C::BM), tiles = nt * (nt + 1) / 2;
  return over_slices(o.K, tiles, C::THREADS, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH(SQUARE ? "ortho square" : "ortho gram", (k_ortho_gram<C, SQUARE>), dim3((unsigned)tiles, (unsigned)count),
                dim3(C::THREADS), C::LDS, st, in, o, (int)m0, b, c, out);
    return (int)HMOE_OK;
  });
}
template <class C, bool LAST>
int ortho_apply(const f16* B, const f16* X, const Ortho& o, float a, f16* out, const OrthoStep& s, hipStream_t st) {
  const int64_t tiles = cdiv(o.r, C::BM) * cdiv(o.lp, C::BN);
  return over_slices(o.K, tiles, C::THREADS, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH("ortho apply", (k_ortho_apply<C, LAST>), dim3((unsigned)tiles, (unsigned)count), dim3(C::THREADS), C::LDS,
                st, B, X, o, (int)m0, a, out, s);
    return (int)HMOE_OK;
  });
}

}  // namespace

size_t ortho_ws(int32_t K, int32_t rows, int32_t cols) {
  Workspace w(nullptr, 0);
  ortho_carve(ortho_of(K, rows, cols), w);
  return w.off;
}

int launch_ortho(const OrthoStep& s, int32_t K, int32_t rows, int32_t cols, int32_t steps, const float* coef,
                 Workspace& ws, hipStream_t st) {
  const Ortho o = ortho_of(K, rows, cols);
  const OrthoSpace w = ortho_carve(o, ws);
  HMOE_TRY(over_slices(K, o.blocks, 256, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH("ortho start", k_ortho_start, dim3(o.blocks, (unsigned)count), dim3(256), 0, st, s, o, (int)m0, w.part);
    return (int)HMOE_OK;
  }));
  const int64_t parts = cdiv(o.rp, 64) * cdiv(o.lp, 64);
  HMOE_TRY(over_slices(K, parts, 256, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH("ortho split", k_ortho_split, dim3((unsigned)parts, (unsigned)count), dim3(256), 0, st, s, o, (int)m0,
                w.part, w.X[0], w.X[1]);
    return (int)HMOE_OK;
  }));
  const auto tiles = [&](int64_t m, int64_t n) { return cdiv(m, 256) * cdiv(n, 256) * K; };
  const bool gram_small = tiles(o.r, o.r) / 2 < device_cus(), apply_small = tiles(o.r, o.lp) < device_cus();
  for (int i = 0; i < steps; ++i) {
    const f16* X = w.X[i & 1];
    f16* next = w.X[1 - (i & 1)];
    if (gram_small) {
      HMOE_TRY((ortho_gram<PairSmall, false>(X, o, 0.f, 0.f, w.A, st)));
      HMOE_TRY((ortho_gram<PairSmall, true>(w.A, o, coef[1], coef[2], w.B, st)));
    } else {
      HMOE_TRY((ortho_gram<PairLarge, false>(X, o, 0.f, 0.f, w.A, st)));
      HMOE_TRY((ortho_gram<PairLarge, true>(w.A, o, coef[1], coef[2], w.B, st)));
    }
    const bool last = i == steps - 1;
    if (apply_small)
      HMOE_TRY(last ? (ortho_apply<PairSmallKS, true>(w.B, X, o, coef[0], next, s, st))
                    : (ortho_apply<PairSmallKS, false>(w.B, X, o, coef[0], next, s, st)));
    else
      HMOE_TRY(last ? (ortho_apply<PairLargeKS, true>(w.B, X, o, coef[0], next, s, st))
                    : (ortho_apply<PairLargeKS, false>(w.B, X, o, coef[0], next, s, st)));
  }
  return HMOE_OK;
}

}  // namespace hmoe
