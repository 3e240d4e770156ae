// ortho.hip -- Newton-Schulz iterations towards the orthogonal factor of K matrices, alone and as the update of a
// step with momentum:  X = U / |U|,  X <- a X + (b A + c A^2) X,  A = X X^T.
//
// With rows <= cols as they are and rows > cols transposed, X is [r][l], r <= l, and A [r][r].  A step is three
// products on the matrix cores, which bound it: r^2 l for A and r^3 for A^2, which are symmetric (the tiles on and
// above the diagonal are computed, the others are their mirror images), and 2 r^2 l for the last.  Two steps can
// be taken at once: with P = a + b A + c A^2 the next A is P A P, and X'' = P' P X -- 3 r^2 l + 5 r^3 instead of
// 6 r^2 l + 2 r^3.
//
// fp32 matrix instructions run at a sixteenth of the rate of fp16 ones.  Small singular values grow by a
// factor of a in every step, and so does what rounding adds to them: iterates of one 16-bit number (an error of
// 8e-2 after five steps where X has a rank of 3, 1.3e-2 with a floor of noise) are not enough.  Values are
// held as two fp16 numbers, hi + lo, 22 bits, and a product is hi hi + hi lo + lo hi, summed in fp32: three
// instructions.  (Emulated on the CPU, five steps in the order taken for fp32 results: 2e-6 for a random 512 x 1024
// matrix, where fp32 products give 4e-6; 9e-6 with a floor of noise and 7e-5 for a rank of 3, 7e-6 and 5e-5 there.)
// fp16 spans little: X is stored times 2^13, A and polynomials of it times 2^12 and products of two of those times 2^8,
// so that entries up to 8, 16 and 256 fit and the smallest lo, 2^-25, is 2^-38 of X -- 2^-25 of the mean entry of
// a matrix of 8192 x 8192.
#include "gemm.hpp"
#include "ortho.hpp"
#include "slices.hpp"

namespace hmoe {

namespace {

struct OrthoSpace {
  f16 *X[2], *A[3];
  double* part;   // [K][blocks]
  floatx4* part4;  // pieces of the products
};
OrthoSpace ortho_carve(const Ortho& o, size_t pieces, Workspace& ws) {
  OrthoSpace s;
  for (f16*& x : s.X) x = ws.take<f16>((size_t)o.K * o.x_size());
  for (f16*& a : s.A) a = ws.take<f16>((size_t)o.K * o.a_size());
  s.part = ws.take<double>((size_t)o.K * o.blocks);
  s.part4 = ws.take<floatx4>(pieces);
  return s;
}

// ------------------------------------------------------------------ the start

// v = momentum v + g, and the sums of squares of U, in fp64 (entries of 1e-30 and of 1e30 have squares there), of
// blockIdx.x's part of matrix m0 + blockIdx.y.
__global__ void __launch_bounds__(256) k_ortho_start(OrthoStep s, Ortho o, int m0, double* __restrict__ part) {
  __shared__ double sh[4];
  const int m = m0 + blockIdx.y;
  const int64_t size = (int64_t)o.rows * o.cols, base = m * size;
  double sum = 0.0;
  // a run of the matrix to a workgroup
  const int64_t run = cdiv(cdiv(size, gridDim.x), 1024) * 1024, first = blockIdx.x * run;
  const int64_t end = first + run < size ? first + run : size, step = 1024;
  const auto add = [&](floatx4 u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = fma((double)u[e], (double)u[e], sum);
  };
  for (int64_t q = first + threadIdx.x * 4; q < end; q += 2 * step) {
    const int64_t at = base + q, next = q + step < end ? at + step : at;
    if (!s.G && s.v) {  // both pairs of loads before the first store
      const floatx4 g0 = *reinterpret_cast<const floatx4*>(s.g + at), g1 = *reinterpret_cast<const floatx4*>(s.g + next);
      const floatx4 v0 = *reinterpret_cast<const floatx4*>(s.v + at), v1 = *reinterpret_cast<const floatx4*>(s.v + next);
      add(ortho_first_u(s, at, g0, v0));
      if (next != at) add(ortho_first_u(s, next, g1, v1));
    } else {
      const floatx4 u0 = ortho_u(s, at), u1 = ortho_u(s, next);
      add(u0);
      if (next != at) add(u1);
    }
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)m * o.blocks + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// X = U / |U| in pairs, 64 x 64 entries to a workgroup, zeros where X is padded.
__global__ void __launch_bounds__(256) k_ortho_split(OrthoStep s, Ortho o, int m0, const double* __restrict__ part,
                                                     f16* __restrict__ X) {
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
  }
}

// ------------------------------------------------------------------ the products

// Four or eight (N) values from column c (a multiple of N) of a row of pairs.
template <int N>
using f16xN = _Float16 __attribute__((ext_vector_type(N)));
template <int N>
__device__ __forceinline__ void put(f16* row, int c, const float* v) {
  f16xN<N> hi, lo;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    f16 h, l;
    pair_of(v[e], h, l);
    hi[e] = h;
    lo[e] = l;
  }
  *reinterpret_cast<f16xN<N>*>(row + pair_at(c)) = hi;
  *reinterpret_cast<f16xN<N>*>(row + pair_at(c) + kPairLo) = lo;
}
__device__ __forceinline__ void get8(const f16* row, int c, float (&v)[8]) {
  const f16x8 hi = *reinterpret_cast<const f16x8*>(row + pair_at(c));
  const f16x8 lo = *reinterpret_cast<const f16x8*>(row + pair_at(c) + kPairLo);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
}

// Tile `b` of those on and above the diagonal, column by column.
__device__ __forceinline__ void upper_tile(int b, int& mi, int& ni) {
  int c = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
  while (c * (c + 1) / 2 > b) --c;
  while ((c + 1) * (c + 2) / 2 <= b) ++c;
  ni = c;
  mi = b - c * (c + 1) / 2;
}

// One product for all matrices:  out = alpha L R + beta E + diag I in the numbers that are stored, L [r][k], and
//   symmetric: R^T [r][k], out [r][r];        otherwise: R [k][l], out [r][l].
struct Product {
  const f16 *L, *R, *E;  // E may be NULL
  f16* out;
  float alpha, beta, diag;
  int k;         // of the reduction, padded: lp or rp
  int64_t step;  // from a matrix' L (and a symmetric product's R) to the next's
  int per;       // tiles of a matrix
  int full;      // tiles of all matrices that are one workgroup's; of the others `split` share the reduction
  int split;
  floatx4* part;  // [tile][piece][accumulator][thread] of those
};

// Row stride of a matrix with `width` (padded) columns, in fp16 numbers.
__device__ __forceinline__ int64_t stride(int width) { return 2 * width; }

template <class C, bool SYM>
struct ProductTile {
  int m, r0, c0;      // matrix, first row and column
  bool mirror;        // off the diagonal
  __device__ __forceinline__ ProductTile(const Ortho& o, const Product& p, int tile) {
    m = tile / p.per;
    const int in = tile - m * p.per;
    if constexpr (SYM) {
      int mi, ni;
      upper_tile(in, mi, ni);
      r0 = mi * C::BM;
      c0 = ni * C::BN;
      mirror = mi != ni;
    } else {
      // rows fastest: the workgroups of a few rows of tiles share B's columns
      const int mt = (o.r + C::BM - 1) / C::BM;
      r0 = in % mt * C::BM;
      c0 = in / mt * C::BN;
      mirror = false;
    }
  }
};

// Accumulators (i, 2 h) and (i, 2 h + 1) of a tile stored; LAST: where `s` says.  Lanes 16 apart trade halves of the two
// blocks of 16 columns, after which each holds eight consecutive columns: 16-byte vectors of hi and of lo.  FULL: the
// tile has no rows or columns that do not exist, and nothing is behind a branch.
template <class C, bool SYM, bool LAST, bool FULL>
__device__ __forceinline__ void product_out(const Ortho& o, const Product& p, const OrthoStep& s,
                                            const ProductTile<C, SYM>& t, const Frag<C>& f, int i, int h, floatx4 a0,
                                            floatx4 a1) {
  const int row = t.r0 + f.row(i, 0), col = t.c0 + f.block(2 * h) + 16 * (f.lg & 1) + 8 * (f.lg >> 1);
  const int width = SYM ? o.rp : o.lp, cols = SYM ? o.r : o.l;
  const int64_t size = SYM ? o.a_size() : o.x_size();
  float v[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(a0[e]), __float_as_uint(a1[e]), false, false);
    v[e] = __uint_as_float(x[0]) * p.alpha;
    v[e + 4] = __uint_as_float(x[1]) * p.alpha;
  }
  if (p.E && (FULL || (row < o.r && col < width))) {
    float x[8];
    get8(p.E + t.m * size + row * stride(width), col, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(p.beta, x[e], v[e]);
  }
  if constexpr (!LAST) {
    // the padding is zeros: rows and columns past the last take part in no product but with zeros
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (SYM) v[e] += row == col + e ? p.diag : 0.f;
      if constexpr (!FULL) v[e] = row < o.r && col + e < cols ? v[e] : 0.f;
    }
    f16* out = p.out + t.m * size;
    if (FULL || (row < (SYM ? o.r : o.rp) && col < width)) put<8>(out + row * stride(width), col, v);
    if constexpr (SYM) {
      if (!t.mirror) return;
#pragma unroll
      for (int z = 0; z < 8; z += 4) {
        float u[4] = {v[z], v[z + 1], v[z + 2], v[z + 3]};
        quad_transpose(u);  // now of column col + z + lane % 4, rows 4 q .. 4 q + 3 of the 16
        const int tr = col + z + (f.lr & 3), tc = row - (f.lr & 3);
        if (FULL || tr < o.r) put<4>(out + tr * stride(width), tc, u);
      }
    }
  } else {
    // four entries in a row of the result: of a row of X, or (tall) of a column, which the quads turn; its rows are
    // cols long, a multiple of 8
    const int64_t base = (int64_t)t.m * o.rows * o.cols;
#pragma unroll
    for (int z = 0; z < 8; z += 4) {
      float u[4] = {v[z], v[z + 1], v[z + 2], v[z + 3]};
      int r = row, c = col + z;
      if (o.tall) {
        quad_transpose(u);
        r -= f.lr & 3;
        c += f.lr & 3;
      }
      if (FULL || (r < o.r && c < o.l)) ortho_put4(s, base + (o.tall ? (int64_t)c * o.cols + r : (int64_t)r * o.cols + c), u);
    }
  }
}
// All accumulators of a tile, or (ROWS = 1) those of row i0 alone.
template <class C, bool SYM, bool LAST, int ROWS>
__device__ __forceinline__ void product_rows(const Ortho& o, const Product& p, const OrthoStep& s,
                                             const ProductTile<C, SYM>& t, int i0, const floatx4 (&acc)[ROWS][C::NJ]) {
  const Frag<C> f;
  const auto rows = [&](auto full) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int h = 0; h < C::NJ / 2; ++h)
        product_out<C, SYM, LAST, decltype(full)::value>(o, p, s, t, f, i0 + i, h, acc[i][2 * h], acc[i][2 * h + 1]);
  };
  if (t.r0 + C::BM <= o.r && t.c0 + C::BN <= (SYM ? o.r : o.l)) rows(std::true_type{});
  else rows(std::false_type{});
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: the b-th of n gets the place that gives each XCD a
// run of its own.  (16 matrices of 2048 x 2048: tiles that share rows of A met in other L2s, and 415 us a square
// instead of 358.)
__device__ __forceinline__ int xcd_run(int b, int n) {
  const int even = n / 8 * 8;
  return b < even ? b % 8 * (even / 8) + b / 8 : b;
}

template <class C, bool SYM, bool LAST>
__global__ void __launch_bounds__(C::THREADS) k_ortho_product(Ortho o, Product p, OrthoStep s) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const bool whole = (int)blockIdx.x < p.full;
  const int b = whole ? xcd_run(blockIdx.x, p.full) : p.full + xcd_run(blockIdx.x - p.full, gridDim.x - p.full);
  const int q = b - p.full;
  const ProductTile<C, SYM> t(o, p, q < 0 ? b : p.full + q / p.split);
  constexpr int kStage = C::BK / 2;  // of the reduction
  const int stages = (p.k + kStage - 1) / kStage, piece = q < 0 ? 0 : q % p.split, pieces = q < 0 ? 1 : p.split;
  const int k0 = stages * piece / pieces * kStage, to = stages * (piece + 1) / pieces * kStage;
  const int k_len = (to < p.k ? to : p.k) - k0;
  const int64_t ldk = stride(p.k);
  const f16* L = p.L + t.m * p.step + t.r0 * ldk + stride(k0);
  const int rows = o.r - t.r0 < C::BM ? o.r - t.r0 : C::BM;
  floatx4 acc[C::MI][C::NJ];
  if constexpr (SYM) {
    const int cols = o.r - t.c0 < C::BN ? o.r - t.c0 : C::BN;
    const f16* R = p.R + t.m * p.step + t.c0 * ldk + stride(k0);
    PipeTile<C, true, true> g;
    g.prime(reinterpret_cast<const bf16*>(L), ldk, rows, reinterpret_cast<const bf16*>(R), ldk, cols, (int)stride(k_len), smem);
    g.run(smem, acc);
  } else {
    const int cols = o.lp - t.c0 < C::BN ? o.lp - t.c0 : C::BN;
    const int64_t ld = stride(o.lp);
    const f16* R = p.R + t.m * o.x_size() + k0 * ld + stride(t.c0);
    PipeTile<C, true, false> g;
    g.prime(reinterpret_cast<const bf16*>(L), ldk, rows, reinterpret_cast<const bf16*>(R), ld, cols, (int)stride(k_len), smem);
    g.run(smem, acc);
  }
  if (q < 0) {
    product_rows<C, SYM, LAST, C::MI>(o, p, s, t, 0, acc);
  } else {
    floatx4* to = p.part + (int64_t)q * C::MI * C::NJ * C::THREADS + threadIdx.x;
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) to[(i * C::NJ + j) * C::THREADS] = acc[i][j];
  }
}

// The same for few tiles and short reductions, where a product is all latency: 64 x 64 tiles of four waves, and 128 values of
// K of both operands to a trip to memory.  The next trip's loads go out before this one's products, but the barrier
// between waits for them, too, so that a trip takes a latency of memory and its products, one after the other.  (152 x
// 152 of 152 on the 128 x 128 tiles, three workgroups: 10 us, and 13 where the result adds A; 152 x 1356 of 152 28.)
// A K-contiguous operand's row is 512 bytes of LDS, chunk c of 16 bytes at c ^ (row & 15).  A K-strided one's 64 columns are 256
// bytes of a row of X, hi and lo of 32 columns and of the next 32, chunk c at c ^ sw(k) (ks_off's swizzle).
struct CfgMid {
  using type = f16;
  static constexpr bool TRANS = true, SPLIT = false, PAIR = true;
  static constexpr int BM = 64, BN = 64, WM = 32, WN = 32, WAVES_N = 2, WAVES_M = 2, WAVES = 4, THREADS = 256, MI = 2, NJ = 2;
  static constexpr int CK = 128;                  // K to a trip
  static constexpr int OPERAND = 64 * CK * 4, LDS = 4 * OPERAND;  // two of each: 128 KB
};
__device__ __forceinline__ int mid_sw(int k) { return ((k & 3) | ((k >> 1) & 4)) << 1; }

template <bool SYM, bool LAST>
__global__ void __launch_bounds__(256) k_ortho_mid(Ortho o, Product p, OrthoStep s) {
  using C = CfgMid;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* const smem = (lds<char>*)smem_raw;
  const int b = blockIdx.x, q = b - p.full;
  const ProductTile<C, SYM> t(o, p, q < 0 ? b : p.full + q / p.split);
  const int steps = p.k / 32, piece = q < 0 ? 0 : q % p.split, pieces = q < 0 ? 1 : p.split;  // p.k: a multiple of 32
  const int k_end = steps * (piece + 1) / pieces * 32;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Frag<C> f;
  floatx4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  // 16 rows to a wave, two to an instruction; rows past the last take a valid row's bytes, chunks past the end of K the
  // first's
  constexpr int LOADS = 16;  // of a wave and trip
  const auto load_rows = [&](const f16* from, int r0, int k0, int len, lds<char>* to) {
    const char* base = reinterpret_cast<const char*>(from) + (int64_t)k0 * 4;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const int row = 16 * w + i + (l >> 5), at = r0 + row < o.r ? r0 + row : o.r - 1, c = (l & 31) ^ (row & 15);
      __builtin_amdgcn_global_load_lds((const void*)(base + (int64_t)at * 4 * p.k + (c * 4 < len ? c : 0) * 16),
                                       (lds<void>*)(to + (16 * w + i) * 512), 16, 0, 0);
    }
  };
  const int k_begin = steps * piece / pieces * 32;
  const auto length = [&](int k0) { return k_end - k0 < C::CK ? k_end - k0 : C::CK; };
  const auto load = [&](int k0, int buffer) {
    lds<char>* const to = smem + buffer * 2 * C::OPERAND;
    const int len = length(k0);
    load_rows(p.L + t.m * p.step, t.r0, k0, len, to);
    if constexpr (SYM) {
      load_rows(p.R + t.m * p.step, t.c0, k0, len, to + C::OPERAND);
    } else {
      const char* base = reinterpret_cast<const char*>(p.R + t.m * o.x_size()) + (int64_t)t.c0 * 4;
      const int groups = (o.lp - t.c0) / 32 < 2 ? 1 : 2;  // of 32 columns
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = 32 * w + 4 * i + (l >> 4), c = (l & 15) ^ mid_sw(k);
        const int64_t row = k0 + (k < len ? k : 0);
        __builtin_amdgcn_global_load_lds((const void*)(base + row * 4 * o.lp + ((c >> 3) < groups ? c : c & 7) * 16),
                                         (lds<void>*)(to + C::OPERAND + (32 * w + 4 * i) * 256), 16, 0, 0);
      }
    }
  };
  load(k_begin, 0);
  int buffer = 0;
  for (int k0 = k_begin; k0 < k_end; k0 += C::CK, buffer ^= 1) {
    const int len = length(k0);
    if (k0 + C::CK < k_end) {
      load(k0 + C::CK, buffer ^ 1);
      wait_vmcnt<LOADS>();
    } else {
      wait_vmcnt<0>();
    }
    __syncthreads();
    lds<char>* const sl = smem + buffer * 2 * C::OPERAND;
    lds<char>* const sr = sl + C::OPERAND;
    for (int ks = 0; ks < len / 32; ++ks) {
      f16x8 a[2][2], bb[2][2];  // [fragment][hi, lo]
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int row = f.wm * 32 + 16 * i + f.lr;
          a[i][z] = *reinterpret_cast<const lds<f16x8>*>(sl + row * 512 + (((8 * ks + 4 * z + f.lg) ^ (row & 15)) << 4));
        }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          if constexpr (SYM) {
            const int row = f.wn * 32 + 16 * j + f.lr;
            bb[j][z] = *reinterpret_cast<const lds<f16x8>*>(sr + row * 512 + (((8 * ks + 4 * z + f.lg) ^ (row & 15)) << 4));
          } else {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef short s8 __attribute__((ext_vector_type(8)));
            const int k = 32 * ks + 8 * f.lg + (f.lr >> 2), c = f.wn * 8 + z * 4 + j * 2 + ((f.lr & 3) >> 1);
            lds<char>* at = sr + k * 256 + ((c ^ mid_sw(k)) << 4) + (f.lr & 1) * 8;
            const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds<s4>*)at);
            const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds<s4>*)(at + 4 * 256));
            bb[j][z] = __builtin_bit_cast(f16x8, s8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
          }
        }
#pragma unroll
      for (int z = 0; z < 3; ++z)  // the small products first
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bb[j][z == 0], a[i][z == 1], acc[i][j], 0, 0, 0);
    }
    __syncthreads();  // before the loads of the trip after the next
  }
  if (q < 0) {
    product_rows<C, SYM, LAST, 2>(o, p, s, t, 0, acc);
  } else {
    floatx4* to = p.part + (int64_t)q * 4 * 256 + threadIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) to[(i * 2 + j) * 256] = acc[i][j];
  }
}

// The pieces of the tiles that are split added in order, and their results: blockIdx.y names the accumulators' row.
template <class C, bool SYM, bool LAST>
__global__ void __launch_bounds__(C::THREADS) k_ortho_join(Ortho o, Product p, OrthoStep s) {
  const ProductTile<C, SYM> t(o, p, p.full + blockIdx.x);
  const int i = blockIdx.y;
  const floatx4* from = p.part + ((int64_t)blockIdx.x * p.split * C::MI + i) * C::NJ * C::THREADS + threadIdx.x;
  floatx4 acc[1][C::NJ];
#pragma unroll
  for (int j = 0; j < C::NJ; ++j) acc[0][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int q = 0; q < p.split; ++q)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) acc[0][j] += from[((int64_t)q * C::MI * C::NJ + j) * C::THREADS];
  product_rows<C, SYM, LAST, 1>(o, p, s, t, i, acc);
}

// Tiles: 256 x 256 of eight waves, or 128 x 128 and 128 x 256 (the swizzle of a K-strided operand spans 256 columns).
template <bool LARGE, bool SYM>
struct PickTile;
template <>
struct PickTile<true, true> { using C = CfgPair<256, 256, 128, 64, false>; };
template <>
struct PickTile<true, false> { using C = CfgPair<256, 256, 128, 64, true>; };
template <>
struct PickTile<false, true> { using C = CfgPair<128, 128, 64, 64, false>; };
template <>
struct PickTile<false, false> { using C = CfgPair<128, 256, 64, 64, true>; };

// How the tiles of a product are dealt out.  Whole rounds of the CUs take a tile each; the tiles of the last round, if
// two or more workgroups are there for each, share their reductions, four stages at least to a piece.
struct Deal {
  bool large, mid;
  int per, full, split, rest;
  size_t part;  // floatx4 of the pieces
};
template <class C>
Deal deal_on(const Ortho& o, int k, bool sym) {
  Deal d;
  const int64_t mt = cdiv(o.r, C::BM);
  d.per = (int)(sym ? mt * (mt + 1) / 2 : mt * cdiv(o.lp, C::BN));
  const int64_t tiles = (int64_t)d.per * o.K;
  const int64_t slots = (int64_t)device_cus() * (C::LDS <= 64 * 1024 ? 2 : 1);
  const int64_t rest = tiles % slots, fit = rest > 0 ? slots / rest : 1, most = k / 32 / 4;
  int64_t split = fit < most ? fit : most;
  split = split < 2 ? 1 : split > 64 ? 64 : split;
  // what sharing saves of a tile's stages against the launch that joins the pieces (16 matrices of 562 x 562: 20 us for the
  // halves and 12 to join them, 22 whole)
  constexpr float stage = C::BM * C::BN == 256 * 256 ? 2.3f : C::BN == 256 ? 1.1f : 0.6f;  // us
  if ((1.f - 1.f / split) * (k / 32) * stage < 12.f) split = 1;
  d.split = (int)split;
  d.full = (int)(d.split > 1 ? tiles - rest : tiles);
  d.rest = (int)(d.split > 1 ? rest : 0);
  d.part = (size_t)d.rest * d.split * C::MI * C::NJ * C::THREADS;
  return d;
}
// For k_ortho_mid: all tiles split, or none; a piece for every two trips if they fit on the chip at once.
Deal deal_mid(const Ortho& o, int k, bool sym) {
  using C = CfgMid;
  Deal d = {};
  d.mid = true;
  const int64_t mt = cdiv(o.r, C::BM);
  d.per = (int)(sym ? mt * (mt + 1) / 2 : mt * cdiv(o.lp, C::BN));
  const int64_t tiles = (int64_t)d.per * o.K, fit = device_cus() / tiles, trips = cdiv(k, 2 * C::CK);
  d.split = (int)(trips <= 2 ? 1 : trips < fit ? trips : fit < 1 ? 1 : fit);  // a trip takes less than a launch
  d.full = (int)(d.split > 1 ? 0 : tiles);
  d.rest = (int)(d.split > 1 ? tiles : 0);
  d.part = (size_t)d.rest * d.split * C::MI * C::NJ * C::THREADS;
  return d;
}
// Whether a problem's products are few tiles and short reductions, by the squares of its small matrices: the Gram matrix
// and the product with X follow them, however long the other side is (five of 512 x 2048: 1280 tiles of X, five rounds of
// the CUs).
bool is_mid(const Ortho& o) {
  const int64_t mt = cdiv(o.r, 128);
  return o.r <= 512 && mt * (mt + 1) / 2 * o.K < device_cus() / 4;
}
// k_ortho_mid also takes the symmetric products of larger matrices whose tiles all run at once (1024 x 1024 in pieces of
// 128 x 128 tiles: 14 us, and 7 to join them).
Deal deal(const Ortho& o, int k, bool sym) {
  if (is_mid(o)) return deal_mid(o, k, sym);
  const int64_t m64 = cdiv(o.r, 64);
  if (sym && k == o.rp && m64 * (m64 + 1) / 2 * o.K <= device_cus()) return deal_mid(o, k, sym);
  using L = PickTile<true, true>::C;
  const int64_t mt = cdiv(o.r, L::BM), tiles = (sym ? mt * (mt + 1) / 2 : mt * cdiv(o.lp, L::BN)) * o.K;
  // enough work for the large tiles: pieces of sixteen stages on every CU
  const bool large = tiles * (k / 32) / 16 >= device_cus();
  Deal d = large ? deal_on<L>(o, k, sym)
                 : sym ? deal_on<PickTile<false, true>::C>(o, k, sym) : deal_on<PickTile<false, false>::C>(o, k, sym);
  d.large = large;
  d.mid = false;
  return d;
}

// What a product is, and by the height of its tiles what its launch is called.
enum Kind { kGram, kSquare, kApply };
const char* label_of(Kind what, int height) {
  static const char* const names[3][3] = {{"ortho gram 64", "ortho gram 128", "ortho gram 256"},
                                          {"ortho square 64", "ortho square 128", "ortho square 256"},
                                          {"ortho apply 64", "ortho apply 128", "ortho apply 256"}};
  return names[what][height / 128];
}
template <class C, bool SYM, bool LAST>
int product_on(Kind what, const Ortho& o, Product p, const Deal& d, const OrthoStep& s, hipStream_t st) {
  p.per = d.per;
  p.full = d.full;
  p.split = d.split;
  HMOE_LAUNCH(label_of(what, C::BM), (k_ortho_product<C, SYM, LAST>),
              dim3((unsigned)(d.full + d.rest * d.split)), dim3(C::THREADS), C::LDS, st, o, p, s);
  if (d.rest)
    HMOE_LAUNCH("ortho join", (k_ortho_join<C, SYM, LAST>), dim3(d.rest, C::MI), dim3(C::THREADS), 0, st, o, p, s);
  return HMOE_OK;
}
template <bool SYM, bool LAST = false>
int product(Kind what, const Ortho& o, const Product& p, const OrthoStep& s, hipStream_t st) {
  const Deal d = deal(o, p.k, SYM);
  if (d.mid) {
    Product m = p;
    m.per = d.per;
    m.full = d.full;
    m.split = d.split;
    HMOE_LAUNCH(label_of(what, CfgMid::BM), (k_ortho_mid<SYM, LAST>), dim3((unsigned)(d.full + d.rest * d.split)),
                dim3(CfgMid::THREADS), CfgMid::LDS, st, o, m, s);
    if (d.rest)
      HMOE_LAUNCH("ortho join", (k_ortho_join<CfgMid, SYM, LAST>), dim3(d.rest, CfgMid::MI), dim3(CfgMid::THREADS), 0, st, o,
                  m, s);
    return HMOE_OK;
  }
  if (d.large) return product_on<typename PickTile<true, SYM>::C, SYM, LAST>(what, o, p, d, s, st);
  return product_on<typename PickTile<false, SYM>::C, SYM, LAST>(what, o, p, d, s, st);
}

size_t part_size(const Ortho& o) {
  size_t most = 0;
  for (const Deal& d : {deal(o, o.lp, true), deal(o, o.rp, true), deal(o, o.rp, false)}) most = d.part > most ? d.part : most;
  return most;
}

// The steps of one call: X in one of two buffers, the small matrices in three.
struct Iterations {
  const Ortho& o;
  const OrthoSpace& w;
  const OrthoStep& s;
  hipStream_t st;
  float a, b, c;
  int at = 0;  // the buffer that holds X

  Product make(const f16* L, const f16* R, const f16* E, f16* out, float alpha, float beta, float diag) const {
    const bool of_x = L == w.X[at];
    return Product{L, R, E, out, alpha, beta, diag, of_x ? o.lp : o.rp, of_x ? o.x_size() : o.a_size(), 0, 0, 1, w.part4};
  }
  int gram(f16* A) {
    return product<true>(kGram, o, make(w.X[at], w.X[at], nullptr, A, kScaleA / (kScaleX * kScaleX), 0.f, 0.f), s, st);
  }
  // diag + b A + c A^2
  int poly(const f16* A, float diag, f16* P) {
    return product<true>(kSquare, o, make(A, A, A, P, c / kScaleA, b, diag * kScaleA), s, st);
  }
  int times(const f16* L, const f16* R, float scale, f16* out) {
    return product<true>(kSquare, o, make(L, R, nullptr, out, scale, 0.f, 0.f), s, st);
  }
  // X = x X + Q X with Q stored times `scale`
  int apply(const f16* Q, float scale, float x, bool last) {
    const float unit = last ? 1.f / kScaleX : 1.f;
    const Product p = make(Q, w.X[at], x != 0.f ? w.X[at] : nullptr, w.X[1 - at], unit / scale, unit * x, 0.f);
    at = 1 - at;
    return last ? product<false, true>(kApply, o, p, s, st) : product<false>(kApply, o, p, s, st);
  }
  int one(bool last) {
    HMOE_TRY(gram(w.A[0]));
    HMOE_TRY(poly(w.A[0], 0.f, w.A[1]));
    return apply(w.A[1], kScaleA, a, last);
  }
  int two(bool last) {
    HMOE_TRY(gram(w.A[0]));
    HMOE_TRY(poly(w.A[0], a, w.A[1]));                                       // P
    HMOE_TRY(times(w.A[1], w.A[0], 1.f / kScaleA, w.A[2]));                  // P A
    HMOE_TRY(times(w.A[2], w.A[1], 1.f / kScaleA, w.A[0]));                  // P A P, the next A
    HMOE_TRY(poly(w.A[0], a, w.A[2]));                                       // P'
    HMOE_TRY(times(w.A[2], w.A[1], kScaleQ / (kScaleA * kScaleA), w.A[0]));  // P' P
    return apply(w.A[0], kScaleQ, 0.f, last);
  }
};

}  // namespace

int launch_ortho_start(const OrthoStep& s, const Ortho& o, double* part, hipStream_t st) {
  return over_slices(o.K, o.blocks, 256, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH("ortho start", k_ortho_start, dim3(o.blocks, (unsigned)count), dim3(256), 0, st, s, o, (int)m0, part);
    return (int)HMOE_OK;
  });
}

size_t ortho_ws(int32_t K, int32_t rows, int32_t cols) {
  Workspace w(nullptr, 0);
  const Ortho o = ortho_of(K, rows, cols);
  if (small_ortho_ws(o) > 0) return small_ortho_ws(o);
  ortho_carve(o, part_size(o), w);
  return w.off;
}

int launch_ortho(const OrthoStep& s, int32_t K, int32_t rows, int32_t cols, int32_t steps, const float* coef,
                 Workspace& ws, hipStream_t st) {
  const Ortho o = ortho_of(K, rows, cols);
  if (small_ortho_ws(o) > 0) return launch_small_ortho(s, o, steps, coef, ws, st);
  const OrthoSpace w = ortho_carve(o, part_size(o), ws);
  HMOE_TRY(launch_ortho_start(s, o, w.part, st));
  const int64_t parts = cdiv(o.rp, 64) * cdiv(o.lp, 64);
  HMOE_TRY(over_slices(K, parts, 256, [&](int64_t m0, int64_t count) {
    HMOE_LAUNCH("ortho split", k_ortho_split, dim3((unsigned)parts, (unsigned)count), dim3(256), 0, st, s, o, (int)m0,
                w.part, w.X[0]);
    return (int)HMOE_OK;
  }));
  Iterations it{o, w, s, st, coef[0], coef[1], coef[2]};
  // Two steps at once where that is less work.  What rounding leaves in A is amplified by a^2 on its way into the
  // second one's, so the first step of all, where the smallest singular values are, is taken alone (rank 3, five
  // steps: 1.0e-4 with the first two together, 6.9e-5 so, 5.0e-5 with none, fp32 products 4.6e-5).
  const bool twos = 2 * o.l >= 3 * o.r;
  for (int i = 0; i < steps;) {
    const int n = twos && i > 0 && steps - i >= 2 ? 2 : 1;
    HMOE_TRY(n == 2 ? it.two(i + n == steps) : it.one(i + n == steps));
    i += n;
  }
  return HMOE_OK;
}

}  // namespace hmoe
