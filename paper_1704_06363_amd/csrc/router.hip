// router.hip -- the learned router of a batch and its gradients:
//   s = R x + b, p = softmax(s), the top_k experts with their weights, counts and mean probabilities of the experts,
//   balance = K sum_e counts_e / (n top_k) mean p_e,  z = mean (ln sum exp s)^2,
// and with ds the gradient of the scores  dX = ds R, dR = ds^T X, db = sum ds.
//
// Bound by HBM: X is read for the scores and for dR, and dX written; the scores (K values a row) lie
// between.  The products are narrow (K columns, or a reduction over K).  ds is fp32 and keeps its accuracy on
// the matrix cores: with bf16 data a value is kept as three bf16 numbers that add up to it, in blocks of 16
// experts -- 16 values, their remainders, and the remainders of those.  The two steps of a block's first 32
// against 16 experts of R taken twice give dX to 2^-16, rounded to bf16 once; dR takes all three.
#include "fewrows.hpp"
#include "gemm.hpp"
#include "primitives.hpp"
#include "train_launch.hpp"

namespace hmoe {

namespace {

constexpr int kParts = 3;
__host__ __device__ inline int padded(int K) { return (K + 15) / 16 * 16; }
template <typename T>
__host__ __device__ inline int ds_width(int K) {
  return sizeof(T) == 2 ? kParts * padded(K) : padded(K);
}

// ------------------------------------------------------------------ scores

// scores [n][K] = X R^T + bias on the ring engine's narrow tiles.
template <class C>
__global__ void __launch_bounds__(C::THREADS)
    k_router_scores(const typename C::type* __restrict__ X, const typename C::type* __restrict__ R,
                    const float* __restrict__ bias, int64_t n, int K, int d, float* __restrict__ scores) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int nt = (K + C::BN - 1) / C::BN;
  const int64_t m0 = (int64_t)(blockIdx.x / nt) * C::BM;
  const int n0 = (int)(blockIdx.x % nt) * C::BN;
  const int rows = n - m0 < C::BM ? (int)(n - m0) : C::BM, cols = K - n0 < C::BN ? K - n0 : C::BN;
  floatx4 acc[C::MI][C::NJ];
  gemm_tile<C, true, true>(X + m0 * d, d, rows, R + (int64_t)n0 * d, d, cols, d, smem, acc);
  const Frag<C> f;
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = f.row(i, r), col = f.col(j, r);
        if (row < rows && col < cols) scores[(m0 + row) * K + n0 + col] = acc[i][j][r] + (bias ? bias[n0 + col] : 0.f);
      }
}

// ------------------------------------------------------------------ choices

// The largest of a key over L lanes, and sums, in each of them.
template <int L>
__device__ __forceinline__ uint64_t lanes_max(uint64_t k) {
  const auto step = [&](uint64_t o) { k = o > k ? o : k; };
  step(lane_xor<1>(k));
  step(lane_xor<2>(k));
  step(lane_xor<4>(k));
  step(lane_xor<8>(k));
  if constexpr (L > 16) {
    step(lane_xor<16>(k));
    step(lane_xor<32>(k));
  }
  return k;
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  return L > 16 ? wave_sum(v) : row_sum(v);
}

// e^(s - mx) where mx is the row's largest number: 0 for -inf in a row of nothing else, and NaN for NaN in any.
__device__ __forceinline__ float row_exp(float s, float mx) { return s == -INFINITY ? 0.f : expf(s - mx); }

// A workgroup's sums over its row groups of L lanes: acc[p] of expert p L + lane.
template <int L, int P, typename V>
__device__ __forceinline__ void experts_out(const V (&acc)[P], V* sh, int K, V* __restrict__ to) {
  constexpr int G = 256 / L, KP = P * L;
  const int g = threadIdx.x / L, lane = threadIdx.x % L;
#pragma unroll
  for (int p = 0; p < P; ++p) sh[g * KP + p * L + lane] = acc[p];
  __syncthreads();
  for (int e = threadIdx.x; e < K; e += 256) {
    V v = sh[e];
    for (int i = 1; i < G; ++i) v += sh[i * KP + e];
    to[e] = v;
  }
  __syncthreads();
}

// L lanes to a row, P scores to a lane.  A workgroup's counts, probabilities' sums and sum of squared lse go to
// its row of the parts.
template <int L, int P>
__global__ void __launch_bounds__(256)
    k_router_choose(const float* __restrict__ scores, int64_t n, int K, int top, int renorm, int32_t* __restrict__ expert,
                    float* __restrict__ weight, float* __restrict__ share_part, int32_t* __restrict__ count_part,
                    double* __restrict__ z_part) {
  constexpr int G = 256 / L;
  __shared__ double s_z[4];
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  const int lane = threadIdx.x % L;
  float share[P];
  int32_t count[P];
#pragma unroll
  for (int p = 0; p < P; ++p) share[p] = 0.f, count[p] = 0;
  double z = 0.0;
  for (int64_t first = (int64_t)blockIdx.x * G; first < n; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < n;
    float s[P];
#pragma unroll
    for (int p = 0; p < P; ++p) s[p] = live && p * L + lane < K ? scores[row * K + p * L + lane] : -INFINITY;
    uint64_t taken = 0;
    float chosen[HMOE_ROUTER_EXPERTS];
    int index[HMOE_ROUTER_EXPERTS];
#pragma unroll
    for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j) {
      if (j >= top) break;
      uint64_t best = 0;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const uint64_t k = p * L + lane < K && !((taken >> p) & 1) ? rank_key(s[p], p * L + lane) : 0;
        best = k > best ? k : best;
      }
      best = lanes_max<L>(best);
      const int e = (int)key_index(best);
      index[j] = e;
      chosen[j] = (uint32_t)(best >> 32) == 0 ? NAN : key_value(best);
      if (e % L == lane) {
        taken |= uint64_t(1) << (e / L);
        if (live && chosen[j] > -INFINITY) {
#pragma unroll
          for (int p = 0; p < P; ++p) count[p] += p == e / L;
        }
      }
    }
    const float mx = chosen[0];  // NaN only where all are
    float p_e[P], tot = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      p_e[p] = row_exp(s[p], mx);
      tot += p_e[p];
    }
    tot = lanes_sum<L>(tot);
    const bool none = tot == 0.f;  // nothing but -inf
    float of = tot;  // the weights' sum
    if (renorm) {
      of = tot != tot ? tot : 0.f;
#pragma unroll
      for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j)
        if (j < top) of += expf(chosen[j] - mx);
    }
    if (!live) continue;
    if (lane == 0) {
#pragma unroll
      for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j)
        if (j < top) {
          expert[row * top + j] = index[j];
          weight[row * top + j] = none ? 0.f : expf(chosen[j] - mx) / of;
        }
      if (!none) {
        const float lse = mx + logf(tot);
        z = fma((double)lse, (double)lse, z);
      }
    }
    if (!none) {
      const float inv = 1.f / tot;
#pragma unroll
      for (int p = 0; p < P; ++p) share[p] = fmaf(p_e[p], inv, share[p]);
    }
  }
  experts_out<L, P>(share, reinterpret_cast<float*>(smem_raw), K, share_part + (int64_t)blockIdx.x * K);
  experts_out<L, P>(count, reinterpret_cast<int32_t*>(smem_raw), K, count_part + (int64_t)blockIdx.x * K);
  z = wave_sum(z);
  if ((threadIdx.x & 63) == 0) s_z[threadIdx.x >> 6] = z;
  __syncthreads();
  if (threadIdx.x == 0) z_part[blockIdx.x] = (s_z[0] + s_z[1]) + (s_z[2] + s_z[3]);
}

// The parts added in order: a wave to 64 experts at a time, and the losses.  One workgroup.
__global__ void __launch_bounds__(1024)
    k_router_finish(const float* __restrict__ share_part, const int32_t* __restrict__ count_part,
                    const double* __restrict__ z_part, int blocks, int64_t n, int K, int top, int32_t* __restrict__ counts,
                    float* __restrict__ share, float* __restrict__ loss) {
  __shared__ double s_sum[16][64];
  __shared__ int32_t s_cnt[16][64];
  __shared__ double s_dot;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (threadIdx.x == 0) s_dot = 0.0;
  for (int e0 = 0; e0 < K; e0 += 64) {
    const int e = e0 + l;
    double p = 0.0;
    int32_t c = 0;
    if (e < K) {
#pragma unroll 8
      for (int b = w; b < blocks; b += 16) {
        p += share_part[(int64_t)b * K + e];
        c += count_part[(int64_t)b * K + e];
      }
    }
    __syncthreads();
    s_sum[w][l] = p;
    s_cnt[w][l] = c;
    __syncthreads();
    if (w == 0) {
      for (int i = 1; i < 16; ++i) {
        p += s_sum[i][l];
        c += s_cnt[i][l];
      }
      const float mean = n > 0 ? (float)(p / (double)n) : 0.f;
      if (e < K) {
        counts[e] = c;
        share[e] = mean;
      }
      const double dot = wave_sum(e < K ? (double)c * (double)mean : 0.0);
      if (l == 0) s_dot += dot;
    }
  }
  if (w == 0) {
    double z = 0.0;
    for (int b = l; b < blocks; b += 64) z += z_part[b];
    z = wave_sum(z);
    if (l == 0) {
      loss[0] = n > 0 ? (float)(s_dot * K / ((double)n * top)) : 0.f;
      loss[1] = n > 0 ? (float)(z / (double)n) : 0.f;
    }
  }
}

// ------------------------------------------------------------------ the scores' gradient

// ds in parts (ds_width) and a workgroup's sums of it.
template <typename T, int L, int P>
__global__ void __launch_bounds__(256)
    k_router_ds(const float* __restrict__ scores, const int32_t* __restrict__ expert, const int32_t* __restrict__ counts,
                const float* __restrict__ g_weight, int64_t n, int K, int top, int renorm, double balance, float z2,
                T* __restrict__ ds, float* __restrict__ bias_part) {
  constexpr int G = 256 / L;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  const int lane = threadIdx.x % L, ld = ds_width<T>(K), kp = padded(K);
  float q[P], sum[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    q[p] = p * L + lane < K ? (float)(balance * counts[p * L + lane]) : 0.f;
    sum[p] = 0.f;
  }
  for (int64_t first = (int64_t)blockIdx.x * G; first < n; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < n;
    float s[P], mx = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      s[p] = live && p * L + lane < K ? scores[row * K + p * L + lane] : -INFINITY;
      mx = fmaxf(mx, s[p]);
    }
    mx = fmaxf(mx, __uint_as_float(lane_xor<1>(__float_as_uint(mx))));
    mx = fmaxf(mx, __uint_as_float(lane_xor<2>(__float_as_uint(mx))));
    mx = fmaxf(mx, __uint_as_float(lane_xor<4>(__float_as_uint(mx))));
    mx = fmaxf(mx, __uint_as_float(lane_xor<8>(__float_as_uint(mx))));
    if constexpr (L > 16) {
      mx = fmaxf(mx, __uint_as_float(lane_xor<16>(__float_as_uint(mx))));
      mx = fmaxf(mx, __uint_as_float(lane_xor<32>(__float_as_uint(mx))));
    }
    float pe[P], g[P], on[P], tot = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      pe[p] = row_exp(s[p], mx);
      tot += pe[p];
      g[p] = on[p] = 0.f;
    }
    tot = lanes_sum<L>(tot);
    const bool none = tot == 0.f;
    if (g_weight && live) {
      for (int j = 0; j < top; ++j) {
        const int e = expert[row * top + j];
        const float gw = g_weight[row * top + j];
#pragma unroll
        for (int p = 0; p < P; ++p)
          if (e == p * L + lane && e < K) {
            g[p] += gw;
            on[p] = 1.f;
          }
      }
    }
    const float inv = none ? 0.f : 1.f / tot, lse = none ? 0.f : mx + logf(tot);
    float dot = 0.f, wt = 0.f, wg = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const float w = pe[p] * on[p];
      if (renorm) {
        wt += w;
        wg = fmaf(w, g[p], wg);
      }
      pe[p] *= inv;
      dot = fmaf(pe[p], renorm ? q[p] : q[p] + g[p], dot);
    }
    dot = lanes_sum<L>(dot);
    float wi = 0.f;
    if (renorm) {
      wt = lanes_sum<L>(wt);
      wg = lanes_sum<L>(wg);
      wi = wt > 0.f ? 1.f / wt : (wt == 0.f ? 0.f : wt);  // NaN stays
      wg *= wi;
    }
    const float zl = z2 * lse;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = p * L + lane;
      // the subtraction first: near p = 1 the sum is close to dot
      float v = pe[p] * (((renorm ? q[p] : q[p] + g[p]) - dot) + zl);
      if (renorm) v = fmaf(pe[p] * tot * on[p] * wi, g[p] - wg, v);
      if (!live || e >= K) v = 0.f;
      sum[p] += v;
      if (live && e < kp) {
        if constexpr (sizeof(T) == 2) {
          const Parts<T, kParts> parts(v);
          T* to = ds + row * ld + e / 16 * (16 * kParts) + e % 16;
#pragma unroll
          for (int i = 0; i < kParts; ++i) to[16 * i] = parts.part[i];
        } else {
          ds[row * ld + e] = v;
        }
      }
    }
  }
  experts_out<L, P>(sum, reinterpret_cast<float*>(smem_raw), K, bias_part + (int64_t)blockIdx.x * K);
}

// Rt [d][padded K] = R [K][d], zeros past K.
template <typename T>
__global__ void __launch_bounds__(256) k_router_transpose(const T* __restrict__ R, int K, int d, T* __restrict__ Rt) {
  __shared__ T s[16][65];
  const int c0 = blockIdx.x * 64, e0 = blockIdx.y * 16, kp = padded(K);
  for (int q = threadIdx.x; q < 16 * 64; q += 256) {
    const int e = q / 64, c = q % 64;
    s[e][c] = e0 + e < K && c0 + c < d ? R[(int64_t)(e0 + e) * d + c0 + c] : from_f32<T>(0.f);
  }
  __syncthreads();
  for (int q = threadIdx.x; q < 16 * 64; q += 256) {
    const int c = q / 16, e = q % 16;
    if (c0 + c < d) Rt[(int64_t)(c0 + c) * kp + e0 + e] = s[e][c];
  }
}

// ------------------------------------------------------------------ the products

// dX = ds R: 64 rows and 256 columns to a workgroup, 64 columns to a wave; fragments straight from memory.
template <typename T>
__global__ void __launch_bounds__(256) k_router_dx(const T* __restrict__ ds, const T* __restrict__ Rt, int64_t n, int K,
                                                   int d, T* __restrict__ dX) {
  const int col_tiles = (d + 255) / 256;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int64_t m0 = (int64_t)(blockIdx.x / col_tiles) * 64;
  const int c0 = (int)(blockIdx.x % col_tiles) * 256 + 64 * w, kp = padded(K), ld = ds_width<T>(K);
  if (c0 >= d) return;
  floatx4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const T *a[4], *b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 16 * i + lr < n ? m0 + 16 * i + lr : n - 1;
    a[i] = ds + row * ld + (sizeof(T) == 2 ? 8 : 4) * lg;
    const int col = c0 + 16 * i + lr < d ? c0 + 16 * i + lr : d - 1;
    b[i] = Rt + (int64_t)col * kp + (sizeof(T) == 2 ? 8 * (lg & 1) : 4 * lg);
  }
  for (int kb = 0; kb < kp / 16; ++kb) {
    i32x4 av[4], bv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      av[i] = *reinterpret_cast<const i32x4*>(a[i] + kb * (sizeof(T) == 2 ? 16 * kParts : 16));
      bv[i] = *reinterpret_cast<const i32x4*>(b[i] + kb * 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) step_mfma<T>(bv[j], av[i], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 16 * i + lr;
    if (row >= n) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = c0 + 16 * j + 4 * lg;
      if (col >= d) continue;
      typedef T quad __attribute__((ext_vector_type(4)));
      quad v;
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = from_f32<T>(acc[i][j][r]);
      *reinterpret_cast<quad*>(dX + row * d + col) = v;
    }
  }
}

// part[piece][K][d] = ds^T X over the piece's rows: 16 or 32 experts of bf16, 32 of fp32 and 256 columns to a workgroup.
template <typename T, int UW>
__global__ void __launch_bounds__(256) k_router_dr(const T* __restrict__ ds, const T* __restrict__ X, int64_t n, int K,
                                                   int d, int piece, float* __restrict__ part) {
  using C = Cfg<T, UW, 256, UW, 64>;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int ld = ds_width<T>(K), chunks = (ld + UW - 1) / UW;
  const int u0 = (int)(blockIdx.x % chunks) * UW, c0 = (int)(blockIdx.x / chunks) * 256;
  const int64_t p0 = (int64_t)blockIdx.y * piece;
  const int rows = n - p0 < piece ? (int)(n - p0) : piece;
  const int uv = ld - u0 < UW ? ld - u0 : UW, cv = d - c0 < 256 ? d - c0 : 256;
  floatx4 acc[C::MI][C::NJ];
  gemm_tile<C, false, false>(ds + p0 * ld + u0, ld, uv, X + p0 * d + c0, d, cv, rows, smem, acc);
  const Frag<C> f;
  float* to = part + (int64_t)blockIdx.y * K * d;
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = c0 + f.col(j, r);
        if constexpr (sizeof(T) == 2) {
          if (i % 3 != 0) continue;
          const int e = u0 / 3 + 16 * (i / 3) + 4 * f.lg + r;
          if (e < K && col < d) to[(int64_t)e * d + col] = (acc[i + 2][j][r] + acc[i + 1][j][r]) + acc[i][j][r];
        } else {
          const int e = u0 + f.row(i, r);
          if (e < K && col < d) to[(int64_t)e * d + col] = acc[i][j][r];
        }
      }
}

// dR and dbias: their parts added in order.
__global__ void __launch_bounds__(256) k_router_join(const float* __restrict__ part, int pieces, int64_t size,
                                                     float* __restrict__ dR, const float* __restrict__ bias_part, int blocks,
                                                     int K, float* __restrict__ dbias) {
  const int64_t groups = dR ? cdiv(size, 1024) : 0;
  if ((int64_t)blockIdx.x < groups) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size) return;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int q = 0; q < pieces; ++q) v += *reinterpret_cast<const floatx4*>(part + q * size + i);
    *reinterpret_cast<floatx4*>(dR + i) = v;
    return;
  }
  __shared__ float s[4][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, e = (int)(blockIdx.x - groups) * 64 + l;
  float v = 0.f;
  if (e < K) {
#pragma unroll 8
    for (int b = w; b < blocks; b += 4) v += bias_part[(int64_t)b * K + e];
  }
  s[w][l] = v;
  __syncthreads();
  if (w == 0 && e < K) dbias[e] = (s[0][l] + s[1][l]) + (s[2][l] + s[3][l]);
}

// ------------------------------------------------------------------ launches

// L and P for K experts.
template <class F>
int router_lanes(int K, F run) {
  using std::integral_constant;
  if (K <= 16) return run(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (K <= 64) return run(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (K <= 256) return run(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (K <= 1024) return run(integral_constant<int, 64>{}, integral_constant<int, 16>{});
  return run(integral_constant<int, 64>{}, integral_constant<int, 64>{});
}
int router_blocks(int64_t n, int K) {
  const int64_t rows = K <= 64 ? 16 : 4, all = cdiv(n, rows), most = 2 * device_cus();
  return (int)(all < most ? all : most);
}

template <typename T>
constexpr int kWide = sizeof(T) == 2 ? 96 : 32;  // columns of ds to a workgroup of k_router_dr
template <typename T>
int router_tiles(int K, int d) {
  const int uw = sizeof(T) == 2 && K <= 16 ? 48 : kWide<T>;
  return (ds_width<T>(K) + uw - 1) / uw * ((d + 255) / 256);
}
// Rows to a piece of dR's reduction.
template <typename T>
int router_piece(int64_t n, int K, int d) {
  int rows = 64;
  const int64_t tiles = router_tiles<T>(K, d);
  while (rows < (1 << 20) && cdiv(n, rows) * tiles > 2 * device_cus()) rows *= 2;
  return rows;
}

struct RouterSpace {
  float *share, *bias, *part;
  int32_t* count;
  double* z;
  void *ds, *Rt;
};
template <typename T>
RouterSpace router_carve(const hmoe_router_t* p, int64_t n, Workspace& ws) {
  RouterSpace s;
  const size_t parts = (size_t)router_blocks(n, p->K) * p->K;
  s.share = ws.take<float>(parts);
  s.bias = s.share;  // of the other direction
  s.count = ws.take<int32_t>(parts);
  s.z = ws.take<double>(router_blocks(n, p->K));
  s.ds = ws.take<T>((size_t)n * ds_width<T>(p->K));
  s.Rt = ws.take<T>((size_t)p->d * padded(p->K));
  s.part = ws.take<float>((size_t)cdiv(n, router_piece<T>(n, p->K, p->d)) * p->K * p->d);
  return s;
}

template <class C>
int router_scores(const hmoe_router_t* p, int64_t n, const void* X, float* scores, hipStream_t st) {
  using T = typename C::type;
  HMOE_LAUNCH("router scores", k_router_scores<C>, dim3((unsigned)(cdiv(n, C::BM) * cdiv(p->K, C::BN))), dim3(C::THREADS),
              C::LDS, st, (const T*)X, (const T*)p->R, p->bias, n, p->K, p->d, scores);
  return HMOE_OK;
}

template <typename T>
int router_forward_t(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight, float* scores,
                     int32_t* counts, float* share, float* loss, Workspace& ws, hipStream_t st) {
  const RouterSpace w = router_carve<T>(p, n, ws);
  const int blocks = n > 0 ? router_blocks(n, p->K) : 0;
  if (n > 0) {
    HMOE_TRY((router_scores<CfgD<T, 128, 64, 32, 64, 3>>(p, n, X, scores, st)));
    HMOE_TRY(router_lanes(p->K, [&](auto l, auto per) {
      constexpr int L = decltype(l)::value, P = decltype(per)::value;
      HMOE_LAUNCH("router choose", (k_router_choose<L, P>), dim3(blocks), dim3(256), 256 / L * P * L * 4, st, scores, n,
                  p->K, p->top_k, p->renorm != 0, expert, weight, w.share, w.count, w.z);
      return (int)HMOE_OK;
    }));
  }
  HMOE_LAUNCH("router finish", k_router_finish, dim3(1), dim3(1024), 0, st, w.share, w.count, w.z, blocks, n, p->K,
              p->top_k, counts, share, loss);
  return HMOE_OK;
}

template <typename T>
int router_backward_t(const hmoe_router_t* p, int64_t n, const void* X, const float* scores, const int32_t* expert,
                      const int32_t* counts, const float* g_weight, float balance, float z, void* dX, float* dR,
                      float* dbias, Workspace& ws, hipStream_t st) {
  const RouterSpace w = router_carve<T>(p, n, ws);
  const int K = p->K, d = p->d, blocks = router_blocks(n, K);
  const double even = (double)balance * K / ((double)n * n * p->top_k);
  const float z2 = (float)(2.0 * z / (double)n);
  T* ds = (T*)w.ds;
  HMOE_TRY(router_lanes(K, [&](auto l, auto per) {
    constexpr int L = decltype(l)::value, P = decltype(per)::value;
    HMOE_LAUNCH("router score gradient", (k_router_ds<T, L, P>), dim3(blocks), dim3(256), 256 / L * P * L * 4, st, scores,
                expert, counts, g_weight, n, K, p->top_k, p->renorm != 0, even, z2, ds, w.bias);
    return (int)HMOE_OK;
  }));
  if (dX) {
    HMOE_LAUNCH("router transpose", k_router_transpose<T>, dim3((unsigned)cdiv(d, 64), padded(K) / 16), dim3(256), 0, st,
                (const T*)p->R, K, d, (T*)w.Rt);
    HMOE_LAUNCH("router dX", k_router_dx<T>, dim3((unsigned)(cdiv(n, 64) * cdiv(d, 256))), dim3(256), 0, st, ds,
                (const T*)w.Rt, n, K, d, (T*)dX);
  }
  const int piece = router_piece<T>(n, K, d), pieces = (int)cdiv(n, piece);
  if (dR) {
    const dim3 grid(router_tiles<T>(K, d), pieces);
    if (sizeof(T) == 2 && K <= 16)
      HMOE_LAUNCH("router dR", (k_router_dr<T, 48>), grid, dim3(256), (Cfg<T, 48, 256, 48, 64>::LDS), st, ds, (const T*)X,
                  n, K, d, piece, w.part);
    else
      HMOE_LAUNCH("router dR", (k_router_dr<T, kWide<T>>), grid, dim3(256), (Cfg<T, kWide<T>, 256, kWide<T>, 64>::LDS), st,
                  ds, (const T*)X, n, K, d, piece, w.part);
  }
  if (dR || dbias) {
    const int64_t size = (int64_t)K * d;
    HMOE_LAUNCH("router join", k_router_join, dim3((unsigned)((dR ? cdiv(size, 1024) : 0) + (dbias ? cdiv(K, 64) : 0))),
                dim3(256), 0, st, w.part, pieces, size, dR, w.bias, blocks, K, dbias);
  }
  return HMOE_OK;
}

}  // namespace

size_t router_ws(const hmoe_router_t* p, int64_t n) {
  Workspace w(nullptr, 0);
  if (p->dt == HMOE_BF16) router_carve<bf16>(p, n, w); else router_carve<float>(p, n, w);
  return w.off;
}

int launch_router_forward(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight,
                          float* scores, int32_t* counts, float* share, float* loss, Workspace& ws, hipStream_t st) {
  if (p->dt == HMOE_BF16) return router_forward_t<bf16>(p, n, X, expert, weight, scores, counts, share, loss, ws, st);
  return router_forward_t<float>(p, n, X, expert, weight, scores, counts, share, loss, ws, st);
}

int launch_router_backward(const hmoe_router_t* p, int64_t n, const void* X, const float* scores,
                           const int32_t* expert, const int32_t* counts, const float* g_weight, float balance, float z,
                           void* dX, float* dR, float* dbias, Workspace& ws, hipStream_t st) {
  if (p->dt == HMOE_BF16)
    return router_backward_t<bf16>(p, n, X, scores, expert, counts, g_weight, balance, z, dX, dR, dbias, ws, st);
  return router_backward_t<float>(p, n, X, scores, expert, counts, g_weight, balance, z, dX, dR, dbias, ws, st);
}

}  // namespace hmoe
