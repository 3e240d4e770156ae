// router.hip -- the learned router of a batch and its gradients:
//   s = R x + b, p = softmax(s), the top_k experts with their weights, counts and mean probabilities of the experts,
//   balance = K sum_e counts_e / (n top_k) mean p_e,  z = mean (ln sum exp s)^2,
// and with ds the gradient of the scores  dX = ds R, dR = ds^T X, db = sum ds.
//
// Bound by HBM: X is read for the scores and for dR, and dX written; the scores (K values a row) lie
// between.  The products are narrow (K columns, or a reduction over K).  ds is fp32 and keeps its accuracy on
// the matrix cores: with bf16 data a value is kept as three bf16 numbers that add up to it, a row's in three planes,
// [values, their remainders, the remainders of those][experts, padded to 16], and both dX and dR take all three, against R
// or X taken three times; dX is rounded to bf16 once.
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

// scores [n][K] = X R^T + bias on the ring engine's narrow tiles; of several pieces of the reduction (gridDim.y) each
// its part in a plane of `scores`, without the bias.
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
  const int units = (d + 63) / 64, s = blockIdx.y, pieces = gridDim.y;
  const int k0 = (int)((int64_t)units * s / pieces) * 64, to = (int)((int64_t)units * (s + 1) / pieces) * 64;
  floatx4 acc[C::MI][C::NJ];
  gemm_tile<C, true, true>(X + m0 * d + k0, d, rows, R + (int64_t)n0 * d + k0, d, cols, (to < d ? to : d) - k0, smem, acc);
  static_assert(C::TRANS, "four consecutive scores to a lane");
  const Frag<C> f;
  float* out = scores + ((int64_t)s * n + m0) * K + n0;
  const bool vec = K % 4 == 0;
#pragma unroll
  for (int j = 0; j < C::NJ; ++j) {
    const int col = f.col(j, 0);
    float b[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) b[r] = bias && pieces == 1 && col + r < cols ? bias[n0 + col + r] : 0.f;
#pragma unroll
    for (int i = 0; i < C::MI; ++i) {
      const int row = f.row(i, 0);
      if (row >= rows || col >= cols) continue;
      float* to = out + (int64_t)row * K + col;
      if (vec) {
        *reinterpret_cast<floatx4*>(to) = acc[i][j] + floatx4{b[0], b[1], b[2], b[3]};
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (col + r < cols) to[r] = acc[i][j][r] + b[r];
      }
    }
  }
}

// ------------------------------------------------------------------ choices

// `op` over L lanes, and sums, in each of them.
template <int L, class Op>
__device__ __forceinline__ uint32_t lanes_reduce(uint32_t k, Op op) {
  if constexpr (L > 16) {
    k = op(k, lane_xor<32>(k));
    k = op(k, lane_xor<16>(k));
  }
  const auto turned = [&](auto ctrl) {  // within the rows of 16 lanes, whose values repeat with the distance then
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)k, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  k = op(k, turned(std::integral_constant<int, 0x128>{}));
  k = op(k, turned(std::integral_constant<int, 0x124>{}));
  k = op(k, turned(std::integral_constant<int, 0x122>{}));
  return op(k, turned(std::integral_constant<int, 0x121>{}));
}
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t k) {
  return lanes_reduce<L>(k, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int L>
__device__ __forceinline__ uint32_t lanes_min(uint32_t k) {
  return lanes_reduce<L>(k, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  return L > 16 ? wave_sum(v) : row_sum(v);
}

// e^(s - mx) where mx is the row's largest number: 0 for -inf in a row of nothing else, and NaN for NaN in any.
__device__ __forceinline__ float row_exp(float s, float mx) { return s == -INFINITY ? 0.f : expf(s - mx); }

// A workgroup's sums over its row groups of L lanes: acc[p] of expert p L + lane.
template <int L, int P, int THREADS, typename V>
__device__ __forceinline__ void experts_out(const V (&acc)[P], V* sh, int K, V* __restrict__ to) {
  constexpr int G = THREADS / L, KP = P * L;
  const int g = threadIdx.x / L, lane = threadIdx.x % L;
#pragma unroll
  for (int p = 0; p < P; ++p) sh[g * KP + p * L + lane] = acc[p];
  __syncthreads();
  for (int e = threadIdx.x; e < K; e += THREADS) {
    V v = sh[e];
#pragma unroll 4
    for (int i = 1; i < G; ++i) v += sh[i * KP + e];
    to[e] = v;
  }
  __syncthreads();
}

// Threads of the kernels that take a row at a time, with P scores to each of L lanes: as many as registers allow.  P = 64,
// for more than 1024 experts, is past them: 1551 registers of the choices and 324 (bf16) and 164 of ds live in scratch
// memory.  (16384 rows: choices 99 us with 1024 experts, 1580 with 2048, 1700 with 4096; ds 84, 577 and 817, by
// events around the launches.)
template <int P>
constexpr int kRowThreads = P <= 4 ? 1024 : P <= 8 ? 512 : 256;

// What becomes of rows of scores, L lanes to a row and P scores to a lane: expert p L + lane.
struct Choices {
  int64_t n;
  int K, top, renorm;
  int32_t* expert;
  float* weight;
  float* share_part;     // [workgroup][K]: a workgroup's sums of probabilities,
  int32_t* count_part;   // counts,
  double* z_part;        // [workgroup] and sums of squared lse
};
template <int L, int P, int THREADS>
struct Chooser {
  float share[P];
  int32_t count[P];
  double z;
  __device__ __forceinline__ Chooser() : z(0.0) {
#pragma unroll
    for (int p = 0; p < P; ++p) share[p] = 0.f, count[p] = 0;
  }
  // Row `row` if `live`; entered by whole waves.
  __device__ __forceinline__ void take(const Choices& c, int64_t row, bool live, const float (&s)[P]) {
    const int lane = threadIdx.x % L;
    uint32_t key[P];  // 0: no entry, or taken; 1: NaN
#pragma unroll
    for (int p = 0; p < P; ++p) key[p] = p * L + lane < c.K ? sortable(s[p]) + 1 : 0;
    float chosen[HMOE_ROUTER_EXPERTS];
    int index[HMOE_ROUTER_EXPERTS];
#pragma unroll
    for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j) {
      if (j >= c.top) break;
      uint32_t best = key[0], at = ~0u;
#pragma unroll
      for (int p = 1; p < P; ++p) best = key[p] > best ? key[p] : best;
      best = lanes_max<L>(best);
#pragma unroll
      for (int p = P - 1; p >= 0; --p) at = key[p] == best ? p * L + lane : at;
      at = lanes_min<L>(at);
      index[j] = (int)at;
      const uint32_t u = best - 1;
      chosen[j] = u == 0 ? NAN : __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const bool mine = at == (uint32_t)(p * L + lane);
        key[p] = mine ? 0 : key[p];
        count[p] += mine && live && chosen[j] > -INFINITY;
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
    if (c.renorm) {
      of = tot != tot ? tot : 0.f;
#pragma unroll
      for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j)
        if (j < c.top) of += expf(chosen[j] - mx);
    }
    if (!live) return;
    if (lane == 0) {
#pragma unroll
      for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j)
        if (j < c.top) {
          c.expert[row * c.top + j] = index[j];
          c.weight[row * c.top + j] = none ? 0.f : expf(chosen[j] - mx) / of;
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
  // The workgroup's sums; `sh` holds THREADS P values.
  __device__ __forceinline__ void leave(const Choices& c, char* sh) {
    __shared__ double s_z[THREADS / 64];
    experts_out<L, P, THREADS>(share, reinterpret_cast<float*>(sh), c.K, c.share_part + (int64_t)blockIdx.x * c.K);
    experts_out<L, P, THREADS>(count, reinterpret_cast<int32_t*>(sh), c.K, c.count_part + (int64_t)blockIdx.x * c.K);
    z = wave_sum(z);
    if ((threadIdx.x & 63) == 0) s_z[threadIdx.x >> 6] = z;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int i = 1; i < THREADS / 64; ++i) z += s_z[i];
      c.z_part[blockIdx.x] = z;
    }
  }
};

// With `planes` the scores are their sum and the bias, and are written, too.
template <int L, int P>
__global__ void __launch_bounds__(kRowThreads<P>)
    k_router_choose(float* __restrict__ scores, const float* __restrict__ planes, int pieces, const float* __restrict__ bias,
                    Choices c) {
  constexpr int THREADS = kRowThreads<P>, G = THREADS / L;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  const int lane = threadIdx.x % L, K = c.K;
  Chooser<L, P, THREADS> choose;
  for (int64_t first = (int64_t)blockIdx.x * G; first < c.n; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < c.n;
    float s[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = p * L + lane;
      s[p] = -INFINITY;
      if (!live || e >= K) continue;
      if (!planes) {
        s[p] = scores[row * K + e];
        continue;
      }
      s[p] = 0.f;
#pragma unroll 4
      for (int z = 0; z < pieces; ++z) s[p] += planes[((int64_t)z * c.n + row) * K + e];
      if (bias) s[p] += bias[e];
      scores[row * K + e] = s[p];
    }
    choose.take(c, row, live, s);
  }
  choose.leave(c, smem_raw);
}

// Scores and choices of up to 16 P experts in one: a tile of scores goes through LDS to 16 lanes a row, and is not read
// again.  Nothing of the next tile is loaded while a tile's rows choose, so that the gain is the launch and the scores' way
// back.  (us a forward of bf16, so and in two kernels: 65536 rows, d = 2048, 16 experts 80.5 and 82.8, 32 84.0 and
// 85.2, 64 91.0 and 91.0; 32768 rows of 128 57.3 and 62.8; 65536 x 512 of 16 25.4 and 28.5; fp32, 32768 x 2048 of 16 135 and 136.)
template <class C>
constexpr int scored_lds() {
  constexpr int rows = C::BM * (C::BN + 4) * 4;
  return rows > C::LDS ? rows : C::LDS;
}
template <class C, int P>
__global__ void __launch_bounds__(C::THREADS)
    k_router_score_choose(const typename C::type* __restrict__ X, const typename C::type* __restrict__ R,
                          const float* __restrict__ bias, int d, float* __restrict__ scores, Choices c) {
  constexpr int L = 16, G = C::THREADS / L, LD = C::BN + 4;
  static_assert(L * P <= C::BN, "scores of the tile");
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  lds<float>* tile = (lds<float>*)smem_raw;
  const int lane = threadIdx.x % L, K = c.K;
  const Frag<C> f;
  Chooser<L, P, C::THREADS> choose;
  for (int64_t m0 = (int64_t)blockIdx.x * C::BM; m0 < c.n; m0 += (int64_t)gridDim.x * C::BM) {
    const int rows = c.n - m0 < C::BM ? (int)(c.n - m0) : C::BM;
    floatx4 acc[C::MI][C::NJ];
    gemm_tile<C, true, true>(X + m0 * d, d, rows, R, d, K, d, smem, acc);
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) {
      const int col = f.col(j, 0);
      floatx4 b;
#pragma unroll
      for (int r = 0; r < 4; ++r) b[r] = bias && col + r < K ? bias[col + r] : 0.f;
#pragma unroll
      for (int i = 0; i < C::MI; ++i) *reinterpret_cast<lds<floatx4>*>(tile + f.row(i, 0) * LD + col) = acc[i][j] + b;
    }
    __syncthreads();
    for (int r = threadIdx.x / L; r < C::BM; r += G) {
      float s[P];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int e = p * L + lane;
        s[p] = e < K ? tile[r * LD + e] : -INFINITY;
        if (r < rows && e < K) scores[(m0 + r) * K + e] = s[p];
      }
      choose.take(c, m0 + r, r < rows, s);
    }
    __syncthreads();  // before the next tile's loads
  }
  choose.leave(c, smem_raw);
}

// The parts added in order, and the losses, by one workgroup: `cols` experts at a time (a power of two up to 1024), the
// workgroups' parts dealt to 1024 / cols threads each.
__global__ void __launch_bounds__(1024)
    k_router_finish(const float* __restrict__ share_part, const int32_t* __restrict__ count_part,
                    const double* __restrict__ z_part, int blocks, int64_t n, int K, int top, int cols,
                    int32_t* __restrict__ counts, float* __restrict__ share, float* __restrict__ loss) {
  __shared__ double s_sum[1024];
  __shared__ int32_t s_cnt[1024];
  __shared__ double s_dot[16], s_z[16];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = threadIdx.x & (cols - 1), slice = threadIdx.x / cols, slices = 1024 / cols;
  double dot = 0.0, z = 0.0;
  for (int b = threadIdx.x; b < blocks; b += 1024) z += z_part[b];
  for (int e0 = 0; e0 < K; e0 += cols) {
    const int e = e0 + col;
    double p = 0.0;
    int32_t c = 0;
    if (e < K) {
#pragma unroll 8
      for (int b = slice; b < blocks; b += slices) {
        p += share_part[(int64_t)b * K + e];
        c += count_part[(int64_t)b * K + e];
      }
    }
    __syncthreads();
    s_sum[threadIdx.x] = p;
    s_cnt[threadIdx.x] = c;
    __syncthreads();
    if (slice == 0 && e < K) {
      for (int i = 1; i < slices; ++i) {
        p += s_sum[i * cols + col];
        c += s_cnt[i * cols + col];
      }
      const float mean = n > 0 ? (float)(p / (double)n) : 0.f;
      counts[e] = c;
      share[e] = mean;
      dot = fma((double)c, (double)mean, dot);
    }
  }
  dot = wave_sum(dot);
  z = wave_sum(z);
  if (l == 0) s_dot[w] = dot, s_z[w] = z;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) dot += s_dot[i], z += s_z[i];
    loss[0] = n > 0 ? (float)(dot * K / ((double)n * top)) : 0.f;
    loss[1] = n > 0 ? (float)(z / (double)n) : 0.f;
  }
}

// ------------------------------------------------------------------ the scores' gradient

// Rt [d][copies][padded K] = R [K][d], zeros past K.
template <typename T>
struct Transposed {
  const T* R;
  T* Rt;
  int d, copies;  // copies 0: not wanted
};
// 64 columns of 16 experts to a workgroup.
template <typename T, int THREADS>
__device__ __forceinline__ void router_transpose(const Transposed<T>& t, int K, int block) {
  __shared__ T s[16][65];
  const int kp = padded(K), d = t.d, c0 = block / (kp / 16) * 64, e0 = block % (kp / 16) * 16;
  for (int q = threadIdx.x; q < 16 * 64; q += THREADS) {
    const int e = q / 64, c = q % 64;
    s[e][c] = e0 + e < K && c0 + c < d ? t.R[(int64_t)(e0 + e) * d + c0 + c] : from_f32<T>(0.f);
  }
  __syncthreads();
  for (int q = threadIdx.x; q < 16 * 64; q += THREADS) {
    const int c = q / 16, e = q % 16;
    if (c0 + c < d)
      for (int i = 0; i < t.copies; ++i) t.Rt[((int64_t)(c0 + c) * t.copies + i) * kp + e0 + e] = s[e][c];
  }
}

// ds in parts (ds_width) and a workgroup's sums of it; workgroups past `blocks` transpose R.
template <typename T, int L, int P>
__global__ void __launch_bounds__(kRowThreads<P>)
    k_router_ds(const float* __restrict__ scores, const int32_t* __restrict__ expert, const int32_t* __restrict__ counts,
                const float* __restrict__ g_weight, int64_t n, int K, int top, int renorm, double balance, float z2,
                T* __restrict__ ds, float* __restrict__ bias_part, int blocks, Transposed<T> t) {
  constexpr int THREADS = kRowThreads<P>, G = THREADS / L;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  if ((int)blockIdx.x >= blocks) {
    router_transpose<T, THREADS>(t, K, blockIdx.x - blocks);
    return;
  }
  const int lane = threadIdx.x % L, ld = ds_width<T>(K), kp = padded(K);
  float q[P], sum[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    q[p] = p * L + lane < K ? (float)(balance * counts[p * L + lane]) : 0.f;
    sum[p] = 0.f;
  }
  for (int64_t first = (int64_t)blockIdx.x * G; first < n; first += (int64_t)blocks * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < n;
    // all of a row's choices before any is looked at: one by one they took a trip to memory each (32768 rows of 128 experts,
    // four choices: 23 us, 22 so)
    int chosen[HMOE_ROUTER_EXPERTS];
    float gw[HMOE_ROUTER_EXPERTS];
#pragma unroll
    for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j) {
      const bool in = j < top && g_weight && live;
      chosen[j] = in ? expert[row * top + j] : -1;
      gw[j] = in ? g_weight[row * top + j] : 0.f;
    }
    float s[P], mx = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      s[p] = live && p * L + lane < K ? scores[row * K + p * L + lane] : -INFINITY;
      mx = fmaxf(mx, s[p]);
    }
    mx = __uint_as_float(lanes_reduce<L>(__float_as_uint(mx), [](uint32_t a, uint32_t b) {
      return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
    float pe[P], g[P], on[P], tot = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      pe[p] = row_exp(s[p], mx);
      tot += pe[p];
      g[p] = on[p] = 0.f;
    }
    tot = lanes_sum<L>(tot);
    const bool none = tot == 0.f;
#pragma unroll
    for (int j = 0; j < HMOE_ROUTER_EXPERTS; ++j) {
      if (j >= top) break;
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (chosen[j] == p * L + lane && chosen[j] < K) {
          g[p] += gw[j];
          on[p] = 1.f;
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
          T* to = ds + row * ld + e;
#pragma unroll
          for (int i = 0; i < kParts; ++i) to[i * kp] = parts.part[i];
        } else {
          ds[row * ld + e] = v;
        }
      }
    }
  }
  experts_out<L, P, THREADS>(sum, reinterpret_cast<float*>(smem_raw), K, bias_part + (int64_t)blockIdx.x * K);
}

// ------------------------------------------------------------------ the products

// dX = ds R: 64 rows and 256 columns to a workgroup, 64 columns to a wave; fragments straight from memory.  bf16, 16
// experts to a step: the last remainders, then values and remainders against the rows of R taken twice.
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
    a[i] = ds + row * ld + (sizeof(T) == 2 ? 8 * (lg & 1) : 4 * lg);
    const int col = c0 + 16 * i + lr < d ? c0 + 16 * i + lr : d - 1;
    b[i] = Rt + (int64_t)col * kp + (sizeof(T) == 2 ? 8 * (lg & 1) : 4 * lg);
  }
  for (int e0 = 0; e0 < kp; e0 += 16) {
    i32x4 av[4], bv[4], last[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      av[i] = *reinterpret_cast<const i32x4*>(a[i] + e0 + (sizeof(T) == 2 ? (lg >> 1) * kp : 0));
      bv[i] = *reinterpret_cast<const i32x4*>(b[i] + e0);
      last[i] = i32x4{0, 0, 0, 0};
      if (sizeof(T) == 2 && lg < 2) last[i] = *reinterpret_cast<const i32x4*>(a[i] + e0 + 2 * kp);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) step_mfma<T>(lg < 2 ? bv[j] : i32x4{0, 0, 0, 0}, last[i], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) step_mfma<T>(bv[j], av[i], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 16 * i + lr;
    if constexpr (sizeof(T) == 2) {
      // lanes 16 apart trade halves of two column blocks, and hold eight columns in a row each
      typedef unsigned int u2v __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x4 va, vb;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          va[r] = (bf16)acc[i][2 * p][r];
          vb[r] = (bf16)acc[i][2 * p + 1][r];
        }
        const u2v x = __builtin_bit_cast(u2v, va), y = __builtin_bit_cast(u2v, vb);
        const u2v s0 = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
        const u2v s1 = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
        const int col = c0 + 32 * p + 16 * (lg & 1) + 8 * (lg >> 1);
        if (row < n && col < d)
          *reinterpret_cast<i32x4*>(dX + row * d + col) = i32x4{(int)s0[0], (int)s1[0], (int)s0[1], (int)s1[1]};
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = c0 + 16 * j + 4 * lg;
        if (row < n && col < d) *reinterpret_cast<floatx4*>(dX + row * d + col) = acc[i][j];
      }
    }
  }
}

// dX = ds R on the engine's tiles, the reduction over the planes: for more experts than the narrow form holds.
template <class C>
__global__ void __launch_bounds__(C::THREADS)
    k_router_dx_wide(const bf16* __restrict__ ds, const bf16* __restrict__ Rt, int64_t n, int K, int d, bf16* __restrict__ dX) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int k = ds_width<bf16>(K);
  const TileCoord tc = tile_plain<C>(n, d, k);
  if (!tc.valid) return;
  floatx4 acc[C::MI][C::NJ];
  gemm_tile<C, true, true>(ds + tc.m0 * k, k, tc.m_rows, Rt + (int64_t)tc.n0 * k, k, tc.n_cols, k, smem, acc);
  store_out<C, bf16>(tc, acc, smem, dX, d, [](int, int, int, float v) { return v; }, RowId{tc.m0}, NoVec{});
}

// part[piece][K][d] = ds^T X over the piece's rows: bf16: all of up to 16 or 32 experts, fp32: 32 experts, and 256
// columns to a workgroup.
template <typename T, int UW>
__global__ void __launch_bounds__(256, 2) k_router_dr(const T* __restrict__ ds, const T* __restrict__ X, int64_t n, int K,
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
  constexpr int B = sizeof(T) == 2 ? C::MI / kParts : C::MI;  // blocks of 16 experts; bf16: and the planes behind them
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = (sizeof(T) == 2 ? 0 : u0) + f.row(i, r), col = c0 + f.col(j, r);
        float v = acc[i][j][r];
        if constexpr (sizeof(T) == 2) v = (acc[i + 2 * B][j][r] + acc[i + B][j][r]) + v;
        if (e < K && col < d) to[(int64_t)e * d + col] = v;
      }
}

// part[piece][planes and experts][d] = ds^T X for more experts, on the engine's tiles; gridDim.y pieces of the rows.
template <class C>
__global__ void __launch_bounds__(C::THREADS) k_router_dr_wide(const bf16* __restrict__ ds, const bf16* __restrict__ X,
                                                               int64_t n, int K, int d, int piece, float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const int ld = ds_width<bf16>(K);
  const int64_t p0 = (int64_t)blockIdx.y * piece;
  const int rows = n - p0 < piece ? (int)(n - p0) : piece;
  const TileCoord tc = tile_plain<C>(ld, d, rows);
  if (!tc.valid) return;
  floatx4 acc[C::MI][C::NJ];
  gemm_tile<C, false, false, false, true>(ds + p0 * ld + tc.m0, ld, tc.m_rows, X + p0 * d + tc.n0, d, tc.n_cols, rows, smem, acc);
  store_out<C, float>(tc, acc, smem, part + (int64_t)blockIdx.y * ld * d, d, [](int, int, int, float v) { return v; },
                      RowId{tc.m0}, NoVec{});
}

// dR and dbias: their parts added in order.  part[piece][plane], `plane` values apart, of which `size` are dR's.
__global__ void __launch_bounds__(256) k_router_join(const float* __restrict__ part, int pieces, int planes,
                                                     int64_t plane, int64_t size, float* __restrict__ dR, const float* __restrict__ bias_part, int blocks,
                                                     int K, float* __restrict__ dbias) {
  const int64_t groups = dR ? cdiv(size, 1024) : 0;
  if ((int64_t)blockIdx.x < groups) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size) return;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    for (int z = planes - 1; z >= 0; --z) {  // the remainders first
#pragma unroll 8
      for (int q = 0; q < pieces; ++q) v += *reinterpret_cast<const floatx4*>(part + (q * planes + z) * plane + i);
    }
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
  if (K <= 32) return run(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (K <= 64) return run(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (K <= 128) return run(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (K <= 256) return run(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (K <= 1024) return run(integral_constant<int, 64>{}, integral_constant<int, 16>{});
  return run(integral_constant<int, 64>{}, integral_constant<int, 64>{});
}
int router_blocks(int64_t n, int K) {
  int rows = 1;
  router_lanes(K, [&](auto l, auto per) {
    rows = kRowThreads<decltype(per)::value> / decltype(l)::value;
    return (int)HMOE_OK;
  });
  const int64_t all = cdiv(n, rows), most = device_cus();
  return (int)(all < most ? all : most);
}
// Tiles of the scores; those of up to 64 and 128 experts choose, too.
template <typename T>
using ScoreNarrow = CfgD<T, 128, 64, 32, 64, 3>;
template <typename T>
using ScoreWide = CfgD<T, 128, 128, 32, 64, 4>;
// Workgroups that score and choose: none where a tile to each leaves CUs idle and a row at a time is what takes long
// (777 rows of 8 experts: 18 us in one, 10 and 8 apart).
int scored_blocks(int64_t n, int K) {
  const int64_t all = cdiv(n, 128), most = (K <= 64 ? 4 : 2) * device_cus();
  if (K > 128 || all < device_cus() / 2) return 0;
  return (int)(all < most ? all : most);
}
// Pieces of the scores' reduction, of 128 products at least, where rows are few.
int router_pieces(int64_t n, int K, int d) {
  if (n == 0) return 1;
  const int64_t tiles = cdiv(n, 64) * cdiv(K, 64), fit = 2 * device_cus() / tiles, most = d / 128;
  const int64_t pieces = fit < most ? fit : most;
  return (int)(pieces < 2 ? 1 : pieces > 16 ? 16 : pieces);
}

// Columns of ds to a workgroup of k_router_dr; bf16 data of more experts takes k_router_dr_wide.
template <typename T>
int router_columns(int K) {
  return sizeof(T) == 4 ? 32 : K <= 16 ? 48 : 96;
}
template <typename T>
bool router_wide(int K) {
  return sizeof(T) == 2 && K > 32;
}
using WideDR = CfgPipeKS;
// Rows to a piece of dR's reduction: whole stages, as many pieces as there are CUs (twice of them where two
// workgroups share one) for the tiles.
template <typename T>
int router_piece(int64_t n, int K, int d) {
  const int width = ds_width<T>(K);
  const bool wide = router_wide<T>(K);
  const int64_t tiles = wide ? cdiv(width, WideDR::BM) * cdiv(d, WideDR::BN) : cdiv(width, router_columns<T>(K)) * cdiv(d, 256);
  const int64_t most = (wide ? 1 : 2) * device_cus() / tiles, pieces = most < 1 ? 1 : most;
  const int64_t rows = cdiv(cdiv(n, pieces), 64) * 64, least = wide ? 256 : 64;
  return (int)(rows < least ? least : rows);
}

struct RouterSpace {
  float *planes, *share, *bias, *part;
  int32_t* count;
  double* z;
  void *ds, *Rt;
};
template <typename T>
RouterSpace router_carve(const hmoe_router_t* p, int64_t n, Workspace& ws) {
  RouterSpace s;
  const int blocks = router_blocks(n, p->K), scored = scored_blocks(n, p->K);
  const size_t most = blocks > scored ? blocks : scored, parts = most * p->K;
  s.share = ws.take<float>(parts);
  s.bias = s.share;  // of the other direction
  s.count = ws.take<int32_t>(parts);
  s.z = ws.take<double>(most);
  const int pieces = router_pieces(n, p->K, p->d);
  s.planes = pieces > 1 ? ws.take<float>((size_t)pieces * n * p->K) : nullptr;
  s.ds = ws.take<T>((size_t)n * ds_width<T>(p->K));
  s.Rt = ws.take<T>((size_t)p->d * padded(p->K) * (router_wide<T>(p->K) ? kParts : 1));
  s.part = ws.take<float>((size_t)cdiv(n, router_piece<T>(n, p->K, p->d)) * (router_wide<T>(p->K) ? ds_width<T>(p->K) : p->K) * p->d);
  return s;
}

template <class C>
int router_scores(const hmoe_router_t* p, int64_t n, const void* X, float* scores, int pieces, hipStream_t st) {
  using T = typename C::type;
  HMOE_LAUNCH("router scores", k_router_scores<C>, dim3((unsigned)(cdiv(n, C::BM) * cdiv(p->K, C::BN)), pieces),
              dim3(C::THREADS), C::LDS, st, (const T*)X, (const T*)p->R, p->bias, n, p->K, p->d, scores);
  return HMOE_OK;
}

template <typename T>
int router_forward_t(const hmoe_router_t* p, int64_t n, const void* X, int32_t* expert, float* weight, float* scores,
                     int32_t* counts, float* share, float* loss, Workspace& ws, hipStream_t st) {
  const RouterSpace w = router_carve<T>(p, n, ws);
  int blocks = 0;
  if (n > 0) {
    const Choices c = {n, p->K, p->top_k, p->renorm != 0, expert, weight, w.share, w.count, w.z};
    const int pieces = router_pieces(n, p->K, p->d);
    const auto score_choose = [&](auto config, auto per) {
      using C = decltype(config);
      constexpr int P = decltype(per)::value;
      blocks = scored_blocks(n, p->K);
      HMOE_LAUNCH("router scores", (k_router_score_choose<C, P>), dim3(blocks), dim3(C::THREADS), scored_lds<C>(), st, (const T*)X,
                  (const T*)p->R, p->bias, p->d, scores, c);
      return (int)HMOE_OK;
    };
    using std::integral_constant;
    if (scored_blocks(n, p->K) > 0) {
      if (p->K <= 16) HMOE_TRY(score_choose(ScoreNarrow<T>{}, integral_constant<int, 1>{}));
      else if (p->K <= 32) HMOE_TRY(score_choose(ScoreNarrow<T>{}, integral_constant<int, 2>{}));
      else if (p->K <= 64) HMOE_TRY(score_choose(ScoreNarrow<T>{}, integral_constant<int, 4>{}));
      else HMOE_TRY(score_choose(ScoreWide<T>{}, integral_constant<int, 8>{}));
    } else {
      if (pieces > 1) HMOE_TRY((router_scores<CfgD<T, 64, 64, 32, 32, 5>>(p, n, X, w.planes, pieces, st)));
      else if (p->K <= 64) HMOE_TRY((router_scores<ScoreNarrow<T>>(p, n, X, scores, 1, st)));
      else HMOE_TRY((router_scores<ScoreWide<T>>(p, n, X, scores, 1, st)));
      blocks = router_blocks(n, p->K);
      HMOE_TRY(router_lanes(p->K, [&](auto l, auto per) {
        constexpr int L = decltype(l)::value, P = decltype(per)::value;
        HMOE_LAUNCH("router choose", (k_router_choose<L, P>), dim3(blocks), dim3(kRowThreads<P>), kRowThreads<P> * P * 4, st,
                    scores, pieces > 1 ? w.planes : nullptr, pieces, p->bias, c);
        return (int)HMOE_OK;
      }));
    }
  }
  int cols = 16;
  while (cols < p->K && cols < 1024) cols *= 2;
  HMOE_LAUNCH("router finish", k_router_finish, dim3(1), dim3(1024), 0, st, w.share, w.count, w.z, blocks, n, p->K,
              p->top_k, cols, counts, share, loss);
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
  constexpr bool BF = sizeof(T) == 2;
  const bool wide = router_wide<T>(K), engine = wide && n > 256;
  const Transposed<T> t = {(const T*)p->R, (T*)w.Rt, d, dX ? (engine ? kParts : 1) : 0};
  const int turning = dX ? (int)cdiv(d, 64) * (padded(K) / 16) : 0;
  HMOE_TRY(router_lanes(K, [&](auto l, auto per) {
    constexpr int L = decltype(l)::value, P = decltype(per)::value;
    HMOE_LAUNCH("router score gradient", (k_router_ds<T, L, P>), dim3(blocks + turning), dim3(kRowThreads<P>), kRowThreads<P> * P * 4, st, scores,
                expert, counts, g_weight, n, K, p->top_k, p->renorm != 0, even, z2, ds, w.bias, blocks, t);
    return (int)HMOE_OK;
  }));
  if (dX) {
    if constexpr (BF) {
      using C = CfgPipe;
      if (engine)
        HMOE_LAUNCH("router dX", k_router_dx_wide<C>, dim3((unsigned)(cdiv(n, C::BM) * cdiv(d, C::BN))), dim3(C::THREADS),
                    C::LDS, st, ds, (const T*)w.Rt, n, K, d, (T*)dX);
    }
    if (!engine)
      HMOE_LAUNCH("router dX", k_router_dx<T>, dim3((unsigned)(cdiv(n, 64) * cdiv(d, 256))), dim3(256), 0, st, ds,
                  (const T*)w.Rt, n, K, d, (T*)dX);
  }
  const int piece = router_piece<T>(n, K, d), pieces = (int)cdiv(n, piece);
  if (dR) {
    const int uw = router_columns<T>(K);
    const dim3 grid((unsigned)(cdiv(ds_width<T>(K), uw) * cdiv(d, 256)), pieces);
    const auto narrow = [&](auto columns) {
      constexpr int UW = decltype(columns)::value;
      HMOE_LAUNCH("router dR", (k_router_dr<T, UW>), grid, dim3(256), (Cfg<T, UW, 256, UW, 64>::LDS), st, ds, (const T*)X, n,
                  K, d, piece, w.part);
      return (int)HMOE_OK;
    };
    if constexpr (BF) {
      using C = WideDR;
      if (wide)
        HMOE_LAUNCH("router dR", k_router_dr_wide<C>, dim3((unsigned)(cdiv(ds_width<T>(K), C::BM) * cdiv(d, C::BN)), pieces),
                    dim3(C::THREADS), C::LDS, st, ds, (const T*)X, n, K, d, piece, w.part);
      else if (K <= 16)
        HMOE_TRY(narrow(std::integral_constant<int, 48>{}));
      else
        HMOE_TRY(narrow(std::integral_constant<int, 96>{}));
    } else {
      HMOE_TRY(narrow(std::integral_constant<int, 32>{}));
    }
  }
  if (dR || dbias) {
    const int64_t size = (int64_t)K * d;
    HMOE_LAUNCH("router join", k_router_join, dim3((unsigned)((dR ? cdiv(size, 1024) : 0) + (dbias ? cdiv(K, 64) : 0))),
                dim3(256), 0, st, w.part, pieces, wide ? kParts : 1, wide ? (int64_t)padded(K) * d : size, size, dR, w.bias,
                blocks, K, dbias);
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
