// join.hip -- the join of a layer's output with the residual stream and the norm before the next layer, and its
// gradients:  x' = c x + sum_j gate_j gamma_y N(y_j),  h = gamma_h N(x'),  N(t) = t r(t), r(t) = (mean t^2 + eps)^-1/2.
// With D the whole gradient of x', t = dh gamma_h and m(a, b) = mean a b:
//   D = dx' + r (t - x' r^2 m(t, x')),  dx = c D,
//   dy_j = g_j r (s - y_j r^2 m(s, y_j)),  s = D gamma_y,  dg_j = r d m(s, y_j),
//   dgamma_y = sum g_j r D y_j,  dgamma_h = sum dh x' r.
//
// Bound by HBM: a row is read once into registers, its sums taken, and its results written; nothing is kept
// from the forward but x', since the row's norms come from numbers that the backward reads anyway.  L lanes
// share a row (8 for the narrowest to a workgroup of 1024), with 16 values each from 16-byte vectors, 32 in the widest
// rows; rows are dealt out to the workgroups round-robin, so that each lane keeps its columns and sums the
// gradients of the gains in registers over all of its rows.  A workgroup's sums go to the workspace, and
// k_join_gains adds them in order.
// The widest rows' registers do not suffice: a lane has 128 of them in a workgroup of 1024, and the backward keeps 44
// (bf16) and 119 (fp32) in scratch memory above 8192 columns, 304 and 519 above 16384; the forward 55 and 61 there.  TB/s
// in bf16 and fp32, 512 MB to a tensor: at 8192 columns forward 5.6 and 5.3, backward 5.3 and 5.3; at 16384 5.6 and
// 5.7, 2.6 and 3.7; at 32768 2.7 and 4.0, 0.85 and 1.5.
#include "primitives.hpp"
#include "train_launch.hpp"

namespace hmoe {

namespace {

struct Join {
  int64_t n;
  int d, k, norm_y;
  float scale, eps, inv_d;
  const void *gamma_y, *gamma_h;
  const void *x, *y;  // forward: x; backward: x'
  const float* gate;
  void *x_out, *h;  // forward
  const void *dx_out, *dh;
  void *dx, *dy;
  float *dgate, *part;  // part[block][gamma_y, gamma_h][d], what is wanted of them
  int want_y, want_h;
};

template <typename T>
constexpr int kVec = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ void unpack(i32x4 v, float (&x)[kVec<T>]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float((uint32_t)v[i] << 16);
      x[2 * i + 1] = __uint_as_float((uint32_t)v[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __int_as_float(v[i]);
  }
}
template <typename T>
__device__ __forceinline__ i32x4 pack(const float (&x)[kVec<T>]) {
  T o[kVec<T>];
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) o[i] = from_f32<T>(x[i]);
  return __builtin_bit_cast(i32x4, o);
}

// Two sums over the L lanes of a row, in each of them.  Rows of several waves meet in LDS, in two places in turn, so
// that one barrier a sum is enough.  Entered by whole workgroups.
template <int L>
struct RowSums {
  float (*s)[16][2];  // [2][waves][2] of LDS, L > 64
  int turn = 0;
  __device__ __forceinline__ static float in_wave(float v) {
    if constexpr (L >= 64) return wave_sum(v);
    if constexpr (L == 32) return row_sum(swap_add<false>(v));
    if constexpr (L == 16) return row_sum(v);
    v += dpp<0xB1>(v);  // eight lanes
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    return v;
  }
  __device__ __forceinline__ void operator()(float& a, float& b) {
    a = in_wave(a);
    b = in_wave(b);
    if constexpr (L > 64) {
      const int w = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) {
        s[turn][w][0] = a;
        s[turn][w][1] = b;
      }
      __syncthreads();
      const int w0 = w / (L / 64) * (L / 64);
      a = b = 0.f;
#pragma unroll
      for (int i = 0; i < L / 64; ++i) {
        a += s[turn][w0 + i][0];
        b += s[turn][w0 + i][1];
      }
      turn ^= 1;
    }
  }
};

template <int L>
constexpr int kThreads = L > 256 ? L : 256;

// A lane's vectors of a row of L * C of them.
template <typename T, int L, int C>
struct Lane {
  static constexpr int V = kVec<T>;
  int nv, lane;
  __device__ __forceinline__ explicit Lane(int d) : nv(d / V), lane(threadIdx.x % L) {}
  __device__ __forceinline__ bool has(int c) const { return c * L + lane < nv; }
  __device__ __forceinline__ void load(const T* row, i32x4 (&v)[C], bool live = true) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
      v[c] = live && has(c) ? reinterpret_cast<const i32x4*>(row)[c * L + lane] : i32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void store(T* row, int c, const float (&x)[V]) const {
    if (has(c)) reinterpret_cast<i32x4*>(row)[c * L + lane] = pack<T>(x);
  }
};
// The gains of a lane's columns; ones without any.
template <typename T, int L, int C>
struct Gains {
  i32x4 g[C];
  __device__ __forceinline__ Gains(const void* gamma, const Lane<T, L, C>& at) {
    float one[kVec<T>];
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) one[e] = 1.f;
    const i32x4 ones = pack<T>(one);
    if (gamma) at.load(static_cast<const T*>(gamma), g);
    else
#pragma unroll
      for (int c = 0; c < C; ++c) g[c] = ones;
  }
  __device__ __forceinline__ void of(int c, float (&x)[kVec<T>]) const { unpack<T>(g[c], x); }
};

template <typename T, int L, int C>
__global__ void __launch_bounds__(kThreads<L>) k_join_forward(Join a) {
  constexpr int V = kVec<T>, G = kThreads<L> / L;
  __shared__ float s_sum[2][16][2];
  RowSums<L> sums{s_sum};
  const Lane<T, L, C> at(a.d);
  const Gains<T, L, C> gy(a.gamma_y, at), gh(a.gamma_h, at);
  const T *x = static_cast<const T*>(a.x), *y = static_cast<const T*>(a.y);
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.n; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < a.n;
    i32x4 raw[C];
    float acc[C][V];
    at.load(x + row * a.d, raw, live);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      unpack<T>(raw[c], acc[c]);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[c][e] *= a.scale;
    }
    for (int j = 0; j < a.k; ++j) {
      at.load(y + (row * a.k + j) * a.d, raw, live);
      float f = live && a.gate ? a.gate[row * a.k + j] : 1.f;
      if (a.norm_y) {
        float sq = 0.f, none = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float v[V];
          unpack<T>(raw[c], v);
#pragma unroll
          for (int e = 0; e < V; ++e) sq = fmaf(v[e], v[e], sq);
        }
        sums(sq, none);
        f *= rsqrtf(sq * a.inv_d + a.eps);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[V], g[V];
        unpack<T>(raw[c], v);
        gy.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[c][e] = fmaf(f * v[e], g[e], acc[c][e]);
      }
    }
    if (a.x_out && live) {
#pragma unroll
      for (int c = 0; c < C; ++c) at.store(static_cast<T*>(a.x_out) + row * a.d, c, acc[c]);
    }
    if (!a.h) continue;
    float sq = 0.f, none = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) sq = fmaf(acc[c][e], acc[c][e], sq);
    sums(sq, none);
    const float r = rsqrtf(sq * a.inv_d + a.eps);
    if (live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float g[V];
        gh.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] *= acc[c][e] * r;
        at.store(static_cast<T*>(a.h) + row * a.d, c, g);
      }
    }
  }
}

template <typename T, int L, int C>
__global__ void __launch_bounds__(kThreads<L>) k_join_backward(Join a) {
  constexpr int V = kVec<T>, G = kThreads<L> / L, WAVES = kThreads<L> / 64;
  __shared__ float s_sum[2][16][2];
  RowSums<L> sums{s_sum};
  const Lane<T, L, C> at(a.d);
  const Gains<T, L, C> gy(a.gamma_y, at), gh(a.gamma_h, at);
  const T *xo = static_cast<const T*>(a.x), *y = static_cast<const T*>(a.y), *dxo = static_cast<const T*>(a.dx_out),
          *dh = static_cast<const T*>(a.dh);
  float of_y[C][V], of_h[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) of_y[c][e] = of_h[c][e] = 0.f;
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.n; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + threadIdx.x / L;
    const bool live = row < a.n;
    i32x4 raw[C], rx[C], rd[C];
    float D[C][V];
    at.load(dxo + row * a.d, raw, live && dxo);
    if (dh) {
      at.load(xo + row * a.d, rx, live);
      at.load(dh + row * a.d, rd, live);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) unpack<T>(raw[c], D[c]);
    if (dh) {
      float sq = 0.f, tx = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[V], t[V], g[V];
        unpack<T>(rx[c], v);
        unpack<T>(rd[c], t);
        gh.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sq = fmaf(v[e], v[e], sq);
          tx = fmaf(t[e] * g[e], v[e], tx);
        }
      }
      sums(sq, tx);
      const float r = rsqrtf(sq * a.inv_d + a.eps), m = r * r * (tx * a.inv_d);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[V], t[V], g[V];
        unpack<T>(rx[c], v);
        unpack<T>(rd[c], t);
        gh.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          D[c][e] = fmaf(r, t[e] * g[e] - v[e] * m, D[c][e]);
          of_h[c][e] = fmaf(t[e], live ? v[e] * r : 0.f, of_h[c][e]);
        }
      }
    }
    if (a.dx && live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = a.scale * D[c][e];
        at.store(static_cast<T*>(a.dx) + row * a.d, c, o);
      }
    }
    for (int j = 0; j < a.k; ++j) {
      const int64_t line = row * a.k + j;
      at.load(y + line * a.d, raw, live);
      const float gate = live && a.gate ? a.gate[line] : 1.f;
      float sq = 0.f, sy = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[V], g[V];
        unpack<T>(raw[c], v);
        gy.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sq = fmaf(v[e], v[e], sq);
          sy = fmaf(D[c][e] * g[e], v[e], sy);
        }
      }
      sums(sq, sy);
      const float r = a.norm_y ? rsqrtf(sq * a.inv_d + a.eps) : 1.f;
      const float m = a.norm_y ? r * r * (sy * a.inv_d) : 0.f, f = gate * r;
      if (a.dgate && live && at.lane == 0) a.dgate[line] = r * sy;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[V], g[V];
        unpack<T>(raw[c], v);
        gy.of(c, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          of_y[c][e] = fmaf(live ? f * v[e] : 0.f, D[c][e], of_y[c][e]);
          g[e] = f * (D[c][e] * g[e] - v[e] * m);
        }
        if (a.dy && live) at.store(static_cast<T*>(a.dy) + line * a.d, c, g);
      }
    }
  }
  // The workgroup's sums of each column: over the rows of a wave, then over the waves in LDS.
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  float* s = reinterpret_cast<float*>(smem_raw);  // [rows of the workgroup, or waves][columns], L < THREADS
  constexpr int ROWS = L >= 64 ? G : WAVES;
  const int cols = C * L * V;
  const auto out = [&](float (&acc)[C][V], float* to) {
    if constexpr (L < 64) {
#pragma unroll
      for (int m = L; m < 64; m *= 2)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) acc[c][e] += shfl_xor(acc[c][e], m);
    }
    if constexpr (ROWS == 1) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (at.has(c))
#pragma unroll
          for (int e = 0; e < V; ++e) to[(c * L + at.lane) * V + e] = acc[c][e];
    } else {
      const int mine = L >= 64 ? threadIdx.x / L : threadIdx.x >> 6;
      if (L >= 64 || (threadIdx.x & 63) < L)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) s[mine * cols + (c * L + at.lane) * V + e] = acc[c][e];
      __syncthreads();
      for (int q = threadIdx.x; q < a.d; q += kThreads<L>) {
        float v = s[q];
#pragma unroll
        for (int i = 1; i < ROWS; ++i) v += s[i * cols + q];
        to[q] = v;
      }
      __syncthreads();
    }
  };
  float* to = a.part + (int64_t)blockIdx.x * (a.want_y + a.want_h) * a.d;
  if (a.want_y) out(of_y, to);
  if (a.want_h) out(of_h, to + (int64_t)a.want_y * a.d);
}

// out[c] = sum over the workgroups of part[.][c], 64 columns to a workgroup of 16 waves; blockIdx.y: which gain.
__global__ void __launch_bounds__(1024) k_join_gains(const float* __restrict__ part, int blocks, int d, int wanted,
                                                     float* __restrict__ first, float* __restrict__ second) {
  __shared__ float s[16][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + l;
  const float* p = part + (int64_t)blockIdx.y * d + c;
  float v = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int b = w; b < blocks; b += 16) v += p[(int64_t)b * wanted * d];
  }
  s[w][l] = v;
  __syncthreads();
  if (w == 0 && c < d) {
    for (int i = 1; i < 16; ++i) v += s[i][l];
    (blockIdx.y == 0 ? first : second)[c] = v;
  }
}

// L and C of a row of d values.
template <typename T, class F>
int join_lanes(int d, F run) {
  constexpr int V = kVec<T>, C = 16 / V;
  using std::integral_constant;
  const auto go = [&](auto l, auto c) { return run(l, c); };
  const integral_constant<int, 1> one{};
  const integral_constant<int, C> few{};
  if (d <= 8 * V) return go(integral_constant<int, 8>{}, one);
  if (d <= 16 * V) return go(integral_constant<int, 16>{}, one);
  if (d <= 32 * V) return go(integral_constant<int, 32>{}, one);
  if (d <= 64 * V) return go(integral_constant<int, 64>{}, one);
  if (d <= 1024) return go(integral_constant<int, 64>{}, few);
  if (d <= 2048) return go(integral_constant<int, 128>{}, few);
  if (d <= 4096) return go(integral_constant<int, 256>{}, few);
  if (d <= 8192) return go(integral_constant<int, 512>{}, few);
  if (d <= 16384) return go(integral_constant<int, 1024>{}, few);
  return go(integral_constant<int, 1024>{}, integral_constant<int, 2 * C>{});
}
// Rows that a workgroup takes at a time.
int join_rows(int d, hmoe_dtype_t dt) {
  int rows = 0;
  const auto run = [&](auto l, auto) {
    rows = kThreads<decltype(l)::value> / decltype(l)::value;
    return (int)HMOE_OK;
  };
  if (dt == HMOE_BF16) join_lanes<bf16>(d, run); else join_lanes<float>(d, run);
  return rows;
}
int join_blocks(int64_t n, int d, hmoe_dtype_t dt) {
  const int64_t all = cdiv(n, join_rows(d, dt)), most = 4 * device_cus();
  return (int)(all < most ? all : most);
}

template <typename T>
int join_forward_t(const Join& a, hipStream_t st) {
  return join_lanes<T>(a.d, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value;
    const int64_t all = cdiv(a.n, kThreads<L> / L), most = 8 * device_cus();
    HMOE_LAUNCH("join", (k_join_forward<T, L, C>), dim3((unsigned)(all < most ? all : most)), dim3(kThreads<L>), 0, st, a);
    return (int)HMOE_OK;
  });
}
template <typename T>
int join_backward_t(const Join& a, float* dgamma_y, float* dgamma_h, hipStream_t st) {
  const int blocks = join_blocks(a.n, a.d, DT<T>::id);
  HMOE_TRY(join_lanes<T>(a.d, [&](auto l, auto c) {
    constexpr int L = decltype(l)::value, C = decltype(c)::value, G = kThreads<L> / L;
    const int rows = L >= 64 ? G : kThreads<L> / 64;
    const int lds = rows > 1 && a.want_y + a.want_h > 0 ? rows * C * L * kVec<T> * 4 : 0;
    HMOE_LAUNCH("join backward", (k_join_backward<T, L, C>), dim3(blocks), dim3(kThreads<L>), lds, st, a);
    return (int)HMOE_OK;
  }));
  if (a.want_y + a.want_h)
    HMOE_LAUNCH("join gains", k_join_gains, dim3((unsigned)cdiv(a.d, 64), a.want_y + a.want_h), dim3(1024), 0, st, a.part,
                blocks, a.d, a.want_y + a.want_h, a.want_y ? dgamma_y : dgamma_h, dgamma_h);
  return HMOE_OK;
}

Join join_of(const hmoe_join_t* p, int64_t n, const void* x, const void* y, const float* gate) {
  Join a = {};
  a.n = n;
  a.d = p->d;
  a.k = p->k;
  a.norm_y = p->norm_y != 0;
  a.scale = p->scale;
  a.eps = p->eps;
  a.inv_d = 1.f / p->d;
  a.gamma_y = p->gamma_y;
  a.gamma_h = p->gamma_h;
  a.x = x;
  a.y = y;
  a.gate = gate;
  return a;
}

}  // namespace

size_t join_ws(const hmoe_join_t* p, int64_t n) { return (size_t)join_blocks(n, p->d, p->dt) * 2 * p->d * sizeof(float); }

int launch_join_forward(const hmoe_join_t* p, int64_t n, const void* x, const void* y, const float* gate, void* x_out,
                        void* h, hipStream_t st) {
  Join a = join_of(p, n, x, y, gate);
  a.x_out = x_out;
  a.h = h;
  return p->dt == HMOE_BF16 ? join_forward_t<bf16>(a, st) : join_forward_t<float>(a, st);
}

int launch_join_backward(const hmoe_join_t* p, int64_t n, const void* x_out, const void* y, const float* gate,
                         const void* dx_out, const void* dh, void* dx, void* dy, float* dgate, float* dgamma_y,
                         float* dgamma_h, Workspace& ws, hipStream_t st) {
  Join a = join_of(p, n, x_out, y, gate);
  a.dx_out = dx_out;
  a.dh = dh;
  a.dx = dx;
  a.dy = dy;
  a.dgate = dgate;
  a.want_y = dgamma_y != nullptr;
  a.want_h = dgamma_h != nullptr;
  if (!dy && !dgate && !dgamma_y) a.k = 0;  // nothing of y is wanted
  a.part = ws.take<float>((size_t)join_blocks(n, p->d, p->dt) * 2 * p->d);
  return p->dt == HMOE_BF16 ? join_backward_t<bf16>(a, dgamma_y, dgamma_h, st) : join_backward_t<float>(a, dgamma_y, dgamma_h, st);
}

}  // namespace hmoe
