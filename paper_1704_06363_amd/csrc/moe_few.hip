// moe_few.hip -- the whole mixture layer for a few samples: routing, experts and combine.
#include <float.h>

#include "fewrows.hpp"
#include "lm_launch.hpp"
#include "slices.hpp"

namespace hmoe {

namespace {

struct FewArgs {
  const void *X, *R, *W1, *b1, *W2, *b2;
  const float* r_bias;
  int n, K, d, h, o, k;  // k experts to a sample
  int32_t* expert;       // [n k]
  float* weight;
  int32_t* chosen;   // [n k]: expert, or -1 where its weight is 0
  float* score;      // [n][K], where one workgroup does not hold them all
  void* hid;         // [n k][Halves][h]
  int splits;        // of the second layer's reduction
  float* part;       // [splits][n k][o], where Y has several
  uint32_t* count;   // per 16 columns of Y: workgroups that have written their part
  int counts;
  void* Y;
};

// ------------------------------------------------------------------ routing

// By the call's first kernel, for its last one.
__device__ __forceinline__ void clear_counts(const FewArgs& a) {
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < a.counts; i += blockDim.x) a.count[i] = 0;
}

// The largest key of the wave, on every lane.
__device__ __forceinline__ uint64_t wave_best(uint64_t k) {
  const auto step = [&](uint64_t o) { k = o > k ? o : k; };
  step(lane_xor<1>(k));
  step(lane_xor<2>(k));
  step(lane_xor<4>(k));
  step(lane_xor<8>(k));
  step(lane_xor<16>(k));
  step(lane_xor<32>(k));
  return k;
}

// The k largest of `best` (k keys on the first lanes, in order, or zeros) and of the scores of 64 M experts
// from b on, one after the other.  (With one sort of 64 keys at a time: 0.6 us for each.)
template <int M, class Score>
__device__ __forceinline__ uint64_t few_best(int k, int K, int b, uint64_t best, Score score) {
  const int l = threadIdx.x & 63;
  uint64_t key[M], next = 0;
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int e = b + 64 * m + l;
    key[m] = e < K ? rank_key(score(e), (uint32_t)e) : 0;
  }
  for (int j = 0; j < k; ++j) {
    uint64_t most = best;
#pragma unroll
    for (int m = 0; m < M; ++m) most = key[m] > most ? key[m] : most;
    most = wave_best(most);
    if (l == j) next = most;
    if (best == most) best = 0;
#pragma unroll
    for (int m = 0; m < M; ++m)
      if (key[m] == most) key[m] = 0;
  }
  return next;
}

// The k best of a sample's K scores, by one wave: weights, and which experts are evaluated.  put(q, expert,
// weight) by the lane that has choice q; true if all weights are 0.
template <class Score, class Put>
__device__ __forceinline__ bool few_choose(const FewArgs& a, int t, Score score, Put put) {
  const int l = threadIdx.x & 63;
  uint64_t best = 0;
  if (a.K <= 128) best = few_best<2>(a.k, a.K, 0, best, score);
  else
    for (int b = 0; b < a.K; b += 512) best = few_best<8>(a.k, a.K, b, best, score);
  const float s = (uint32_t)(best >> 32) == 0 ? NAN : key_value(best);
  const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s)));
  float p = l < a.k ? (s == -INFINITY ? 0.f : __expf(s - top)) : 0.f;
  const float sum = wave_sum(p);
  if (sum > 0.f || sum != sum) p /= sum;
  if (p < FLT_MIN) p = 0.f;  // NaN stays
  if (l < a.k) {
    a.expert[t * a.k + l] = (int32_t)key_index(best);
    a.weight[t * a.k + l] = p;
    put(l, (int32_t)key_index(best), p);
  }
  return sum == 0.f;
}

// For the kernels that follow.
template <typename T, class Score>
__device__ __forceinline__ void few_choose_row(const FewArgs& a, int t, Score score) {
  const bool none = few_choose(a, t, score, [&](int q, int e, float p) { a.chosen[t * a.k + q] = p == 0.f ? -1 : e; });
  if (a.counts == 0 && none)  // nobody else writes the row
    for (int c = threadIdx.x & 63; c < a.o; c += 64) static_cast<T*>(a.Y)[(int64_t)t * a.o + c] = from_f32<T>(0.f);
}

// A workgroup to a sample: the scores of all experts, four at a time to a wave, and the k best.  One CU
// draws some 40 GB/s from its L2 here, so this is for small routers.
constexpr int kRouteWaves = 16, kRouteEach = 4, kRouteMost = 128;
template <typename T>
__global__ void __launch_bounds__(64 * kRouteWaves) k_few_route(FewArgs a) {
  constexpr int N = 16 / sizeof(T), G = kRouteEach;
  __shared__ float s_score[kRouteMost];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, t = blockIdx.x;
  clear_counts(a);
  const T* x = static_cast<const T*>(a.X) + (int64_t)t * a.d;
  for (int e0 = w * G; e0 < a.K; e0 += kRouteWaves * G) {
    const T* r[G];
    float s[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      r[g] = static_cast<const T*>(a.R) + (int64_t)(e0 + g < a.K ? e0 + g : a.K - 1) * a.d;
      s[g] = 0.f;
    }
#pragma unroll 4
    for (int v = l; v < a.d / N; v += 64) {
      const i32x4 xv = *reinterpret_cast<const i32x4*>(x + v * N);
      i32x4 rv[G];
#pragma unroll
      for (int g = 0; g < G; ++g) rv[g] = *reinterpret_cast<const i32x4*>(r[g] + v * N);
      const T* xe = reinterpret_cast<const T*>(&xv);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const T* re = reinterpret_cast<const T*>(&rv[g]);
#pragma unroll
        for (int z = 0; z < N; ++z) s[g] = fmaf(to_f32(xe[z]), to_f32(re[z]), s[g]);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) s[g] = wave_sum(s[g]);
    if (l == 0) {
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (e0 + g < a.K) s_score[e0 + g] = s[g];
    }
  }
  __syncthreads();
  if (w == 0) few_choose_row<T>(a, t, [&](int e) { return s_score[e] + (a.r_bias ? a.r_bias[e] : 0.f); });
}

// Scores of 16 samples against 16 experts; eight waves split the reduction.
constexpr int kScoreWaves = 8;
template <typename T>
__global__ void __launch_bounds__(64 * kScoreWaves) k_few_score(FewArgs a) {
  constexpr int NW = kScoreWaves;
  __shared__ floatx4 s_acc[NW][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16, t = t0 + lr;
  clear_counts(a);
  uint32_t xo[1][4], ro[1][4];
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int row = group_row(f);
    xo[0][f] = (uint32_t)(t0 + row < a.n ? row : a.n - 1 - t0) * a.d * sizeof(T);
    ro[0][f] = (uint32_t)(e0 + row < a.K ? row : a.K - 1 - e0) * a.d * sizeof(T);
  }
  const int groups = groups_of<T>(a.d);
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  stream_groups<T, 2>({static_cast<const T*>(a.R) + (int64_t)e0 * a.d}, ro, static_cast<const T*>(a.X) + (int64_t)t0 * a.d, xo,
                      a.d, groups * w / NW, groups * (w + 1) / NW,
                      [&](const i32x4(&rv)[1], const i32x4(&xv)[1]) { step_mfma<T>(rv[0], xv[0], acc); });
  s_acc[w][l] = acc;
  __syncthreads();
  if (w != 0 || t >= a.n) return;
#pragma unroll
  for (int q = 1; q < NW; ++q) acc += s_acc[q][l];
#pragma unroll
  for (int z = 0; z < 4; ++z)
    if (e0 + 4 * lg + z < a.K) a.score[(int64_t)t * a.K + e0 + 4 * lg + z] = acc[z];
}

template <typename T>
__global__ void __launch_bounds__(64) k_few_choose(FewArgs a) {
  const int t = blockIdx.x;
  few_choose_row<T>(a, t, [&](int e) { return a.score[(int64_t)t * a.K + e] + (a.r_bias ? a.r_bias[e] : 0.f); });
}

// ------------------------------------------------------------------ all of a small layer

// The sum over groups of `lanes` (a power of two) adjacent lanes, on every one of them.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  if (lanes > 1) v += dpp<0xB1>(v);   // quad_perm [1,0,3,2]
  if (lanes > 2) v += dpp<0x4E>(v);   // quad_perm [2,3,0,1]
  if (lanes > 4) v += dpp<0x141>(v);  // half mirror: quads hold their sums
  if (lanes > 8) v += dpp<0x140>(v);  // row mirror
  if (lanes > 16) v += __shfl_xor(v, 16, 64);
  if (lanes > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

// done(row, products, before(row)) with the MI products of each row < rows of W, W + rows kd, ... with the kd
// values of x (LDS); by all THREADS, 16 bytes of a row to a lane, the loads of two rows and of what
// before() takes together.  done runs on one lane of a row's, the same one in every call with the same kd.
template <typename T, int THREADS, int MI, class Before, class Done>
__device__ __forceinline__ void few_rows_dot(const T* __restrict__ W, int rows, int kd, const float* x, Before before,
                                             Done done) {
  constexpr int N = 16 / sizeof(T), R = 2 / MI;
  const int nv = kd / N;
  int lanes = 1;
  while (lanes < nv && lanes < 64) lanes <<= 1;
  const int sub = threadIdx.x & (lanes - 1), r0 = threadIdx.x / lanes, step = THREADS / lanes;
  for (int base = 0; base < rows; base += R * step) {
    float s[R][MI];
    decltype(before(0)) pre[R];
    const T* w[R][MI];
#pragma unroll
    for (int g = 0; g < R; ++g) {
      const int r = base + g * step + r0 < rows ? base + g * step + r0 : rows - 1;
      pre[g] = before(r);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        w[g][i] = W + ((int64_t)i * rows + r) * kd;
        s[g][i] = 0.f;
      }
    }
    for (int v = sub; v < nv; v += lanes) {
      i32x4 wv[R][MI];
#pragma unroll
      for (int g = 0; g < R; ++g)
#pragma unroll
        for (int i = 0; i < MI; ++i) wv[g][i] = *reinterpret_cast<const i32x4*>(w[g][i] + v * N);
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        const floatx4 xv = *reinterpret_cast<const floatx4*>(x + v * N + q);
#pragma unroll
        for (int z = 0; z < 4; ++z)
#pragma unroll
          for (int g = 0; g < R; ++g)
#pragma unroll
            for (int i = 0; i < MI; ++i)
              s[g][i] = fmaf(to_f32(reinterpret_cast<const T*>(&wv[g][i])[q + z]), xv[z], s[g][i]);
      }
    }
#pragma unroll
    for (int g = 0; g < R; ++g) {
      const int r = base + g * step + r0;
#pragma unroll
      for (int i = 0; i < MI; ++i) s[g][i] = lanes_sum(s[g][i], lanes);
      if (sub == 0 && r < rows) done(r, s[g], pre[g]);
    }
  }
}

__device__ __forceinline__ float few_silu(float g, float up) { return g / (1.f + __expf(-g)) * up; }
__device__ __forceinline__ float few_relu(float v) { return v < 0.f ? 0.f : v; }  // NaN stays

// A workgroup to a sample, routing, experts and combine, h and Y's row in LDS in fp32: nothing goes through
// HBM between the steps and there is one launch, but a sample's weights come through one CU.  5 samples,
// fp32, 64 -> 128 -> 64 with one of 8 experts (66 KB a sample): 5.8 us, as the launches of larger layers
// 12.9; bf16, one of 16 experts, 132 / 200 KB a sample: 8.2 / 10.2 us; 264 KB as those launches: 11.9.
// (16 waves with two rows' loads each; with four rows' 7.6, 8 waves with two / four 6.4 / 6.5 us.)
constexpr int kSampleThreads = 1024, kSampleBytes = 224 << 10, kSampleFloats = 12 << 10;
template <typename T, bool GATED>
__global__ void __launch_bounds__(kSampleThreads) k_few_sample(FewArgs a) {
  constexpr int THREADS = kSampleThreads, MI = GATED ? 2 : 1;
  extern __shared__ floatx4 s_values[];
  __shared__ int s_expert[HMOE_FEW_EXPERTS];
  __shared__ float s_weight[HMOE_FEW_EXPERTS];
  float *s_x = reinterpret_cast<float*>(s_values), *s_hid = s_x + a.d, *s_y = s_hid + a.h, *s_score = s_y + a.o;
  const int t = blockIdx.x;
  const T* x = static_cast<const T*>(a.X) + (int64_t)t * a.d;
  for (int c = threadIdx.x; c < a.d; c += THREADS) s_x[c] = to_f32(x[c]);
  for (int c = threadIdx.x; c < a.o; c += THREADS) s_y[c] = 0.f;
  __syncthreads();
  few_rows_dot<T, THREADS, 1>(
      static_cast<const T*>(a.R), a.K, a.d, s_x, [&](int e) { return a.r_bias ? a.r_bias[e] : 0.f; },
      [&](int e, const float(&s)[1], float bias) { s_score[e] = s[0] + bias; });
  __syncthreads();
  if (threadIdx.x < 64)
    few_choose(a, t, [&](int e) { return s_score[e]; }, [&](int q, int e, float p) {
      s_expert[q] = e;
      s_weight[q] = p;
    });
  __syncthreads();
  for (int j = 0; j < a.k; ++j) {
    const float weight = s_weight[j];
    if (weight == 0.f) continue;
    const int e = s_expert[j];
    const T* b1 = static_cast<const T*>(a.b1) + (int64_t)e * MI * a.h;
    const T* b2 = static_cast<const T*>(a.b2) + (int64_t)e * a.o;
    few_rows_dot<T, THREADS, MI>(
        static_cast<const T*>(a.W1) + (int64_t)e * MI * a.h * a.d, a.h, a.d, s_x,
        [&](int r) {
          return a.b1 ? float2{to_f32(b1[r]), GATED ? to_f32(b1[a.h + r]) : 0.f} : float2{0.f, 0.f};
        },
        [&](int r, const float(&s)[MI], float2 bias) {
          if constexpr (GATED) s_hid[r] = few_silu(s[0] + bias.x, s[1] + bias.y);
          else s_hid[r] = few_relu(s[0] + bias.x);
        });
    __syncthreads();
    few_rows_dot<T, THREADS, 1>(
        static_cast<const T*>(a.W2) + (int64_t)e * a.o * a.h, a.o, a.h, s_hid,
        [&](int c) { return a.b2 ? to_f32(b2[c]) : 0.f; },
        [&](int c, const float(&s)[1], float bias) { s_y[c] += weight * (s[0] + bias); });
    __syncthreads();
  }
  T* y = static_cast<T*>(a.Y) + (int64_t)t * a.o;
  for (int c = threadIdx.x; c < a.o; c += THREADS) y[c] = from_f32<T>(s_y[c]);
}

// What a sample reads and computes is a workgroup's work.
bool few_small(const hmoe_few_params_t* p) {
  const int64_t mi = p->act == HMOE_ACT_SILU_GATED ? 2 : 1, size = p->dt == HMOE_BF16 ? 2 : 4;
  const int64_t d = p->d_in, h = p->d_hid, o = p->d_out;
  return d + h + o + p->K <= kSampleFloats &&
         (p->K * d + p->top_k * (mi * h * d + o * h)) * size <= kSampleBytes;
}

// ------------------------------------------------------------------ experts

// Four floats that workgroups of other XCDs read later in the same launch: stored and loaded past the
// L2s (which are not coherent with each other), so that neither side has to write back or drop what its
// L2 holds -- as the fences of a release and an acquire do: 93 us instead of 17 for the second layer of 8
// samples with two of 128 experts each.
__device__ __forceinline__ void store_through(float* p, floatx4 v) {
  uint64_t* q = reinterpret_cast<uint64_t*>(p);
  const uint64_t lo = ((uint64_t)__float_as_uint(v[1]) << 32) | __float_as_uint(v[0]);
  const uint64_t hi = ((uint64_t)__float_as_uint(v[3]) << 32) | __float_as_uint(v[2]);
  __hip_atomic_store(q, lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(q + 1, hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ floatx4 load_through(const float* p) {
  const uint64_t* q = reinterpret_cast<const uint64_t*>(p);
  const uint64_t lo = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const uint64_t hi = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return floatx4{__uint_as_float((uint32_t)lo), __uint_as_float((uint32_t)(lo >> 32)), __uint_as_float((uint32_t)hi),
                 __uint_as_float((uint32_t)(hi >> 32))};
}

// LAYER 1: hid[q] = act(W1_e x + b1_e).   LAYER 2: Y, the combine included.   For the slots from slot0 on, of `slots`
// in all.
// A workgroup has 16 outputs (GATED: and the 16 they are gated with) of one expert, or of a split of
// its reduction; its four waves split that further and join in LDS.  In layer 2 with several parts to an
// output the workgroup that is the last to store its part of 16 columns adds them up, in the order of the
// choices and splits: the result does not depend on which one that is.
// U steps of loads go out together: more of them keep fewer waves on a CU.  64 samples with four of 128
// experts each, U = 4 / 8: 334 / 343 us for the first layer (2048 -> 2 x 2048), 114 / 132 for the second
// (2048 -> 1024); one sample with one of 16, U = 4 / 8 / 16: 6.9 / 6.5 / 5.3 us for the first
// (2048 -> 4096), whose waves have 16 steps each.
template <typename T, int LAYER, bool GATED, int UG>
__global__ void __launch_bounds__(256) k_few_layer(FewArgs a, int tiles, int slots, int slot0) {
  constexpr int MI = LAYER == 1 && GATED ? 2 : 1;
  constexpr int NX = LAYER == 2 ? Halves<T>::N : 1;  // operands of an activation
  __shared__ int s_expert, s_count, s_rows[HMOE_FEW_ROWS];
  __shared__ floatx4 s_acc[4][MI][64];
  const int splits = LAYER == 1 ? 1 : a.splits;
  const int slot = slot0 + blockIdx.x / (tiles * splits), tile = blockIdx.x % tiles, split = blockIdx.x / tiles % splits;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int c0 = tile * 16 + 4 * lg;
  // the choices of one sample are groups of their own
  const bool any = a.n == 1 ? a.chosen[slot] >= 0
                            : few_group<256>(a.chosen, a.n * a.k, a.K, slot, &s_expert, s_rows, &s_count);
  if (LAYER == 1 && !any) return;
  if (any) {
    const int e = uniform_int(a.n == 1 ? a.chosen[slot] : s_expert), count = a.n == 1 ? 1 : s_count;
    const int kd = LAYER == 1 ? a.d : a.h, rows = LAYER == 1 ? a.h : a.o;
    const T* W[MI];
    uint32_t wo[MI][4];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      W[i] = LAYER == 1 ? static_cast<const T*>(a.W1) + ((int64_t)(e * MI + i) * a.h + tile * 16) * kd
                        : static_cast<const T*>(a.W2) + ((int64_t)e * a.o + tile * 16) * kd;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int r = group_row(f);
        wo[i][f] = (uint32_t)(tile * 16 + r < rows ? r : rows - 1 - tile * 16) * kd * sizeof(T);
      }
    }
    const int groups = groups_of<T>(kd), shares = 4 * splits, share = split * 4 + w;
    const int g0 = (int)((int64_t)groups * share / shares), g1 = (int)((int64_t)groups * (share + 1) / shares);
    for (int t0 = 0; t0 < count; t0 += 16) {
      const auto row_of = [&](int i) { return a.n == 1 ? slot : s_rows[t0 + i < count ? t0 + i : count - 1]; };
      const int q = row_of(lr);
      uint32_t xo[NX][4];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int qf = row_of(group_row(f));
#pragma unroll
        for (int j = 0; j < NX; ++j) xo[j][f] = (uint32_t)(LAYER == 1 ? qf / a.k : qf * NX + j) * kd * sizeof(T);
      }
      floatx4 acc[MI];
#pragma unroll
      for (int i = 0; i < MI; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      stream_groups<T, UG>(W, wo, static_cast<const T*>(LAYER == 1 ? a.X : a.hid), xo, kd, g0, g1,
                           [&](const i32x4(&wv)[MI], const i32x4(&xv)[NX]) {
#pragma unroll
                             for (int i = 0; i < MI; ++i)
#pragma unroll
                               for (int j = 0; j < NX; ++j) step_mfma<T>(wv[i], xv[j], acc[i]);
                           });
#pragma unroll
      for (int i = 0; i < MI; ++i) s_acc[w][i][l] = acc[i];
      __syncthreads();
      if (w == 0 && t0 + lr < count && c0 < rows) {  // rows are a multiple of 8: four at a time
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i] = (acc[i] + s_acc[1][i][l]) + (s_acc[2][i][l] + s_acc[3][i][l]);
        if constexpr (LAYER == 1) {
          const T* b = static_cast<const T*>(a.b1) + (int64_t)e * MI * a.h;
          T* out = static_cast<T*>(a.hid) + (int64_t)q * Halves<T>::N * a.h + c0;
          quad<T> hid[Halves<T>::N];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            float v = acc[0][z] + (a.b1 ? to_f32(b[c0 + z]) : 0.f);
            if constexpr (GATED) {
              const float up = acc[1][z] + (a.b1 ? to_f32(b[a.h + c0 + z]) : 0.f);
              v = few_silu(v, up);
            } else {
              v = few_relu(v);
            }
            const Halves<T> p(v);
#pragma unroll
            for (int j = 0; j < Halves<T>::N; ++j) hid[j][z] = p.part[j];
          }
#pragma unroll
          for (int j = 0; j < Halves<T>::N; ++j) *reinterpret_cast<quad<T>*>(out + j * a.h) = hid[j];
        } else {
          const T* b = static_cast<const T*>(a.b2) + (int64_t)e * a.o;
          if (a.b2 && split == 0)
#pragma unroll
            for (int z = 0; z < 4; ++z) acc[0][z] += to_f32(b[c0 + z]);
          if (a.counts == 0) {
            const float weight = a.weight[q];
            quad<T> y;
#pragma unroll
            for (int z = 0; z < 4; ++z) y[z] = from_f32<T>(weight * acc[0][z]);
            *reinterpret_cast<quad<T>*>(static_cast<T*>(a.Y) + (int64_t)q * a.o + c0) = y;
          } else {
            store_through(a.part + ((int64_t)split * a.n * a.k + q) * a.o + c0, acc[0]);
          }
        }
      }
      __syncthreads();
    }
  }
  if constexpr (LAYER == 2) {
    if (a.counts == 0) return;
    if (w == 0) {
      // this wave's parts have arrived (it alone stores them) before they are counted
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (l == 0)
        s_count = __hip_atomic_fetch_add(&a.count[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                  (uint32_t)(slots * splits) - 1;
    }
    __syncthreads();
    if (!s_count) return;
    for (int i = threadIdx.x; i < a.n * 4; i += 256) {
      const int t = i >> 2, c = tile * 16 + 4 * (i & 3);
      if (c >= a.o) continue;
      floatx4 y = {0.f, 0.f, 0.f, 0.f};
      for (int j = 0; j < a.k; ++j) {
        const int q = t * a.k + j;
        if (a.chosen[q] < 0) continue;
        floatx4 v = load_through(a.part + (int64_t)q * a.o + c);
        for (int s = 1; s < splits; ++s) v += load_through(a.part + ((int64_t)s * a.n * a.k + q) * a.o + c);
        y += a.weight[q] * v;
      }
      quad<T> out;
#pragma unroll
      for (int z = 0; z < 4; ++z) out[z] = from_f32<T>(y[z]);
      *reinterpret_cast<quad<T>*>(static_cast<T*>(a.Y) + (int64_t)t * a.o + c) = out;
    }
  }
}

int64_t few_slots(int64_t n, int k, int K) { return n * k < K ? n * k : K; }

// Splits of the second layer's reduction: where there are fewer workgroups than CUs (one sample, 4096 ->
// 1024: 64 of them 8.2 us, split in four 5.7).
int few_splits(const hmoe_few_params_t* p, int64_t n) {
  const int64_t s = device_cus() / (few_slots(n, p->top_k, p->K) * cdiv(p->d_out, 16)), steps = p->d_hid / 256;
  const int64_t most = s < steps ? s : steps;
  return (int)(most < 1 ? 1 : (most > 8 ? 8 : most));
}

template <typename T, int LAYER, bool GATED>
int few_layer(const FewArgs& a, hipStream_t st) {
  const int slots = (int)few_slots(a.n, a.k, a.K), tiles = (int)cdiv(LAYER == 1 ? a.h : a.o, 16);
  const char* label = LAYER == 1 ? "few layer 1" : "few layer 2";
  const int per = tiles * (LAYER == 1 ? 1 : a.splits);  // workgroups of a slot
  return over_slices(slots, per, 256, [&](int64_t slot0, int64_t count) {
    const dim3 grid((unsigned)(count * per)), block(256);
    if (LAYER == 1 && (int64_t)slots * tiles <= 2 * device_cus() && groups_of<T>(a.d) > 8)
      HMOE_LAUNCH(label, (k_few_layer<T, LAYER, GATED, (GATED ? 2 : 4)>), grid, block, 0, st, a, tiles, slots, (int)slot0);
    else
      HMOE_LAUNCH(label, (k_few_layer<T, LAYER, GATED, 1>), grid, block, 0, st, a, tiles, slots, (int)slot0);
    return (int)HMOE_OK;
  });
}

template <typename T>
int moe_few_t(const FewArgs& a, bool gated, bool small, hipStream_t st) {
  if (small) {
    const size_t bytes = (size_t)(a.d + a.h + a.o + a.K) * sizeof(float);
    if (gated) HMOE_LAUNCH("few sample", (k_few_sample<T, true>), dim3(a.n), dim3(kSampleThreads), bytes, st, a);
    else HMOE_LAUNCH("few sample", (k_few_sample<T, false>), dim3(a.n), dim3(kSampleThreads), bytes, st, a);
    return HMOE_OK;
  }
  // a router of up to 128 KB in one launch (64 KB: 4.1 us, 512 KB: 13), larger ones in two
  if (a.K <= kRouteMost && (int64_t)a.K * a.d * sizeof(T) <= (128 << 10)) {
    HMOE_LAUNCH("few route", k_few_route<T>, dim3(a.n), dim3(64 * kRouteWaves), 0, st, a);
  } else {
    HMOE_LAUNCH("few score", k_few_score<T>, dim3((unsigned)cdiv(a.K, 16), (unsigned)cdiv(a.n, 16)),
                dim3(64 * kScoreWaves), 0, st, a);
    HMOE_LAUNCH("few choose", k_few_choose<T>, dim3(a.n), dim3(64), 0, st, a);
  }
  HMOE_TRY(gated ? few_layer<T, 1, true>(a, st) : few_layer<T, 1, false>(a, st));
  return few_layer<T, 2, false>(a, st);
}

void few_carve(const hmoe_few_params_t* p, int64_t n, Workspace& ws, FewArgs& a) {
  const size_t rows = (size_t)n * p->top_k;
  a.splits = few_splits(p, n);
  const bool parts = p->top_k > 1 || a.splits > 1;
  a.counts = parts ? (int)cdiv(p->d_out, 16) : 0;
  a.chosen = ws.take<int32_t>(rows);
  a.score = ws.take<float>((size_t)n * p->K);
  a.hid = ws.take<char>(rows * p->d_hid * 4);  // two bf16 or one fp32
  a.part = ws.take<float>(parts * a.splits * rows * p->d_out);
  a.count = ws.take<uint32_t>(a.counts);
}

}  // namespace

size_t moe_few_ws(const hmoe_few_params_t* p, int64_t n) {
  Workspace w(nullptr, 0);
  FewArgs a;
  few_carve(p, n, w, a);
  return w.off;
}

int launch_moe_few(const hmoe_few_params_t* p, int64_t n, const void* X, int32_t* expert, float* weight, void* Y,
                   Workspace& ws, hipStream_t st) {
  FewArgs a = {X, p->R, p->W1, p->b1, p->W2, p->b2, p->r_bias, (int)n, p->K, p->d_in, p->d_hid, p->d_out, p->top_k,
               expert, weight, nullptr, nullptr, nullptr, 1, nullptr, nullptr, 0, Y};
  few_carve(p, n, ws, a);
  const bool gated = p->act == HMOE_ACT_SILU_GATED, small = few_small(p);
  return p->dt == HMOE_BF16 ? moe_few_t<bf16>(a, gated, small, st) : moe_few_t<float>(a, gated, small, st);
}

}  // namespace hmoe
