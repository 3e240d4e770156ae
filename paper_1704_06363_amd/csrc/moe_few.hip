// moe_few.hip -- the whole mixture layer for a few samples: routing, experts and combine.
#include <float.h>

#include "fewrows.hpp"
#include "lm_launch.hpp"

namespace hmoe {

namespace {

struct FewArgs {
  const void *X, *R, *W1, *b1, *W2, *b2;
  const float* r_bias;
  int n, K, d, h, o, k;  // k experts to a sample
  int32_t* expert;       // [n k]
  float* weight;
  int32_t* chosen;  // [n k]: expert, or -1 where its weight is 0
  void* hid;        // [n k][Halves][h]
  float* part;      // [splits][n k][o]
  int splits;       // of the second layer's reduction
  void* Y;
};

// ------------------------------------------------------------------ routing

// The k best of K keys, by one wave: weights, and which experts are evaluated.
__device__ __forceinline__ void few_choose(const FewArgs& a, int t, const lds<uint64_t>* key) {
  const int l = threadIdx.x & 63;
  uint64_t best = 0;
  for (int b = 0; b < a.K; b += 64) wave_merge(best, b + l < a.K ? key[b + l] : 0);
  const float s = (uint32_t)(best >> 32) == 0 ? NAN : key_value(best);
  const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s)));
  float p = l < a.k ? (s == -INFINITY ? 0.f : __expf(s - top)) : 0.f;
  const float sum = wave_sum(p);
  if (sum > 0.f || sum != sum) p /= sum;
  if (p < FLT_MIN) p = 0.f;  // NaN stays
  if (l < a.k) {
    const int q = t * a.k + l;
    a.expert[q] = (int32_t)key_index(best);
    a.weight[q] = p;
    a.chosen[q] = p == 0.f ? -1 : (int32_t)key_index(best);
  }
}

// A workgroup to a sample: the scores of all experts, four at a time to a wave, and the k best.
constexpr int kRouteWaves = 16, kRouteEach = 4;
template <typename T>
__global__ void __launch_bounds__(64 * kRouteWaves) k_few_route(FewArgs a) {
  constexpr int N = 16 / sizeof(T), G = kRouteEach;
  __shared__ uint64_t s_key[4096];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, t = blockIdx.x;
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
        if (e0 + g < a.K) s_key[e0 + g] = rank_key(s[g] + (a.r_bias ? a.r_bias[e0 + g] : 0.f), (uint32_t)(e0 + g));
    }
  }
  __syncthreads();
  if (w == 0) few_choose(a, t, (const lds<uint64_t>*)s_key);
}

// ------------------------------------------------------------------ experts

// LAYER 1: hid[q] = act(W1_e x + b1_e).   LAYER 2: part[split][q] = W2_e hid[q] over a split of the reduction.
// A workgroup has 16 outputs (GATED: and the 16 they are gated with) of one expert; its four waves split
// the reduction and join in LDS.
template <typename T, int LAYER, bool GATED>
__global__ void __launch_bounds__(256) k_few_layer(FewArgs a, int tiles) {
  constexpr int STEP = 64 / sizeof(T);
  constexpr int MI = LAYER == 1 && GATED ? 2 : 1;
  constexpr int NX = LAYER == 2 ? Halves<T>::N : 1;  // operands of an activation
  __shared__ int s_expert, s_count, s_rows[HMOE_FEW_ROWS];
  __shared__ floatx4 s_acc[4][MI][64];
  const int splits = LAYER == 1 ? 1 : a.splits;
  const int slot = blockIdx.x / (tiles * splits);
  const int tile = blockIdx.x % tiles, split = blockIdx.x / tiles % splits;
  if (!few_group<256>(a.chosen, a.n * a.k, a.K, slot, &s_expert, s_rows, &s_count)) return;
  const int e = s_expert, count = s_count;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int kd = LAYER == 1 ? a.d : a.h, rows = LAYER == 1 ? a.h : a.o;
  const int r = tile * 16 + lr < rows ? tile * 16 + lr : rows - 1;
  const T* W = LAYER == 1 ? static_cast<const T*>(a.W1) + ((int64_t)e * MI * a.h + r) * kd
                          : static_cast<const T*>(a.W2) + ((int64_t)e * a.o + r) * kd;
  const int steps = (kd + STEP - 1) / STEP, parts = 4 * splits, part = split * 4 + w;
  const int s0 = (int)((int64_t)steps * part / parts), s1 = (int)((int64_t)steps * (part + 1) / parts);
  for (int t0 = 0; t0 < count; t0 += 16) {
    const int q = s_rows[t0 + lr < count ? t0 + lr : count - 1];
    const T* x = LAYER == 1 ? static_cast<const T*>(a.X) + (int64_t)(q / a.k) * kd
                            : static_cast<const T*>(a.hid) + (int64_t)q * NX * kd;
    floatx4 acc[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    const T *wp[MI], *xp[NX];
#pragma unroll
    for (int i = 0; i < MI; ++i) wp[i] = W + (int64_t)i * a.h * kd;
#pragma unroll
    for (int j = 0; j < NX; ++j) xp[j] = x + j * kd;
    stream_steps<T, 8 / (MI + NX - 1)>(wp, xp, kd, s0, s1, [&](const i32x4(&wv)[MI], const i32x4(&xv)[NX]) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NX; ++j) step_mfma<T>(wv[i], xv[j], acc[i]);
    });
#pragma unroll
    for (int i = 0; i < MI; ++i) s_acc[w][i][l] = acc[i];
    __syncthreads();
    if (w == 0 && t0 + lr < count) {
#pragma unroll
      for (int i = 0; i < MI; ++i) acc[i] = (s_acc[0][i][l] + s_acc[1][i][l]) + (s_acc[2][i][l] + s_acc[3][i][l]);
      const int c0 = tile * 16 + 4 * lg;
      if (c0 < rows) {  // rows are a multiple of 8: four at a time
        if constexpr (LAYER == 1) {
          const T* b = static_cast<const T*>(a.b1) + (int64_t)e * MI * a.h;
          T* out = static_cast<T*>(a.hid) + (int64_t)q * Halves<T>::N * a.h + c0;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            float v = acc[0][z] + (a.b1 ? to_f32(b[c0 + z]) : 0.f);
            if constexpr (GATED) {
              const float up = acc[1][z] + (a.b1 ? to_f32(b[a.h + c0 + z]) : 0.f);
              v = v / (1.f + __expf(-v)) * up;
            } else {
              v = v < 0.f ? 0.f : v;  // NaN stays
            }
            const Halves<T> p(v);
#pragma unroll
            for (int j = 0; j < Halves<T>::N; ++j) out[j * a.h + z] = p.part[j];
          }
        } else {
          *reinterpret_cast<floatx4*>(a.part + ((int64_t)split * a.n * a.k + q) * a.o + c0) = acc[0];
        }
      }
    }
    __syncthreads();
  }
}

// Y = sum over the choices, in their order, of weight (sum of the splits + b2).
template <typename T>
__global__ void __launch_bounds__(256) k_few_combine(FewArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.n * a.o) return;
  const int t = (int)(i / a.o), c = (int)(i - (int64_t)t * a.o);
  float y = 0.f;
  for (int j = 0; j < a.k; ++j) {
    const int q = t * a.k + j, e = a.chosen[q];
    if (e < 0) continue;
    float v = a.b2 ? to_f32(static_cast<const T*>(a.b2)[(int64_t)e * a.o + c]) : 0.f;
    for (int s = 0; s < a.splits; ++s) v += a.part[((int64_t)s * a.n * a.k + q) * a.o + c];
    y = fmaf(a.weight[q], v, y);
  }
  static_cast<T*>(a.Y)[i] = from_f32<T>(y);
}

int few_splits(const hmoe_few_params_t* p, int64_t n) {
  const int64_t slots = n * p->top_k < p->K ? n * p->top_k : p->K;
  const int64_t s = 1024 / (slots * cdiv(p->d_out, 16));
  return (int)(s < 1 ? 1 : (s > 8 ? 8 : s));
}

template <typename T>
int moe_few_t(const FewArgs& a, bool gated, hipStream_t st) {
  const int64_t slots = (int64_t)a.n * a.k < a.K ? (int64_t)a.n * a.k : a.K;
  const int t1 = (int)cdiv(a.h, 16), t2 = (int)cdiv(a.o, 16);
  HMOE_LAUNCH("few route", k_few_route<T>, dim3(a.n), dim3(64 * kRouteWaves), 0, st, a);
  if (gated)
    HMOE_LAUNCH("few layer 1", (k_few_layer<T, 1, true>), dim3((unsigned)(slots * t1)), dim3(256), 0, st, a, t1);
  else
    HMOE_LAUNCH("few layer 1", (k_few_layer<T, 1, false>), dim3((unsigned)(slots * t1)), dim3(256), 0, st, a, t1);
  HMOE_LAUNCH("few layer 2", (k_few_layer<T, 2, false>), dim3((unsigned)(slots * t2 * a.splits)), dim3(256), 0, st, a,
              t2);
  HMOE_LAUNCH("few combine", k_few_combine<T>, dim3((unsigned)cdiv((int64_t)a.n * a.o, 256)), dim3(256), 0, st, a);
  return HMOE_OK;
}

void few_carve(const hmoe_few_params_t* p, int64_t n, Workspace& ws, FewArgs& a) {
  const size_t rows = (size_t)n * p->top_k;
  a.splits = few_splits(p, n);
  a.chosen = ws.take<int32_t>(rows);
  a.hid = ws.take<char>(rows * p->d_hid * 4);  // two bf16 or one fp32
  a.part = ws.take<float>(rows * p->d_out * a.splits);
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
               expert, weight, nullptr, nullptr, nullptr, 1, Y};
  few_carve(p, n, ws, a);
  const bool gated = p->act == HMOE_ACT_SILU_GATED;
  return p->dt == HMOE_BF16 ? moe_few_t<bf16>(a, gated, st) : moe_few_t<float>(a, gated, st);
}

}  // namespace hmoe
