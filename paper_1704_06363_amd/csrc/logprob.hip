// logprob.hip -- log-probabilities of given tokens, entropies and the most probable alternatives
// of rows of logits, and the gradient of the first two.
//
// With x a row's logits, s the scale, M = max x:  S = sum e^(s (x - M)),  T = sum e^(s (x - M)) (x - M),
//   ln sum e^(s x) = s M + ln S,   ln p_v = s (x_v - M) - ln S,   entropy = ln S - s T / S.
// All three sums come out of one pass: a lane keeps (M, S, T) of the entries it has seen and, when a
// later step brings a larger M, multiplies them into it (RowSums); lanes, waves and the pieces of a row are
// joined the same way.  Differences to M are formed before they are scaled, so that rows around the
// type's lowest value (a finite mask) and rows of large logits lose nothing.  Each step adds its own
// entries first and then one number to S and T, so no sum runs over more than a few hundred terms.
//
// The alternatives: a wave keeps a bound on its m-th best entry, lists what is above it in LDS, and sorts the
// list 64 keys at a time (lanes.hpp).  The first bound is the m-th largest of the lanes' maxima over
// the first step, which m entries reach; the best of the row's waves' bounds is everyone's, so that the
// waves with the tail of a vocabulary in order of frequency list next to nothing.
//
// Bound: HBM, the logits are read once (a bf16 entry costs 10 to 11 vector cycles of a lane, which
// 256 CUs have time for at 7 TB/s).
#include <float.h>

#include "lanes.hpp"
#include "lm_launch.hpp"
#include "slices.hpp"

namespace hmoe {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kLpTop = 16;    // most alternatives
constexpr int kLpList = 192;  // keys a wave lists before it sorts them
constexpr int kLpUnroll = 4;  // vectors of a lane and step

// 16 bytes of a row, which may start at any element.
typedef int32_t vec_of_bf16 __attribute__((ext_vector_type(4), aligned(2)));
typedef int32_t vec_of_f32 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct RowVec {
  using type = typename std::conditional<sizeof(T) == 2, vec_of_bf16, vec_of_f32>::type;
  static constexpr int N = 16 / sizeof(T);
};

struct RowSums {
  float M, S, T;
  // Neutral: no entry is below -FLT_MAX but -inf, whose terms are 0.
  __device__ __forceinline__ void clear() {
    M = -FLT_MAX;
    S = T = 0.f;
  }
  // The sums relative to a larger maximum (c2 = s log2 e).  A factor of 0 takes the T term's product
  // with it only if that is finite; a NaN stays.
  __device__ __forceinline__ void raise(float to, float c2) {
    const float d = fmaxf(M - to, -FLT_MAX);
    const float f = __builtin_amdgcn_exp2f(d * c2);
    S *= f;
    T = fmaf(S, d, T * f);
    M = to;
  }
  __device__ __forceinline__ void join(RowSums o, float c2) {
    const float m = fmaxf(M, o.M);
    raise(m, c2);
    o.raise(m, c2);
    S += o.S;
    T += o.T;
  }
};

// One piece of a row, as the join reads it: the sums, and the m best keys.
struct Piece {
  float M, S, T, pad;
};

struct LogprobArgs {
  const void* L;
  int64_t ld, n;
  const float* anc;
  int V, m;
  float scale;
  const int32_t* token;
  float *logp, *entropy, *lse, *stat;
  int32_t* top_idx;
  float* top_logp;
  int64_t row0, n_end;  // the rows of this launch
  int pieces;         // of a row
  Piece* part;        // [n][pieces]
  uint64_t* part_key; // [n][pieces][m]
};

template <typename T, bool ANC>
__device__ __forceinline__ float entry(const LogprobArgs& a, int64_t row, int64_t v) {
  const float x = to_f32(static_cast<const T*>(a.L)[row * a.ld + v]);
  return ANC ? a.anc[anchor_index(a.n, row, v)] + x : x;
}

// A wave's list of candidates for the m best entries.
struct TopList {
  uint64_t best = 0;   // sorted over the lanes
  uint64_t floor = 0;  // keys above it may be among the m best
  int count = 0;       // listed since the last sort

  __device__ __forceinline__ void sort_in(lds<uint64_t>* buf, int m) {
    const int l = threadIdx.x & 63;
    wave_lds_fence();
    for (int b = 0; b < count; b += 64) wave_merge(best, b + l < count ? buf[b + l] : 0);
    wave_lds_fence();
    count = 0;
    const uint64_t last = lane_value(best, m - 1);
    floor = last > floor ? last : floor;
  }
  // A bound found by another wave of the row: entries equal to it may still be among the m best.
  __device__ __forceinline__ void raise_to(uint32_t value) {
    const uint64_t k = (uint64_t)value << 32;
    floor = k > floor ? k : floor;
  }
  // Entries not above this are not listed (of -inf none are: finish_row finds those).
  __device__ __forceinline__ float below() const {
    const uint32_t hi = (uint32_t)(floor >> 32);
    // entries equal to a bound's value pass, to one that has its own index do not; what precedes +0 is -0, which
    // is not below it
    const uint32_t step = (uint32_t)floor != 0 ? 0u : (hi == 0x80000000u ? 2u : 1u);
    return hi <= kKeyMinusInf ? -INFINITY : key_value((uint64_t)(hi - step) << 32);
  }
  // Lists the lanes' entries x at `index` that are `in` and above the floor.
  __device__ __forceinline__ void add(float x, uint32_t index, bool in, lds<uint64_t>* buf, int m) {
    const uint64_t key = rank_key(x, index);
    const uint64_t hit = __ballot(in && key > floor);
    if (hit == 0) return;
    const int c = __popcll(hit);
    if (count + c > kLpList) sort_in(buf, m);
    if ((hit >> (threadIdx.x & 63)) & 1) buf[count + lanes_below(hit)] = key;
    count += c;
  }
};

// The row's results from its sums and its best keys (sorted over the lanes), by one wave.
template <typename T, bool ANC>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int64_t row, const RowSums& r, uint64_t best) {
  const int l = threadIdx.x & 63;
  const float ls = kLn2 * __builtin_amdgcn_logf(r.S);
  const bool empty = r.S == 0.f;
  if (l == 0) {
    if (a.logp) {
      const int32_t t = a.token[row];
      float lp = 0.f;
      if (t >= 0 && t < a.V) lp = empty ? -INFINITY : a.scale * (entry<T, ANC>(a, row, t) - r.M) - ls;
      a.logp[row] = lp;
    }
    if (a.entropy) a.entropy[row] = empty ? 0.f : ls - a.scale * (r.T / r.S);
    if (a.lse) a.lse[row] = empty ? -INFINITY : fmaf(a.scale, r.M, ls);
    if (a.stat) {
      a.stat[2 * row] = r.M;
      a.stat[2 * row + 1] = ls;
    }
  }
  if (a.m == 0) return;
  // Entries of -inf and NaN are not all listed: where the m best need them, they are taken in order of
  // their indexes, first the ones and then the others.
  const int found = __popcll(__ballot(l < a.m && (uint32_t)(best >> 32) > kKeyMinusInf));
  if (found < a.m) {
    int have = found;
    for (int nan = 0; nan < 2 && have < a.m; ++nan)
      for (int64_t v0 = 0; v0 < a.V && have < a.m; v0 += 64) {
        const float x = v0 + l < a.V ? entry<T, ANC>(a, row, v0 + l) : 0.f;
        uint64_t hit = __ballot(nan ? x != x : x == -INFINITY);
        while (hit != 0 && have < a.m) {
          const int at = __builtin_ctzll(hit);
          hit &= hit - 1;
          if (l == have) best = rank_key(nan ? NAN : -INFINITY, (uint32_t)(v0 + at));
          ++have;
        }
      }
  }
  if (l < a.m) {
    a.top_idx[row * (int64_t)a.m + l] = (int32_t)key_index(best);
    const bool nan = (uint32_t)(best >> 32) == 0;
    if (a.top_logp)
      a.top_logp[row * (int64_t)a.m + l] =
          r.S != r.S || nan ? NAN : (empty ? -INFINITY : a.scale * (key_value(best) - r.M) - ls);
  }
}

// W waves to a piece of a row, 4 / W pieces to a workgroup.
template <typename T, bool ANC, bool TOP, int W>
__global__ void __launch_bounds__(256) k_token_logprob(LogprobArgs a) {
  using Vec = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N, U = kLpUnroll;
  __shared__ uint64_t s_list[TOP ? 4 : 1][TOP ? kLpList : 1];
  __shared__ float s_sum[4][3];
  __shared__ uint32_t s_floor[1];
  if constexpr (TOP && W > 1) {
    if (threadIdx.x == 0) *s_floor = 0;
    __syncthreads();
  }
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t job = a.row0 * a.pieces + (int64_t)blockIdx.x * (4 / W) + w / W;
  const int64_t row = job / a.pieces;
  const int piece = (int)(job - row * a.pieces);
  if (row >= a.n_end) return;  // whole waves, and with W > 1 whole workgroups
  const T* x = static_cast<const T*>(a.L) + row * a.ld;
  const float c2 = a.scale * kLog2e;
  const int nvec = a.V / N;
  const int per = (nvec + a.pieces - 1) / a.pieces;
  const int first = piece * per;
  const int end = first + per < nvec ? first + per : nvec;
  lds<uint64_t>* buf = (lds<uint64_t>*)s_list[TOP ? w : 0];
  RowSums r;
  r.clear();
  TopList top;
  Vec raw[U];
  float an[U];
  const int step = 64 * U * W, b0 = first + (w % W) * 64 * U;
  // 64 vectors are whole tiles of anchors, so this lane's move by the same distance with each
  constexpr int TILES = 64 * N / kAnchorTile;
  const int64_t tile = a.n * kAnchorSlots;
  const float* anc = nullptr;
  if constexpr (ANC) anc = a.anc + anchor_index(a.n, row, (int64_t)(b0 + l) * N);
  const auto load = [&](int b) {  // each step once, in order
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = b + 64 * u + l;
      if (v < end) {
        raw[u] = *reinterpret_cast<const Vec*>(x + (int64_t)v * N);
        if constexpr (ANC) an[u] = anc[u * TILES * tile];
      }
    }
    if constexpr (ANC) anc += U * W * TILES * tile;
  };
  if (b0 < end) load(b0);
  for (int b = b0; b < end; b += step) {
    // the entries, as fp32 sums with their anchors, and each vector's largest
    float f[U][N], cm[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = b + 64 * u + l < end;
      constexpr int kNone = sizeof(T) == 2 ? (int)0xff80ff80u : (int)0xff800000u;  // -inf
      i32x4 q = raw[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = in ? q[i] : kNone;
      const T* e = reinterpret_cast<const T*>(&q);
      const float base = ANC && in ? an[u] : 0.f;
#pragma unroll
      for (int z = 0; z < N; ++z) {
        f[u][z] = ANC ? base + to_f32(e[z]) : to_f32(e[z]);
        cm[u] = z == 0 ? f[u][0] : fmaxf(cm[u], f[u][z]);
      }
    }
    if (b + step < end) load(b + step);
    float mx = r.M;
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(mx, cm[u]);
    r.raise(mx, c2);
    float S = 0.f, Tn = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int z = 0; z < N; ++z) {
        const float d = f[u][z] - mx;
        const float e = __builtin_amdgcn_exp2f(d * c2);
        S += e;
        Tn = fmaf(e, fmaxf(d, -FLT_MAX), Tn);
      }
    r.S += S;
    r.T += Tn;
    if constexpr (TOP) {
      if (b == b0) {  // the m-th largest of the lanes' maxima
        float best = cm[0];
#pragma unroll
        for (int u = 1; u < U; ++u) best = fmaxf(best, cm[u]);
        top.floor = (uint64_t)sortable(mth_lane_value(best, a.m, l)) << 32;
        if (W > 1 && l == 0) atomicMax(s_floor, (uint32_t)(top.floor >> 32));
      }
      if (W > 1) top.raise_to(*(volatile uint32_t*)s_floor);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float below = top.below();
        if (__ballot(cm[u] > below) == 0) continue;
        // the lanes' entries that may enter, one of each lane at a time
        const int v = b + 64 * u + l;
        uint32_t bits = 0;
#pragma unroll
        for (int z = 0; z < N; ++z) bits |= (f[u][z] > below && v < end ? 1u : 0u) << z;
        while (__ballot(bits != 0) != 0) {
          const int z = __builtin_ctz(bits | 256u);
          float y = f[u][0];
#pragma unroll
          for (int q = 1; q < N; ++q) y = z == q ? f[u][q] : y;
          top.add(y, (uint32_t)(v * N + z), bits != 0, buf, a.m);
          bits &= bits - 1;
        }
      }
    }
  }
  if (piece == a.pieces - 1 && w % W == 0) {  // the last entries, less than a vector
    const int v = nvec * N + l;
    const bool in = v < a.V;
    const float y = in ? entry<T, ANC>(a, row, v) : -INFINITY;
    const float mx = fmaxf(r.M, y);
    r.raise(mx, c2);
    const float d = y - mx;
    const float e = __builtin_amdgcn_exp2f(d * c2);
    r.S += e;
    r.T = fmaf(e, fmaxf(d, -FLT_MAX), r.T);
    if constexpr (TOP) top.add(y, (uint32_t)v, in, buf, a.m);
  }
  // lanes, then waves
  float M = r.M;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, shfl_xor(M, o));
  r.raise(M, c2);
  r.S = wave_sum(r.S);
  r.T = wave_sum(r.T);
  if constexpr (TOP) top.sort_in(buf, a.m);
  if constexpr (W > 1) {
    if (l == 0) {
      s_sum[w][0] = r.M;
      s_sum[w][1] = r.S;
      s_sum[w][2] = r.T;
    }
    if constexpr (TOP)
      if (l < kLpTop) buf[l] = top.best;
    __syncthreads();
    if (w != 0) return;
#pragma unroll
    for (int q = 1; q < W; ++q) r.join(RowSums{s_sum[q][0], s_sum[q][1], s_sum[q][2]}, c2);
    if constexpr (TOP) {
      uint64_t k = l / kLpTop < W ? ((lds<uint64_t>*)s_list[l / kLpTop])[l % kLpTop] : 0;
      wave_sort(k, true);
      top.best = k;
    }
  }
  if (a.pieces == 1) {
    finish_row<T, ANC>(a, row, r, top.best);
  } else {
    if (l == 0) a.part[job] = Piece{r.M, r.S, r.T, 0.f};
    if constexpr (TOP)
      if (l < a.m) a.part_key[job * a.m + l] = top.best;
  }
}

// The pieces of a row joined, a workgroup to a row: the waves sort the keys 64 at a time, the first the best
// of theirs.
template <typename T, bool ANC>
__global__ void __launch_bounds__(256) k_logprob_join(LogprobArgs a) {
  __shared__ uint64_t s_key[4][kLpTop];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t row = a.row0 + blockIdx.x;
  const int keys = a.pieces * a.m;
  const float c2 = a.scale * kLog2e;
  uint64_t best = 0;
  for (int b = 64 * w; b < keys; b += 256) wave_merge(best, b + l < keys ? a.part_key[row * keys + b + l] : 0);
  if (l < kLpTop) s_key[w][l] = best;
  __syncthreads();
  if (w != 0) return;
  RowSums r;
  r.clear();
  if (l < a.pieces) {
    const Piece q = a.part[row * a.pieces + l];
    r = RowSums{q.M, q.S, q.T};
  }
  float M = r.M;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, shfl_xor(M, o));
  r.raise(M, c2);
  r.S = wave_sum(r.S);
  r.T = wave_sum(r.T);
  if (keys > 64) {
    best = s_key[l / kLpTop][l % kLpTop];
    wave_sort(best, true);
  }
  finish_row<T, ANC>(a, row, r, best);
}

// ------------------------------------------------------------------ gradient

struct LogprobGrad {
  const void* L;
  int64_t ld, n;
  const float* anc;
  int V;
  float scale;
  const int32_t* token;
  const float *stat, *entropy, *g_logp, *g_entropy;
  void* dL;
  int64_t ldo;
  int64_t row0;  // first row of this launch
  int chunks;    // workgroups to a row
};

// 256 threads, U vectors each.  dL may be L: every thread reads what it writes.
template <typename T, bool ANC>
__global__ void __launch_bounds__(256) k_logprob_grad(LogprobGrad a) {
  using Vec = typename RowVec<T>::type;
  constexpr int N = RowVec<T>::N, U = kLpUnroll;
  const int64_t row = a.row0 + blockIdx.x / a.chunks;
  const int chunk = blockIdx.x % a.chunks;
  const T* x = static_cast<const T*>(a.L) + row * a.ld;
  T* y = static_cast<T*>(a.dL) + row * a.ldo;
  const int nvec = a.V / N;
  const int v0 = chunk * 256 * U + threadIdx.x;
  Vec raw[U];
  float an[U];
  const float* anc = nullptr;
  if constexpr (ANC) anc = a.anc + anchor_index(a.n, row, (int64_t)v0 * N);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int v = v0 + 256 * u;
    if (v < nvec) {
      raw[u] = *reinterpret_cast<const Vec*>(x + (int64_t)v * N);
      if constexpr (ANC) an[u] = anc[u * (256 * N / kAnchorTile) * a.n * kAnchorSlots];
    }
  }
  const float M = a.stat[2 * row], ls = a.stat[2 * row + 1];
  const float ge = a.g_entropy ? a.g_entropy[row] : 0.f;
  const float H = a.g_entropy ? a.entropy[row] : 0.f;
  int t = -1;
  float gl = 0.f;
  if (a.g_logp) {
    t = a.token[row];
    if (t >= 0 && t < a.V) gl = a.g_logp[row]; else t = -1;
  }
  const bool empty = ls == -INFINITY;
  const float base = gl + ge * H;
  // ln p below -200 has p = 0: the bound keeps 0 times -inf out of the sum.  p is the square of e^(ln p / 2): v_exp_f32
  // gives 0 below 2^-126, the product does not, and near 1 it keeps all bits.  (e^(ln p + 32 ln 2) 2^-32 was off by
  // 6e-7 there, 5% of a gradient 1 - p of 1e-5.)
  const auto grad = [&](float z, int v) {
    const float lp = a.scale * (z - M) - ls;
    const float root = __builtin_amdgcn_exp2f(lp * (0.5f * kLog2e));
    const float p = root * root;
    const float g = (v == t ? gl : 0.f) - p * fmaf(ge, fmaxf(lp, -200.f), base);
    return empty ? 0.f : a.scale * g;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int v = v0 + 256 * u;
    if (v >= nvec) break;
    const T* e = reinterpret_cast<const T*>(&raw[u]);
    Vec out;
    T* o = reinterpret_cast<T*>(&out);
#pragma unroll
    for (int z = 0; z < N; ++z) o[z] = from_f32<T>(grad(ANC ? an[u] + to_f32(e[z]) : to_f32(e[z]), v * N + z));
    *reinterpret_cast<Vec*>(y + (int64_t)v * N) = out;
  }
  if (chunk == 0 && threadIdx.x < a.V - nvec * N) {
    const int v = nvec * N + threadIdx.x;
    const float z = ANC ? a.anc[anchor_index(a.n, row, v)] + to_f32(x[v]) : to_f32(x[v]);
    y[v] = from_f32<T>(grad(z, v));
  }
}

// Pieces of a row: where there are fewer rows than workgroups that fill the chip, rows are split down to
// one step of a workgroup each.
int logprob_pieces(int64_t n, int V, hmoe_dtype_t dt) {
  const int64_t most = cdiv(V, (int64_t)(16 / dtype_size(dt)) * 256 * kLpUnroll);
  const int64_t want = n > 0 ? cdiv(2 * 256, n) : 1;
  const int64_t p = want < most ? want : most;
  return (int)(p < 1 ? 1 : (p > 64 ? 64 : p));
}

template <typename T, bool ANC, bool TOP>
int logprob_t(LogprobArgs a, hipStream_t st) {
  const int64_t n = a.n;
  return over_slices(n, a.pieces, 256, [&](int64_t row0, int64_t rows) {
    a.row0 = row0;
    a.n_end = row0 + rows;
    const dim3 block(256);
    // Short rows of which there are many: a wave to each
    if (a.pieces == 1 && a.V <= 8192 && n >= 1024)
      HMOE_LAUNCH("token logprob", (k_token_logprob<T, ANC, TOP, 1>), dim3((unsigned)cdiv(rows, 4)), block, 0, st, a);
    else
      HMOE_LAUNCH("token logprob", (k_token_logprob<T, ANC, TOP, 4>), dim3((unsigned)(rows * a.pieces)), block, 0, st,
                  a);
    if (a.pieces > 1)
      HMOE_LAUNCH("token logprob join", (k_logprob_join<T, ANC>), dim3((unsigned)rows), block, 0, st, a);
    return (int)HMOE_OK;
  });
}

template <typename T, bool ANC>
int logprob_grad_t(LogprobGrad a, hipStream_t st) {
  return over_slices(a.n, a.chunks, 256, [&](int64_t row0, int64_t rows) {
    a.row0 = row0;
    HMOE_LAUNCH("token logprob gradient", (k_logprob_grad<T, ANC>), dim3((unsigned)(rows * a.chunks)), dim3(256), 0, st,
                a);
    return (int)HMOE_OK;
  });
}

}  // namespace

size_t token_logprob_ws(int64_t n, int V, int m, hmoe_dtype_t dt) {
  const int p = logprob_pieces(n, V, dt);
  if (p == 1) return 0;
  Workspace w(nullptr, 0);
  w.take<Piece>((size_t)n * p);
  w.take<uint64_t>((size_t)n * p * m);
  return w.off;
}

int launch_token_logprob(const void* L, int64_t ld, const float* anc, hmoe_dtype_t dt, int64_t n, int V, float scale,
                         const int32_t* token, int m, float* logp, float* entropy, float* lse, float* stat,
                         int32_t* top_idx, float* top_logp, Workspace& ws, hipStream_t st) {
  const int p = logprob_pieces(n, V, dt);
  Piece* part = nullptr;
  uint64_t* key = nullptr;
  if (p > 1) {
    part = ws.take<Piece>((size_t)n * p);
    key = ws.take<uint64_t>((size_t)n * p * m);
  }
  const LogprobArgs a = {L, ld, n, anc, V, m, scale, token, token ? logp : nullptr, entropy, lse, stat, top_idx,
                         top_logp, 0, n, p, part, key};
  const bool bf = dt == HMOE_BF16;
  if (anc) {
    if (m > 0) return bf ? logprob_t<bf16, true, true>(a, st) : logprob_t<float, true, true>(a, st);
    return bf ? logprob_t<bf16, true, false>(a, st) : logprob_t<float, true, false>(a, st);
  }
  if (m > 0) return bf ? logprob_t<bf16, false, true>(a, st) : logprob_t<float, false, true>(a, st);
  return bf ? logprob_t<bf16, false, false>(a, st) : logprob_t<float, false, false>(a, st);
}

int launch_token_logprob_backward(const void* L, int64_t ld, const float* anc, hmoe_dtype_t dt, int64_t n, int V,
                                  float scale, const int32_t* token, const float* stat, const float* entropy,
                                  const float* g_logp, const float* g_entropy, void* dL, int64_t ldo, hipStream_t st) {
  const int nvec = V / (int)(16 / dtype_size(dt));
  int64_t chunks = cdiv(nvec, 256 * kLpUnroll);
  if (chunks < 1) chunks = 1;
  const LogprobGrad a = {L,     ld,      n,      anc,       V,  scale, token,       stat, entropy,
                         g_logp, g_entropy, dL, ldo, 0, (int)chunks};
  const bool bf = dt == HMOE_BF16;
  if (anc) return bf ? logprob_grad_t<bf16, true>(a, st) : logprob_grad_t<float, true>(a, st);
  return bf ? logprob_grad_t<bf16, false>(a, st) : logprob_grad_t<float, false>(a, st);
}

}  // namespace hmoe
