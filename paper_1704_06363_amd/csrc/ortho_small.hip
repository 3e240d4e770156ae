// ortho_small.hip -- the iterations of ortho.hip for matrices whose short side is up to 128: a launch to a step, or all
// of a call in one, where a launch to a product is mostly launching (8 matrices of 128 x 64: 17 launches, 140 us).
//
// A workgroup of eight waves holds 128 NG columns of X (padded to RB rows): in registers, 16 columns to a wave and
// group, as the matrix cores give and take them, fp32; and in LDS in pairs, row by row, for the Gram matrix.
//   A = X X^T     16 x 16 tiles of A are dealt to the waves; both operands from LDS, over the workgroup's columns
//   B = b A + c A^2  A in LDS in pairs; B takes its place
//   X = a X + B X  each wave for its columns: lane (c, g) of the matrix core's result holds rows 16 t + 4 g .. + 3 of
//                  column c, and as an operand eight values of K for column c.  The order of K is free as long as both
//                  operands have the same: a step of 32 takes rows 16 t + 4 g .. + 3 of tiles 2 s and 2 s + 1
//                  from group g, which it holds already; B's columns are stored in that order.
// Matrices of more columns are cut into chunks of them, one to a workgroup: each adds up the chunks' Gram matrices of
// the launch before, computes B for itself, and leaves its part of the next one.
#include "ortho.hpp"
#include "primitives.hpp"

namespace hmoe {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Small {
  int chunks;
  float a, b, c;
  int steps;
  const double* norm;     // sums of squares, [K][blocks]
  floatx4* X;             // [K][chunk][group, tile][thread]
  const floatx4* gram;    // [K][chunk][tile][lane]: of the launch before
  floatx4* next;          // of this one
  int first, last;        // U is taken; the result is left
};

template <int RB, int NG, bool WHOLE>
__global__ void __launch_bounds__(512) k_ortho_small(Ortho o, OrthoStep s, Small q) {
  constexpr int T = RB / 16, S = RB / 32, CW = 128 * NG;
  constexpr int NT = T * T > 8 ? T * T / 8 : 1;  // tiles of A to a wave
  constexpr int XROW = CW * 2, XPLANE = RB * XROW, AROW = RB * 2, APLANE = RB * AROW;
  constexpr int AMASK = RB / 8 - 1, ASHIFT = RB == 32 ? 2 : RB == 64 ? 1 : 0;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* const sx = (lds<char>*)smem_raw;  // X: hi [RB][CW], lo
  lds<char>* const sa = sx + 2 * XPLANE;       // A, then B: hi [RB][RB], lo
  __shared__ double s_sum[8];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int lr = l & 15, lg = l >> 4;
  const int m = blockIdx.y, chunk = blockIdx.x;
  const int64_t base = (int64_t)m * o.rows * o.cols;
  const bool owner = w < T * T;
  const int tj = w % T, ti0 = w / T;
  const auto ti = [&](int n) { return ti0 + n * (8 / T); };
  const auto col0 = [&](int g) { return chunk * CW + (g * 8 + w) * 16; };
  // LDS addresses: 16-byte chunk `at` of a row, spread over the banks by the row
  const auto x_at = [&](int row, int at) { return row * XROW + ((at ^ (row & 15)) << 4); };
  const auto a_at = [&](int row, int at) { return row * AROW + ((at ^ ((row >> ASHIFT) & AMASK)) << 4); };
  const auto put = [&](lds<char>* to, int plane, const float (&v)[4]) {
    f16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f16 h, k;
      pair_of(v[e], h, k);
      hi[e] = h;
      lo[e] = k;
    }
    *reinterpret_cast<lds<f16x4>*>(to) = hi;
    *reinterpret_cast<lds<f16x4>*>(to + plane) = lo;
  };
  const auto frag = [&](lds<char>* from) { return *reinterpret_cast<const lds<f16x8>*>(from); };
  const auto mfma = [](f16x8 a, f16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); };
  const auto mfma3 = [&](f16x8 ah, f16x8 al, f16x8 bh, f16x8 bl, floatx4 c) {
    return mfma(ah, bh, mfma(ah, bl, mfma(al, bh, c)));
  };

  floatx4 x[NG][T];  // X times kScaleX
  floatx4 af[NT];    // this wave's tiles of A times kScaleA

  const auto load = [&] {  // U, or U / |U| where the norm is known
    double sum = 0.0;
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t) {
        // 16 bytes along the rows of U to a lane, turned by the quads if those are the rows of X
        const int row = 16 * t + 4 * lg + (o.tall ? 0 : lr & 3), col = col0(g) + (o.tall ? lr : lr & 12);
        const int64_t at = base + (o.tall ? (int64_t)col * o.cols + row : (int64_t)row * o.cols + col);
        floatx4 u = {0.f, 0.f, 0.f, 0.f};
        if (row < o.r && col < o.l) {  // the vector is along cols, a multiple of 8
          u = WHOLE ? ortho_first_u(s, at) : ortho_u(s, at);
        }
        float v[4] = {u[0], u[1], u[2], u[3]};
        if (!o.tall) quad_transpose(v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[g][t][e] = v[e];
          if constexpr (WHOLE) sum = fma((double)v[e], (double)v[e], sum);
        }
      }
    if constexpr (WHOLE) {
      sum = wave_sum(sum);
      if (l == 0) s_sum[w] = sum;
      __syncthreads();
      sum = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += s_sum[i];
    } else {
      for (int b = l; b < o.blocks; b += 64) sum += q.norm[(int64_t)m * o.blocks + b];
      sum = wave_sum(sum);
    }
    const double norm = sqrt(sum);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[g][t][e] = norm == 0.0 ? 0.f : (float)((double)x[g][t][e] / norm * (double)kScaleX);
  };
  const auto gram = [&] {
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float v[4] = {x[g][t][0], x[g][t][1], x[g][t][2], x[g][t][3]};
        quad_transpose(v);  // row 4 lg + lr % 4 of the tile, columns lr & 12 .. + 3
        const int col = (g * 8 + w) * 16 + (lr & 12);
        put(sx + x_at(16 * t + 4 * lg + (lr & 3), col >> 3) + (col & 4) * 2, XPLANE, v);
      }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) af[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (owner) {
#pragma unroll 2
      for (int k = 0; k < CW / 32; ++k) {
        const int rj = 16 * tj + lr;
        const f16x8 bh = frag(sx + x_at(rj, 4 * k + lg)), bl = frag(sx + XPLANE + x_at(rj, 4 * k + lg));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int ri = 16 * ti(n) + lr;
          const f16x8 ah = frag(sx + x_at(ri, 4 * k + lg)), al = frag(sx + XPLANE + x_at(ri, 4 * k + lg));
          af[n] = mfma3(ah, al, bh, bl, af[n]);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) af[n] *= kScaleA / (kScaleX * kScaleX);
  };
  const auto step = [&] {
    // A, whose tile (i, j) is the mirror image of (j, i): lane (c, g) writes row 16 j + c, columns 16 i + 4 g .. + 3
    if (owner) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float v[4] = {af[n][0], af[n][1], af[n][2], af[n][3]};
        put(sa + a_at(16 * tj + lr, 2 * ti(n) + (lg >> 1)) + (lg & 1) * 8, APLANE, v);
      }
    }
    __syncthreads();
    floatx4 bf[NT];
    if (owner) {
#pragma unroll
      for (int n = 0; n < NT; ++n) bf[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const int rj = 16 * tj + lr;
        const f16x8 bh = frag(sa + a_at(rj, 4 * k + lg)), bl = frag(sa + APLANE + a_at(rj, 4 * k + lg));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int ri = 16 * ti(n) + lr;
          const f16x8 ah = frag(sa + a_at(ri, 4 * k + lg)), al = frag(sa + APLANE + a_at(ri, 4 * k + lg));
          bf[n] = mfma3(ah, al, bh, bl, bf[n]);
        }
      }
    }
    __syncthreads();
    if (owner) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(q.b, af[n][e], q.c / kScaleA * bf[n][e]);
        // columns 16 i + 4 g .. + 3 of K's order
        put(sa + a_at(16 * tj + lr, ti(n) / 2 * 4 + lg) + (ti(n) & 1) * 8, APLANE, v);
      }
    }
    __syncthreads();
    f16x8 xh[NG][S], xl[NG][S];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int k = 0; k < S; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f16 h, lo;
          pair_of(x[g][2 * k + e / 4][e & 3], h, lo);
          xh[g][k][e] = h;
          xl[g][k][e] = lo;
        }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      floatx4 acc[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) acc[g] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const f16x8 bh = frag(sa + a_at(16 * t + lr, 4 * k + lg)), bl = frag(sa + APLANE + a_at(16 * t + lr, 4 * k + lg));
#pragma unroll
        for (int g = 0; g < NG; ++g) acc[g] = mfma3(bh, bl, xh[g][k], xl[g][k], acc[g]);
      }
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[g][t][e] = fmaf(q.a, x[g][t][e], acc[g][e] * (1.f / kScaleA));
    }
  };
  const auto leave = [&] {
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[g][t][e] * (1.f / kScaleX);
        if (!o.tall) quad_transpose(v);
        const int row = 16 * t + 4 * lg + (o.tall ? 0 : lr & 3), col = col0(g) + (o.tall ? lr : lr & 12);
        if (row < o.r && col < o.l)
          ortho_put4(s, base + (o.tall ? (int64_t)col * o.cols + row : (int64_t)row * o.cols + col), v);
      }
  };

  if constexpr (WHOLE) {
    load();
    for (int i = 0; i < q.steps; ++i) {
      gram();
      step();
    }
    leave();
  } else {
    floatx4* mine = q.X + ((int64_t)m * q.chunks + chunk) * NG * T * 512 + threadIdx.x;
    if (q.first) {
      load();
    } else {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int t = 0; t < T; ++t) x[g][t] = mine[(g * T + t) * 512];
      if (owner) {
        // all tiles of a chunk at a time, and several chunks: what these loads take is their latency
        const floatx4* from = q.gram + ((int64_t)m * q.chunks * T * T + ti0 * T + tj) * 64 + l;
#pragma unroll
        for (int n = 0; n < NT; ++n) af[n] = floatx4{0.f, 0.f, 0.f, 0.f};
        constexpr int AHEAD = NT >= 8 ? 4 : 8;
        for (int k0 = 0; k0 < q.chunks; k0 += AHEAD) {
          floatx4 v[AHEAD][NT];
#pragma unroll
          for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              v[k][n] = k0 + k < q.chunks ? from[((int64_t)(k0 + k) * T * T + n * (8 / T) * T) * 64] : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int n = 0; n < NT; ++n) af[n] += v[k][n];
        }
      }
      step();
    }
    if (q.last) {
      leave();
      return;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t) mine[(g * T + t) * 512] = x[g][t];
    gram();
    if (owner) {
#pragma unroll
      for (int n = 0; n < NT; ++n) q.next[(((int64_t)m * q.chunks + chunk) * T * T + ti(n) * T + tj) * 64 + l] = af[n];
    }
  }
}

// Rows and groups of columns for a problem: RB = 0 where it is not for these kernels.
struct Plan {
  int RB, NG, chunks;
};
Plan plan_of(const Ortho& o) {
  const auto chunks = [&](int ng) { return (int)cdiv(o.l, 128 * ng); };
  const auto groups = [&](int most) {  // the fewest that hold all columns, or the most
    int ng = 1;
    while (ng < most && chunks(ng) > 1) ng = ng < 3 ? ng + 1 : ng * 2 - 2;  // 1, 2, 3, 4, 6 ..
    return ng;
  };
  Plan p = {0, 1, 0};
  if (o.r <= 32) p = {32, groups(6), 0};
  else if (o.r <= 64) p = {64, groups(3), 0};
  else if (o.r <= 128) p = {128, 1, 0};
  else return p;
  p.chunks = chunks(p.NG);
  // Every workgroup adds up all chunks' Gram matrices, which takes longer than a launch to a product for many chunks of 64
  // KB each (us for five steps here and on k_ortho_mid: 128 x 1024 98 and 110, 128 x 2048 124 and 112; eight of 128 x
  // 1024 111 and 126; 32 of 128 x 512 108 and 145, of 128 x 1024 184 and 178; 64 x 4096 70 and 101, 32 of them 180 and 191).
  if (p.RB == 32 ? p.chunks > 64 : p.RB == 64 ? p.chunks > 16 : p.chunks > 8 || p.chunks * o.K >= device_cus()) p.RB = 0;
  return p;
}

struct SmallSpace {
  double* norm;
  floatx4 *X, *gram[2];
};
SmallSpace small_carve(const Ortho& o, const Plan& p, Workspace& ws) {
  SmallSpace w = {};
  w.norm = ws.take<double>((size_t)o.K * o.blocks);
  if (p.chunks > 1) {
    const size_t T = p.RB / 16, all = (size_t)o.K * p.chunks;
    w.X = ws.take<floatx4>(all * p.NG * T * 512);
    for (floatx4*& g : w.gram) g = ws.take<floatx4>(all * T * T * 64);
  }
  return w;
}

template <int RB, int NG>
int small_on(const OrthoStep& s, const Ortho& o, const Plan& p, Small q, const SmallSpace& w, hipStream_t st) {
  constexpr int LDS = RB * 128 * NG * 4 + RB * RB * 4;
  static_assert(LDS <= 159 * 1024, "fits beside the norm's sums");
  if (p.chunks == 1) {
    HMOE_LAUNCH("ortho small", (k_ortho_small<RB, NG, true>), dim3(1, o.K), dim3(512), LDS, st, o, s, q);
    return HMOE_OK;
  }
  HMOE_TRY(launch_ortho_start(s, o, w.norm, st));
  for (int i = 0; i <= q.steps; ++i) {
    q.first = i == 0;
    q.last = i == q.steps;
    q.gram = w.gram[(i + 1) & 1];
    q.next = w.gram[i & 1];
    HMOE_LAUNCH("ortho small", (k_ortho_small<RB, NG, false>), dim3(p.chunks, o.K), dim3(512), LDS, st, o, s, q);
  }
  return HMOE_OK;
}

}  // namespace

size_t small_ortho_ws(const Ortho& o) {
  const Plan p = plan_of(o);
  if (p.RB == 0) return 0;
  Workspace w(nullptr, 0);
  small_carve(o, p, w);
  return w.off;
}

int launch_small_ortho(const OrthoStep& s, const Ortho& o, int steps, const float* coef, Workspace& ws, hipStream_t st) {
  const Plan p = plan_of(o);
  const SmallSpace w = small_carve(o, p, ws);
  Small q = {p.chunks, coef[0], coef[1], coef[2], steps, w.norm, w.X, nullptr, nullptr, 0, 0};
  if (p.RB == 32) {
    switch (p.NG) {
      case 1: return small_on<32, 1>(s, o, p, q, w, st);
      case 2: return small_on<32, 2>(s, o, p, q, w, st);
      case 3: return small_on<32, 3>(s, o, p, q, w, st);
      case 4: return small_on<32, 4>(s, o, p, q, w, st);
      default: return small_on<32, 6>(s, o, p, q, w, st);
    }
  }
  if (p.RB == 64) {
    switch (p.NG) {
      case 1: return small_on<64, 1>(s, o, p, q, w, st);
      case 2: return small_on<64, 2>(s, o, p, q, w, st);
      default: return small_on<64, 3>(s, o, p, q, w, st);
    }
  }
  return small_on<128, 1>(s, o, p, q, w, st);
}

}  // namespace hmoe
