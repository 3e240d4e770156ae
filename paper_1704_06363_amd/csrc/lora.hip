// lora.hip -- a shared projection with a low-rank adapter for each group of rows:
//   Y_i = W x_i + b + s_a B_a (A_a x_i),  a the adapter of row i (or none),
// and its gradients with W fixed:  with V_i = s_a B_a^T dY_i,
//   dX_i = W^T dY_i + A_a^T V_i,   dB_a = sum_i dY_i (s_a A_a x_i)^T,   dA_a = sum_i V_i x_i^T.
//
// The narrow products U = s A x and V keep their fp32 accuracy: for bf16 data each value is kept as bf16
// numbers that add up to it.  The fragments of one MFMA step hold 32 values of K, so 16 values of U with
// their remainders fill exactly one step against 16 values of B taken twice: the products that Y and dX
// take, which are rounded to bf16 once, are good to 2^-16 at no instruction more than rounded values would cost.
// The adapters' gradients are fp32, and take a third number: all bits of U and V.
#include "fewrows.hpp"
#include "gemm.hpp"
#include "lm_launch.hpp"
#include "primitives.hpp"
#include "slices.hpp"

namespace hmoe {

namespace {

// A row of U or V: bf16: blocks of 16 M, 16 values of the rank (zeros past it), then their remainders, and (M = 3)
// the remainders of those; fp32: the values.  Few rows, which have no gradient, take M = 2.
constexpr int kUParts = 3;
__host__ __device__ inline int u_blocks(int rank) { return (rank + 15) / 16; }
template <typename T, int M = kUParts>
__host__ __device__ inline int u_width(int rank) {
  return sizeof(T) == 2 ? 16 * M * u_blocks(rank) : rank;
}

// This lane's 16 bytes of step kb of row `row` of U.
template <typename T>
__device__ __forceinline__ i32x4 u_frag(const T* __restrict__ U, int64_t row, int ldu, int kb, int lg, int rank) {
  if constexpr (sizeof(T) == 2) return *reinterpret_cast<const i32x4*>(U + row * ldu + 16 * kUParts * kb + 8 * lg);
  return 16 * kb + 4 * lg < rank ? *reinterpret_cast<const i32x4*>(U + row * ldu + 16 * kb + 4 * lg) : i32x4{0, 0, 0, 0};
}
// And of the row of `rank` values that multiplies it (bf16: the same for the value and its remainder).
template <typename T>
__device__ __forceinline__ i32x4 r_frag(const T* __restrict__ row, int kb, int lg, int rank) {
  const int c = sizeof(T) == 2 ? 16 * kb + 8 * (lg & 1) : 16 * kb + 4 * lg;
  return c < rank ? *reinterpret_cast<const i32x4*>(row + c) : i32x4{0, 0, 0, 0};
}
// The same fragments for 16 rows at once, loaded with adjacent lanes in one row (64 contiguous bytes of each, cf.
// fewrows.hpp) and moved through LDS' crossbar: rank_load j of the row l / 4 feeds the steps of rank_steps.
template <typename T>
__host__ __device__ constexpr int rank_steps() {  // steps to a load
  return sizeof(T) == 2 ? 2 : 1;
}
template <typename T>
__device__ __forceinline__ i32x4 rank_load(const T* __restrict__ row, int j, int rank) {
  const int c = (4 * j + (threadIdx.x & 3)) * (16 / (int)sizeof(T));
  return *reinterpret_cast<const i32x4*>(row + (c < rank ? c : 0));
}
template <typename T>
__device__ __forceinline__ i32x4 rank_pick(i32x4 v, int kb, int lr, int lg, int rank) {
  const int from = 4 * (4 * lr + (sizeof(T) == 2 ? 2 * (kb & 1) + (lg & 1) : lg));
  const bool in = (sizeof(T) == 2 ? 16 * kb + 8 * (lg & 1) : 16 * kb + 4 * lg) < rank;
  i32x4 o;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int x = __builtin_amdgcn_ds_bpermute(from, v[d]);
    o[d] = in ? x : 0;
  }
  return o;
}

// Stores four values 16 kb + 4 lg .. of a row of U (those past the rank as zeros).
template <typename T, int M>
__device__ __forceinline__ void u_store(T* __restrict__ U, int64_t row, int ldu, int kb, int lg, int rank, floatx4 v) {
  const bool in = 16 * kb + 4 * lg < rank;  // the rank is a multiple of 8
  if constexpr (sizeof(T) == 2) {
    quad<T> q[M];
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const Parts<T, M> p(in ? v[z] : 0.f);
#pragma unroll
      for (int i = 0; i < M; ++i) q[i][z] = p.part[i];
    }
#pragma unroll
    for (int i = 0; i < M; ++i) *reinterpret_cast<quad<T>*>(U + row * ldu + 16 * (M * kb + i) + 4 * lg) = q[i];
  } else if (in) {
    *reinterpret_cast<floatx4*>(U + row * ldu + 16 * kb + 4 * lg) = v;
  }
}

// The index-th of the runs of at most `height` rows that segments 0 .. G - 1 are cut into: its segment and its
// number in it, false past the last.  Found by each wave for itself: a lane counts the runs of an equal
// share of the segments, a scan over the lanes names the share and a second one the segment -- two trips to
// memory for up to 64 segments a lane (a binary search in a table takes one for each halving, 3 us of
// them for 128 segments, and a launch before it for the table).  Entered by whole waves.
struct Run {
  int segment;
  int64_t local;
};
__device__ __forceinline__ bool find_run(const int32_t* __restrict__ seg, int G, int height, int64_t index, Run& run) {
  const int l = threadIdx.x & 63, per = (G + 63) / 64;
  const auto runs = [&](int e) { return e < G ? (int64_t)((seg[e + 1] - seg[e] + height - 1) / height) : (int64_t)0; };
  int64_t mine = 0;
#pragma unroll 8
  for (int i = 0; i < per; ++i) mine += runs(l * per + i);
  int64_t end = wave_incl_scan(mine);
  uint64_t past = __ballot(end > index);
  if (past == 0) return false;
  int at = __builtin_ctzll(past);
  const int first = at * per;
  const int64_t before = lane_value((uint64_t)(end - mine), at);
  mine = l < per ? runs(first + l) : 0;
  end = before + wave_incl_scan(mine);
  at = __builtin_ctzll(__ballot(end > index));
  run.segment = first + at;
  run.local = index - (int64_t)lane_value((uint64_t)(end - mine), at);
  return true;
}

// ------------------------------------------------------------------ few rows

struct LoraFew {
  const void *X, *W, *b, *A, *B;
  const float* scale;
  const int32_t* adapter;
  int n, E, d, o, rank;
  void* U;
  void* Y;
};

// U of 16 values of the rank for the rows of one adapter; the waves split d.
constexpr int kFewShrinkWaves = 8;
template <typename T>
__global__ void __launch_bounds__(64 * kFewShrinkWaves) k_lora_few_shrink(LoraFew a) {
  constexpr int NW = kFewShrinkWaves;
  __shared__ int s_group, s_count, s_rows[HMOE_FEW_ROWS];
  __shared__ floatx4 s_acc[NW][64];
  const int blocks = u_blocks(a.rank), kb = blockIdx.x % blocks;
  if (!few_group<64 * NW>(a.adapter, a.n, a.E, blockIdx.x / blocks, &s_group, s_rows, &s_count)) return;
  const int e = s_group, count = s_count, ldu = u_width<T, 2>(a.rank);
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const T* A = static_cast<const T*>(a.A) + ((int64_t)uniform_int(e) * a.rank + 16 * kb) * a.d;
  uint32_t ao[1][4];
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int r = group_row(f);
    ao[0][f] = (uint32_t)(16 * kb + r < a.rank ? r : a.rank - 1 - 16 * kb) * a.d * sizeof(T);
  }
  const int groups = groups_of<T>(a.d), g0 = groups * w / NW, g1 = groups * (w + 1) / NW;
  const float scale = a.scale ? a.scale[e] : 1.f;
  for (int t0 = 0; t0 < count; t0 += 16) {
    const auto row_of = [&](int i) { return s_rows[t0 + i < count ? t0 + i : count - 1]; };
    const int row = row_of(lr);
    uint32_t xo[1][4];
#pragma unroll
    for (int f = 0; f < 4; ++f) xo[0][f] = (uint32_t)row_of(group_row(f)) * a.d * sizeof(T);
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    stream_groups<T, 2>({A}, ao, static_cast<const T*>(a.X), xo, a.d, g0, g1,
                        [&](const i32x4(&av)[1], const i32x4(&xv)[1]) { step_mfma<T>(av[0], xv[0], acc); });
    s_acc[w][l] = acc;
    __syncthreads();
    if (w == 0 && t0 + lr < count) {
      acc = s_acc[0][l];
#pragma unroll
      for (int q = 1; q < NW; ++q) acc += s_acc[q][l];
      u_store<T, 2>(static_cast<T*>(a.U), row, ldu, kb, lg, a.rank, acc * scale);
    }
    __syncthreads();
  }
}

// Waves to a SIMD that the registers are kept to for wide outputs: what fits without spilling.  (48 rows, 50000
// columns of 1024, 16 adapters of rank 32: 50 us, with two waves to a SIMD 61, with four and 16 spilled registers, a load of B at a time, 59.)
constexpr int few_waves(int mi, int nt) { return mi == 1 ? 1 : (nt == 4 ? 2 : (nt == 3 ? 3 : 4)); }

// 16 MI columns of Y for all rows (16 NT at most); the waves split d, and the adapters of the rows.
// RB > 0: one row, whose 16 RB values of U the workgroup forms itself, the rows of A going past x with its rows
// of W: for a narrow A the reads of it (from L2) take less than the launch that U otherwise comes from.
template <typename T, int MI, int NT, int RB, int NW>
__global__ void __launch_bounds__(64 * NW, few_waves(MI, NT)) k_lora_few(LoraFew a) {
  static_assert(RB == 0 || (MI == 1 && NT == 1), "one row");
  constexpr int UROW = HMOE_LORA_RANK * 4 + 16;  // bytes of a row of U at most, and a bank shift
  constexpr int ACC = NW * MI * NT * 64 * 16, ULDS = 16 * NT * UROW;
  __shared__ __attribute__((aligned(16))) char s_mem[ACC > ULDS ? ACC : ULDS];
  __shared__ floatx4 s_a[RB > 0 ? NW : 1][RB > 0 ? RB : 1][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int c0 = blockIdx.x * 16 * MI;
  const int ldu = u_width<T, 2>(a.rank), blocks = u_blocks(a.rank), urow = ldu * (int)sizeof(T) + 16;
  const int all = a.adapter[l < a.n ? l : a.n - 1];  // a lane to a row
  lds<char>* s_u = (lds<char>*)s_mem;
  if constexpr (RB == 0) {  // U, 16-byte pieces
    const int per = ldu * (int)sizeof(T) / 16;
    for (int q = threadIdx.x; q < per * a.n; q += 64 * NW) {
      const int r = q / per, v = q - r * per;
      *reinterpret_cast<lds<i32x4>*>(s_u + r * urow + 16 * v) =
          *reinterpret_cast<const i32x4*>(static_cast<const char*>(a.U) + (int64_t)r * ldu * sizeof(T) + 16 * v);
    }
  }
  const T* W[MI + RB];
  uint32_t wo[MI + RB][4], xo[NT][4];
  int col[MI], row[NT], mine[NT];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int ci = c0 + 16 * i < a.o ? c0 + 16 * i : a.o - 1;  // a tile past the columns repeats the last
    col[i] = ci;
    W[i] = static_cast<const T*>(a.W) + (int64_t)ci * a.d;
#pragma unroll
    for (int f = 0; f < 4; ++f)
      wo[i][f] = (uint32_t)(ci + group_row(f) < a.o ? group_row(f) : a.o - 1 - ci) * a.d * sizeof(T);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    row[t] = 16 * t + lr < a.n ? 16 * t + lr : a.n - 1;
    mine[t] = a.adapter[row[t]];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int r = 16 * t + group_row(f);
      xo[t][f] = (uint32_t)(r < a.n ? r : a.n - 1) * a.d * sizeof(T);
    }
  }
  if constexpr (RB > 0) {
    const int e = uniform_int(all);
    const bool some = e >= 0 && e < a.E;
#pragma unroll
    for (int i = 0; i < RB; ++i) {  // without an adapter: any rows, for sums that are not used
      W[MI + i] = some ? static_cast<const T*>(a.A) + (int64_t)e * a.rank * a.d : static_cast<const T*>(a.A);
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int r = 16 * i + group_row(f);
        wo[MI + i][f] = (uint32_t)(r < a.rank ? r : a.rank - 1) * a.d * sizeof(T);
      }
    }
  }
  floatx4 acc[MI + RB][NT];
#pragma unroll
  for (int i = 0; i < MI + RB; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int groups = groups_of<T>(a.d);
  stream_groups<T, (RB > 0 ? 2 : (MI * NT > 1 ? 1 : 4))>(
      W, wo, static_cast<const T*>(a.X), xo, a.d, groups * w / NW, groups * (w + 1) / NW,
      [&](const i32x4(&wv)[MI + RB], const i32x4(&xv)[NT]) {
#pragma unroll
        for (int i = 0; i < MI + RB; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t) step_mfma<T>(wv[i], xv[t], acc[i][t]);
      });
  if constexpr (RB > 0) {
#pragma unroll
    for (int i = 0; i < RB; ++i) s_a[w][i][l] = acc[MI + i][0];
    __syncthreads();
    if (w < RB && lr == 0) {
      const int e = all >= 0 && all < a.E ? all : 0;
      floatx4 u = s_a[0][w][l];
#pragma unroll
      for (int q = 1; q < NW; ++q) u += s_a[q][w][l];
      u_store<T, 2>((T*)s_mem, 0, ldu, w, lg, a.rank, u * (a.scale ? a.scale[e] : 1.f));
    }
  }
  __syncthreads();
  // The adapters in the order of their first rows, one to a wave in turn, with sums of their own, which only
  // their rows take: another row's zeros times an infinite B would not be zeros.
  // Four loads of B go out together, of one adapter or of several (one at a time: 53 us for the 50).
  constexpr int PER = rank_steps<T>(), BATCH = 4;
  const int loads = (blocks + PER - 1) / PER;
  uint64_t left = __ballot(l < a.n && all >= 0 && all < a.E), with = 0;
  int turn = 0, e = -1, j = loads;  // what is loaded next: load j of adapter e
  floatx4 own[MI][NT];
  while (true) {
    i32x4 raw[BATCH][MI];
    int be[BATCH], bj[BATCH];
    uint64_t bw[BATCH];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      if (j == loads) {
        j = 0;
        e = -1;
        while (left != 0 && e < 0) {
          const int c = __builtin_amdgcn_readlane(all, __builtin_ctzll(left));
          const uint64_t m = __ballot(all == c) & left;
          left &= ~m;
          if (turn++ % NW != uniform_int(w)) continue;
          e = c;
          with = m;
        }
      }
      be[q] = e;
      bj[q] = j;
      bw[q] = with;
      if (e < 0) {  // no more
        j = loads;
        continue;
      }
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int c = col[i] + (l >> 2);
        raw[q][i] = rank_load(static_cast<const T*>(a.B) + ((int64_t)e * a.o + (c < a.o ? c : a.o - 1)) * a.rank, j, a.rank);
      }
      ++j;
    }
    if (be[0] < 0) break;
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      if (be[q] < 0) break;
      if (bj[q] == 0) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t) own[i][t] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int kb = bj[q] * PER + p;
        if (kb >= blocks) break;
        i32x4 bv[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) bv[i] = rank_pick<T>(raw[q][i], kb, lr, lg, a.rank);
        const int at = 64 * kb + 16 * lg;  // bytes of the row of U
        const bool in = at < ldu * (int)sizeof(T);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (((bw[q] >> (16 * t)) & 0xffff) == 0) continue;
          i32x4 uv = *reinterpret_cast<const lds<i32x4>*>(s_u + row[t] * urow + (in ? at : 0));
          uv = in && mine[t] == be[q] ? uv : i32x4{0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < MI; ++i) step_mfma<T>(bv[i], uv, own[i][t]);
        }
      }
      if (bj[q] == loads - 1) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (mine[t] == be[q]) acc[i][t] += own[i][t];
      }
    }
  }
  __syncthreads();
  floatx4(*s_acc)[MI][NT][64] = reinterpret_cast<floatx4(*)[MI][NT][64]>(s_mem);
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) s_acc[w][i][t][l] = acc[i][t];
  __syncthreads();
  for (int q = w; q < MI * NT; q += NW) {
    const int i = q / NT, t = q % NT, c = c0 + 16 * i + 4 * lg;
    floatx4 v = s_acc[0][i][t][l];
#pragma unroll
    for (int p = 1; p < NW; ++p) v += s_acc[p][i][t][l];
    if (16 * t + lr >= a.n || c >= a.o) continue;
    quad<T> y;
#pragma unroll
    for (int z = 0; z < 4; ++z) y[z] = from_f32<T>(v[z] + (a.b ? to_f32(static_cast<const T*>(a.b)[c + z]) : 0.f));
    *reinterpret_cast<quad<T>*>(static_cast<T*>(a.Y) + (int64_t)(16 * t + lr) * a.o + c) = y;
  }
}

template <typename T, int MI, int NW>
int lora_few_mi(const LoraFew& a, hipStream_t st) {
  const dim3 grid((unsigned)cdiv(a.o, 16 * MI)), block(64 * NW);
  switch ((a.n + 15) / 16) {
    case 1: HMOE_LAUNCH("lora few", (k_lora_few<T, MI, 1, 0, 4>), grid, dim3(256), 0, st, a); break;
    case 2: HMOE_LAUNCH("lora few", (k_lora_few<T, MI, 2, 0, NW>), grid, block, 0, st, a); break;
    case 3: HMOE_LAUNCH("lora few", (k_lora_few<T, MI, 3, 0, NW>), grid, block, 0, st, a); break;
    default: HMOE_LAUNCH("lora few", (k_lora_few<T, MI, 4, 0, NW>), grid, block, 0, st, a); break;
  }
  return HMOE_OK;
}

template <typename T>
int lora_few_t(const LoraFew& a, hipStream_t st) {
  const int slots = a.n < a.E ? a.n : a.E, blocks = u_blocks(a.rank);
  // Eight waves to a workgroup rather than four where there is one on each CU at most, for more than 16 rows
  // (bf16, 2048 -> 4096, 16 adapters: 48 rows 17.4 -> 15.2 us, 64 rows of rank 128 31 -> 24; 4 rows 10.2 ->
  // 10.6; 64 rows, 8192 columns 24 -> 27), and for one row whose reduction gives each two groups (2048 -> 4096
  // 7.6 -> 7.1 us with W in the caches, 9.4 -> 9.7 from HBM; 1024 -> 1024, one group, 4.5 -> 4.7).
  const bool narrow = cdiv(a.o, 16) <= device_cus();
  // One row: in one launch where reading A for every 16 columns (up to 20 MB from L2 per 16 of the rank,
  // 4 us) takes less than a second one.
  if (a.n == 1 && blocks <= 2 && (int64_t)a.o * a.d * sizeof(T) * blocks <= (20 << 20)) {
    const dim3 grid((unsigned)cdiv(a.o, 16));
    const bool eight = narrow && groups_of<T>(a.d) >= 16;
    if (blocks == 1 && eight) HMOE_LAUNCH("lora few", (k_lora_few<T, 1, 1, 1, 8>), grid, dim3(512), 0, st, a);
    else if (blocks == 1) HMOE_LAUNCH("lora few", (k_lora_few<T, 1, 1, 1, 4>), grid, dim3(256), 0, st, a);
    else if (eight) HMOE_LAUNCH("lora few", (k_lora_few<T, 1, 1, 2, 8>), grid, dim3(512), 0, st, a);
    else HMOE_LAUNCH("lora few", (k_lora_few<T, 1, 1, 2, 4>), grid, dim3(256), 0, st, a);
    return HMOE_OK;
  }
  HMOE_LAUNCH("lora few shrink", k_lora_few_shrink<T>, dim3((unsigned)(slots * blocks)), dim3(64 * kFewShrinkWaves), 0,
              st, a);
  // wide outputs: two blocks of columns to a workgroup, which halves the reads of X
  if (a.o >= 16 * 1024) return lora_few_mi<T, 2, 4>(a, st);
  return narrow && a.n > 16 ? lora_few_mi<T, 1, 8>(a, st) : lora_few_mi<T, 1, 4>(a, st);
}

// ------------------------------------------------------------------ rows in adapter order

// U = s_e rows A_e^T for 16 MT rows of one adapter and 16 RT values of the rank: rows [n][K] (row map[p] for slot
// p, if there is a map), A [E][rank][K].
// The four waves split K.  blockIdx.x: the runs from run0 on.
template <typename T, int RT, int MT>
__global__ void __launch_bounds__(256) k_lora_shrink(const T* __restrict__ X, int K, const T* __restrict__ A, int rank,
                                                     const float* __restrict__ scale, const int32_t* __restrict__ seg,
                                                     int E, const int32_t* __restrict__ map, T* __restrict__ U,
                                                     int64_t run0) {
  __shared__ floatx4 s_acc[4][RT][MT][64];
  Run run;
  if (!find_run(seg, E, 16 * MT, run0 + blockIdx.x, run)) return;
  const int e = run.segment;
  const int64_t r0 = seg[e] + run.local * (16 * MT);
  const int rows = seg[e + 1] - r0 < 16 * MT ? (int)(seg[e + 1] - r0) : 16 * MT;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, lr = l & 15, lg = l >> 4;
  const int kb0 = blockIdx.y * RT;
  const T* Ab[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) Ab[i] = A + (int64_t)uniform_int(e) * rank * K;
  // rows by 64-bit distance from the tile's first, which offsets below 2^32 from the least of them cannot
  // always hold once they are scattered
  const T* xr[MT][4];
  uint32_t ao[RT][4];
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int r = group_row(f);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t slot = r0 + (16 * t + r < rows ? 16 * t + r : rows - 1);
      xr[t][f] = X + (map ? map[slot] : slot) * K;
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) ao[i][f] = (uint32_t)(16 * (kb0 + i) + r < rank ? 16 * (kb0 + i) + r : rank - 1) * K * sizeof(T);
  }
  floatx4 acc[RT][MT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[i][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int groups = groups_of<T>(K);
  stream_groups<T, (RT == 1 ? 2 : 1)>(Ab, ao, xr, K, groups * w / 4,
                                      groups * (w + 1) / 4, [&](const i32x4(&av)[RT], const i32x4(&xv)[MT]) {
#pragma unroll
                                        for (int i = 0; i < RT; ++i)
#pragma unroll
                                          for (int t = 0; t < MT; ++t) step_mfma<T>(av[i], xv[t], acc[i][t]);
                                      });
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < MT; ++t) s_acc[w][i][t][l] = acc[i][t];
  __syncthreads();
  const float sc = scale ? scale[e] : 1.f;
  for (int q = w; q < RT * MT; q += 4) {
    const int i = q / MT, t = q % MT;
    if (kb0 + i >= u_blocks(rank) || 16 * t + lr >= rows) continue;
    const floatx4 v = (s_acc[0][i][t][l] + s_acc[1][i][t][l]) + (s_acc[2][i][t][l] + s_acc[3][i][t][l]);
    u_store<T, kUParts>(U, r0 + 16 * t + lr, u_width<T>(rank), kb0 + i, lg, rank, v * sc);
  }
}

// acc += U B_e^T over the adapters of this wave's rows, fragments straight from memory.
template <class C>
__device__ __forceinline__ void lora_extend(const TileCoord& tc, floatx4 (&acc)[C::MI][C::NJ],
                                            const typename C::type* __restrict__ U, const typename C::type* __restrict__ B,
                                            int rank, int cols, const int32_t* __restrict__ seg, int E) {
  using T = typename C::type;
  const Frag<C> f;
  const int l = threadIdx.x & 63;
  const int64_t lo = tc.m0 + f.wm * C::WM;
  const int64_t hi = lo + C::WM < tc.m0 + tc.m_rows ? lo + C::WM : tc.m0 + tc.m_rows;
  int e = -1;  // the last adapter whose rows start at or before lo
  for (int b = 0; b < E; b += 64) e += __popcll(__ballot(b + l < E && seg[b + l < E ? b + l : 0] <= lo));
  if (e < 0 || lo >= hi) return;
  const int ldu = u_width<T>(rank), blocks = u_blocks(rank);
  for (; e < E; ++e) {
    const int64_t s = seg[e] > lo ? seg[e] : lo, t = seg[e + 1] < hi ? seg[e + 1] : hi;
    if (seg[e] >= hi) break;
    if (s >= t) continue;
    const int i0 = (int)(s - lo) / 16, i1 = (int)(t - 1 - lo) / 16;
    for (int kb = 0; kb < blocks; ++kb) {
      i32x4 bv[C::NJ];
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) {
        const int col = f.block(j) + f.lr;
        bv[j] = col < tc.n_cols ? r_frag(B + ((int64_t)e * cols + tc.n0 + col) * rank, kb, f.lg, rank) : i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < C::MI; ++i) {
        if (i < i0 || i > i1) continue;
        const int64_t first = lo + 16 * i, row = first + f.lr;
        i32x4 uv = {0, 0, 0, 0};
        if (row >= s && row < t) uv = u_frag(U, row, ldu, kb, f.lg, rank);
        const bool whole = first >= s && first + 16 <= t;
#pragma unroll
        for (int j = 0; j < C::NJ; ++j) {
          // where rows of others share the fragment only the adapter's take the product: their zeros
          // times an infinite B would not be zeros
          floatx4 own = whole ? acc[i][j] : floatx4{0.f, 0.f, 0.f, 0.f};
          if constexpr (C::TRANS) step_mfma<T>(bv[j], uv, own);
          else step_mfma<T>(uv, bv[j], own);
          if (whole) {
            acc[i][j] = own;
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int64_t at = C::TRANS ? row : first + 4 * f.lg + r;
              acc[i][j][r] += at >= s && at < t ? own[r] : 0.f;
            }
          }
        }
      }
    }
  }
}

struct LoraRow {  // destination row
  const int32_t* __restrict__ map;
  int64_t m0;
  __device__ __forceinline__ int64_t operator()(int r) const { return map ? map[m0 + r] : m0 + r; }
};

// The pipelined engine's tile with row map[m0 + r] of A as its row r; A below 4 GB (32-bit offsets).
template <class C, bool B_KC>
struct GatherTile : PipeTile<C, true, B_KC> {
  using P = PipeTile<C, true, B_KC>;
  __device__ __forceinline__ void prime(const bf16* __restrict__ A_, int64_t lda_, const int32_t* __restrict__ map,
                                        int a_rows_, const bf16* __restrict__ B_, int64_t ldb_, int b_rows_, int k_len,
                                        lds<char>* smem) {
    this->A = uniform(reinterpret_cast<const char*>(A_));
    this->B = uniform(reinterpret_cast<const char*>(B_));
    this->lda = lda_;
    this->ldb = ldb_;
    this->a_rows = a_rows_;
    this->b_rows = b_rows_;
    k_len = __builtin_amdgcn_readfirstlane(k_len);
    this->nk = (k_len + C::BK - 1) / C::BK;
    this->k_last = k_len - (this->nk - 1) * C::BK;
    this->step_a = C::BK * 2;
    this->step_b = B_KC ? C::BK * 2 : C::BK * 2 * ldb_;
    const int t = thread_id();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < P::OA::NQ; ++q) {
        const int piece = q * C::THREADS + t, tr = P::OA::tile_row(h, piece >> 3);
        const int64_t row = map[tr < a_rows_ ? tr : a_rows_ - 1];
        this->oa.off[h][q] = (uint32_t)((row * lda_ + P::OA::k_of(piece)) * 2);
      }
    this->ob.init(ldb_, b_rows_);
    this->template load_b<0>(0, P::slot_b(smem, 0, 0));
    this->template load_a<0>(0, P::slot_a(smem, 0, 0));
    this->template load_b<1>(0, P::slot_b(smem, 0, 1));
    this->template load_a<1>(0, P::slot_a(smem, 0, 1));
    if (this->nk > 1) {
      this->template load_b<0>(1, P::slot_b(smem, 1, 0));
      this->template load_a<0>(1, P::slot_a(smem, 1, 0));
      this->template load_b<1>(1, P::slot_b(smem, 1, 1));
    }
  }
};

// out[map[m]] = A[m] W^T + bias + U[m] B_e^T.   W_KC: W [cols][Kd], otherwise [Kd][cols].  GATHER: A's rows are
// in out's order, too.  blockIdx.y: the split of the reduction where gridDim.y > 1; the sums of split s then go to
// part[s][n][cols], for k_lora_gemm_join.
template <class C, bool W_KC, bool GATHER>
__global__ void __launch_bounds__(C::THREADS)
    k_lora_gemm(const typename C::type* __restrict__ A, const typename C::type* __restrict__ W,
                const typename C::type* __restrict__ bias, const typename C::type* __restrict__ U,
                const typename C::type* __restrict__ B, int rank, const int32_t* __restrict__ seg, int E, int64_t n,
                int cols, int Kd, const int32_t* __restrict__ map, typename C::type* __restrict__ out,
                float* __restrict__ part) {
  using T = typename C::type;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  const TileCoord tc = tile_plain<C>(n, cols, Kd);
  if (!tc.valid) return;
  floatx4 acc[C::MI][C::NJ];
  const T* Wt = W_KC ? W + (int64_t)tc.n0 * Kd : W + tc.n0;
  if constexpr (GATHER) {
    GatherTile<C, W_KC> g;
    g.prime(A, Kd, map + tc.m0, tc.m_rows, Wt, W_KC ? Kd : cols, tc.n_cols, Kd, smem);
    g.run(smem, acc);
  } else if (C::PIPE || gridDim.y == 1) {
    gemm_tile<C, true, W_KC>(A + tc.m0 * Kd, Kd, tc.m_rows, Wt, W_KC ? Kd : cols, tc.n_cols, Kd, smem, acc);
  } else {
    const int stages = (Kd + C::BK - 1) / C::BK, s = blockIdx.y;
    const int k0 = stages * s / gridDim.y * C::BK, to = stages * (s + 1) / gridDim.y * C::BK, k1 = to < Kd ? to : Kd;
    gemm_tile<C, true, W_KC>(A + tc.m0 * Kd + k0, Kd, tc.m_rows, W_KC ? Wt + k0 : Wt + (int64_t)k0 * cols,
                             W_KC ? Kd : cols, tc.n_cols, k1 - k0, smem, acc);
    if (s == 0) lora_extend<C>(tc, acc, U, B, rank, cols, seg, E);
    store_out<C, float>(tc, acc, smem, part + s * n * cols, cols, [](int, int, int, float v) { return v; }, RowId{tc.m0},
                        NoVec{});
    return;
  }
  lora_extend<C>(tc, acc, U, B, rank, cols, seg, E);
  using F = Frag<C>;
  const F f;
  float bv[F::NCOL];
#pragma unroll
  for (int q = 0; q < F::NCOL; ++q) {
    const int col = f.colq(q);
    bv[q] = (bias && col < tc.n_cols) ? to_f32(bias[tc.n0 + col]) : 0.f;
  }
  store_out<C, T>(tc, acc, smem, out, cols, [&](int, int j, int r, float v) { return v + bv[F::qidx(j, r)]; },
                  LoraRow{map, tc.m0}, NoVec{});
}

// Four columns to a thread.
template <typename T>
__global__ void __launch_bounds__(256) k_lora_gemm_join(const float* __restrict__ part, int splits, int64_t n, int cols,
                                                        const T* __restrict__ bias, const int32_t* __restrict__ map,
                                                        T* __restrict__ out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, size = n * cols;
  if (i >= size) return;
  const int64_t m = i / cols;
  const int c = (int)(i - m * cols);
  floatx4 v = *reinterpret_cast<const floatx4*>(part + i);
  for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const floatx4*>(part + s * size + i);
  quad<T> y;
#pragma unroll
  for (int z = 0; z < 4; ++z) y[z] = from_f32<T>(v[z] + (bias ? to_f32(bias[c + z]) : 0.f));
  *reinterpret_cast<quad<T>*>(out + (map ? map[m] : m) * cols + c) = y;
}

// Bt [E][rank][o] = B [E][o][rank] and At [E][d][rank] = A [E][rank][d] for the adapters that have rows, one to
// a blockIdx.y; blockIdx.x: 64 of o, then 64 of d.  A workgroup takes all of the rank, in 16-byte vectors.
template <typename T>
__global__ void __launch_bounds__(256) k_lora_transpose(const T* __restrict__ B, T* __restrict__ Bt, int o,
                                                        const T* __restrict__ A, T* __restrict__ At, int d, int rank,
                                                        const int32_t* __restrict__ seg) {
  constexpr int N = 16 / sizeof(T);
  __shared__ T s[64 * (HMOE_LORA_RANK + 1)];  // [long][rank], odd rows of it
  const int e = blockIdx.y;
  if (seg[e] == seg[e + 1]) return;
  const int of_b = (o + 63) / 64;
  const bool tall = (int)blockIdx.x < of_b;  // the long side is the rows
  const int size = tall ? o : d, p0 = (tall ? blockIdx.x : blockIdx.x - of_b) * 64;
  const int valid = size - p0 < 64 ? size - p0 : 64, ld = rank + 1;
  const T* in = (tall ? B : A) + (int64_t)e * size * rank;
  T* out = (tall ? Bt : At) + (int64_t)e * size * rank;
  const auto walk = [&](bool along_rank, auto body) {  // vectors along the rank, or along the long side
    const int vecs = along_rank ? rank / N : valid / N, lines = along_rank ? valid : rank;
    for (int q = threadIdx.x; q < vecs * lines; q += 256) {
      const int line = q / vecs, v = (q - line * vecs) * N;
      const int64_t at = along_rank ? (int64_t)(p0 + line) * rank + v : (int64_t)line * size + p0 + v;
      body(at, along_rank ? line * ld + v : v * ld + line, along_rank ? 1 : ld);
    }
  };
  walk(tall, [&](int64_t at, int first, int step) {
    const i32x4 v = *reinterpret_cast<const i32x4*>(in + at);
    const T* x = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int z = 0; z < N; ++z) s[first + z * step] = x[z];
  });
  __syncthreads();
  walk(!tall, [&](int64_t at, int first, int step) {
    i32x4 v;
    T* x = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int z = 0; z < N; ++z) x[z] = s[first + z * step];
    *reinterpret_cast<i32x4*>(out + at) = v;
  });
}

// ------------------------------------------------------------------ gradients of the adapters

// Rows of one adapter that a workgroup sums over; adapters with more have several pieces, joined
// in order by k_lora_grad_join.  A 64th of all rows, so that no workgroup has much more than the others (with
// 1024 for 16384 rows the few long ones took 69 us for dB and 57 for dA) and 130 pieces at most are kept.
// Smaller ones, of 64 at least, where they leave CUs idle (a step on 777 rows of 8 adapters of 64 and 1000 columns:
// 54 us with 256 rows, 49 with 64).
inline int lora_piece(int64_t n, int E, int d_in, int d_out) {
  const int64_t tiles = cdiv(d_in, 64) + cdiv(d_out, 64);
  int rows = 256;
  while (rows > 64 && (n / rows + (E < n ? E : n)) * tiles < 2 * device_cus()) rows /= 2;
  while (rows < (1 << 20) && (int64_t)rows * 64 < n) rows *= 2;
  return rows;
}
// Where a piece's sums are kept: every adapter of more than `piece` rows advances seg / piece by at least
// half of its pieces.
__device__ __forceinline__ int64_t lora_piece_slot(int64_t seg_e, int64_t local, int piece) {
  return 2 * (seg_e / piece) + local;
}

// Tiles of the gradients: BW columns of D by UW of U, four waves.  The reduction over an adapter's rows is
// often short, a stage or two, and then a workgroup is all latency: 256 columns rather than 64 (111 us for
// dB and 74 for dA at 16384 rows of 128 adapters of rank 16, 4096 and 2048 columns; with 256, and both in one
// launch, 84) keep 36 KB of loads in flight in each.  64 where 256 leave CUs idle.
template <typename T, int UW, int BW, bool U_LEFT>
struct GradTile {
  using type = typename std::conditional<U_LEFT, Cfg<T, UW, BW, UW, BW / 4>, Cfg<T, BW, UW, BW / 4, UW>>::type;
};

// A K-strided operand (gemm.hpp's Stager) whose K row k is at base + rows[k] ld.
template <typename T, int ROWS, int THREADS>
struct MapStager : Stager<T, ROWS, THREADS, false> {
  using S = Stager<T, ROWS, THREADS, false>;
  __device__ __forceinline__ void load(const T* __restrict__ base, int64_t ld, int cols_valid, int k0, int k_valid,
                                       const lds<int32_t>* rows) {
    constexpr int RQ = ROWS / 4;
#pragma unroll
    for (int q = 0; q < S::NPIECE; ++q) {
      const int pc = threadIdx.x + THREADS * q;
      if (S::SPARE && pc >= S::PIECES) continue;
      const int r = pc % RQ * 4, kb = pc / RQ;
      if constexpr (S::BF) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 8 * kb + 2 * i;  // of the stage
          uint2 e = make_uint2(0u, 0u), o = make_uint2(0u, 0u);
          if (r < cols_valid && k0 + k < k_valid) e = *reinterpret_cast<const uint2*>(base + (int64_t)rows[k] * ld + r);
          if (r < cols_valid && k0 + k + 1 < k_valid)
            o = *reinterpret_cast<const uint2*>(base + (int64_t)rows[k + 1] * ld + r);
          this->v[q * 4 + i] = i32x4{(int)e.x, (int)e.y, (int)o.x, (int)o.y};
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 4 * kb + i;
          if (r < cols_valid && k0 + k < k_valid)
            this->v[q * 4 + i] = *reinterpret_cast<const i32x4*>(base + (int64_t)rows[k] * ld + r);
          else
            this->v[q * 4 + i] = i32x4{0, 0, 0, 0};
        }
      }
    }
  }
};

// acc = U^T D or D^T U over `rows` slots from p0 on (pu is there already), on the register-staged engine.  A
// stage's rows of D are looked up a stage before its loads go out: s_row holds those of two stages.  LDS holds
// one stage, the next one's loads are in registers: with two stages in LDS there are fewer workgroups
// to a CU to hide each other's latency (64 values of the rank, 16 adapters, 16384 rows: 214 us, 141 with
// one; and of rank 16 with three workgroups to a CU rather than two 84 us instead of 103).
template <class C, int BW, int UW, bool U_LEFT>
__device__ __forceinline__ void grad_tile(const typename C::type* __restrict__ D, int width, int dv,
                                          const int32_t* __restrict__ map, int64_t p0,
                                          const typename C::type* __restrict__ pu, int ldu, int uv, int rows,
                                          lds<char>* smem, floatx4 (&acc)[C::MI][C::NJ]) {
  using T = typename C::type;
  __shared__ int32_t s_row[2][C::BK];
  MapStager<T, BW, C::THREADS> sd;
  Stager<T, UW, C::THREADS, false> su;
  constexpr int D_BYTES = BW * kStageRowBytes, U_BYTES = UW * kStageRowBytes;
  lds<char>* const bd = smem;
  lds<char>* const bu = smem + D_BYTES;
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int nk = (rows + C::BK - 1) / C::BK, t = threadIdx.x;
  const auto look_up = [&](int s) {
    const int k = s * C::BK + t;
    return t < C::BK && k < rows ? (map ? map[p0 + k] : (int32_t)(p0 + k)) : 0;
  };
  const auto load = [&](int s) {
    sd.load(D, width, dv, s * C::BK, rows, (const lds<int32_t>*)s_row[s & 1]);
    su.load(pu, ldu, uv, s * C::BK, rows);
  };
  const auto store = [&] {
    sd.store(bd);
    su.store(bu);
  };
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int32_t r = look_up(s);
    if (t < C::BK) s_row[s][t] = r;
  }
  __syncthreads();
  load(0);
  store();
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + 1 < nk) load(kt + 1);
    const int32_t r = look_up(kt + 2);
    if constexpr (U_LEFT) mfma_stage<C>((const lds<char>*)bu, (const lds<char>*)bd, acc);
    else mfma_stage<C>((const lds<char>*)bd, (const lds<char>*)bu, acc);
    __syncthreads();
    if (kt + 1 < nk) store();
    if (t < C::BK) s_row[kt & 1][t] = r;  // stage kt's rows: last read before the last barrier
    __syncthreads();
  }
}

// One of the two gradients.
struct GradSide {
  const void* D;       // [n][width]
  const int32_t* map;  // D's row of slot p is map[p], or p without a map
  const void* U;       // U or V, as u_width says
  int width;           // 0: not wanted
  float *out, *part;
};

// For one piece of adapter e's rows:  U_LEFT: out[c][m] = sum_rows U[c] D[m] (dA: [rank][width]),
// otherwise out[m][c] = sum_rows D[m] U[c] (dB: [width][rank]), m from d0 and U's columns from u0 on.
template <typename T, int UW, int BW, bool U_LEFT>
__device__ __forceinline__ void lora_grad_side(const GradSide& g, int d0, int u0, int rank,
                                               const int32_t* __restrict__ seg, int E, int piece) {
  using C = typename GradTile<T, UW, BW, U_LEFT>::type;
  static_assert(C::THREADS == 256, "four waves");
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds<char>* smem = (lds<char>*)smem_raw;
  Run run;
  if (!find_run(seg, E, piece, blockIdx.x, run)) return;
  const int e = run.segment;
  const int64_t local = run.local, p0 = seg[e] + local * piece;
  const int64_t len = seg[e + 1] - p0;
  const int rows = (int)(len < piece ? len : piece);
  const int ldu = u_width<T>(rank);
  const int width = g.width;
  const T *D = static_cast<const T*>(g.D), *U = static_cast<const T*>(g.U);
  const int dv = width - d0 < BW ? width - d0 : BW, uv = ldu - u0 < UW ? ldu - u0 : UW;
  floatx4 acc[C::MI][C::NJ];
  grad_tile<C, BW, UW, U_LEFT>(D + d0, width, dv, g.map, p0, U + p0 * ldu + u0, ldu, uv, rows, smem, acc);
  const int64_t size = (int64_t)width * rank;
  float* to = seg[e + 1] - seg[e] > piece ? g.part + lora_piece_slot(seg[e], local, piece) * size : g.out + e * size;
  const Frag<C> f;
  const auto put = [&](int c, int m, float v) {  // value c of the rank, column m of D
    if (c < rank && m < width) to[U_LEFT ? (int64_t)c * width + m : (int64_t)m * rank + c] = v;
  };
  constexpr bool BF = sizeof(T) == 2;  // the sums with 16 values and with their remainders are one
  static_assert(!BF || UW % (16 * kUParts) == 0, "whole blocks of U");
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (BF && U_LEFT) {
          if (i % 3 == 0)
            put(u0 / 3 + 16 * (i / 3) + 4 * f.lg + r, d0 + f.col(j, r), (acc[i + 2][j][r] + acc[i + 1][j][r]) + acc[i][j][r]);
        } else if constexpr (BF) {
          if (j % 3 == 0)
            put(u0 / 3 + 16 * (j / 3) + f.lr, d0 + f.row(i, r), (acc[i][j + 2][r] + acc[i][j + 1][r]) + acc[i][j][r]);
        } else {
          if constexpr (U_LEFT) put(u0 + f.row(i, r), d0 + f.col(j, r), acc[i][j][r]);
          else put(u0 + f.col(j, r), d0 + f.row(i, r), acc[i][j][r]);
        }
      }
}

// Both gradients: blockIdx.y runs over dB's tiles and then dA's.  (One launch each: 24 us for 777 rows of the tiny
// decoder, 13 together.)  The chunks of the rank that read the same part of D come one after the other on
// the same XCD, gridDim.x being a multiple of 8 (rank 128, 16 adapters of 16384 rows: 270 us, 254 so).
template <typename T>
constexpr int kNarrow = sizeof(T) == 2 ? 48 : 32;  // of U: rank 16, 32
template <typename T, int UW, int BW>
__global__ void __launch_bounds__(256, UW == kNarrow<T> ? 3 : 2)
    k_lora_grad(GradSide b, GradSide a, int rank, const int32_t* __restrict__ seg, int E, int piece) {
  const int tiles_b = (b.width + BW - 1) / BW, chunks = (u_width<T>(rank) + UW - 1) / UW;
  const int y = blockIdx.y / chunks, u0 = blockIdx.y % chunks * UW;
  if (y < tiles_b) lora_grad_side<T, UW, BW, false>(b, y * BW, u0, rank, seg, E, piece);
  else lora_grad_side<T, UW, BW, true>(a, (y - tiles_b) * BW, u0, rank, seg, E, piece);
}

// The pieces of an adapter added in their order; adapters without rows get zeros.  Both gradients in one launch:
// blockIdx.x runs over dB's outputs and then dA's (either may be missing: size 0), four to a thread.
__global__ void __launch_bounds__(256) k_lora_grad_join(GradSide b, GradSide a, int rank, const int32_t* __restrict__ seg,
                                                        int piece) {
  const int e = blockIdx.y;
  const int64_t pieces = cdiv(seg[e + 1] - seg[e], piece), first = cdiv((int64_t)b.width * rank, 1024);
  if (pieces == 1) return;
  const bool is_b = blockIdx.x < first;
  const GradSide& g = is_b ? b : a;
  const int64_t size = (int64_t)g.width * rank;
  const int64_t i = ((blockIdx.x - (is_b ? 0 : first)) * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  floatx4 s = {0.f, 0.f, 0.f, 0.f};
  const float* p = g.part + lora_piece_slot(seg[e], 0, piece) * size + i;
  for (int64_t q = 0; q < pieces; ++q) s += *reinterpret_cast<const floatx4*>(p + q * size);
  *reinterpret_cast<floatx4*>(g.out + e * size + i) = s;
}

template <typename T>
int lora_shrink(const T* X, int K, const T* A, int rank, const float* scale, const int32_t* seg, int E,
                int64_t n, const int32_t* map, T* U, hipStream_t st) {
  const int blocks = u_blocks(rank);
  const int rows = blocks == 1 ? 16 : 32;
  return over_slices(n / rows + (E < n ? E : n), 1, 256, [&](int64_t run0, int64_t runs) {
    const dim3 grid((unsigned)runs, (unsigned)cdiv(blocks, 4)), block(256);
    if (blocks == 1)
      HMOE_LAUNCH("lora shrink", (k_lora_shrink<T, 1, 1>), grid, block, 0, st, X, K, A, rank, scale, seg, E, map, U, run0);
    else if (blocks == 2)
      HMOE_LAUNCH("lora shrink", (k_lora_shrink<T, 2, 2>), grid, block, 0, st, X, K, A, rank, scale, seg, E, map, U, run0);
    else
      HMOE_LAUNCH("lora shrink", (k_lora_shrink<T, 4, 2>), grid, block, 0, st, X, K, A, rank, scale, seg, E, map, U, run0);
    return (int)HMOE_OK;
  });
}

// Tiles for the type (gemm.hpp), quarter tiles where there are fewer of them than half of the CUs (bf16, rows of
// 1024 into 1024: 4096 rows, 64 tiles, 37 us with whole tiles and 25 with quarter tiles; 8192 rows 36 and 43).
template <typename T, bool W_KC>
using LoraTile = typename std::conditional<W_KC, typename Pick<T>::C, typename Pick<T>::CK>::type;
template <typename T, bool W_KC>
bool lora_small(int64_t n, int cols) {
  using C = LoraTile<T, W_KC>;
  return cdiv(n, C::BM) * cdiv(cols, C::BN) * 2 < device_cus();
}
// Splits of the reduction, of three stages at least, up to four workgroups to a CU, where that makes three or
// more of them worth the launch that joins them (4 us): 777 x 64 fp32 outputs of 1000 products, 13 tiles: 36 us,
// 10 in eight splits; 4814 x 200 bf16 of 3528, 304 tiles: 60 us, 31 in three.
template <typename T>
int lora_gemm_splits(int64_t n, int cols, int Kd) {
  using Q = CfgQuarter<T>;
  const int64_t tiles = cdiv(n, Q::BM) * cdiv(cols, Q::BN);
  const int64_t fill = 4 * device_cus() / tiles, stages = Kd / (3 * Q::BK), s = fill < stages ? fill : stages;
  return s < 3 ? 1 : (s > 8 ? 8 : (int)s);
}
template <typename T>
size_t lora_gemm_part(int64_t n, int cols, int Kd) {
  const int s = lora_gemm_splits<T>(n, cols, Kd);
  return s > 1 ? (size_t)s * n * cols : 0;
}
template <class C, bool W_KC, bool GATHER, typename T>
int lora_gemm_on(const T* A, const T* W, const T* bias, const T* U, const T* B, int rank, const int32_t* seg, int E,
                 int64_t n, int cols, int Kd, const int32_t* map, T* out, int splits, float* part, hipStream_t st) {
  HMOE_LAUNCH(W_KC ? "lora forward" : "lora input gradient", (k_lora_gemm<C, W_KC, GATHER>),
              dim3((unsigned)(cdiv(n, C::BM) * cdiv(cols, C::BN)), (unsigned)splits), dim3(C::THREADS), C::LDS, st, A, W,
              bias, U, B, rank, seg, E, n, cols, Kd, map, out, part);
  return HMOE_OK;
}
template <typename T, bool W_KC>
int lora_gemm(const T* A, const T* W, const T* bias, const T* U, const T* B, int rank, const int32_t* seg, int E,
              int64_t n, int cols, int Kd, const int32_t* map, T* out, float* part, hipStream_t st) {
  if (!lora_small<T, W_KC>(n, cols))
    return lora_gemm_on<LoraTile<T, W_KC>, W_KC, false>(A, W, bias, U, B, rank, seg, E, n, cols, Kd, map, out, 1, nullptr, st);
  const int splits = lora_gemm_splits<T>(n, cols, Kd);
  HMOE_TRY((lora_gemm_on<CfgQuarter<T>, W_KC, false>(A, W, bias, U, B, rank, seg, E, n, cols, Kd, map, out, splits, part, st)));
  if (splits > 1)
    HMOE_LAUNCH("lora join", k_lora_gemm_join<T>, dim3((unsigned)cdiv(n * cols, 1024)), dim3(256), 0, st, part, splits, n,
                cols, bias, map, out);
  return HMOE_OK;
}

template <typename T, int UW, int BW>
int lora_grad_tiles(const GradSide& b, const GradSide& a, int rank, const int32_t* seg, int E, int64_t n, int piece,
                    hipStream_t st) {
  using C = typename GradTile<T, UW, BW, false>::type;
  static_assert(C::LDS == GradTile<T, UW, BW, true>::type::LDS, "one launch for both");
  HMOE_LAUNCH("lora gradients", (k_lora_grad<T, UW, BW>),
              dim3((unsigned)(cdiv(n / piece + (E < n ? E : n), 8) * 8),
                   (unsigned)((cdiv(b.width, BW) + cdiv(a.width, BW)) * cdiv(u_width<T>(rank), UW))),
              dim3(256), C::LDS / 2, st, b, a, rank, seg, E, piece);
  return HMOE_OK;
}
template <typename T>
int lora_grad(const GradSide& b, const GradSide& a, int rank, const int32_t* seg, int E, int64_t n, int piece,
                    hipStream_t st) {
  constexpr int NARROW = kNarrow<T>;
  const int64_t pieces = n / piece + (E < n ? E : n);
  if (pieces * (cdiv(b.width, 256) + cdiv(a.width, 256)) < device_cus())
    HMOE_TRY((lora_grad_tiles<T, NARROW, 64>(b, a, rank, seg, E, n, piece, st)));
  else if (u_width<T>(rank) <= NARROW)
    HMOE_TRY((lora_grad_tiles<T, NARROW, 256>(b, a, rank, seg, E, n, piece, st)));
  else
    HMOE_TRY((lora_grad_tiles<T, 2 * NARROW, 256>(b, a, rank, seg, E, n, piece, st)));
  HMOE_LAUNCH("lora gradient join", k_lora_grad_join,
              dim3((unsigned)(cdiv((int64_t)b.width * rank, 1024) + cdiv((int64_t)a.width * rank, 1024)), (unsigned)E),
              dim3(256), 0, st, b, a, rank, seg, piece);
  return HMOE_OK;
}

struct LoraSpace {
  void *dYs, *Bt, *At, *V;
  float *part_a, *part_b, *split;  // of the adapters' gradients' sums, and of the products'
};

LoraSpace lora_carve(const hmoe_lora_t* p, int64_t n, Workspace& ws) {
  const size_t s = dtype_size(p->dt), ldu = p->dt == HMOE_BF16 ? u_width<bf16>(p->rank) : u_width<float>(p->rank);
  LoraSpace x;
  x.dYs = ws.take<char>((size_t)n * p->d_out * s);
  x.Bt = ws.take<char>((size_t)p->E * p->rank * p->d_out * s);
  x.At = ws.take<char>((size_t)p->E * p->rank * p->d_in * s);
  x.V = ws.take<char>((size_t)n * ldu * s);
  const int64_t piece = lora_piece(n, p->E, p->d_in, p->d_out);
  const size_t pieces = n > piece ? 2 * (n / piece) + 2 : 0;
  x.part_a = ws.take<float>(pieces * p->d_in * p->rank);
  x.part_b = ws.take<float>(pieces * p->d_out * p->rank);
  const size_t fwd = p->dt == HMOE_BF16 ? lora_gemm_part<bf16>(n, p->d_out, p->d_in) : lora_gemm_part<float>(n, p->d_out, p->d_in);
  const size_t bwd = p->dt == HMOE_BF16 ? lora_gemm_part<bf16>(n, p->d_in, p->d_out) : lora_gemm_part<float>(n, p->d_in, p->d_out);
  x.split = ws.take<float>(fwd > bwd ? fwd : bwd);
  return x;
}

template <typename T>
int lora_forward_t(const hmoe_lora_t* p, int64_t n, const T* X, const int32_t* offsets, const int32_t* perm, T* U, T* Y,
                   const LoraSpace& w, hipStream_t st) {
  HMOE_TRY(lora_shrink<T>(X, p->d_in, (const T*)p->A, p->rank, p->scale, offsets, p->E, n, nullptr, U, st));
  return lora_gemm<T, true>(X, (const T*)p->W, (const T*)p->b, U, (const T*)p->B, p->rank, offsets, p->E, n, p->d_out,
                            p->d_in, perm, Y, w.split, st);
}

template <typename T>
int lora_backward_t(const hmoe_lora_t* p, int64_t n, const T* X, const int32_t* offsets, const int32_t* perm, const T* U,
                    const T* dY, T* dX, float* dA, float* dB, const LoraSpace& w, hipStream_t st) {
  // dY's rows are gathered by whoever reads them (a copy in slot order took 45 us of 670 at 16384 rows of
  // 4096), but for the input gradient on tiles that cannot
  const bool gather = perm && (!dX || (sizeof(T) == 2 && !lora_small<T, false>(n, p->d_in) &&
                                       (int64_t)n * p->d_out * (int64_t)sizeof(T) < (int64_t(1) << 32)));
  const int32_t* map = gather ? perm : nullptr;
  if (perm && !gather) {
    HMOE_TRY(launch_permute(dY, w.dYs, perm, n, p->d_out, p->dt, st));
    dY = (const T*)w.dYs;
  }
  if (dX || dA) {
    HMOE_LAUNCH("lora transpose", k_lora_transpose<T>,
                dim3((unsigned)(cdiv(p->d_out, 64) + (dX ? cdiv(p->d_in, 64) : 0)), (unsigned)p->E), dim3(256), 0, st,
                (const T*)p->B, (T*)w.Bt, p->d_out, (const T*)p->A, (T*)w.At, p->d_in, p->rank, offsets);
    HMOE_TRY(lora_shrink<T>(dY, p->d_out, (const T*)w.Bt, p->rank, p->scale, offsets, p->E, n, map, (T*)w.V, st));
  }
  if (dX) {
    const T *W = (const T*)p->W, *V = (const T*)w.V, *At = (const T*)w.At;
    if constexpr (sizeof(T) == 2) {
      if (gather)
        HMOE_TRY(lora_gemm_on<LoraTile<T, false>, false, true>(dY, W, (const T*)nullptr, V, At, p->rank, offsets, p->E, n,
                                                               p->d_in, p->d_out, perm, dX, 1, nullptr, st));
    }
    if (!gather)
      HMOE_TRY(lora_gemm<T, false>(dY, W, nullptr, V, At, p->rank, offsets, p->E, n, p->d_in, p->d_out, perm, dX, w.split, st));
  }
  if (dA || dB) {
    const GradSide b = {dY, map, U, dB ? p->d_out : 0, dB, w.part_b}, a = {X, nullptr, w.V, dA ? p->d_in : 0, dA, w.part_a};
    return lora_grad<T>(b, a, p->rank, offsets, p->E, n, lora_piece(n, p->E, p->d_in, p->d_out), st);
  }
  return HMOE_OK;
}

}  // namespace

int lora_saved_width(int rank, hmoe_dtype_t dt) { return dt == HMOE_BF16 ? u_width<bf16>(rank) : u_width<float>(rank); }

static int lora_few_width(const hmoe_lora_t* p) {
  return p->dt == HMOE_BF16 ? u_width<bf16, 2>(p->rank) : u_width<float>(p->rank);
}

size_t lora_few_ws(const hmoe_lora_t* p, int64_t n) {
  Workspace w(nullptr, 0);
  w.take<char>((size_t)n * lora_few_width(p) * dtype_size(p->dt));
  return w.off;
}

size_t lora_ws(const hmoe_lora_t* p, int64_t n) {
  Workspace w(nullptr, 0);
  lora_carve(p, n, w);
  return w.off;
}

int launch_lora_few(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* adapter, void* Y, Workspace& ws,
                    hipStream_t st) {
  LoraFew a = {X, p->W, p->b, p->A, p->B, p->scale, adapter, (int)n, p->E, p->d_in, p->d_out, p->rank, nullptr, Y};
  a.U = ws.take<char>((size_t)n * lora_few_width(p) * dtype_size(p->dt));
  return p->dt == HMOE_BF16 ? lora_few_t<bf16>(a, st) : lora_few_t<float>(a, st);
}

int launch_lora_forward(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* offsets, const int32_t* perm,
                        void* U, void* Y, Workspace& ws, hipStream_t st) {
  const LoraSpace w = lora_carve(p, n, ws);
  if (p->dt == HMOE_BF16)
    return lora_forward_t<bf16>(p, n, (const bf16*)X, offsets, perm, (bf16*)U, (bf16*)Y, w, st);
  return lora_forward_t<float>(p, n, (const float*)X, offsets, perm, (float*)U, (float*)Y, w, st);
}

int launch_lora_backward(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* offsets, const int32_t* perm,
                         const void* U, const void* dY, void* dX, float* dA, float* dB, Workspace& ws, hipStream_t st) {
  const LoraSpace w = lora_carve(p, n, ws);
  if (p->dt == HMOE_BF16)
    return lora_backward_t<bf16>(p, n, (const bf16*)X, offsets, perm, (const bf16*)U, (const bf16*)dY, (bf16*)dX, dA, dB,
                                 w, st);
  return lora_backward_t<float>(p, n, (const float*)X, offsets, perm, (const float*)U, (const float*)dY, (float*)dX, dA,
                                dB, w, st);
}

}  // namespace hmoe
