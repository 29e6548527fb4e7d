// Layer norm over the rows of a matrix, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh gamma + beta
//   q = dy gamma, dx = r (q - mean(q) - xh mean(q xh)), dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Every pass is bound by memory: a row is read once into registers, its mean and then its centred square sum (no
// difference of large sums) are taken there in fp32, and its result is rounded once, when it is stored.  A row belongs
// to G threads, 16 elements each (up to 24 in bf16, a run of 16 bytes of short rows): 8 to 64 lanes of a wavefront, or 128 to 1024 threads of a workgroup; longer
// rows are read again from the cache.  The backward pass keeps dgamma and dbeta of a thread's columns in registers over
// all the rows that its workgroup takes, so the sums over rows cost one row of partial sums for each workgroup and a
// second, small pass that adds them in a fixed order.
//
// Measured, bf16: 16384 x 4096 forward 47 us (5.7 TB/s from and to memory and the last cache; a large copy 4.9), backward 79 + 5 (5.1);
// 8192 x 1024 8.6, 11.5 + 3.8; 1027 x 1501 (rows at odd addresses) 4.8, 7.6 + 3.4; 100000 x 128 10, 18 together.  The next row in
// flight, kept whole accesses and fewer partial sums made the backward pass of 16384 x 4096 136 -> 84 us.
#include <algorithm>
#include <type_traits>

#include "rows.hpp"

namespace ard {

struct NormRows {
  int R, D;        // rows; elements that take part
  int wide;        // columns stored: D, or pad8(D) with zeros behind D
  int64_t ldx, ldy;
  float eps, d;       // d = D
};


// sum over the up to 64 lanes of a row that lie in one wavefront (16: a row of the cross-lane moves, 8: half of one)
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
  static_assert(G == 8 || G == 16 || G == 32 || G >= 64, "");
  if constexpr (G >= 64) return wave_sum(v);
  if constexpr (G == 8) return half_row_sum(v);
  v = row_sum(v);
  if constexpr (G == 32) v += __shfl_xor(v, 16);
  return v;
}
// sum over the G threads of a row; `slot`: LDS of this sum alone (one float for each wavefront)
template <int G> __device__ __forceinline__ float group_sum(float v, float* slot) {
  v = lanes_sum<G>(v);
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x % G >> 6] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) v += slot[w];
  }
  return v;
}

template <int N, typename WT> __device__ __forceinline__ void load_weight(const WT* w, int col, int n, float dflt, float (&x)[N]) {
  if (w) {
    load_some<N>(w + col, n, x);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = dflt;
  }
}

// Where a thread's k-th run of CE elements lies: the run that the row's end cuts lies back from it, so that every access is a
// whole one inside the row (rows have CE elements at least).  Its first `skip` elements are other threads' too: sums over the row leave
// them out, results are the same bits and are stored twice (335544 x 100 bf16 forward + backward 29.7 + 43.7 us; with the last ones stored one
// by one 40.5 + 50.7).  Runs behind the end store nothing.
template <int CE, int G> struct RunAt {
  int col, skip;
  __device__ __forceinline__ RunAt(int k, int lane, int D) {
    const int c = (k * G + lane) * CE;
    col = imin(c, D - CE), skip = c - col;
  }
};
template <int CE, typename T> __device__ __forceinline__ void store_twice(T* p, int skip, const float (&x)[CE]) {
  if (skip < CE) store_run<CE>(p, x);
}
// The same where the first `skip` values are not the other thread's.
template <int CE, typename T> __device__ __forceinline__ void store_own(T* p, int skip, const float (&x)[CE]) {
  if (skip == 0) {
    store_run<CE>(p, x);
  } else if (skip < CE) {
#pragma unroll
    for (int j = 1; j < CE; ++j)
      if (j >= skip) p[j] = ElemTraits<T>::from_f32(x[j]);
  }
}
// zeros behind the D elements of a compact row
template <typename T> __device__ __forceinline__ void store_padding(const NormRows& a, T* y, int lane) {
  if (lane < a.wide - a.D) y[a.D + lane] = ElemTraits<T>::from_f32(0.0f);
}

constexpr int norm_fwd_threads(int G) { return G > 256 ? G : 256; }

template <typename T, typename WT, int G, int CE, int NV>
__global__ __launch_bounds__(norm_fwd_threads(G)) void norm_fwd_kernel(NormRows a, const T* X, const WT* gamma, const WT* beta, T* Y, float* mean,
                                                                      float* rstd) {
  constexpr int GROUPS = norm_fwd_threads(G) / G;  // rows at a time
  __shared__ float slots[2][GROUPS][G > 64 ? G / 64 : 1];
  const int lane = threadIdx.x % G, group = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // a row is asked for while the one before it is worked on; the weights are held for all
  typename Run<T, CE>::V rx[NV];
  typename Run<WT, CE>::V rg[NV], rb[NV];
  auto ask = [&](int64_t row) {
    if (GROUPS > 1) row = row < a.R ? row : a.R - 1;  // (a group without a row of its own reads the last one)
#pragma unroll
    for (int k = 0; k < NV; ++k) rx[k] = load_whole<CE>(X + row * a.ldx + RunAt<CE, G>(k, lane, a.D).col);
  };
  ask((int64_t)blockIdx.x * GROUPS + group);
  if (gamma) {
#pragma unroll
    for (int k = 0; k < NV; ++k) rg[k] = load_whole<CE>(gamma + RunAt<CE, G>(k, lane, a.D).col);
  }
  if (beta) {
#pragma unroll
    for (int k = 0; k < NV; ++k) rb[k] = load_whole<CE>(beta + RunAt<CE, G>(k, lane, a.D).col);
  }
  for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < a.R; row0 += step) {
    const int64_t row = row0 + group;
    const bool mine = GROUPS == 1 || row < a.R;
    T* y = Y + row * a.ldy;
    float v[NV][CE], s = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) values_of<CE, T>(rx[k], v[k]);
    if (row0 + step < a.R) ask(row + step);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int skip = RunAt<CE, G>(k, lane, a.D).skip;
#pragma unroll
      for (int j = 0; j < CE; ++j) s += j >= skip ? v[k][j] : 0.0f;
    }
    const float mu = group_sum<G>(s, slots[0][group]) / a.d;
    float q = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int skip = RunAt<CE, G>(k, lane, a.D).skip;
#pragma unroll
      for (int j = 0; j < CE; ++j) {
        v[k][j] -= mu;
        const float d = j >= skip ? v[k][j] : 0.0f;
        q = fmaf(d, d, q);
      }
    }
    const float r = 1.0f / sqrtf(group_sum<G>(q, slots[1][group]) / a.d + a.eps);
    if (!mine) break;  // (the last turn)
    if (lane == 0) mean[row] = mu, rstd[row] = r;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const RunAt<CE, G> at(k, lane, a.D);
      float w[CE], u[CE];
      if (gamma) {
        values_of<CE, WT>(rg[k], w);
      } else {
#pragma unroll
        for (int j = 0; j < CE; ++j) w[j] = 1.0f;
      }
      if (beta) {
        values_of<CE, WT>(rb[k], u);
      } else {
#pragma unroll
        for (int j = 0; j < CE; ++j) u[j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < CE; ++j) w[j] = fmaf(v[k][j] * r, w[j], u[j]);
      store_twice<CE>(y + at.col, at.skip, w);
    }
    store_padding(a, y, lane);
    // (the next row's first sum is written after every wavefront has passed this row's second barrier, hence has read the
    // first; its second sum after the next row's first barrier: the slots need no barrier of their own)
  }
}

// Rows too long for the registers of a workgroup: read three times, the second and third time from the cache.  A run's elements are added
// up before their sum joins the thread's: one by one, 32768 squares of a thread (rows of 2^25 bf16 elements) came out
// 1e-5 too large, each being ever less beside the growing sum.  2048 x 20480 bf16 forward 50 us, backward 112 (3.3, 2.2 TB/s of inputs and results;
// 2048 x 16384, held in registers, 29 and 63), 2048 x 32768 84 and 170; fp32 97 and 195, 159 and 317.
template <typename T, typename WT>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(NormRows a, const T* X, const WT* gamma, const WT* beta, T* Y, float* mean, float* rstd) {
  constexpr int CE = ElemTraits<T>::CE;
  __shared__ float slots[2][16];
  for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
    const T* x = X + row * a.ldx;
    T* y = Y + row * a.ldy;
    float s = 0.0f, v[CE];
    for (int64_t col = threadIdx.x * CE; col < a.D; col += 1024 * CE) {
      load_some<CE>(x + col, (int)(a.D - col), v);
      float of_run = 0.0f;
  #pragma unroll
      for (int j = 0; j < CE; ++j) of_run += v[j];
      s += of_run;
    }
    const float mu = group_sum<1024>(s, slots[0]) / a.d;
    float q = 0.0f;
    for (int64_t col = threadIdx.x * CE; col < a.D; col += 1024 * CE) {
      load_some<CE>(x + col, (int)(a.D - col), v);
      float of_run = 0.0f;
  #pragma unroll
      for (int j = 0; j < CE; ++j) {
        const float d = j < a.D - col ? v[j] - mu : 0.0f;
        of_run = fmaf(d, d, of_run);
      }
      q += of_run;
    }
    const float r = 1.0f / sqrtf(group_sum<1024>(q, slots[1]) / a.d + a.eps);
    if (threadIdx.x == 0) mean[row] = mu, rstd[row] = r;
    for (int64_t col = threadIdx.x * CE; col < a.wide; col += 1024 * CE) {
      const int n = (int)(a.D - col);
      float g[CE], b[CE];
      load_some<CE>(x + col, n, v);
      load_weight<CE>(gamma, (int)col, n, 1.0f, g);
      load_weight<CE>(beta, (int)col, n, 0.0f, b);
  #pragma unroll
      for (int j = 0; j < CE; ++j) g[j] = j < n ? fmaf((v[j] - mu) * r, g[j], b[j]) : 0.0f;
      store_some<CE>(y + col, (int)(a.wide - col), g);
    }
  }
}

struct NormBack {
  NormRows a;      // ldx: of X
  int64_t lddy, lddx;
};

// One row of partial sums [2][D] for each workgroup: dgamma, dbeta of the rows it took.  A workgroup of 8 wavefronts (16 for
// rows of 1024 threads) works on as many rows at a time as it has groups of G threads and adds up their sums in LDS: a partial
// row for every group would be a third of the traffic of 8192 rows of 1024.
constexpr int norm_bwd_threads(int G, int N) { return G > 512 || N <= 8 ? 1024 : 512; }
template <typename T, typename WT, int G, int CE, int NV>
__global__ __launch_bounds__(norm_bwd_threads(G, NV * CE)) void norm_bwd_kernel(NormBack b, const T* dY, const T* X, const WT* gamma, const float* mean,
                                                                     const float* rstd, T* dX, float* part) {
  constexpr int GROUPS = norm_bwd_threads(G, NV * CE) / G, N = NV * CE, W = G > 64 ? G / 64 : 1;  // rows at a time, elements of a thread, wavefronts of a row
  constexpr int PARTS = GROUPS / (G < 64 ? 64 / G : 1);  // sums of groups that do not share a wavefront
  constexpr bool AHEAD = G < 1024;  // the next row is asked for while one is worked on, and gamma is held (16 wavefronts have no registers for either)
  __shared__ float slots[2][2][GROUPS][W];
  __shared__ float sums[PARTS > 1 ? PARTS - 1 : 1][PARTS > 1 ? 2 * G * N : 1];
  const int lane = threadIdx.x % G, group = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G, D = b.a.D;
  float g[NV][CE], ag[NV][CE] = {}, ab[NV][CE] = {};
  auto weights = [&] {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (gamma) {
        values_of<CE, WT>(load_whole<CE>(gamma + RunAt<CE, G>(k, lane, D).col), g[k]);
      } else {
#pragma unroll
        for (int j = 0; j < CE; ++j) g[k][j] = 1.0f;
      }
    }
  };
  if (AHEAD) weights();
  const int64_t first = (int64_t)blockIdx.x * GROUPS, step = (int64_t)gridDim.x * GROUPS;
  typename Run<T, CE>::V nx[NV], ny[NV];
  float nmu = 0.0f, nr = 0.0f;
  auto ask = [&](int64_t row) {
    if (GROUPS > 1) row = row < b.a.R ? row : b.a.R - 1;  // (a group without a row of its own reads the last one)
    const T *x = X + row * b.a.ldx, *dy = dY + row * b.lddy;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = RunAt<CE, G>(k, lane, D).col;
      nx[k] = load_whole<CE>(x + col);
      ny[k] = load_whole<CE>(dy + col);
    }
    nmu = mean[row], nr = rstd[row];
  };
  if (AHEAD) ask(first + group);
  int turn = 0;
  // (every group takes as many turns, so all meet at the barriers; one without a row of its own in the last turn adds nothing)
  for (int64_t row0 = first; row0 < b.a.R; row0 += step, turn ^= 1) {
    const int64_t row = row0 + group;
    const bool mine = GROUPS == 1 || row < b.a.R;
    if (!AHEAD) ask(row), weights();
    float v[NV][CE], u[NV][CE];
#pragma unroll
    for (int k = 0; k < NV; ++k) values_of<CE, T>(nx[k], v[k]), values_of<CE, T>(ny[k], u[k]);
    const float mu = nmu, r = nr;
    if (AHEAD && row0 + step < b.a.R) ask(row + step);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int skip = RunAt<CE, G>(k, lane, D).skip;
#pragma unroll
      for (int j = 0; j < CE; ++j) {
        v[k][j] = mine ? (v[k][j] - mu) * r : 0.0f;
        u[k][j] = mine ? u[k][j] : 0.0f;
        ag[k][j] = fmaf(u[k][j], v[k][j], ag[k][j]);
        ab[k][j] += u[k][j];
        u[k][j] *= g[k][j];
        const float d = j >= skip ? u[k][j] : 0.0f;
        s1 += d;
        s2 = fmaf(d, j >= skip ? v[k][j] : 0.0f, s2);
      }
    }
    s1 = lanes_sum<G>(s1), s2 = lanes_sum<G>(s2);
    if constexpr (G > 64) {  // (two sums at one barrier; the next row's go to the other slots, so none is read while it is written)
      if ((threadIdx.x & 63) == 0) slots[turn][0][group][lane >> 6] = s1, slots[turn][1][group][lane >> 6] = s2;
      __syncthreads();
      s1 = slots[turn][0][group][0], s2 = slots[turn][1][group][0];
#pragma unroll
      for (int w = 1; w < W; ++w) s1 += slots[turn][0][group][w], s2 += slots[turn][1][group][w];
    }
    if (!mine) break;  // (the last turn)
    s1 /= b.a.d, s2 /= b.a.d;
    T* dx = dX + row * b.lddx;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const RunAt<CE, G> at(k, lane, D);
#pragma unroll
      for (int j = 0; j < CE; ++j) u[k][j] = r * (u[k][j] - s1 - v[k][j] * s2);
      store_twice<CE>(dx + at.col, at.skip, u[k]);
    }
    store_padding(b.a, dx, lane);
  }
  if (!part) return;
  float* out = part + (int64_t)blockIdx.x * 2 * D;
  if constexpr (G < 64) {  // those of a wavefront's groups, lane to lane
#pragma unroll
    for (int o = G; o < 64; o *= 2)
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < CE; ++j) ag[k][j] += __shfl_xor(ag[k][j], o), ab[k][j] += __shfl_xor(ab[k][j], o);
  }
  if constexpr (PARTS > 1) {  // the groups' sums, added in order
    const int of = G < 64 ? threadIdx.x >> 6 : group;
    const bool speaks = G >= 64 || (threadIdx.x & 63) < G;
    if (of && speaks) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < CE; ++j) sums[of - 1][(k * CE + j) * G + lane] = ag[k][j], sums[of - 1][(N + k * CE + j) * G + lane] = ab[k][j];
    }
    __syncthreads();
    if (of || !speaks) return;
#pragma unroll 1
    for (int o = 0; o < PARTS - 1; ++o)
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < CE; ++j) ag[k][j] += sums[o][(k * CE + j) * G + lane], ab[k][j] += sums[o][(N + k * CE + j) * G + lane];
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const RunAt<CE, G> at(k, lane, D);
    store_twice<CE>(out + at.col, at.skip, ag[k]);
    store_twice<CE>(out + D + at.col, at.skip, ab[k]);
  }
}

// Few rows: one launch in place of two.  The first `row_blocks` workgroups take a row a group, the others 16 runs of columns
// each, whose sums over the rows they make from the inputs themselves (which the caches hold): dealt to threads / 16 lanes,
// added in order.  128 x 1000 bf16 takes 4.2 us of calls in a row (the host's time), 6.7 in two launches.  Where dX takes the place of an
// input the two kinds of workgroups are two launches, sums first.
constexpr int norm_few_threads(int G) { return G > 512 ? G : 512; }
template <typename T, typename WT, int G, int CE, int NV>
__global__ __launch_bounds__(norm_few_threads(G)) void norm_bwd_few_kernel(NormBack b, const T* dY, const T* X, const WT* gamma, const float* mean,
                                                                         const float* rstd, T* dX, WT* dgamma, WT* dbeta, int row_blocks) {
  constexpr int THREADS = norm_few_threads(G), GROUPS = THREADS / G, W = G > 64 ? G / 64 : 1;
  __shared__ float slots[2][GROUPS][W];
  __shared__ float sums[THREADS / 64][16][2 * CE];
  const int D = b.a.D, R = b.a.R;
  if ((int)blockIdx.x >= row_blocks) {
    const int lane = threadIdx.x & 15;
    const RunAt<CE, 16> at(blockIdx.x - row_blocks, lane, D);
    float ag[CE] = {}, ab[CE] = {};
#pragma unroll 4
    for (int row = threadIdx.x >> 4; row < R; row += THREADS / 16) {
      float v[CE], u[CE];
      load_run<CE>(X + row * b.a.ldx + at.col, v);
      load_run<CE>(dY + row * b.lddy + at.col, u);
      const float mu = mean[row], r = rstd[row];
#pragma unroll
      for (int j = 0; j < CE; ++j) ag[j] = fmaf(u[j], (v[j] - mu) * r, ag[j]), ab[j] += u[j];
    }
#pragma unroll
    for (int j = 0; j < CE; ++j) {
      ag[j] += __shfl_xor(ag[j], 16), ab[j] += __shfl_xor(ab[j], 16);
      ag[j] += __shfl_xor(ag[j], 32), ab[j] += __shfl_xor(ab[j], 32);
    }
    if ((threadIdx.x & 63) < 16) {
#pragma unroll
      for (int j = 0; j < CE; ++j) sums[threadIdx.x >> 6][lane][j] = ag[j], sums[threadIdx.x >> 6][lane][CE + j] = ab[j];
    }
    __syncthreads();
    if (threadIdx.x >= 16) return;
    for (int w = 1; w < THREADS / 64; ++w)
#pragma unroll
      for (int j = 0; j < CE; ++j) ag[j] += sums[w][lane][j], ab[j] += sums[w][lane][CE + j];
    if (dgamma) store_own<CE>(dgamma + at.col, at.skip, ag);
    if (dbeta) store_own<CE>(dbeta + at.col, at.skip, ab);
    return;
  }
  const int lane = threadIdx.x % G, group = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
  const int64_t mine = (int64_t)blockIdx.x * GROUPS + group, row = GROUPS == 1 || mine < R ? mine : R - 1;
  typename Run<T, CE>::V rx[NV], ry[NV];
  typename Run<WT, CE>::V rg[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int col = RunAt<CE, G>(k, lane, D).col;
    rx[k] = load_whole<CE>(X + row * b.a.ldx + col), ry[k] = load_whole<CE>(dY + row * b.lddy + col);
    if (gamma) rg[k] = load_whole<CE>(gamma + col);
  }
  const float mu = mean[row], r = rstd[row];
  float v[NV][CE], u[NV][CE], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int skip = RunAt<CE, G>(k, lane, D).skip;
    float g[CE];
    values_of<CE, T>(rx[k], v[k]), values_of<CE, T>(ry[k], u[k]);
    if (gamma) {
      values_of<CE, WT>(rg[k], g);
    } else {
#pragma unroll
      for (int j = 0; j < CE; ++j) g[j] = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < CE; ++j) {
      v[k][j] = j >= skip ? (v[k][j] - mu) * r : 0.0f;
      u[k][j] = j >= skip ? u[k][j] * g[j] : 0.0f;
      s1 += u[k][j];
      s2 = fmaf(u[k][j], v[k][j], s2);
    }
  }
  s1 = group_sum<G>(s1, slots[0][group]) / b.a.d, s2 = group_sum<G>(s2, slots[1][group]) / b.a.d;
  if (GROUPS > 1 && mine >= R) return;
  T* dx = dX + row * b.lddx;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const RunAt<CE, G> at(k, lane, D);
#pragma unroll
    for (int j = 0; j < CE; ++j) u[k][j] = r * (u[k][j] - s1 - v[k][j] * s2);
    store_own<CE>(dx + at.col, at.skip, u[k]);
  }
  store_padding(b.a, dx, lane);
}

// long rows: the data gradient, reading its row twice
template <typename T, typename WT>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(NormBack b, const T* dY, const T* X, const WT* gamma, const float* mean, const float* rstd,
                                                             T* dX) {
  constexpr int CE = ElemTraits<T>::CE;
  __shared__ float slots[2][16];
  const int D = b.a.D;
  for (int64_t row = blockIdx.x; row < b.a.R; row += gridDim.x) {
    const T *x = X + row * b.a.ldx, *dy = dY + row * b.lddy;
    const float mu = mean[row], r = rstd[row];
    float s1 = 0.0f, s2 = 0.0f, v[CE], u[CE], g[CE];
    for (int64_t col = threadIdx.x * CE; col < D; col += 1024 * CE) {
      const int n = (int)(D - col);
      load_some<CE>(x + col, n, v);
      load_some<CE>(dy + col, n, u);
      load_weight<CE>(gamma, (int)col, n, 1.0f, g);
      float of_run1 = 0.0f, of_run2 = 0.0f;
  #pragma unroll
      for (int j = 0; j < CE; ++j) {
        const float q = j < n ? u[j] * g[j] : 0.0f;
        of_run1 += q;
        of_run2 = fmaf(q, j < n ? (v[j] - mu) * r : 0.0f, of_run2);
      }
      s1 += of_run1, s2 += of_run2;
    }
    s1 = group_sum<1024>(s1, slots[0]) / b.a.d, s2 = group_sum<1024>(s2, slots[1]) / b.a.d;
    T* dx = dX + row * b.lddx;
    for (int64_t col = threadIdx.x * CE; col < b.a.wide; col += 1024 * CE) {
      const int n = (int)(D - col);
      load_some<CE>(x + col, n, v);
      load_some<CE>(dy + col, n, u);
      load_weight<CE>(gamma, (int)col, n, 1.0f, g);
  #pragma unroll
      for (int j = 0; j < CE; ++j) u[j] = j < n ? r * (u[j] * g[j] - s1 - (v[j] - mu) * r * s2) : 0.0f;
      store_some<CE>(dx + col, (int)(b.a.wide - col), u);
    }
  }
}
// long rows: partial sums of the weight's gradient, a wavefront's columns over every gridDim.y-th row
template <typename T>
__global__ __launch_bounds__(64) void norm_bwd_cols_kernel(NormBack b, const T* dY, const T* X, const float* mean, const float* rstd, float* part) {
  constexpr int CE = ElemTraits<T>::CE;
  const int64_t col = ((int64_t)blockIdx.x * 64 + threadIdx.x) * CE;
  if (col >= b.a.D) return;
  const int n = (int)(b.a.D - col);
  float ag[CE] = {}, ab[CE] = {}, v[CE], u[CE];
  for (int64_t row = blockIdx.y; row < b.a.R; row += gridDim.y) {
    load_some<CE>(X + row * b.a.ldx + col, n, v);
    load_some<CE>(dY + row * b.lddy + col, n, u);
    const float mu = mean[row], r = rstd[row];
#pragma unroll
    for (int j = 0; j < CE; ++j) ag[j] = fmaf(u[j], (v[j] - mu) * r, ag[j]), ab[j] += u[j];
  }
  float* out = part + (int64_t)blockIdx.y * 2 * b.a.D + col;
  store_some<CE>(out, n, ag);
  store_some<CE>(out + b.a.D, n, ab);
}

// dgamma (columns 0..D-1 of the partial sums) and dbeta (the others): 16 columns a workgroup, the P rows dealt to 64 lanes of
// it each; the sums of a wavefront's four lanes of a column, then those of the 16 wavefronts, are added in order.  Few columns
// a workgroup make many workgroups with a few loads in flight a lane.
template <typename WT>
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(int D, int P, const float* part, WT* dgamma, WT* dbeta) {
  __shared__ float sums[16][16];
  const int c = threadIdx.x & 15, at = threadIdx.x >> 4;
  const int64_t cols = 2 * (int64_t)D, col = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 16 + c;
  float s = 0.0f;
  if (col < cols) {
#pragma unroll 4
    for (int p = at; p < P; p += 64) s += part[p * cols + col];
  }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if ((threadIdx.x & 63) < 16) sums[threadIdx.x >> 6][c] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || col >= cols) return;
  float parts[16];
#pragma unroll
  for (int w = 0; w < 16; ++w) parts[w] = sums[w][c];
  s = parts[0];
#pragma unroll
  for (int w = 1; w < 16; ++w) s += parts[w];
  if (col < D) {
    if (dgamma) dgamma[col] = ElemTraits<WT>::from_f32(s);
  } else if (dbeta) {
    dbeta[col - D] = ElemTraits<WT>::from_f32(s);
  }
}

// How a row is dealt: `threads`, each with `runs` runs of 16 bytes (a row too short for one: of single elements).  No threads: rows
// too long for registers.
struct NormShape {
  int threads, runs;
};
// 16 elements a thread.  bf16, whose lanes hold fewer bytes, also 24 in place of twice the threads (forward + backward, 2^25 elements in rows of
// 1100: 29.5 + 45.5 us, 36.6 + 61.4 as 16 of 128 threads; 2100: 31 + 47, 37 + 64; 9000: 28 + 49, 38 + 64; at the other end of the range,
// 1400 and 6000, 28 + 44, 28 + 42 and 29 + 47, 28 + 45), if that leaves two rows a group to the backward pass's 256 workgroups
// (8000 x 600 6.1 + 12.7, 6.6 + 11.9; 2000 x 300 4.7 + 10.7, 4.7 + 8.8) or the alternative is 1024 threads (300 x 9000 6.0 + 8.1, 7.1 + 12.2), and 8 of the shortest rows (466033 x 72: 39 + 49, 54 + 73; 2500 x 100 5.2 + 8.5, 4.7 + 8.9).
// fp32 lost nothing there (1100 and 2100: 5.0 TB/s and more).
template <typename T> static NormShape norm_shape(int R, int D) {
  constexpr int CE = ElemTraits<T>::CE;
  const int runs = (D + CE - 1) / CE;
  if (runs <= 8 || D < CE) return {8, 1};
  if (runs <= 16) return {16, 1};
  if (CE == 4 && runs <= 32) return {16, 2};
  for (int g = 16; g <= 1024; g *= 2) {
    if (runs <= g * 16 / CE) return {g, 16 / CE};
    if (CE == 8 && g < 1024 && runs <= g * 3 && (g == 512 || (int64_t)R * g >= 1 << 18)) return {g, 3};
  }
  return {0, 0};
}
// workgroups of the backward pass, each with a row of partial sums
template <typename T> static int norm_parts(int R, int D) {
  const NormShape s = norm_shape<T>(R, D);
  const int rows = s.threads ? norm_bwd_threads(s.threads, s.runs * ElemTraits<T>::CE) / s.threads : 1;  // rows a workgroup takes at a time
  return imin(R / rows + (R % rows != 0), s.threads ? 256 : 64);
}

// Few rows take one launch: up to 512, bf16 or fp32, 100 to 8192 elements, it was faster throughout (512 x 1000 bf16 5.6 us against
// 6.8, 512 x 8192 10.0 against 16.0); at 1024 rows of 1000 it was not (10.4 against 7.5).
static bool norm_few(int R, int D) { return R <= 512 && D <= 16384; }

// (one answer for all types, whose partial rows are not equally many)
static size_t norm_ws_bytes(int R, int D) {
  return norm_few(R, D) ? 0 : (size_t)std::max(norm_parts<float>(R, D), norm_parts<uint16_t>(R, D)) * 2 * D * sizeof(float);
}

// Calls with<threads of a row, elements of a run, runs>.
template <typename T, class F> static void norm_instance(int R, int D, F&& with) {
  constexpr int CE = ElemTraits<T>::CE;
  using std::integral_constant;
  if (D < CE) return with(integral_constant<int, 8>(), integral_constant<int, 1>(), integral_constant<int, 1>());
  const NormShape s = norm_shape<T>(R, D);
#define ARD_NORM_SHAPE(G, NV) \
  if (s.threads == G && s.runs == NV) return with(integral_constant<int, G>(), integral_constant<int, CE>(), integral_constant<int, NV>());
#define ARD_NORM_SHAPES(NV) ARD_NORM_SHAPE(16, NV) ARD_NORM_SHAPE(32, NV) ARD_NORM_SHAPE(64, NV) ARD_NORM_SHAPE(128, NV) ARD_NORM_SHAPE(256, NV) ARD_NORM_SHAPE(512, NV)
  ARD_NORM_SHAPE(8, 1)
  ARD_NORM_SHAPE(16, 1)
  ARD_NORM_SHAPES(16 / CE)
  ARD_NORM_SHAPE(1024, 16 / CE)
  if constexpr (CE == 8) {
    ARD_NORM_SHAPES(3)
  } else {
    ARD_NORM_SHAPE(16, 2)
  }
#undef ARD_NORM_SHAPES
#undef ARD_NORM_SHAPE
}

// (the rows beyond a grid of this size are taken in turns: HIP counts a grid's threads in 32 bits)
static unsigned norm_grid(int R) { return (unsigned)imin(R, 1 << 20); }
// workgroups of the forward pass: 16 wavefronts a CU, which then go through their rows
static unsigned norm_fwd_grid(int R, int G, int N) {
  const int rows = norm_fwd_threads(G) / G;
  return (unsigned)imin(R / rows + (R % rows != 0), (N <= 8 ? 2048 : 1024) * 256 / norm_fwd_threads(G));
}

static int32_t norm_check(int32_t dtype, int32_t wdtype, int32_t R, int32_t D, int32_t flags, std::initializer_list<int64_t> lds, std::initializer_list<int64_t> out_lds) {
  if (dtype != ARD_F32 && dtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", dtype);
  if (wdtype != ARD_F32 && wdtype != dtype) return fail(ARD_EDTYPE, "weights are fp32 or of the activations' dtype (got %d)", wdtype);
  if (R <= 0 || D <= 0) return fail(ARD_ESHAPE, "R and D must be positive (got %d, %d)", R, D);
  if (D > 1 << 30) return fail(ARD_ESHAPE, "D = %d is too large", D);
  if (flags & ~ARD_OUT_COMPACT) return fail(ARD_EINVAL, "unknown flags 0x%x", flags);
  const int wide = flags & ARD_OUT_COMPACT ? pad8(D) : D;
  for (int64_t ld : lds)
    if (ld < D) return fail(ARD_ESHAPE, "leading dimension %lld of rows of %d elements", (long long)ld, D);
  for (int64_t ld : out_lds)
    if (ld < wide) return fail(ARD_ESHAPE, "leading dimension %lld of rows of %d stored elements", (long long)ld, wide);
  return ARD_OK;
}

template <typename T, typename WT>
static int32_t norm_fwd_t(const NormRows& a, const void* X, const void* gamma, const void* beta, void* Y, float* mean, float* rstd, hipStream_t st) {
  const T* x = (const T*)X;
  const WT *g = (const WT*)gamma, *b = (const WT*)beta;
  T* y = (T*)Y;
  if (norm_shape<T>(a.R, a.D).threads)
    norm_instance<T>(a.R, a.D, [&](auto G, auto CE, auto NV) {
      ARD_LAUNCH((norm_fwd_kernel<T, WT, G.value, CE.value, NV.value>), dim3(norm_fwd_grid(a.R, G.value, NV.value * CE.value)),
                 dim3(norm_fwd_threads(G.value)), 0, st, a, x, g, b, y, mean, rstd);
    });
  else
    ARD_LAUNCH((norm_fwd_long_kernel<T, WT>), dim3(norm_grid(a.R)), dim3(1024), 0, st, a, x, g, b, y, mean, rstd);
  ARD_LAUNCH_CHECK("norm_fwd_kernel");
  return ARD_OK;
}

// in_place: dX lies where dY or X does.  A row's threads have read it before they store it, so only the sums over rows, where they
// are made from the inputs once more, have to be made before dX is stored: a launch of their own then.
template <typename T, typename WT>
static int32_t norm_bwd_t(const NormBack& b, const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd, void* dX,
                          void* dgamma, void* dbeta, float* part, bool in_place, hipStream_t st) {
  const T *dy = (const T*)dY, *x = (const T*)X;
  const WT* g = (const WT*)gamma;
  T* dx = (T*)dX;
  const int P = norm_parts<T>(b.a.R, b.a.D), D = b.a.D;
  if (norm_few(b.a.R, D)) {
    norm_instance<T>(b.a.R, D, [&](auto G, auto CE, auto NV) {
      constexpr int rows = norm_few_threads(G.value) / G.value;
      const int row_blocks = ceil_div(b.a.R, rows), col_blocks = dgamma || dbeta ? ceil_div(D, 16 * CE.value) : 0;
      auto launch = [&](int of_rows, int of_cols) {
        ARD_LAUNCH((norm_bwd_few_kernel<T, WT, G.value, CE.value, NV.value>), dim3(of_rows + of_cols), dim3(norm_few_threads(G.value)), 0, st, b, dy, x, g,
                   mean, rstd, dx, (WT*)dgamma, (WT*)dbeta, of_rows);
      };
      if (in_place && col_blocks) launch(0, col_blocks), launch(row_blocks, 0);
      else launch(row_blocks, col_blocks);
    });
    ARD_LAUNCH_CHECK("norm_bwd_few_kernel");
    return ARD_OK;
  }
  if (norm_shape<T>(b.a.R, D).threads) {
    norm_instance<T>(b.a.R, D, [&](auto G, auto CE, auto NV) {
      ARD_LAUNCH((norm_bwd_kernel<T, WT, G.value, CE.value, NV.value>), dim3(P), dim3(norm_bwd_threads(G.value, NV.value * CE.value)), 0, st, b, dy, x, g, mean, rstd, dx, part);
    });
  } else {
    auto sums = [&] { ARD_LAUNCH((norm_bwd_cols_kernel<T>), dim3(ceil_div(D, 64 * ElemTraits<T>::CE), P), dim3(64), 0, st, b, dy, x, mean, rstd, part); };
    if (part && in_place) sums();
    ARD_LAUNCH((norm_bwd_long_kernel<T, WT>), dim3(norm_grid(b.a.R)), dim3(1024), 0, st, b, dy, x, g, mean, rstd, dx);
    ARD_LAUNCH_CHECK("norm_bwd_long_kernel");
    if (part && !in_place) sums();
  }
  ARD_LAUNCH_CHECK("norm_bwd_kernel");
  if (!part) return ARD_OK;
  const int blocks = (int)((2 * (int64_t)D + 15) / 16), planes = ceil_div(blocks, 1 << 20);  // (HIP counts a grid's threads along an axis in 32 bits)
  ARD_LAUNCH_NAMED(launch_instance("norm_weight_grad_kernel", ceil_div(blocks, planes), planes, 1024), (norm_weight_grad_kernel<WT>),
                   dim3(ceil_div(blocks, planes), planes), dim3(1024), 0, st, D, P, part, (WT*)dgamma, (WT*)dbeta);
  ARD_LAUNCH_CHECK("norm_weight_grad_kernel");
  return ARD_OK;
}

}  // namespace ard

using namespace ard;

extern "C" size_t ard_layer_norm_workspace_bytes(int32_t R, int32_t D) {
  if (R <= 0 || D <= 0 || D > 1 << 30) return 0;
  return norm_ws_bytes(R, D);
}

extern "C" int32_t ard_layer_norm_fwd(int32_t dtype, int32_t wdtype, int32_t R, int32_t D, const void* X, int64_t ldx, const void* gamma,
                                      const void* beta, float eps, void* Y, int64_t ldy, float* mean, float* rstd, int32_t flags, void* stream) {
  if (int32_t st = norm_check(dtype, wdtype, R, D, flags, {ldx}, {ldy})) return st;
  if (!X || !Y || !mean || !rstd) return fail(ARD_EINVAL, "null tensor pointer");
  if (!(eps > 0.0f) || !(eps <= 3.0e38f)) return fail(ARD_EINVAL, "eps must be positive and finite (got %g)", (double)eps);
  const size_t es = dtype == ARD_F32 ? 4 : 2, ws = wdtype == ARD_F32 ? 4 : 2;
  if (misaligned(X, es) || misaligned(Y, es) || misaligned(gamma, ws) || misaligned(beta, ws) || misaligned(mean, 4) || misaligned(rstd, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  if (R > 1 && X == Y && ldx != ldy) return fail(ARD_EINVAL, "Y in the place of X has its leading dimension");
  const NormRows a{R, D, flags & ARD_OUT_COMPACT ? pad8(D) : D, ldx, ldy, eps, (float)D};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == ARD_F32) return norm_fwd_t<float, float>(a, X, gamma, beta, Y, mean, rstd, st);
  if (wdtype == ARD_F32) return norm_fwd_t<uint16_t, float>(a, X, gamma, beta, Y, mean, rstd, st);
  return norm_fwd_t<uint16_t, uint16_t>(a, X, gamma, beta, Y, mean, rstd, st);
}

extern "C" int32_t ard_layer_norm_bwd(int32_t dtype, int32_t wdtype, int32_t R, int32_t D, const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                      const void* gamma, const float* mean, const float* rstd, void* dX, int64_t lddx, void* dgamma, void* dbeta,
                                      int32_t flags, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = norm_check(dtype, wdtype, R, D, flags, {lddy, ldx}, {lddx})) return st;
  if (!dY || !X || !mean || !rstd || !dX) return fail(ARD_EINVAL, "null tensor pointer");
  const size_t es = dtype == ARD_F32 ? 4 : 2, wes = wdtype == ARD_F32 ? 4 : 2;
  if (misaligned(X, es) || misaligned(dY, es) || misaligned(dX, es) || misaligned(gamma, wes) || misaligned(dgamma, wes) || misaligned(dbeta, wes) ||
      misaligned(mean, 4) || misaligned(rstd, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const NormBack b{{R, D, flags & ARD_OUT_COMPACT ? pad8(D) : D, ldx, 0, 0.0f, (float)D}, lddy, lddx};
  const bool in_place = dX == dY || dX == X;
  if (R > 1 && ((dX == dY && lddx != lddy) || (dX == X && lddx != ldx))) return fail(ARD_EINVAL, "dX in the place of an input has its leading dimension");
  float* part = nullptr;
  if ((dgamma || dbeta) && !norm_few(R, D)) {
    const size_t need = norm_ws_bytes(R, D);
    if (!ws || ws_bytes < need || misaligned(ws, 4)) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws ? ws_bytes : 0);
    part = (float*)ws;
  }
  hipStream_t st = (hipStream_t)stream;
  if (dtype == ARD_F32) return norm_bwd_t<float, float>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, in_place, st);
  if (wdtype == ARD_F32) return norm_bwd_t<uint16_t, float>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, in_place, st);
  return norm_bwd_t<uint16_t, uint16_t>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, in_place, st);
}
