// Layer norm over the rows of a matrix, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh gamma + beta
//   q = dy gamma, dx = r (q - mean(q) - xh mean(q xh)), dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Every pass is bound by memory: a row is read once into registers, its mean and then its centred square sum (no
// difference of large sums) are taken there in fp32, and its result is rounded once, when it is stored.  A row belongs
// to G threads: a wavefront where its elements fit that one's registers, else a workgroup of 256 or 1024 threads; longer
// rows are read again from the cache.  The backward pass keeps dgamma and dbeta of a thread's columns in registers over
// all the rows that its workgroup takes, so the sums over rows cost one row of partial sums for each workgroup and a
// second, small pass that adds them in a fixed order.
#include "rows.hpp"

namespace ard {

struct NormRows {
  int R, D;        // rows; elements that take part
  int wide;        // columns stored: D, or pad8(D) with zeros behind D
  int64_t ldx, ldy;
  float eps, d;       // d = D
};

constexpr int kNormElems = 16;  // elements of a row a thread holds (a wavefront: 1024, 256 threads: 4096, 1024: 16384)

// sum over the G threads of a row; `slot`: LDS of this sum alone (one float for each wavefront)
template <int G> __device__ __forceinline__ float group_sum(float v, float* slot) {
  v = wave_sum(v);
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
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

template <typename T, typename WT, int G>
__global__ __launch_bounds__(G == 64 ? 256 : G) void norm_fwd_kernel(NormRows a, const T* X, const WT* gamma, const WT* beta, T* Y, float* mean,
                                                                     float* rstd) {
  constexpr int CE = ElemTraits<T>::CE, NV = kNormElems / CE;
  __shared__ float slots[2][G > 64 ? G / 64 : 1];
  constexpr int WAVES = G == 64 ? 4 : 1;
  const int lane = threadIdx.x % G;
  for (int64_t row = (int64_t)blockIdx.x * WAVES + (G == 64 ? threadIdx.x >> 6 : 0); row < a.R; row += (int64_t)gridDim.x * WAVES) {
    const T* x = X + row * a.ldx;
    T* y = Y + row * a.ldy;
    float v[NV][CE], s = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = (k * G + lane) * CE;
      load_some<CE>(x + col, a.D - col, v[k]);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < CE; ++j) s += v[k][j];
    const float mu = group_sum<G>(s, slots[0]) / a.d;
    float q = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int n = a.D - (k * G + lane) * CE;
#pragma unroll
      for (int j = 0; j < CE; ++j) {
        v[k][j] = j < n ? v[k][j] - mu : 0.0f;
        q = fmaf(v[k][j], v[k][j], q);
      }
    }
    const float r = 1.0f / sqrtf(group_sum<G>(q, slots[1]) / a.d + a.eps);
    if (lane == 0) mean[row] = mu, rstd[row] = r;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = (k * G + lane) * CE, n = a.D - col;
      if (col >= a.wide) continue;
      float g[CE], b[CE];
      load_weight<CE>(gamma, col, n, 1.0f, g);
      load_weight<CE>(beta, col, n, 0.0f, b);
#pragma unroll
      for (int j = 0; j < CE; ++j) g[j] = j < n ? fmaf(v[k][j] * r, g[j], b[j]) : 0.0f;
      store_some<CE>(y + col, a.wide - col, g);
    }
    // (the next row's first sum is written after every wavefront has passed this row's second barrier, hence has read the
    // first; its second sum after the next row's first barrier: the slots need no barrier of their own)
  }
}

// rows too long for the registers of a workgroup: read three times, the second and third time from the cache
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
  #pragma unroll
      for (int j = 0; j < CE; ++j) s += v[j];
    }
    const float mu = group_sum<1024>(s, slots[0]) / a.d;
    float q = 0.0f;
    for (int64_t col = threadIdx.x * CE; col < a.D; col += 1024 * CE) {
      load_some<CE>(x + col, (int)(a.D - col), v);
  #pragma unroll
      for (int j = 0; j < CE; ++j) {
        const float d = j < a.D - col ? v[j] - mu : 0.0f;
        q = fmaf(d, d, q);
      }
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

// One row of partial sums [2][D] for each workgroup: dgamma, dbeta of the rows it took.
template <typename T, typename WT, int G>
__global__ __launch_bounds__(G == 64 ? 256 : G) void norm_bwd_kernel(NormBack b, const T* dY, const T* X, const WT* gamma, const float* mean,
                                                                     const float* rstd, T* dX, float* part) {
  constexpr int CE = ElemTraits<T>::CE, NV = kNormElems / CE, WAVES = G == 64 ? 4 : 1;
  __shared__ float slots[2][2][G > 64 ? G / 64 : 1];
  __shared__ float sums[G == 64 ? 3 : 1][G == 64 ? 2 * 64 * kNormElems : 1];
  const int lane = threadIdx.x % G, D = b.a.D;
  float g[NV][CE], ag[NV][CE] = {}, ab[NV][CE] = {};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int col = (k * G + lane) * CE;
    load_weight<CE>(gamma, col, D - col, 1.0f, g[k]);
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * WAVES + (G == 64 ? threadIdx.x >> 6 : 0); row < b.a.R; row += (int64_t)gridDim.x * WAVES, turn ^= 1) {
    const T *x = X + row * b.a.ldx, *dy = dY + row * b.lddy;
    float v[NV][CE], u[NV][CE];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = (k * G + lane) * CE;
      load_some<CE>(x + col, D - col, v[k]);
      load_some<CE>(dy + col, D - col, u[k]);
    }
    const float mu = mean[row], r = rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int n = D - (k * G + lane) * CE;
#pragma unroll
      for (int j = 0; j < CE; ++j) {
        v[k][j] = j < n ? (v[k][j] - mu) * r : 0.0f;
        ag[k][j] = fmaf(u[k][j], v[k][j], ag[k][j]);
        ab[k][j] += u[k][j];
        u[k][j] = j < n ? u[k][j] * g[k][j] : 0.0f;
        s1 += u[k][j];
        s2 = fmaf(u[k][j], v[k][j], s2);
      }
    }
    if constexpr (G == 64) {
      s1 = wave_sum(s1) / b.a.d, s2 = wave_sum(s2) / b.a.d;
    } else {  // (two sums at one barrier; the next row's go to the other slots, so none is read while it is written)
      s1 = wave_sum(s1), s2 = wave_sum(s2);
      if ((threadIdx.x & 63) == 0) slots[turn][0][threadIdx.x >> 6] = s1, slots[turn][1][threadIdx.x >> 6] = s2;
      __syncthreads();
      s1 = slots[turn][0][0], s2 = slots[turn][1][0];
#pragma unroll
      for (int w = 1; w < G / 64; ++w) s1 += slots[turn][0][w], s2 += slots[turn][1][w];
      s1 /= b.a.d, s2 /= b.a.d;
    }
    T* dx = dX + row * b.lddx;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = (k * G + lane) * CE, n = D - col;
      if (col >= b.a.wide) continue;
#pragma unroll
      for (int j = 0; j < CE; ++j) u[k][j] = j < n ? r * (u[k][j] - s1 - v[k][j] * s2) : 0.0f;
      store_some<CE>(dx + col, b.a.wide - col, u[k]);
    }
  }
  if (!part) return;
  float* out = part + (int64_t)blockIdx.x * 2 * D;
  if constexpr (G == 64) {  // the four wavefronts' sums, added in order
    const int w = threadIdx.x >> 6;
    if (w) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < CE; ++j) sums[w - 1][(k * CE + j) * 64 + lane] = ag[k][j], sums[w - 1][(kNormElems + k * CE + j) * 64 + lane] = ab[k][j];
    }
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int o = 0; o < 3; ++o)
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < CE; ++j) ag[k][j] += sums[o][(k * CE + j) * 64 + lane], ab[k][j] += sums[o][(kNormElems + k * CE + j) * 64 + lane];
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int col = (k * G + lane) * CE;
    if (col >= D) continue;
    store_some<CE>(out + col, D - col, ag[k]);
    store_some<CE>(out + D + col, D - col, ab[k]);
  }
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
  #pragma unroll
      for (int j = 0; j < CE; ++j) {
        const float q = j < n ? u[j] * g[j] : 0.0f;
        s1 += q;
        s2 = fmaf(q, j < n ? (v[j] - mu) * r : 0.0f, s2);
      }
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

// dgamma (columns 0..D-1 of the partial sums) and dbeta (the others): 64 columns a workgroup, P rows dealt to its 16
// wavefronts, their sums added in order
template <typename WT>
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(int D, int P, const float* part, WT* dgamma, WT* dbeta) {
  __shared__ float sums[16][64];
  const int64_t col = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63), cols = 2 * (int64_t)D;
  float s = 0.0f;
  if (col < cols)
    for (int p = threadIdx.x >> 6; p < P; p += 16) s += part[p * cols + col];
  sums[threadIdx.x >> 6][threadIdx.x & 63] = s;
  __syncthreads();
  if (threadIdx.x >= 64 || col >= cols) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) s += sums[w][threadIdx.x];
  if (col < D) {
    if (dgamma) dgamma[col] = ElemTraits<WT>::from_f32(s);
  } else if (dbeta) {
    dbeta[col - D] = ElemTraits<WT>::from_f32(s);
  }
}

// threads a row belongs to; 0: rows too long for registers
static int norm_group(int wide) { return wide <= 64 * kNormElems ? 64 : wide <= 256 * kNormElems ? 256 : wide <= 1024 * kNormElems ? 1024 : 0; }
// workgroups of the backward pass, each with a row of partial sums
static int norm_parts(int R, int wide) {
  const int g = norm_group(wide);
  return g == 64 ? imin(R / 4 + (R % 4 != 0), 512) : g == 256 ? imin(R, 512) : g == 1024 ? imin(R, 256) : imin(R, 64);
}

// (the rows beyond a grid of this size are taken in turns: HIP counts a grid's threads in 32 bits)
static unsigned norm_grid(int R) { return (unsigned)imin(R, 1 << 20); }

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
  switch (norm_group(a.wide)) {
    case 64: ARD_LAUNCH((norm_fwd_kernel<T, WT, 64>), dim3(norm_grid(a.R / 4 + (a.R % 4 != 0))), dim3(256), 0, st, a, x, g, b, y, mean, rstd); break;
    case 256: ARD_LAUNCH((norm_fwd_kernel<T, WT, 256>), dim3(norm_grid(a.R)), dim3(256), 0, st, a, x, g, b, y, mean, rstd); break;
    case 1024: ARD_LAUNCH((norm_fwd_kernel<T, WT, 1024>), dim3(norm_grid(a.R)), dim3(1024), 0, st, a, x, g, b, y, mean, rstd); break;
    default: ARD_LAUNCH((norm_fwd_long_kernel<T, WT>), dim3(norm_grid(a.R)), dim3(1024), 0, st, a, x, g, b, y, mean, rstd);
  }
  ARD_LAUNCH_CHECK("norm_fwd_kernel");
  return ARD_OK;
}

template <typename T, typename WT>
static int32_t norm_bwd_t(const NormBack& b, const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd, void* dX,
                          void* dgamma, void* dbeta, float* part, hipStream_t st) {
  const T *dy = (const T*)dY, *x = (const T*)X;
  const WT* g = (const WT*)gamma;
  T* dx = (T*)dX;
  const int P = norm_parts(b.a.R, b.a.wide), D = b.a.D;
  switch (norm_group(b.a.wide)) {
    case 64: ARD_LAUNCH((norm_bwd_kernel<T, WT, 64>), dim3(P), dim3(256), 0, st, b, dy, x, g, mean, rstd, dx, part); break;
    case 256: ARD_LAUNCH((norm_bwd_kernel<T, WT, 256>), dim3(P), dim3(256), 0, st, b, dy, x, g, mean, rstd, dx, part); break;
    case 1024: ARD_LAUNCH((norm_bwd_kernel<T, WT, 1024>), dim3(P), dim3(1024), 0, st, b, dy, x, g, mean, rstd, dx, part); break;
    default:
      ARD_LAUNCH((norm_bwd_long_kernel<T, WT>), dim3(norm_grid(b.a.R)), dim3(1024), 0, st, b, dy, x, g, mean, rstd, dx);
      ARD_LAUNCH_CHECK("norm_bwd_long_kernel");
      if (part) ARD_LAUNCH((norm_bwd_cols_kernel<T>), dim3(ceil_div(D, 64 * ElemTraits<T>::CE), P), dim3(64), 0, st, b, dy, x, mean, rstd, part);
  }
  ARD_LAUNCH_CHECK("norm_bwd_kernel");
  if (!part) return ARD_OK;
  ARD_LAUNCH((norm_weight_grad_kernel<WT>), dim3((unsigned)((2 * (int64_t)D + 63) / 64)), dim3(1024), 0, st, D, P, part, (WT*)dgamma, (WT*)dbeta);
  ARD_LAUNCH_CHECK("norm_weight_grad_kernel");
  return ARD_OK;
}

}  // namespace ard

using namespace ard;

extern "C" size_t ard_layer_norm_workspace_bytes(int32_t R, int32_t D) {
  if (R <= 0 || D <= 0 || D > 1 << 30) return 0;
  // (a row may be stored in D or in pad8(D) columns: whichever needs more partial sums)
  return (size_t)imax(norm_parts(R, D), norm_parts(R, pad8(D))) * 2 * D * sizeof(float);
}

extern "C" int32_t ard_layer_norm_fwd(int32_t dtype, int32_t wdtype, int32_t R, int32_t D, const void* X, int64_t ldx, const void* gamma,
                                      const void* beta, float eps, void* Y, int64_t ldy, float* mean, float* rstd, int32_t flags, void* stream) {
  if (int32_t st = norm_check(dtype, wdtype, R, D, flags, {ldx}, {ldy})) return st;
  if (!X || !Y || !mean || !rstd) return fail(ARD_EINVAL, "null tensor pointer");
  if (!(eps > 0.0f) || !(eps <= 3.0e38f)) return fail(ARD_EINVAL, "eps must be positive and finite (got %g)", (double)eps);
  const size_t es = dtype == ARD_F32 ? 4 : 2, ws = wdtype == ARD_F32 ? 4 : 2;
  if (misaligned(X, es) || misaligned(Y, es) || misaligned(gamma, ws) || misaligned(beta, ws) || misaligned(mean, 4) || misaligned(rstd, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
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
  float* part = nullptr;
  if (dgamma || dbeta) {
    const size_t need = (size_t)norm_parts(R, b.a.wide) * 2 * D * sizeof(float);
    if (!ws || ws_bytes < need || misaligned(ws, 4)) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws ? ws_bytes : 0);
    part = (float*)ws;
  }
  hipStream_t st = (hipStream_t)stream;
  if (dtype == ARD_F32) return norm_bwd_t<float, float>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, st);
  if (wdtype == ARD_F32) return norm_bwd_t<uint16_t, float>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, st);
  return norm_bwd_t<uint16_t, uint16_t>(b, dY, X, gamma, mean, rstd, dX, dgamma, dbeta, part, st);
}
