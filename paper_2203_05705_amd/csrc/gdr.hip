// Gated delta rule: a recurrence whose state of a head is a matrix.
//   S_t = a_t S_{t-1} + w_t kh_t (v_t - a_t S_{t-1}^T kh_t)^T,  o_t = scale S_t^T qh_t
//
// Few steps (a generation step above all) go one by one.  More steps are taken in chunks of 64.  With
// G_i the sum of log(a) inside the chunk up to step i, Gamma_ij = exp(G_i - G_j), K and Q the unit keys and queries by rows, S the state before the chunk:
//   A_ij = w_i Gamma_ij K_i.K_j (j < i),  P_ij = scale Gamma_ij Q_i.K_j (j <= i),  M = (I + A)^-1
//   X_i = w_i (v_i - exp(G_i) S^T K_i),  U = M X                  (the rows that the steps write beside their keys)
//   o_i = scale exp(G_i) S^T Q_i + sum_j P_ij U_j,   S' = exp(G_last) S + sum_j exp(G_last - G_j) K_j U_j^T
// All factors are at most 1 and every G_i - G_j comes from fp64 sums, so no decay loses digits, however fast.
//
// A first launch, over all chunks at once, makes what does not depend on the states: A, P, M (blocks of 16 by substitution, the rest by
// fp32 matrix instructions), written as operands of the second.  The second walks the chunks; a wavefront holds 16 columns of S in registers and
// needs no other's: everything a chunk does to a column is a chain of products in its own registers (gdr.hpp).
#include <algorithm>
#include <type_traits>

#include "gdr.hpp"

namespace ard {

// ---- step by step ---------------------------------------------------------------
// A wavefront holds 32 columns of a head's S: V of them (4, if rows are whole runs of 4) and a share of the rows a lane, which has these rows' keys and queries too; sums
// over rows go round the lanes.  Reading and writing the states bounds a generation step: 128-byte pieces of rows, 64 registers a lane for them, so that
// four wavefronts a SIMD have theirs on the way.  Measured, bf16, 128 sequences x 8 heads of 128 x 128: 26.1 us, 5.1 TB/s, what a copy reaches (a column a lane, 4-byte
// accesses: 53.7).
template <typename T, int DK, int V>
__global__ __launch_bounds__(256) void gdr_steps_kernel(GdrArgs a, const float* S0, ard_steps o, float* ST, float* ckpt, int slices) {
  constexpr int ACROSS = 32 / V, R = DK * ACROSS / 64;  // lanes of a row; rows of a lane
  const int index = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), unit = index / slices;
  if (unit >= a.B * a.H) return;
  const int lane = threadIdx.x & 63, col = (index - unit * slices) * 32 + lane % ACROSS * V, row = lane / ACROSS * R;
  const int n = unit / a.H, h = unit - n * a.H, hk = h / a.group;
  const int64_t matrix = (int64_t)a.Dk * a.Dv, plane = (int64_t)a.B * a.H * matrix;
  const uint32_t at = col < a.Dv ? (uint32_t)(row * a.Dv + col) * 4u : 0x80000000u, step = a.Dv * 4u;
  const auto states = [&](const float* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p + unit * matrix), 0, (int)matrix * 4, 0x00020000); };
  float S[R][V];
  const auto store = [&](float* p) {
    const auto buffer = states(p);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if constexpr (V == 4) __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(S[i][0]), __float_as_uint(S[i][1]), __float_as_uint(S[i][2]), __float_as_uint(S[i][3])}, buffer, at + i * step, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[i][0]), buffer, at + i * step, 0, 0);
    }
  };
  const auto over_rows = [&](float x) {
#pragma unroll
    for (int d = ACROSS; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
  };
  float k[R], q[R], v[V], f, b;
  const auto inputs = [&](int t) {
    const T *kp = (const T*)a.k.p + t * a.k.t + n * a.k.b + hk * a.Dk + row, *qp = (const T*)a.q.p + t * a.q.t + n * a.q.b + hk * a.Dk + row;
#pragma unroll
    for (int i = 0; i < R; i += 8) load_some<8>(kp + i, a.Dk - row - i, reinterpret_cast<float(&)[8]>(k[i])), load_some<8>(qp + i, a.Dk - row - i, reinterpret_cast<float(&)[8]>(q[i]));
    load_some<V>((const T*)a.v.p + t * a.v.t + n * a.v.b + h * a.Dv + col, a.Dv - col, v);
    f = ElemTraits<T>::to_f32(((const T*)a.f.p)[t * a.f.t + n * a.f.b + h]), b = ElemTraits<T>::to_f32(((const T*)a.b.p)[t * a.b.t + n * a.b.b + h]);
  };
  const int live = live_steps(a, n);
  if (S0) {
    const auto buffer = states(S0);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if constexpr (V == 4) {
        const f32x4 x = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, at + i * step, 0, 0));
        S[i][0] = x[0], S[i][1] = x[1], S[i][2] = x[2], S[i][3] = x[3];
      } else {
        S[i][0] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer, at + i * step, 0, 0));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) S[i][e] = 0.0f;
  }
  for (int t = 0; t < a.T; ++t) {
    if (ckpt && t % kChunk == 0) store(ckpt + (t / kChunk) * plane);
    T* out = (T*)o.p + t * o.t + n * o.b + h * a.Dv + col;
    float y[V] = {};
    if (t < live) {
      inputs(t);
      float ks = 0.0f, qs = 0.0f, e[V] = {};
#pragma unroll
      for (int i = 0; i < R; ++i) ks = fmaf(k[i], k[i], ks), qs = fmaf(q[i], q[i], qs);
      const float al = logistic(f), w = logistic(b), rk = 1.0f / sqrtf(over_rows(ks) + a.eps), rq = a.scale / sqrtf(over_rows(qs) + a.eps);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        k[i] *= rk, q[i] *= rq;
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = fmaf(k[i], S[i][j], e[j]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) e[j] = w * (v[j] - al * over_rows(e[j]));
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          S[i][j] = fmaf(k[i], e[j], al * S[i][j]);
          y[j] = fmaf(q[i], S[i][j], y[j]);
        }
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = over_rows(y[j]);
    }
    if (row == 0 && col < a.Dv) store_some<V>(out, a.Dv - col, y);
  }
  if (ST) store(ST);
}

// ---- what does not depend on the states -------------------------------------------
template <typename T, int DK> struct PrepShared {
  union {
    struct {
      T k[kChunk][DK + 16 / sizeof(T)], q[kChunk][DK + 16 / sizeof(T)];  // as they are stored
    };
    struct {
      float A[kChunk][kChunk + 4], M[kChunk][kChunk + 4], P[kChunk][kChunk + 4];
    };
  };
  double G[kChunk];
  float w[kChunk], rk[kChunk], rq[kChunk];
};

// 8 values of row `row` of a matrix in LDS, columns kb * 32 + {4 g + 0..3, 16 + 4 g + 0..3}
template <int N, int LD> __device__ __forceinline__ Parts<N> row_parts(const float (*m)[LD], int row, int kb, int g) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(&m[row][kb * 32 + 4 * g]), hi = *reinterpret_cast<const f32x4*>(&m[row][kb * 32 + 16 + 4 * g]);
  return parts_of<N>(lo, hi);
}
template <int N, int LD> __device__ __forceinline__ Parts<N> row_parts(const uint16_t (*m)[LD], int row, int kb, int g) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  static_assert(N == 1, "");
  const u32x2 lo = *reinterpret_cast<const u32x2*>(&m[row][kb * 32 + 4 * g]), hi = *reinterpret_cast<const u32x2*>(&m[row][kb * 32 + 16 + 4 * g]);
  return Parts<1>{{u32x4{lo[0], lo[1], hi[0], hi[1]}}};
}
// the same of the transpose: of column `col`, rows in that order
template <int N, int LD> __device__ __forceinline__ Parts<N> col_parts(const float (*m)[LD], int col, int kb, int g) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = m[kb * 32 + 4 * g + (j & 3) + 16 * (j >> 2)][col];
  return parts_of<N>(x);
}
template <int N, int LD> __device__ __forceinline__ Parts<N> col_parts(const uint16_t (*m)[LD], int col, int kb, int g) {
  static_assert(N == 1, "");
  Parts<1> s;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = kb * 32 + 4 * g + (2 * j & 3) + 16 * (j >> 1);
    s.p[0][j] = m[row][col] | (uint32_t)m[row + 1][col] << 16;
  }
  return s;
}

// A workgroup of four wavefronts makes the operands of a chunk and a key head, then of its heads, or a share of them, in turn; wavefront w has rows 16 w .. 16 w + 15.  Phases of few
// instructions with barriers between them bound it, more than its stores do (2.5 TB/s), so three workgroups share a compute unit, which takes keys and
// queries as stored (not as fp32) in LDS; the gates' sums are made where their wavefront has least else to do.  Measured, bf16, forward / backward: 4096 x 4 x 16 heads of
// 64 x 64 74 / 84 us, 16384 x 1 x 8 of 128 x 128 61; two workgroups, diagonal blocks inverted by way of LDS: 91 / 102, 77.  Without its loads, its stores, the inverses or
// the products each it would take 0.75 to 0.95 of its time: no one of them.
template <typename T, int DK, bool BWD> __global__ __launch_bounds__(256, sizeof(T) == 2 || DK == 64 ? 3 : 2) void gdr_prep_kernel(GdrArgs a, int splits) {
  constexpr int IN = kInput<T>, KB = DK / 32;
  __shared__ PrepShared<T, DK> sh;
  const int unit = blockIdx.x / splits, part = blockIdx.x - unit * splits, chunk = unit / (a.B * a.Hk), n = (unit - chunk * a.B * a.Hk) / a.Hk, hk = unit % a.Hk;
  const int t0 = chunk * kChunk, live = imin(live_steps(a, n) - t0, kChunk);
  if (live <= 0) return;  // (nobody reads this chunk's operands)
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  // sums of log(a) and write strengths of a head, by one wavefront
  const auto gates = [&](int h) {
    const int64_t t = t0 + lane;
    double G = 0.0;
    float wr = 0.0f;
    if (lane < live) {
      const float f = ElemTraits<T>::to_f32(((const T*)a.f.p)[t * a.f.t + n * a.f.b + h]);
      wr = logistic(ElemTraits<T>::to_f32(((const T*)a.b.p)[t * a.b.t + n * a.b.b + h]));
      // log(sg(f)); below -1e4 its exponential is 0 as well, and sums stay finite
      const float l = fminf(f, 0.0f) - log1pf(expf(-fabsf(f)));
      G = (double)(l < -1e4f ? -1e4f : l);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double before = __shfl_up(G, d);
      if (lane >= d) G += before;
    }
    sh.G[lane] = G, sh.w[lane] = wr;
  };
  const int first = part * a.group / splits, end = (part + 1) * a.group / splits;  // of the key head's heads
  if (w == 3) gates(hk * a.group + first);
  {
    const int row = threadIdx.x >> 2, part = threadIdx.x & 3;
    const int64_t t = t0 + row;
    const T *kp = (const T*)a.k.p + t * a.k.t + n * a.k.b + hk * a.Dk, *qp = (const T*)a.q.p + t * a.q.t + n * a.q.b + hk * a.Dk;
    float ks = 0.0f, qs = 0.0f;
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      const int at = (part + 4 * i) * 8;
      float x[8] = {}, y[8] = {};
      if (row < live) load_some<8>(kp + at, a.Dk - at, x), load_some<8>(qp + at, a.Dk - at, y);
      store_run<8>(&sh.k[row][at], x), store_run<8>(&sh.q[row][at], y);
#pragma unroll
      for (int j = 0; j < 8; ++j) ks = fmaf(x[j], x[j], ks), qs = fmaf(y[j], y[j], qs);
    }
    ks += __shfl_xor(ks, 1), qs += __shfl_xor(qs, 1);
    ks += __shfl_xor(ks, 2), qs += __shfl_xor(qs, 2);
    if (part == 0) sh.rk[row] = row < live ? 1.0f / sqrtf(ks + a.eps) : 0.0f, sh.rq[row] = row < live ? 1.0f / sqrtf(qs + a.eps) : 0.0f;
  }
  __syncthreads();
  f32x4 kk[4] = {}, qk[4] = {};
  {
    constexpr int KF = 4 * KB * IN, KTF = DK / 8 * IN;
    u32x4 *kf = a.rows + (int64_t)unit * 2 * KF * 64 + lane, *qf = kf + KF * 64;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const Parts<IN> ka = row_parts<IN>(sh.k, w * 16 + c, kb, g), qa = row_parts<IN>(sh.q, w * 16 + c, kb, g);
      if (part == 0) store_parts(kf, w * KB + kb, ka), store_parts(qf, w * KB + kb, qa);
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
        if (ct <= w) {
          const Parts<IN> b = row_parts<IN>(sh.k, ct * 16 + c, kb, g);
          mul_add(ka, b, kk[ct]);
          mul_add(qa, b, qk[ct]);
        }
    }
    u32x4 *ktf = a.cols + (int64_t)unit * (BWD ? 2 : 1) * KTF * 64 + lane, *qtf = ktf + KTF * 64;
    for (int i = w; part == 0 && i < DK / 8; i += 4) {
      store_parts(ktf, i, col_parts<IN>(sh.k, (i >> 1) * 16 + c, i & 1, g));
      if (BWD) store_parts(qtf, i, col_parts<IN>(sh.q, (i >> 1) * 16 + c, i & 1, g));
    }
  }
  for (int s = first; s < end; ++s) {
    const int h = hk * a.group + s;
    const int64_t out = ((int64_t)chunk * a.B + n) * a.H + h;
    __syncthreads();  // keys and queries, or the head before, have been read
    if (w == 3) {  // (it has the fewest blocks to multiply)
      Steps64& st = a.steps[out];
      const double G = sh.G[lane], last = sh.G[63];
      const float wr = sh.w[lane], rk = sh.rk[lane], rq = sh.rq[lane], since = expf((float)G), still = expf((float)(last - G));
      st.G[lane] = G, st.since[lane] = since, st.still[lane] = still, st.w[lane] = wr, st.rk[lane] = rk, st.rq[lane] = rq;
      st.ka[lane] = rk * since, st.qa[lane] = a.scale * rq * since, st.ke[lane] = rk * still;
      if (lane == 63) st.whole = since;
    }
    f32x4 own = {};  // of A's diagonal block
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const int j = ct * 16 + c;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = w * 16 + 4 * g + r;
        float A = 0.0f, P = 0.0f;
        if (j <= i) {
          const float fade = exp_of((float)(sh.G[i] - sh.G[j])) * sh.rk[j];
          A = j < i ? sh.w[i] * sh.rk[i] * fade * kk[ct][r] : 0.0f;
          P = a.scale * sh.rq[i] * fade * qk[ct][r];
        }
        sh.A[i][j] = A, sh.P[i][j] = P;
        if (ct == w) own[r] = A;
        else sh.M[i][j] = 0.0f;
      }
    }
    {  // the diagonal blocks' inverses, a column a lane; A's elements go from the lanes that made them to the scalar registers, without LDS
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float s0 = i == c ? 1.0f : 0.0f, s1 = 0.0f;
#pragma unroll
        for (int j = 0; j < i; ++j) {
          const float m = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own[i & 3]), 16 * (i >> 2) + j));
          if (j & 1) s1 = fmaf(-m, x[j], s1);
          else s0 = fmaf(-m, x[j], s0);
        }
        x[i] = s0 + s1;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (g == 0) sh.M[w * 16 + i][w * 16 + c] = x[i];
    }
#pragma unroll
    for (int d = 1; d < 4; ++d) {  // the blocks d below: M_rc = -M_rr sum_m A_rm M_mc
      __syncthreads();
      if (w + d < 4) {
        const int rb = w + d, cb = w;
        f32x4 s = {}, y = {};
#pragma unroll
        for (int m = 0; m < d; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(sh.A[rb * 16 + c][(cb + m) * 16 + 4 * e + g], sh.M[(cb + m) * 16 + 4 * e + g][cb * 16 + c], s, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_16x16x4f32(sh.M[rb * 16 + c][rb * 16 + 4 * g + e], -s[e], y, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) sh.M[rb * 16 + 4 * g + e][cb * 16 + c] = y[e];
      }
    }
    __syncthreads();
    if (w == 3 && s + 1 < end) gates(h + 1);  // (it has one operand less to store)
    u32x4 *mf = a.tri + out * (BWD ? 54 : 18 + 6 * Operands<true>::PER) * 64 + lane, *pf = mf + 18 * 64, *mtf = mf + 18 * 64, *ptf = mf + 36 * 64;
    for (int i = w; i < 6; i += 4) {
      const int rt = i < 2 ? i : 1 + i / 2, kb = i < 2 ? 0 : i & 1;  // (lower_frag's)
      store_parts(mf, i, row_parts<3>(sh.M, rt * 16 + c, kb, g));
      if (!BWD) Operands<true>::store(pf, i, *reinterpret_cast<const f32x4*>(&sh.P[rt * 16 + c][kb * 32 + 4 * g]), *reinterpret_cast<const f32x4*>(&sh.P[rt * 16 + c][kb * 32 + 16 + 4 * g]));
      if (BWD) {
        const int ut = i < 4 ? i / 2 : i - 2, ub = i < 4 ? i & 1 : 1;  // (upper_frag's)
        store_parts(mtf, i, col_parts<3>(sh.M, ut * 16 + c, ub, g));
        store_parts(ptf, i, col_parts<3>(sh.P, ut * 16 + c, ub, g));
      }
    }
  }
}

// ---- a wavefront's columns ----------------------------------------------------------
struct Columns {
  int unit, n, h, hk, first;  // first: the lane's column
  int segment;
  // Workgroups of four wavefronts, each of 64 of one head's columns, in one segment: `groups` of them a head (a wavefront behind the last column has columns outside,
  // which are 0 and stay unwritten, and helps to load).  Those of one segment that read the same keys take turns of 8 in the grid, which goes round
  // the 8 dies: what one has loaded, the others find in their die's cache.
  __device__ __forceinline__ Columns(const GdrArgs& a, int groups, int* taken) {
    const int team = groups * a.group, heads = a.B * a.Hk, teams = gridDim.x / team, turned = teams & ~7, id = blockIdx.x;
    const int beyond = id - turned * team, turn = id >> 3;
    const int which = beyond < 0 ? turn / team * 8 + (id & 7) : turned + beyond / team, member = beyond < 0 ? turn % team : beyond % team;
    segment = which / heads;
    const int head = which - segment * heads, part = member / groups;
    *taken = member - part * groups;
    n = head / a.Hk, hk = head - n * a.Hk, h = hk * a.group + part, unit = n * a.H + h;
  }
  __device__ __forceinline__ void take(int group) { first = group * 64 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 16 + (threadIdx.x & 15); }
  // wavefronts counted through the heads
  __device__ __forceinline__ Columns(const GdrArgs& a, int index, int slices) {
    unit = index / slices, segment = 0;
    first = (index - unit * slices) * 16 + (threadIdx.x & 15);
    n = unit / a.H, h = unit - n * a.H, hk = h / a.group;
  }
};
// Rows of a matrix (steps of a chunk, or of a state) as the lanes hold them: rows 16 rt + 4 g + r at the lane's column.  Of `rows` x `wide` elements; what
// lies outside is 0 / is not written.  NEAR: as a buffer whose end the hardware checks, so that no access needs a branch or a 64-bit address (rows that do not
// overlap, all within 2 GB).
template <typename T, bool NEAR> struct Window {
  T* p;
  int64_t step;
  int rows;
  bool on;
  uint32_t at[4], tile;  // bytes: of the lane's element in the first four rows, and from a tile of rows to the next
  __amdgpu_buffer_rsrc_t buffer;
  __device__ __forceinline__ Window(const void* base, int64_t step_, int rows_, int wide, int first) : step(step_), rows(rows_) {
    const int g = (threadIdx.x & 63) >> 4;
    on = first < wide;
    if constexpr (NEAR) {
      const uint32_t row = (uint32_t)step * sizeof(T);
      tile = 16 * row;
      at[0] = on ? 4 * g * row + first * (uint32_t)sizeof(T) : 0x80000000u;
      at[1] = at[0] + row, at[2] = at[1] + row, at[3] = at[2] + row;
      buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, rows > 0 ? rows * (int)row : 0, 0x00020000);
    } else {
      p = (T*)const_cast<void*>(base) + 4 * g * step + first;
      rows -= 4 * g;
    }
  }
  // as it is stored (T's bits): what is made of it has to wait for it
  __device__ __forceinline__ uint32_t load(int rt, int r) const {
    const int i = rt * 16 + r;
    if constexpr (!NEAR) return on && i < rows ? __builtin_bit_cast(std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>, p[i * step]) : 0u;
    else if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(buffer, at[r] + rt * tile, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(buffer, at[r] + rt * tile, 0, 0);
  }
  __device__ __forceinline__ static float value(uint32_t bits) { return __uint_as_float(sizeof(T) == 2 ? bits << 16 : bits); }
  __device__ __forceinline__ void store(int rt, int r, float x) const {
    const int i = rt * 16 + r;
    if constexpr (!NEAR) {
      if (on && i < rows) p[i * step] = ElemTraits<T>::from_f32(x);
    } else if constexpr (sizeof(T) == 2) {
      __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bf16_pair(x, 0.0f), buffer, at[r] + rt * tile, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), buffer, at[r] + rt * tile, 0, 0);
    }
  }
};
template <int TILES, typename W> __device__ __forceinline__ void load_tiles(const W& w, f32x4 (&S)[TILES]) {
#pragma unroll
  for (int rt = 0; rt < TILES; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[rt][r] = W::value(w.load(rt, r));
}
// a chunk's rows as they are stored, and their values
struct RawRows {
  uint32_t v[4][4];
};
template <typename W> __device__ __forceinline__ void load_raw(const W& w, RawRows& x) {
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) x.v[rt][r] = w.load(rt, r);
}
template <typename W> __device__ __forceinline__ void values_of_rows(const RawRows& x, f32x4 (&S)[4]) {
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[rt][r] = W::value(x.v[rt][r]);
}
template <int TILES, typename W> __device__ __forceinline__ void store_tiles(const W& w, const f32x4 (&S)[TILES]) {
#pragma unroll
  for (int rt = 0; rt < TILES; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) w.store(rt, r, S[rt][r]);
}
// the same of steps of which only `live` count: the others are stored as 0
template <typename W> __device__ __forceinline__ void store_live(const W& w, int live, const f32x4 (&S)[4]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) w.store(rt, r, rt * 16 + 4 * g + r < live ? S[rt][r] : 0.0f);
}
typedef Window<float, true> StateWindow;
__device__ __forceinline__ f32x4 row_weights(const float* w, int rt) { return *reinterpret_cast<const f32x4*>(w + rt * 16 + 4 * ((threadIdx.x & 63) >> 4)); }

// Weighed rows for the products with M: x = w (v - ka (K S)); k: operands of K, st: w, ka, qa, ke of the chunk
template <int IN, int DK>
__device__ __forceinline__ void unwritten(const u32x4* kf, const float* w, const float* ka, const Parts<3> (&Sp)[DK / 32], const f32x4 (&v)[4], f32x4 (&x)[4]) {
  constexpr int KB = DK / 32;
  f32x4 y[4] = {};
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    Parts<IN> k[4];
    load_parts(kf, kb, KB, k);
    mul_add(k, Sp[kb], y);
  }
#pragma unroll
  for (int rt = 0; rt < 4; ++rt) x[rt] = row_weights(w, rt) * (v[rt] - row_weights(ka, rt) * y[rt]);
}
// y += L x of a lower triangular L (64 x 64), or of its transpose
template <bool UPPER, bool FLOATS, int M> __device__ __forceinline__ void triangle(const u32x4* f, const Parts<M> (&x)[2], f32x4 (&y)[4]) {
  using L = Operands<FLOATS>;
  Parts<3> two[2], four[4];
  if (UPPER) {  // of all rows the last 32 columns, of the first two tiles of rows the first 32 as well
    L::load(f, 0, 2, two);
    mul_add(two, x[0], reinterpret_cast<f32x4(&)[2]>(y[0]));
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) four[rt] = L::load(f, upper_frag(rt, 1));
    mul_add(four, x[1], y);
  } else {
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) four[rt] = L::load(f, lower_frag(rt, 0));
    mul_add(four, x[0], y);
    L::load(f, 3, 2, two);
    mul_add(two, x[1], reinterpret_cast<f32x4(&)[2]>(y[2]));
  }
}
template <int N, int TILES> __device__ __forceinline__ void column_parts(const f32x4 (&x)[TILES], Parts<N> (&p)[TILES / 2]) {
#pragma unroll
  for (int kb = 0; kb < TILES / 2; ++kb)
  p[kb] = parts_of<N>(x[2 * kb], x[2 * kb + 1]);
}
// S += (operands of DK rows x 64 steps) x (y, weighed by rows)
template <int IN, int DK> __device__ __forceinline__ void add_outer(const u32x4* f, const float* weights, float sign, const f32x4 (&y)[4], f32x4 (&S)[DK / 16]) {
  Parts<3> p[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const f32x4 lo = sign * row_weights(weights, 2 * kb), hi = sign * row_weights(weights, 2 * kb + 1);
    p[kb] = parts_of<3>(lo * y[2 * kb], hi * y[2 * kb + 1]);
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int rt = 0; rt < DK / 16; rt += 4) {
      Parts<IN> k[4];
      load_parts(f, rt * 2 + kb, 2, k);
      mul_add(k, p[kb], reinterpret_cast<f32x4(&)[4]>(S[rt]));
    }
}

// Four wavefronts with columns of one head walk its chunks.  They share the operands in LDS, in two groups: what the first half of a
// chunk reads is loaded for the next chunk while the second half is worked on, and the other way about.  Operands that LDS does not hold
// (fp32, wide heads) are read from the caches.
// P lies there as values, which become parts where they are used: so the operands of heads of 128 take 80 KB, and two workgroups share a compute unit where nothing is kept
// (bf16, 512 x 32 x 16 heads of 128 x 128: 262 us with the operands' launch, one workgroup, or P in parts, 300).
// KEEP: the states before the chunks are stored, in ckpt.
// A chunk is a chain of products that wait for each other: 4.3 us with few workgroups on the chip, 5.2 with 128 that keep their states.  Measured, bf16: 8 x 1024 x 8 heads of
// 128 x 128 83 us; 16384 x 1 x 8 of 128 x 128 in 16 segments 75 + 41 + 80, at once 1108; 4096 x 4 x 16 of 64 x 64 in 4 segments 53 + 6 + 77, at once 221.
//
// Few heads leave most of the chip idle, and their chunks follow one another.  So a long sequence is cut into segments.  A segment is linear in the
// state before it: S' = F S + Z.  SUM walks all but the last segment at once, for Z (from a state of zeros) and F (DK more columns, from the
// unit matrix, without values); gdr_join_kernel makes the states between the segments of them, and then all segments are walked at once.
enum { DROP, KEEP, SUM };
template <int DK> __device__ __forceinline__ void unit_columns(int first, f32x4 (&S)[DK / 16]) {
  const int row = 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
  for (int rt = 0; rt < DK / 16; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[rt][r] = rt * 16 + row + r == first ? 1.0f : 0.0f;
}
template <int DK> __device__ __forceinline__ StateWindow sum_window(const GdrArgs& a, int index, const Columns& at, bool transition) {
  const int wide = a.dvp + DK;
  return StateWindow(a.sums + ((int64_t)index * a.B * a.H + at.unit) * DK * wide, wide, DK, wide, transition ? a.dvp + at.first : at.first);
}
template <int DK> __device__ __forceinline__ StateWindow start_window(const GdrArgs& a, int index, const Columns& at) {
  return StateWindow(a.starts + ((int64_t)index * a.B * a.H + at.unit) * DK * a.dvp, a.dvp, DK, a.dvp, at.first);
}
// The states before all segments but the first, one behind the other: S_{i + 1} = F_i S_i + Z_i, where Z_0 holds what S_0 gave; S_0 is copied (the last
// segment may write where it lies).  A workgroup takes 16 columns, each of its four wavefronts a quarter of the rows, for which it has the next F and Z
// on the way; the state goes round through LDS, in parts.  Segments count in the order of the walk.
template <int DK> __global__ __launch_bounds__(256) void gdr_join_kernel(GdrArgs a, const float* S0, int slices) {
  constexpr int KB = DK / 32, TILES = DK / 64;
  __shared__ u32x4 parts[2][KB * 3 * 64];
  const int lane = threadIdx.x & 63, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wide = a.dvp + DK, row = wave * (DK / 4);
  const int unit = blockIdx.x / slices, column = (blockIdx.x - unit * slices) * 16 + (lane & 15), units = a.B * a.H;
  f32x4 S[TILES] = {}, Z[TILES], F[TILES][KB][2];
  const auto starts = [&](int index) { return StateWindow(a.starts + (((int64_t)index * units + unit) * DK + row) * a.dvp, a.dvp, DK / 4, a.dvp, column); };
  const float* sums = a.sums + ((int64_t)unit * DK + row) * wide;
  const int64_t step = (int64_t)units * DK * wide;
  if (S0 && row < a.Dk) load_tiles(StateWindow(S0 + ((int64_t)unit * a.Dk + row) * a.Dv, a.Dv, a.Dk - row, a.Dv, column), S);
  store_tiles(starts(0), S);
  load_tiles(StateWindow(sums, wide, DK / 4, wide, column), S);
  store_tiles(starts(1), S);
  const auto load = [&](int index) {
    const float *z = sums + index * step, *f = z + a.dvp + (lane & 15) * wide + 4 * g;
    load_tiles(StateWindow(z, wide, DK / 4, wide, column), Z);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < KB * 2; ++i) F[t][i >> 1][i & 1] = *reinterpret_cast<const f32x4*>(f + t * 16 * wide + i * 16);
  };
  const int last = a.segments - 1;
  if (last > 1) load(1);
  for (int index = 1; index < last; ++index) {
    // rows 16 or 32 of the state are half or all of an operand of 32
    if constexpr (TILES == 2) {
      store_parts(parts[index & 1] + lane, wave, parts_of<3>(S[0], S[1]));
    } else {
      const float x[8] = {S[0][0], S[0][1], S[0][2], S[0][3]};
      const Parts<3> p = parts_of<3>(x);
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 3; ++i) reinterpret_cast<u32x2*>(&parts[index & 1][((wave >> 1) * 3 + i) * 64 + lane])[wave & 1] = u32x2{p.p[i][0], p.p[i][1]};
    }
    Parts<3> f[KB][TILES];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int t = 0; t < TILES; ++t) f[kb][t] = parts_of<3>(F[t][kb][0], F[t][kb][1]);
#pragma unroll
    for (int t = 0; t < TILES; ++t) S[t] = Z[t];
    load(imin(index + 1, last - 1));
    __syncthreads();  // (one a segment: the other half of `parts` was last read before the one before)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) mul_add(f[kb], load_parts<3>(parts[index & 1] + lane, kb), S);
    store_tiles(starts(index + 1), S);
  }
}

template <typename T, int DK, bool NEAR, int MODE>
__global__ __launch_bounds__(256, MODE == DROP && sizeof(T) == 2 ? 2 : 1) void gdr_fwd_kernel(GdrArgs a, const float* S0, ard_steps o, float* ST, float* ckpt, int groups) {
  constexpr int IN = kInput<T>, KB = DK / 32, KF = 4 * KB * IN, KTF = DK / 8 * IN, MF = 6 * 3, PF = 6 * Operands<true>::PER;
  constexpr bool KEPT = MODE == KEEP, OUTPUT = MODE != SUM;
  constexpr int RF = OUTPUT ? 2 * KF : KF, TF = OUTPUT ? MF + PF : MF;  // (the operands of Q and P are read for o alone)
  constexpr bool STAGED = walk_operands(false, MODE == SUM, DK, IN) > 0;
  static_assert(!STAGED || walk_operands(false, MODE == SUM, DK, IN) == RF + KTF + TF, "");
  __shared__ u32x4 one[STAGED ? RF * 64 : 1], two[STAGED ? (KTF + TF) * 64 : 1];  // what the halves read
  __shared__ f32x4 weights[2][64];  // w, ka, qa, ke of a chunk
  int group;
  Columns at(a, OUTPUT ? groups : groups + DK / 64, &group);  // (a sum's transition is the last columns)
  const bool transition = !OUTPUT && group >= groups;
  at.take(transition ? group - groups : group);
  const int segment = at.segment, begin = segment * a.span, end = imin(begin + a.span, a.chunks);
  if (transition && segment == 0) return;  // (all wavefronts: the first segment's state is S0's)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t matrix = (int64_t)a.Dk * a.Dv, plane = (int64_t)a.B * a.H * matrix;
  f32x4 S[DK / 16] = {}, v[4] = {};
  if (OUTPUT && a.segments > 1) load_tiles(start_window<DK>(a, segment, at), S);
  else if (transition) unit_columns<DK>(at.first, S);
  else if (S0 && segment == 0) load_tiles(StateWindow(S0 + at.unit * matrix, a.Dv, a.Dk, a.Dv, at.first), S);
  const int all = live_steps(a, at.n), chunks = imin((all + kChunk - 1) / kChunk, end), given = transition ? 0 : all;
  const auto ku = [&](int chunk) { return (int64_t)((chunk * a.B + at.n) * a.Hk + at.hk); };
  const auto hu = [&](int chunk) { return (int64_t)((chunk * a.B + at.n) * a.H + at.h); };
  const T* vp = (const T*)a.v.p + at.n * a.v.b + at.h * a.Dv;
  T* op = (T*)o.p + at.n * o.b + at.h * a.Dv + (int64_t)begin * kChunk * o.t;
  float* kept = ckpt + at.unit * matrix + begin * plane;
  RawRows next;
  f32x4 sw;  // the chunk's weights, which go to LDS by way of a register: loads straight into an array let every later read of it wait for them
  float next_whole = 0.0f;
  int zero = 0;
  asm volatile("" : "+v"(zero));  // (a vector load: one by the scalar unit would let every read of LDS wait for it)
  const auto first_half = [&](int chunk) {  // loads of what it reads
    if (STAGED) stage<RF>(a.rows + ku(chunk) * (2 * KF * 64), one, wave);
    sw = *reinterpret_cast<const f32x4*>(a.steps[hu(chunk)].w + (threadIdx.x & 63) * 4);
    load_raw(Window<T, NEAR>(vp + (int64_t)chunk * kChunk * a.v.t, a.v.t, imin(given - chunk * kChunk, kChunk), a.Dv, at.first), next);
    next_whole = (&a.steps[hu(chunk)].whole)[zero];
  };
  const auto second_half = [&](int chunk) {
    if (STAGED) stage<KTF>(a.cols + ku(chunk) * (KTF * 64), two, wave), stage<TF>(a.tri + hu(chunk) * ((MF + PF) * 64), two + KTF * 64, wave);
  };
  constexpr int COUNT = STAGED && NEAR;  // (elsewhere accesses are not counted: all are waited for)
  if (begin < chunks) {
    first_half(begin);
    staged();
    weights[begin & 1][threadIdx.x & 63] = sw;
    all_landed<0>();
    second_half(begin);
    staged();
  }
  for (int chunk = begin; chunk < chunks; ++chunk) {
    const int steps = imin(a.T - chunk * kChunk, kChunk), live = imin(all - chunk * kChunk, steps);
    const float *w = (const float*)weights[chunk & 1], *ka = w + kChunk, *qa = w + 2 * kChunk, *ke = w + 3 * kChunk;
    const int lane = threadIdx.x & 63;
    const u32x4 *rows = (STAGED ? one : a.rows + ku(chunk) * (2 * KF * 64)) + lane, *cols = (STAGED ? two : a.cols + ku(chunk) * (KTF * 64)) + lane,
                *tri = (STAGED ? two + KTF * 64 : a.tri + hu(chunk) * ((MF + PF) * 64)) + lane;
    const float whole = next_whole;
    values_of_rows<Window<T, NEAR>>(next, v);
    if (KEPT) {
      store_tiles(StateWindow(kept, a.Dv, a.Dk, a.Dv, at.first), S);
      kept += plane;
    }
    f32x4 x[4], y[4] = {}, u[4] = {};
    {
      Parts<3> Sp[KB];
      column_parts<3>(S, Sp);
      unwritten<IN, DK>(rows, w, ka, Sp, v, x);
      if constexpr (OUTPUT) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          Parts<IN> q[4];
          load_parts(rows + KF * 64, kb, KB, q);
          mul_add(q, Sp[kb], y);
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) y[rt] *= row_weights(qa, rt);
      }
    }
    all_landed<KEPT * COUNT * (DK / 4)>();
    first_half(imin(chunk + 1, chunks - 1));  // (behind the last chunk its own once more: accesses that are counted are made on every way)
    staged();
    {
      Parts<3> xp[2];
      column_parts<3>(x, xp);
      triangle<false, false>(tri, xp, u);
    }
    if constexpr (OUTPUT) {
      Parts<3> up[2];
      column_parts<3>(u, up);
      triangle<false, true>(tri + MF * 64, up, y);
    }
    weights[(chunk + 1) & 1][threadIdx.x & 63] = sw;  // (waits for all accesses: in front of the stores)
    if constexpr (OUTPUT) store_live(Window<T, NEAR>(op, o.t, steps, a.Dv, at.first), live, y);
    op += kChunk * o.t;
#pragma unroll
    for (int rt = 0; rt < DK / 16; ++rt) S[rt] *= whole;
    add_outer<IN, DK>(cols, ke, 1.0f, u, S);
    all_landed<OUTPUT * COUNT * 16>();
    second_half(imin(chunk + 1, chunks - 1));
    staged();
  }
  all_landed<0>();  // (nothing may arrive in LDS once the wavefront has ended)
  if constexpr (!OUTPUT) {
    store_tiles(sum_window<DK>(a, segment, at, transition), S);
    return;
  }
  for (int chunk = imax(chunks, begin); chunk < end; ++chunk) {  // behind the sequence's end
    const f32x4 none[4] = {};
    if (KEPT) store_tiles(StateWindow(kept, a.Dv, a.Dk, a.Dv, at.first), S);
    store_tiles(Window<T, NEAR>(op, o.t, imin(a.T - chunk * kChunk, kChunk), a.Dv, at.first), none);
    kept += plane, op += kChunk * o.t;
  }
  if (ST && end == a.chunks) store_tiles(StateWindow(ST + at.unit * matrix, a.Dv, a.Dk, a.Dv, at.first), S);
}

// ---- backward -----------------------------------------------------------------------
// With dS' the gradient of the state behind a chunk, E = dX U^T, F = dO U^T:
//   dX = M^T (P^T dO + still K dS'),  dV = w dX,  dS = exp(G_last) dS' + scale Q^T (since dO) - K^T (since w dX)
//   dA = -E (j < i),  dP = F (j <= i), and with N_ij = -E_ij w_i Gamma_ij, R_ij = F_ij scale Gamma_ij:
//   dQ_i = scale since_i S dO_i + sum_j R_ij K_j
//   dK_i = sum_j N_ij K_j - w_i since_i S dX_i + sum_j N_ji K_j + sum_j R_ji Q_j + still_i dS' U_i
//   dw_i / w_i = E_ii  (dX_i . X_i less what A's own w_i takes back; no division by a small w)
//   d log(a_t) = sum_{i >= t > j} (N_ij K_i.K_j + R_ij Q_i.K_j) + sum_{i >= t} (scale since_i Q_i.S dO_i - w_i since_i K_i.S dX_i)
//                + sum_{j < t} still_j K_j.dS' U_j + exp(G_last) <S, dS'>,
// terms that all have a_t as a factor (as differences of sums over i and over j, K.dK and Q.dQ, a step that forgets all would be left with their rounding).
// Three launches after the first: U of every chunk from the states kept; the chunks from the last to the first, which leaves dX and dS' of each; and
// all other gradients, every chunk for itself.

// U of every chunk.  Reading the states bounds it: bf16 8 x 1024 x 8 heads of 128 x 128 43 us, 2.8 TB/s.
template <typename T, int DK, bool NEAR> __global__ __launch_bounds__(256) void gdr_rows_kernel(GdrArgs a, const float* ckpt, int slices, int waves) {
  constexpr int IN = kInput<T>, KB = DK / 32;
  const int index = __builtin_amdgcn_readfirstlane(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6));
  const int chunk = index / waves;
  if (chunk >= a.chunks) return;
  const Columns at(a, index - chunk * waves, slices);
  const int t0 = chunk * kChunk, live = imin(live_steps(a, at.n) - t0, kChunk);
  if (live <= 0) return;
  const int64_t ku = ((int64_t)chunk * a.B + at.n) * a.Hk + at.hk, hu = ((int64_t)chunk * a.B + at.n) * a.H + at.h;
  f32x4 S[DK / 16], v[4], x[4], u[4] = {};
  load_tiles(StateWindow(ckpt + hu * a.Dk * a.Dv, a.Dv, a.Dk, a.Dv, at.first), S);
  load_tiles(Window<T, NEAR>((const T*)a.v.p + t0 * a.v.t + at.n * a.v.b + at.h * a.Dv, a.v.t, live, a.Dv, at.first), v);
  const Steps64& st = a.steps[hu];
  {
    Parts<3> Sp[KB];
    column_parts<3>(S, Sp);
    unwritten<IN, DK>(a.rows + ku * 2 * 4 * KB * IN * 64 + (threadIdx.x & 63), st.w, st.ka, Sp, v, x);
  }
  Parts<3> xp[2];
  column_parts<3>(x, xp);
  triangle<false, false>(a.tri + hu * 54 * 64 + (threadIdx.x & 63), xp, u);
  store_tiles(StateWindow(a.u + hu * kChunk * a.dvp, a.dvp, kChunk, a.dvp, at.first), u);
}

// SUM: as forward, of segments from the last on.  Measured, bf16: 8 x 1024 x 8 heads of 128 x 128 88 us; 4096 x 4 x 16 of 64 x 64 in 4 segments 82 + 6 + 79, at once 240.
template <typename T, int DK, bool NEAR, int MODE>
__global__ __launch_bounds__(256) void gdr_back_kernel(GdrArgs a, ard_steps d_o, const float* dST, ard_steps dv, float* dS0, int groups) {
  constexpr int IN = kInput<T>, KB = DK / 32, KF = 4 * KB * IN, KTF = DK / 8 * IN, MF = 6 * 3;
  constexpr bool STAGED = walk_operands(true, MODE == SUM, DK, IN) > 0;
  static_assert(!STAGED || walk_operands(true, MODE == SUM, DK, IN) == KF + 2 * KTF + 2 * MF, "");
  constexpr bool OUTPUT = MODE != SUM;
  __shared__ u32x4 one[STAGED ? (KF + MF) * 64 : 1], two[STAGED ? (2 * KTF + MF) * 64 : 1];
  __shared__ f32x4 weights[2][64];  // w, ka, qa, ke of a chunk
  int group;
  Columns at(a, OUTPUT ? groups : groups + DK / 64, &group);  // (a sum's transition is the last columns)
  const bool transition = !OUTPUT && group >= groups;
  at.take(transition ? group - groups : group);
  const int segment = at.segment, begin = (a.segments - 1 - segment) * a.span, end = imin(begin + a.span, a.chunks);
  if (transition && segment == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t matrix = (int64_t)a.Dk * a.Dv;
  f32x4 S[DK / 16] = {}, x[4] = {};
  if (OUTPUT && a.segments > 1) load_tiles(start_window<DK>(a, segment, at), S);
  else if (transition) unit_columns<DK>(at.first, S);
  else if (dST && segment == 0) load_tiles(StateWindow(dST + at.unit * matrix, a.Dv, a.Dk, a.Dv, at.first), S);
  const int all = live_steps(a, at.n), chunks = imin((all + kChunk - 1) / kChunk, end), given = transition ? 0 : all;
  const auto ku = [&](int chunk) { return (int64_t)((chunk * a.B + at.n) * a.Hk + at.hk); };
  const auto hu = [&](int chunk) { return (int64_t)((chunk * a.B + at.n) * a.H + at.h); };
  const T* gp = (const T*)d_o.p + at.n * d_o.b + at.h * a.Dv;
  T* vp = (T*)dv.p + at.n * dv.b + at.h * a.Dv;
  RawRows next;
  f32x4 sw;
  float next_whole = 0.0f;
  int zero = 0;
  asm volatile("" : "+v"(zero));
  const auto first_half = [&](int chunk) {
    if (STAGED) stage<KF>(a.rows + ku(chunk) * (2 * KF * 64), one, wave), stage<MF>(a.tri + hu(chunk) * (3 * MF * 64) + 2 * MF * 64, one + KF * 64, wave);
    sw = *reinterpret_cast<const f32x4*>(a.steps[hu(chunk)].w + (threadIdx.x & 63) * 4);
    load_raw(Window<T, NEAR>(gp + (int64_t)chunk * kChunk * d_o.t, d_o.t, imin(given - chunk * kChunk, kChunk), a.Dv, at.first), next);
    next_whole = (&a.steps[hu(chunk)].whole)[zero];
  };
  const auto second_half = [&](int chunk) {
    if (STAGED) stage<MF>(a.tri + hu(chunk) * (3 * MF * 64) + MF * 64, two, wave), stage<2 * KTF>(a.cols + ku(chunk) * (2 * KTF * 64), two + MF * 64, wave);
  };
  for (int chunk = OUTPUT ? imax(chunks, begin) : end; chunk < end; ++chunk) {  // behind the sequence's end
    const f32x4 none[4] = {};
    store_tiles(Window<T, NEAR>(vp + (int64_t)chunk * kChunk * dv.t, dv.t, imin(a.T - chunk * kChunk, kChunk), a.Dv, at.first), none);
  }
  constexpr int COUNT = STAGED && NEAR;
  if (begin < chunks) {
    first_half(chunks - 1);
    staged();
    weights[(chunks - 1) & 1][threadIdx.x & 63] = sw;
    all_landed<0>();
    second_half(chunks - 1);
    staged();
  }
  for (int chunk = chunks - 1; chunk >= begin; --chunk) {
    const int steps = imin(a.T - chunk * kChunk, kChunk), live = imin(all - chunk * kChunk, steps);
    const float *w = (const float*)weights[chunk & 1], *ka = w + kChunk, *qa = w + 2 * kChunk, *ke = w + 3 * kChunk;
    const int lane = threadIdx.x & 63;
    const u32x4 *kf = (STAGED ? one : a.rows + ku(chunk) * (2 * KF * 64)) + lane, *cols = (STAGED ? two + MF * 64 : a.cols + ku(chunk) * (2 * KTF * 64)) + lane,
                *ptf = (STAGED ? one + KF * 64 : a.tri + hu(chunk) * (3 * MF * 64) + 2 * MF * 64) + lane,
                *mtf = (STAGED ? two : a.tri + hu(chunk) * (3 * MF * 64) + MF * 64) + lane;
    const float whole = next_whole;
    values_of_rows<Window<T, NEAR>>(next, x);
    if constexpr (OUTPUT) store_tiles(StateWindow(a.ds + hu(chunk) * DK * a.dvp, a.dvp, DK, a.dvp, at.first), S);
    f32x4 y[4] = {}, dx[4] = {}, od[4];
    {
      Parts<3> Sp[KB];
      column_parts<3>(S, Sp);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Parts<IN> k[4];
        load_parts(kf, kb, KB, k);
        mul_add(k, Sp[kb], y);
      }
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) y[rt] *= row_weights(ke, rt);
    }
    {
      Parts<IN> p[2];
      column_parts<IN>(x, p);
      triangle<true, false>(ptf, p, y);
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) od[rt] = x[rt];
    all_landed<OUTPUT * COUNT * (DK / 4)>();
    first_half(imax(chunk - 1, begin));
    staged();
    {
      Parts<3> p[2];
      column_parts<3>(y, p);
      triangle<true, false>(mtf, p, dx);
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) y[rt] = row_weights(w, rt) * dx[rt];
    weights[(chunk + 1) & 1][threadIdx.x & 63] = sw;
    if constexpr (OUTPUT) {
      store_tiles(StateWindow(a.dx + hu(chunk) * kChunk * a.dvp, a.dvp, kChunk, a.dvp, at.first), dx);
      store_live(Window<T, NEAR>(vp + (int64_t)chunk * kChunk * dv.t, dv.t, steps, a.Dv, at.first), live, y);
    }
#pragma unroll
    for (int rt = 0; rt < DK / 16; ++rt) S[rt] *= whole;
    add_outer<IN, DK>(cols + KTF * 64, qa, 1.0f, od, S);
    add_outer<IN, DK>(cols, ka, -1.0f, y, S);
    all_landed<OUTPUT * COUNT * 32>();
    second_half(imax(chunk - 1, begin));
    staged();
  }
  all_landed<0>();
  if constexpr (!OUTPUT) {
    store_tiles(sum_window<DK>(a, segment, at, transition), S);
    return;
  }
  if (dS0 && begin == 0) store_tiles(StateWindow(dS0 + at.unit * matrix, a.Dv, a.Dk, a.Dv, at.first), S);
}

__device__ __forceinline__ float over_rows(float x) {  // the sum over the lanes that share a column
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Neighbouring elements of a lane's rows, 0 where they are outside.  QUICK: by one access whose end the hardware checks, without a branch: for rows whose runs of
// N are inside or outside as a whole, and within 2 GB.
template <typename T, int N, bool QUICK> struct Runs {
  const T* p;
  int64_t step;
  int rows, wide;
  __amdgpu_buffer_rsrc_t buffer;
  __device__ __forceinline__ Runs(const void* base, int64_t step_, int rows_, int wide_) : p((const T*)base), step(step_), rows(rows_), wide(wide_) {
    if constexpr (QUICK) buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, rows > 0 ? rows * (int)step * (int)sizeof(T) : 0, 0x00020000);
  }
  __device__ __forceinline__ void load(int row, int at, float (&x)[N]) const {
    if constexpr (QUICK) {
      const uint32_t from = at < wide ? ((uint32_t)row * (uint32_t)step + (uint32_t)at) * (uint32_t)sizeof(T) : 0x80000000u;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          const auto v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, from + j * 4, 0, 0));
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j + e] = v[e];
        }
      } else if constexpr (N == 8) {
        const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, from, 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(v[e] << 16), x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
      } else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(buffer, from, 0, 0));
#pragma unroll
        for (int e = 0; e < 2; ++e) x[2 * e] = __uint_as_float(v[e] << 16), x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
      }
    } else {
      load_some<N>(p + row * step + at, row < rows ? wide - at : 0, x);
    }
  }
  // eight as an operand's parts will be made of: bf16 is one already, and taken apart on the way its loads would be waited for
  struct Eight {
    std::conditional_t<sizeof(T) == 2, u32x4, float[8]> v;
    __device__ __forceinline__ Parts<kInput<T>> parts() const {
      if constexpr (sizeof(T) == 2) return Parts<1>{{v}};
      else return parts_of<3>(v);
    }
  };
  __device__ __forceinline__ void load(int row, int at, Eight& x) const {
    if constexpr (sizeof(T) == 4) {
      load(row, at, x.v);
    } else if constexpr (QUICK) {
      x.v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, at < wide ? ((uint32_t)row * (uint32_t)step + (uint32_t)at) * 2u : 0x80000000u, 0, 0));
    } else {
      float y[8];
      load(row, at, y);
      x.v = parts_of<1>(y).p[0];
    }
  }
};

// Four values as they were stored.  again(): they are taken apart anew from here on, not kept so.
template <typename T> struct Four;
template <> struct Four<float> {
  float v[4];
  __device__ __forceinline__ void set(const float (&x)[4]) { v[0] = x[0], v[1] = x[1], v[2] = x[2], v[3] = x[3]; }
  __device__ __forceinline__ float at(int r) const { return v[r]; }
  __device__ __forceinline__ void again() {}
};
template <> struct Four<uint16_t> {
  uint32_t v[2];
  __device__ __forceinline__ void set(const float (&x)[4]) { v[0] = bf16_pair(x[0], x[1]), v[1] = bf16_pair(x[2], x[3]); }
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(v[0]), "+v"(v[1])); }
  __device__ __forceinline__ float at(int r) const { return __uint_as_float(r & 1 ? v[r / 2] & 0xffff0000u : v[r / 2] << 16); }
};

// The gradients of queries, keys and gates of a chunk and a key head, by four wavefronts, or eight for wide keys.  Wavefront w has the steps of tile w % 4 as columns, and all
// rows of Dk or half of them.  U, dX and dO go around through LDS, each tile the right hand operand of its own wavefronts and the left hand one of the others; S and dS' follow there in
// pieces of 32 columns, a tile of rows from each wavefront, one stored while the one before it is multiplied.  Operands are read from LDS where they are used, for all of a wavefront's
// rows at once: its registers hold sums, not operands (with those of its own steps in registers too, 256 were not enough, and what was spilled took most of the time).  They are parts, made
// once; where LDS does not hold all of them so, dX, then U, then dO are values there (bf16, heads of 128 x 128: whole states and all three as values 240 us, so 184).
// What later and earlier steps give is made apart, each before its own products, so that the operands of one are gone when the other's come.
// Measured, bf16: 8 x 1024 x 8 heads of 128 x 128 184 us, 4096 x 4 x 16 of 64 x 64 with 8 key heads 219; matrix and vector instructions follow one another in
// the same phases, and one workgroup a compute unit (LDS, registers) cannot fill the waits between them.
template <typename T, int DK, int DV, bool QUICK>
__global__ __launch_bounds__(DK * 4) void gdr_grads_kernel(GdrArgs a, ard_steps d_o, const float* ckpt, ard_steps dq, ard_steps dk, ard_steps df, ard_steps db) {
  constexpr int IN = kInput<T>, VB = DV / 32, RT = DK / 16, HALVES = DK / 64, WAVES = 4 * HALVES, OWN = RT / HALVES;
  static_assert(RT == WAVES && VB % 2 == 0, "a tile of a state's rows each, and two slots in turn");
  // KB of LDS: two slots of a state's pieces; dX, U and dO as parts, or, one after the other as far as need be, as values
  constexpr int SLOT = RT * 3, TILES = 4 * VB, ROOM = 152 - 2 * SLOT;
  constexpr bool VALUES_X = TILES * (6 + IN) > ROOM, VALUES_U = TILES * (5 + IN) > ROOM, VALUES_O = IN == 3 && TILES * (4 + IN) > ROOM;
  using HeldX = Operands<VALUES_X>;
  using HeldU = Operands<VALUES_U>;
  using HeldO = Operands<VALUES_O>;
  constexpr int ROWS = TILES * (HeldU::PER + HeldX::PER + (IN == 3 ? HeldO::PER : IN));
  static_assert(ROWS <= ROOM, "");
  __shared__ u32x4 lds[(ROWS + 2 * SLOT) * 64];
  __shared__ double dG[HALVES][2][kChunk];
  __shared__ float ends[WAVES], dots[2][HALVES][kChunk];
  __shared__ float crossing[WAVES][kChunk];
  __shared__ Steps64 st;
  const int unit = blockIdx.x, chunk = unit / (a.B * a.Hk), n = (unit - chunk * a.B * a.Hk) / a.Hk, hk = unit % a.Hk;
  const int t0 = chunk * kChunk, steps = imin(a.T - t0, kChunk), live = imin(live_steps(a, n) - t0, steps);
  const int w8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = w8 & 3, half = HALVES > 1 ? w8 >> 2 : 0, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, mine = w * 16 + c;
  f32x4 sumq[OWN] = {}, sumk[OWN] = {};
  if (live > 0) {
    const Runs<T, 4, QUICK> keys((const T*)a.k.p + t0 * a.k.t + n * a.k.b + hk * a.Dk, a.k.t, live, a.Dk), queries((const T*)a.q.p + t0 * a.q.t + n * a.q.b + hk * a.Dk, a.q.t, live, a.Dk);
    Four<T> kx[OWN], qx[OWN];  // of the wavefront's own steps, where its sums lie
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int at = (half * OWN + i) * 16 + 4 * g;
      float x[4], y[4];
      keys.load(mine, at, x), queries.load(mine, at, y);
      kx[i].set(x), qx[i].set(y);
    }
    const Steps64& any = a.steps[((int64_t)chunk * a.B + n) * a.H + hk * a.group];
    const float rkm = any.rk[mine], rqm = any.rq[mine];
    // products of keys and of queries (rows) with the lane's step's key; of two halves the first has the keys', the second the queries'
    f32x4 pairs[HALVES == 1 ? 2 : 1][4] = {};
    {
      const u32x4* rows = a.rows + (int64_t)unit * (DK / 4) * IN * 64 + lane;
#pragma unroll
      for (int kb = 0; kb < DK / 32; ++kb) {
        const Parts<IN> own = load_parts<IN>(rows, w * (DK / 32) + kb);
        Parts<IN> m[4];
        load_parts(rows + half * (DK / 8) * IN * 64, kb, DK / 32, m);
        mul_add(m, own, pairs[0]);
        if (HALVES == 1) {
          load_parts(rows + (DK / 8) * IN * 64, kb, DK / 32, m);
          mul_add(m, own, pairs[HALVES == 1]);
        }
      }
    }
    for (int s = 0; s < a.group; ++s) {
      const int h = hk * a.group + s;
      const int64_t hu = ((int64_t)chunk * a.B + n) * a.H + h;
      // (what is made from these is made in the loop: taken out of it, it alone would not fit the registers)
      int at_lane = threadIdx.x & 63;
      asm volatile("" : "+v"(at_lane));
      const int lane = at_lane, g = lane >> 4, c = lane & 15;
#pragma unroll
      for (int i = 0; i < OWN; ++i) kx[i].again(), qx[i].again();
      const u32x4 *ktf = a.cols + (int64_t)unit * (DK / 4) * IN * 64 + at_lane, *qtf = ktf + DK / 8 * IN * 64;
      u32x4 *lu = lds + at_lane, *lx = lu + TILES * HeldU::PER * 64, *lo = lx + TILES * HeldX::PER * 64, *ls = lu + ROWS * 64;
      const int mine = w * 16 + c;
      const Runs<float, 8, QUICK> S(ckpt + hu * a.Dk * a.Dv, a.Dv, a.Dk, a.Dv);
      const Runs<float, 8, true> ds(a.ds + hu * DK * a.dvp, a.dvp, DK, a.dvp);
      // the gates whose slopes the end needs, as they are stored: f for the first wavefront, b for those of the first half (by all lanes and without a
      // branch, of the last step for lanes behind it: registers that are moved aside where lanes come together again have lost those lanes' values)
      T fg, bg;
      {
        // (of two halves the second takes dX)
        const Runs<float, 8, true> rows_of_mine((half ? a.dx : a.u) + hu * kChunk * a.dvp, a.dvp, kChunk, a.dvp), dx(a.dx + hu * kChunk * a.dvp, a.dvp, kChunk, a.dvp);
        const Runs<T, 8, QUICK> go((const T*)d_o.p + t0 * d_o.t + n * d_o.b + h * a.Dv, d_o.t, live, a.Dv);
        float x[VB][8], z[HALVES > 1 ? 1 : VB][8];
        typename Runs<T, 8, QUICK>::Eight y[VB];
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) rows_of_mine.load(mine, vb * 32 + 8 * g, x[vb]);
        if (HALVES == 1) {
#pragma unroll
          for (int vb = 0; vb < VB; ++vb) dx.load(mine, vb * 32 + 8 * g, z[HALVES > 1 ? 0 : vb]);
        }
        if (half == 0) {
#pragma unroll
          for (int vb = 0; vb < VB; ++vb) go.load(mine, vb * 32 + 8 * g, y[vb]);
        }
        const u32x4 weights = w8 < 3 ? ((const u32x4*)&a.steps[hu])[w8 * 64 + lane] : u32x4{};
        fg = ((const T*)a.f.p)[(int64_t)(t0 + imin(63 - lane, live - 1)) * a.f.t + n * a.f.b + h];
        bg = ((const T*)a.b.p)[(int64_t)(t0 + imin(mine, live - 1)) * a.b.t + n * a.b.b + h];
        __syncthreads();  // (the head before has been read)
        if (w8 < 3) ((u32x4*)&st)[w8 * 64 + lane] = weights;
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
          if (half) HeldX::store(lx, w * VB + vb, x[vb]);
          else HeldU::store(lu, w * VB + vb, x[vb]);
          if (HALVES == 1) HeldX::store(lx, w * VB + vb, z[HALVES > 1 ? 0 : vb]);
        }
        if (half == 0) {
#pragma unroll
          for (int vb = 0; vb < VB; ++vb) {
            if constexpr (IN == 3) HeldO::store(lo, w * VB + vb, y[vb].v);
            else store_parts<IN>(lo, w * VB + vb, y[vb].parts());
          }
        }
      }
      float Sx[VB][8], Dx[VB][8];  // S and dS' by pieces of 32 columns, a tile of rows a wavefront
#pragma unroll
      for (int vb = 0; vb < VB; ++vb) S.load(w8 * 16 + c, vb * 32 + 8 * g, Sx[vb]);
      const auto piece = [&](int vb) { return ls + (vb & 1) * SLOT * 64; };
      __syncthreads();
      const auto given = [&](int frag) {
        if constexpr (IN == 3) return HeldO::load(lo, frag);
        else return load_parts<IN>(lo, frag);
      };
      const auto of_u = [&](int vb) { return HeldU::load(lu, w * VB + vb); };
      const auto of_x = [&](int vb) { return HeldX::load(lx, w * VB + vb); };
      const auto of_o = [&](int vb) { return given(w * VB + vb); };
      const double Gm = st.G[mine];
      const float wm = st.w[mine];
      float dw = 0.0f;
      // By pairs of row tiles, ready as operands: N_ij and R_ij of earlier rows j, and of later rows i; each shortly before its products.  (All tiles
      // are multiplied, though some are not needed: a branch around each would make the next one's operands wait for it.)
      Parts<3> below[2], belowq[2], above[2], aboveq[2];
      // sums of keys or queries with these weights
      const auto weighed = [&](const u32x4* columns, const Parts<3> (&weights)[2], f32x4 (&sum)[OWN]) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          Parts<IN> k[OWN];
          load_parts(columns, half * OWN * 2 + kb, 2, k);
          mul_add(k, weights[kb], sum);
        }
      };
      const auto earlier = [&] {
        f32x4 up[4] = {}, upq[4] = {};
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
          Parts<3> y[4];
          HeldU::load(lu, vb, VB, y);
          mul_add(y, of_x(vb), up);
          mul_add(y, of_o(vb), upq);
          __builtin_amdgcn_sched_barrier(0);  // (operands read further ahead would not fit the registers)
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
          const f32x4 rk = row_weights(st.rk, rt);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = rt * 16 + 4 * g + r;
            const float fade = rk[r] * exp_of(-(float)fabs(st.G[i] - Gm));
            up[rt][r] = i < mine ? -up[rt][r] * (wm * fade) : 0.0f;
            upq[rt][r] = i <= mine ? upq[rt][r] * (a.scale * fade) : 0.0f;
          }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) above[kb] = parts_of<3>(up[2 * kb], up[2 * kb + 1]), aboveq[kb] = parts_of<3>(upq[2 * kb], upq[2 * kb + 1]);
      };
      const auto later = [&] {
        f32x4 dn[4] = {}, dnq[4] = {};
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
          Parts<3> y[4];
          Parts<IN> z[4];
          const Parts<3> u = of_u(vb);
          HeldX::load(lx, vb, VB, y);
          mul_add(y, u, dn);
#pragma unroll
          for (int t = 0; t < 4; ++t) z[t] = given(t * VB + vb);
          mul_add(z, u, dnq);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
          const f32x4 rk = row_weights(st.rk, rt), rq = row_weights(st.rq, rt), wr = row_weights(st.w, rt);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = rt * 16 + 4 * g + r;
            const float fade = exp_of(-(float)fabs(st.G[i] - Gm));
            if (i == mine) dw = dn[rt][r];
            dn[rt][r] = i > mine ? -dn[rt][r] * (wr[r] * rk[r] * fade) : 0.0f;
            dnq[rt][r] = i >= mine ? dnq[rt][r] * (a.scale * rq[r] * fade) : 0.0f;
          }
        }
        // what the pairs (i, the lane's step j) give to every step from behind j up to i
        f32x4 cross[4];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) cross[rt] = HALVES == 1 ? dn[rt] * pairs[0][rt] + dnq[rt] * pairs[HALVES == 1][rt] : (half ? dnq[rt] : dn[rt]) * pairs[0][rt];
        float behind = 0.0f, crossed = 0.0f;  // of later tiles of rows; of the step whose sum the lane keeps
#pragma unroll
        for (int rt = 3; rt >= 0; --rt) {
          f32x4 x = cross[rt] * rkm;
          x[2] += x[3], x[1] += x[2], x[0] += x[1];
          const float whole = x[0], n1 = __shfl_down(whole, 16), n2 = __shfl_down(whole, 32), n3 = __shfl_down(whole, 48);
          const float more = behind + ((g < 3 ? n1 : 0.0f) + (g < 2 ? n2 : 0.0f) + (g < 1 ? n3 : 0.0f));
          behind += over_rows(whole);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float sum = row_sum(rt * 16 + 4 * g + r > mine ? x[r] + more : 0.0f);
            crossed = c == rt * 4 + r ? sum : crossed;
          }
        }
        crossing[w8][(c >> 2) * 16 + 4 * g + (c & 3)] = crossed;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) below[kb] = parts_of<3>(dn[2 * kb], dn[2 * kb + 1]), belowq[kb] = parts_of<3>(dnq[2 * kb], dnq[2 * kb + 1]);
      };
      earlier();
      const float since = st.since[mine], still = st.still[mine];
      float moved = 0.0f, into = 0.0f, both = 0.0f;
      // A piece is stored while the one before it, in the other slot, is multiplied.
      const auto next_of_S = [&](int vb) {
        store_parts<3>(piece(vb), w8, parts_of<3>(Sx[vb]));
        ds.load(w8 * 16 + c, vb * 32 + 8 * g, Dx[vb]);
      };
      const auto product = [&](int vb) {
#pragma unroll
        for (int e = 0; e < 8; ++e) both = fmaf(Sx[vb][e], Dx[vb][e], both);
      };
      const auto next_of_dS = [&](int vb) { store_parts<3>(piece(vb), w8, parts_of<3>(Dx[vb])); };
      next_of_S(0);
      // (at once where registers are short, so that the weights are gone when the states' pieces come: 8 x 1024 x 8 heads of 128 x 128 353 us of backward pass, behind the pieces 394; else
      // behind them, whose products the keys' loads are waited for beside: 4096 x 4 x 16 of 64 x 64 531, at once 552)
      constexpr bool AT_ONCE = HALVES > 1;
      if (AT_ONCE) weighed(ktf, above, sumk), weighed(ktf, aboveq, sumq);
      {
        f32x4 tq[OWN] = {}, tp[OWN] = {};
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
          __syncthreads();
          if (vb + 1 < VB) next_of_S(vb + 1);
          else next_of_dS(0);
          if (vb > 0) product(vb - 1);
          const Parts<3> x = of_x(vb);
          const Parts<IN> o = of_o(vb);
          Parts<3> y[OWN];
          load_parts(piece(vb), half * OWN, 1, y);
          mul_add(y, o, tq);
          mul_add(y, x, tp);
        }
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
          tq[i] *= a.scale * since, tp[i] *= -wm * since;
          float mk = 0.0f, mq = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) mk = fmaf(kx[i].at(r), tp[i][r], mk), mq = fmaf(qx[i].at(r), tq[i][r], mq);
          moved += rkm * mk + rqm * mq;
          sumq[i] += tq[i], sumk[i] += tp[i];
        }
        product(VB - 1);
      }
      if (!AT_ONCE) weighed(ktf, above, sumk), weighed(ktf, aboveq, sumq);
      later();
      if (AT_ONCE) weighed(ktf, below, sumk), weighed(qtf, belowq, sumk);
      {
        f32x4 te[OWN] = {};
#pragma unroll
        for (int vb = 0; vb < VB; ++vb) {
          __syncthreads();
          if (vb + 1 < VB) next_of_dS(vb + 1);
          const Parts<3> u = of_u(vb);
          Parts<3> y[OWN];
          load_parts(piece(vb), half * OWN, 1, y);
          mul_add(y, u, te);
        }
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
          float me = 0.0f;
          te[i] *= still;
#pragma unroll
          for (int r = 0; r < 4; ++r) me = fmaf(kx[i].at(r), te[i][r], me);
          into += rkm * me;
          sumk[i] += te[i];
        }
      }
      if (!AT_ONCE) weighed(ktf, below, sumk), weighed(qtf, belowq, sumk);
      dw = over_rows(dw), moved = over_rows(moved), into = over_rows(into);
      both = wave_sum(both);
      if (g == 0) dG[half][0][mine] = moved, dG[half][1][mine] = into;
      if (lane == 0) ends[w8] = both * st.whole;
      __syncthreads();
      if (w8 == 0) {
        // lane t' = 63 - t: what later steps read, and what earlier ones wrote
        double x = dG[0][0][63 - lane], y = lane < 63 ? dG[0][1][62 - lane] : 0.0;
        if (HALVES > 1) x += dG[HALVES - 1][0][63 - lane], y += lane < 63 ? dG[HALVES - 1][1][62 - lane] : 0.0;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const double before = __shfl_up(x, d), after = __shfl_down(y, d);
          if (lane >= d) x += before;
          if (lane + d < 64) y += after;
        }
        x += y;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) x += (double)ends[i] + (double)crossing[i][63 - lane];
        const int i = 63 - lane;
        const int64_t t = t0 + i;
        float grad = 0.0f;
        if (i < live) grad = (float)x * logistic(-ElemTraits<T>::to_f32(fg));
        if (i < steps) ((T*)df.p)[t * df.t + n * df.b + h] = ElemTraits<T>::from_f32(grad);
      }
      if (half == 0 && g == 0 && mine < steps) {
        const int64_t t = t0 + mine;
        float grad = 0.0f;
        if (mine < live) grad = dw * logistic(-ElemTraits<T>::to_f32(bg));
        ((T*)db.p)[t * db.t + n * db.b + h] = ElemTraits<T>::from_f32(grad);
      }
    }
    // through the division by the length
    float kd = 0.0f, qd = 0.0f;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
#pragma unroll
      for (int r = 0; r < 4; ++r) kd = fmaf(kx[i].at(r), sumk[i][r], kd), qd = fmaf(qx[i].at(r), sumq[i][r], qd);
    }
    kd = over_rows(kd), qd = over_rows(qd);
    if (g == 0) dots[0][half][mine] = kd, dots[1][half][mine] = qd;
    __syncthreads();
    kd = rkm * rkm * (dots[0][0][mine] + (HALVES > 1 ? dots[0][HALVES - 1][mine] : 0.0f)), qd = rqm * rqm * (dots[1][0][mine] + (HALVES > 1 ? dots[1][HALVES - 1][mine] : 0.0f));
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // (of a single element only eps is left of 1 - kh^2, which a difference would lose)
        sumk[i][r] = rkm * (a.Dk == 1 ? a.eps * rkm * rkm * sumk[i][r] : fmaf(-kx[i].at(r), kd, sumk[i][r]));
        sumq[i][r] = rqm * (a.Dk == 1 ? a.eps * rqm * rqm * sumq[i][r] : fmaf(-qx[i].at(r), qd, sumq[i][r]));
      }
    }
  } else if ((int)threadIdx.x < steps) {
    const int64_t t = t0 + threadIdx.x;
    for (int s = 0; s < a.group; ++s) {
      const int h = hk * a.group + s;
      ((T*)df.p)[t * df.t + n * df.b + h] = ElemTraits<T>::from_f32(0.0f);
      ((T*)db.p)[t * db.t + n * db.b + h] = ElemTraits<T>::from_f32(0.0f);
    }
  }
  if (mine >= steps) return;
  T *dqp = (T*)dq.p + (int64_t)(t0 + mine) * dq.t + n * dq.b + hk * a.Dk, *dkp = (T*)dk.p + (int64_t)(t0 + mine) * dk.t + n * dk.b + hk * a.Dk;
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int at = (half * OWN + i) * 16 + 4 * g;
    float x[4], y[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = mine < live ? sumq[i][r] : 0.0f, y[r] = mine < live ? sumk[i][r] : 0.0f;
    if (QUICK) {
      if (at < a.Dk) store_run<4>(dqp + at, x), store_run<4>(dkp + at, y);
    } else {
      store_some<4>(dqp + at, a.Dk - at, x);
      store_some<4>(dkp + at, a.Dk - at, y);
    }
  }
}

// ---- host ---------------------------------------------------------------------------
struct GdrPlan {
  GdrArgs a;
  int dk, slices;  // padded key size; wavefronts' worth of 16 columns of a head
  size_t bytes;
};
// Chunks of a segment: all, or, where the workgroups of all heads' columns leave compute units idle, what is estimated (in chunks' times) to end first: a segment's chunks,
// before them 0.7 of their time for the sums, as often as their workgroups (`sums` of a segment) fill the chip, and a product of a state for every segment.
// Measured, in segments against at once, forward / backward, us: bf16 1 x 8 heads of 64 x 64, 512 steps (not cut) 43 / 58, 1024 steps 40 / 64 and 71 / 82, 4096 66 / 110 and
// 241 / 252; 4 x 16 of 64 x 64, 1024 70 / 158 and 87 / 158, 4096 221 / 618 and 348 / 690; 2 x 8 of 128 x 128, 768 59 / 111 and 71 / 120, 4096 134 / 418 and 312 / 535; fp32 1 x 8 of
// 128 x 128, 1024 84 / 180 and 180 / 307; backward fp32, of whose sums LDS holds one workgroup: 4096 steps, 2 x 4 of 64 x 128 172 (11 segments; 13, as if it held two, 188) and 361,
// 4 x 4 of 64 x 64 264 (8; 13: 269) and 448.
static int segment_span(int chunks, int workgroups, int sums, int resident) {
  constexpr int kUnits = 256;
  int best = chunks;
  float least = 0.85f * chunks;
  for (int n = 2; n * workgroups <= kUnits && n <= chunks; ++n) {
    const int span = ceil_div(chunks, n);
    const float cost = span * (1.0f + 0.7f * ceil_div((n - 1) * sums, kUnits * resident)) + 0.7f * ceil_div(chunks, span) + 2.0f;
    if (cost < least) least = cost, best = span;
  }
  return best;
}
// The workspace's parts, one behind the other; `base` may be NULL, when only the size is asked for.
static GdrPlan gdr_plan(int32_t dtype, int T, int B, int Hk, int H, int Dk, int Dv, bool backward, void* base) {
  GdrPlan p{};
  GdrArgs& a = p.a;
  a.T = T, a.B = B, a.Hk = Hk, a.H = H, a.Dk = Dk, a.Dv = Dv, a.group = H / Hk, a.chunks = ceil_div(T, kChunk);
  p.dk = Dk <= 64 ? 64 : 128;
  p.slices = ceil_div(Dv, 16);
  a.dvp = Dv <= 64 ? 64 : 128;
  const size_t in = dtype == ARD_F32 ? 3 : 1, ku = (size_t)a.chunks * B * Hk, hu = (size_t)a.chunks * B * H;
  size_t at = 0;
  const auto take = [&](auto*& ptr, size_t n) {
    ptr = (std::decay_t<decltype(ptr)>)((char*)base + at);
    at = align_up(at + n, 256);
  };
  const size_t rows = (size_t)4 * (p.dk / 32) * in * 1024, cols = (size_t)(p.dk / 8) * in * 1024;
  take(a.steps, hu * sizeof(Steps64));
  take(a.rows, ku * rows * 2), take(a.cols, ku * cols * (backward ? 2 : 1)), take(a.tri, hu * 6 * (backward ? 9 : 3 + Operands<true>::PER) * 1024);
  // (the backward pass's wavefronts cover the padded columns)
  const int groups = ceil_div(backward ? a.dvp / 16 : p.slices, 4);
  // workgroups of sums that a compute unit holds: their registers allow two, LDS (with 2 KB of weights each) one or two
  const int resident = imin(2, 160 / (walk_operands(backward, true, p.dk, (int)in) + 2));
  a.span = segment_span(a.chunks, B * H * groups, B * H * (groups + p.dk / 64), resident);
  a.segments = ceil_div(a.chunks, a.span);
  if (a.segments > 1) {
    const size_t n = (size_t)a.segments * B * H * p.dk * 4;
    take(a.sums, n * (a.dvp + p.dk)), take(a.starts, n * a.dvp);
  }
  if (backward) {
    take(a.u, hu * kChunk * a.dvp * 4), take(a.dx, hu * kChunk * a.dvp * 4), take(a.ds, hu * p.dk * a.dvp * 4);
  }
  p.bytes = at;
  return p;
}

// Up to this many steps go one by one, as a chunk costs as much with few steps as with 64.  Measured, one by one against a chunk, 8 steps, us: bf16 16.1 and 18.2
// (8 sequences x 8 heads of 64 x 64), 17.2 and 27.0 (32 x 16 of 64 x 64), 19.4 and 19.8 (1 x 8 of 128 x 128), 59 and 77 (128 x 8 of 128 x 128); 12 steps 22.5 and 18.2,
// 23.1 and 27.3, 27.3 and 20.0, 77 and 77.  fp32 gains until 12 to 32.
constexpr int kFewSteps = 8;

static int32_t gdr_check(int32_t dtype, int32_t T, int32_t B, int32_t Hk, int32_t H, int32_t Dk, int32_t Dv) {
  if (dtype != ARD_F32 && dtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", dtype);
  if (T <= 0 || B <= 0 || Hk <= 0 || H <= 0 || Dk <= 0 || Dv <= 0)
    return fail(ARD_ESHAPE, "T, B, Hk, H, Dk and Dv must be positive (got %d, %d, %d, %d, %d, %d)", T, B, Hk, H, Dk, Dv);
  if (H % Hk) return fail(ARD_ESHAPE, "H = %d is no multiple of Hk = %d", H, Hk);
  if (Dk > ARD_GDR_MAX || Dv > ARD_GDR_MAX) return fail(ARD_EUNSUPPORTED, "Dk = %d and Dv = %d may be %d at most", Dk, Dv, ARD_GDR_MAX);
  // (HIP counts a grid's threads in 32 bits)
  if (T > 1 << 30 || (int64_t)B * H > 1 << 20 || (int64_t)ceil_div(T, kChunk) * B * H > 1 << 21) return fail(ARD_ESHAPE, "T = %d, B = %d, H = %d are too large", T, B, H);
  return ARD_OK;
}
static int32_t gdr_tensors(int32_t dtype, const ard_steps* s, int n, const char* what) {
  if (!s) return fail(ARD_EINVAL, "%s: null pointer", what);
  for (int i = 0; i < n; ++i) {
    if (!s[i].p) return fail(ARD_EINVAL, "%s: null tensor pointer", what);
    if (misaligned(s[i].p, dtype == ARD_F32 ? 4 : 2)) return fail(ARD_EINVAL, "%s: a tensor does not start at a whole element", what);
  }
  return ARD_OK;
}
static int32_t gdr_numbers(float scale, float eps) {
  if (!(eps >= 0x1p-100f && eps < INFINITY)) return fail(ARD_EINVAL, "eps must be finite and at least 2^-100 (got %g)", eps);  // (1 / eps, times the scale, meets a product of zeros)
  if (!(scale > -INFINITY && scale < INFINITY)) return fail(ARD_EINVAL, "scale must be finite (got %g)", scale);
  return ARD_OK;
}

// Workgroups of the operands of a chunk and a key head: more than one, each with a share of its heads, where one each would not fill the chip (keys' and
// queries' products are made by each of them).  Measured, shared out against one each, forward / backward of 64 steps x 16 x 8 heads of 128 x 128, 2 key heads, bf16: 26 / 154 and
// 45 / 172 us; 2048 x 1 x 32 of 64 x 64, 4 key heads: 72 / 169 and 104 / 204; 256 x 8 x 24 of 64 x 64, 12 key heads (384 workgroups): 41 / 99 and 43 / 105.
static int prep_splits(const GdrArgs& a) {
  const int64_t units = (int64_t)a.chunks * a.B * a.Hk;
  return units * 2 <= 768 ? (int)std::min<int64_t>(a.group, 768 / units) : 1;
}

template <class F> static int32_t gdr_instance(int32_t dtype, int dk, bool near, F&& with) {
  const auto sized = [&](auto t) {
    using Wide = std::integral_constant<int, 128>;
    using Narrow = std::integral_constant<int, 64>;
    if (near) return dk == 64 ? with(t, Narrow{}, std::true_type{}) : with(t, Wide{}, std::true_type{});
    return dk == 64 ? with(t, Narrow{}, std::false_type{}) : with(t, Wide{}, std::false_type{});
  };
  return dtype == ARD_F32 ? sized(0.0f) : sized((uint16_t)0);
}
// (a single step's stride says nothing)
static ard_steps gdr_steps(const ard_steps& s, int T, int wide) { return T == 1 ? ard_steps{s.p, wide, s.b} : s; }
// Window's NEAR: the steps of a chunk do not overlap and lie within 2 GB
static bool gdr_near(const ard_steps& s, int wide) { return s.t >= wide && s.t < (int64_t)INT32_MAX / 4 / kChunk; }

}  // namespace ard

using namespace ard;

extern "C" int32_t ard_gdr_chunk(void) { return kChunk; }

extern "C" size_t ard_gdr_workspace_bytes(int32_t dtype, int32_t T, int32_t B, int32_t Hk, int32_t H, int32_t Dk, int32_t Dv, int32_t backward) {
  if (gdr_check(dtype, T, B, Hk, H, Dk, Dv) != ARD_OK || (!backward && T <= kFewSteps)) return 0;
  return gdr_plan(dtype, T, B, Hk, H, Dk, Dv, backward != 0, nullptr).bytes;
}

extern "C" int32_t ard_gdr_fwd(int32_t dtype, int32_t T, int32_t B, int32_t Hk, int32_t H, int32_t Dk, int32_t Dv, const ard_steps* in, float scale, float eps,
                               const float* S0, const int32_t* d_lengths, const ard_steps* o, float* ST, float* ckpt, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = gdr_check(dtype, T, B, Hk, H, Dk, Dv)) return st;
  if (int32_t st = gdr_tensors(dtype, in, 5, "inputs")) return st;
  if (int32_t st = gdr_tensors(dtype, o, 1, "o")) return st;
  if (int32_t st = gdr_numbers(scale, eps)) return st;
  if (misaligned(S0, 4) || misaligned(ST, 4) || misaligned(ckpt, 4) || misaligned(d_lengths, 4)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const bool few = T <= kFewSteps;
  GdrPlan p = gdr_plan(dtype, T, B, Hk, H, Dk, Dv, false, ws);
  if (!few && (!ws || ws_bytes < p.bytes || misaligned(ws, 16))) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", p.bytes, ws ? ws_bytes : 0);
  GdrArgs& a = p.a;
  a.q = gdr_steps(in[0], T, Hk * Dk), a.k = gdr_steps(in[1], T, Hk * Dk), a.v = gdr_steps(in[2], T, H * Dv), a.f = in[3], a.b = in[4], a.scale = scale, a.eps = eps, a.len = d_lengths;
  hipStream_t st = (hipStream_t)stream;
  const ard_steps out = gdr_steps(*o, T, H * Dv);
  const int splits = prep_splits(a);
  return gdr_instance(dtype, p.dk, gdr_near(a.v, Dv) && gdr_near(out, Dv), [&](auto t, auto dk, auto near) {
    using E = decltype(t);
    constexpr int DK = decltype(dk)::value;
    constexpr bool NEAR = decltype(near)::value;
    if (few) {
      const int slices = ceil_div(Dv, 32);
      const dim3 grid(ceil_div(B * H * slices, 4));
      if (Dv % 4 == 0) ARD_LAUNCH_NAMED("gdr_steps_kernel", (gdr_steps_kernel<E, DK, 4>), grid, dim3(256), 0, st, a, S0, out, ST, ckpt, slices);
      else ARD_LAUNCH_NAMED("gdr_steps_kernel", (gdr_steps_kernel<E, DK, 1>), grid, dim3(256), 0, st, a, S0, out, ST, ckpt, slices);
      ARD_LAUNCH_CHECK("gdr_steps_kernel");
      return (int32_t)ARD_OK;
    }
    ARD_LAUNCH_NAMED("gdr_prep_kernel", (gdr_prep_kernel<E, DK, false>), dim3(a.chunks * B * Hk * splits), dim3(256), 0, st, a, splits);
    ARD_LAUNCH_CHECK("gdr_prep_kernel");
    const int groups = ceil_div(p.slices, 4);
    if (a.segments > 1) {
      const int sums = B * H * (groups + DK / 64) * (a.segments - 1);
      ARD_LAUNCH_NAMED(launch_instance("gdr_fwd_kernel", sums, a.segments, a.span), (gdr_fwd_kernel<E, DK, NEAR, SUM>), dim3(sums), dim3(256), 0, st, a, S0, out, ST, ckpt, groups);
      ARD_LAUNCH_CHECK("gdr_fwd_kernel");
      ARD_LAUNCH_NAMED("gdr_join_kernel", (gdr_join_kernel<DK>), dim3(B * H * p.slices), dim3(256), 0, st, a, S0, p.slices);
      ARD_LAUNCH_CHECK("gdr_join_kernel");
    }
    const dim3 grid(B * H * groups * a.segments);
    if (ckpt) ARD_LAUNCH_NAMED("gdr_fwd_kernel", (gdr_fwd_kernel<E, DK, NEAR, KEEP>), grid, dim3(256), 0, st, a, S0, out, ST, ckpt, groups);
    else ARD_LAUNCH_NAMED("gdr_fwd_kernel", (gdr_fwd_kernel<E, DK, NEAR, DROP>), grid, dim3(256), 0, st, a, S0, out, ST, ckpt, groups);
    ARD_LAUNCH_CHECK("gdr_fwd_kernel");
    return (int32_t)ARD_OK;
  });
}

extern "C" int32_t ard_gdr_bwd(int32_t dtype, int32_t T, int32_t B, int32_t Hk, int32_t H, int32_t Dk, int32_t Dv, const ard_steps* in, float scale, float eps,
                               const int32_t* d_lengths, const float* ckpt, const ard_steps* d_o, const float* dST, const ard_steps* grads, float* dS0,
                               void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = gdr_check(dtype, T, B, Hk, H, Dk, Dv)) return st;
  if (int32_t st = gdr_tensors(dtype, in, 5, "inputs")) return st;
  if (int32_t st = gdr_tensors(dtype, d_o, 1, "the gradient of o")) return st;
  if (int32_t st = gdr_tensors(dtype, grads, 5, "gradients")) return st;
  if (int32_t st = gdr_numbers(scale, eps)) return st;
  if (!ckpt) return fail(ARD_EINVAL, "null tensor pointer");
  if (misaligned(ckpt, 4) || misaligned(dST, 4) || misaligned(dS0, 4) || misaligned(d_lengths, 4)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  GdrPlan p = gdr_plan(dtype, T, B, Hk, H, Dk, Dv, true, ws);
  if (!ws || ws_bytes < p.bytes || misaligned(ws, 16)) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", p.bytes, ws ? ws_bytes : 0);
  GdrArgs& a = p.a;
  a.q = gdr_steps(in[0], T, Hk * Dk), a.k = gdr_steps(in[1], T, Hk * Dk), a.v = gdr_steps(in[2], T, H * Dv), a.f = in[3], a.b = in[4], a.scale = scale, a.eps = eps, a.len = d_lengths;
  hipStream_t st = (hipStream_t)stream;
  // dX and U are read in whole operands of 32 columns: the wavefronts of the padded columns write them as zeros
  const int slices = a.dvp / 16, waves = B * H * slices;
  const ard_steps od = gdr_steps(*d_o, T, H * Dv), dv = gdr_steps(grads[2], T, H * Dv);
  const int splits = prep_splits(a);
  return gdr_instance(dtype, p.dk, gdr_near(a.v, Dv) && gdr_near(od, Dv) && gdr_near(dv, Dv), [&](auto t, auto dk, auto near) {
    using E = decltype(t);
    constexpr int DK = decltype(dk)::value;
    constexpr bool NEAR = decltype(near)::value;
    ARD_LAUNCH_NAMED("gdr_prep_kernel", (gdr_prep_kernel<E, DK, true>), dim3(a.chunks * B * Hk * splits), dim3(256), 0, st, a, splits);
    ARD_LAUNCH_CHECK("gdr_prep_kernel");
    ARD_LAUNCH_NAMED("gdr_rows_kernel", (gdr_rows_kernel<E, DK, NEAR>), dim3((unsigned)(((int64_t)a.chunks * waves + 3) / 4)), dim3(256), 0, st, a, ckpt, slices, waves);
    ARD_LAUNCH_CHECK("gdr_rows_kernel");
    const int groups = ceil_div(slices, 4);
    if (a.segments > 1) {
      const int sums = B * H * (groups + DK / 64) * (a.segments - 1);
      ARD_LAUNCH_NAMED(launch_instance("gdr_back_kernel", sums, a.segments, a.span), (gdr_back_kernel<E, DK, NEAR, SUM>), dim3(sums), dim3(256), 0, st, a, od, dST, dv, dS0, groups);
      ARD_LAUNCH_CHECK("gdr_back_kernel");
      ARD_LAUNCH_NAMED("gdr_join_kernel", (gdr_join_kernel<DK>), dim3(B * H * slices), dim3(256), 0, st, a, dST, slices);
      ARD_LAUNCH_CHECK("gdr_join_kernel");
    }
    ARD_LAUNCH_NAMED("gdr_back_kernel", (gdr_back_kernel<E, DK, NEAR, KEEP>), dim3(B * H * groups * a.segments), dim3(256), 0, st, a, od, dST, dv, dS0, groups);
    ARD_LAUNCH_CHECK("gdr_back_kernel");
    const auto grads_of = [&](auto dv_, auto quick) {
      constexpr int DV = decltype(dv_)::value;
      constexpr bool QUICK = decltype(quick)::value;
      ARD_LAUNCH_NAMED("gdr_grads_kernel", (gdr_grads_kernel<E, DK, DV, QUICK>), dim3(a.chunks * B * Hk), dim3(DK * 4), 0, st, a, od, ckpt, grads[0], grads[1], grads[3], grads[4]);
    };
    const bool quick = Dk % 4 == 0 && Dv % 8 == 0 && gdr_near(a.q, Dk) && gdr_near(a.k, Dk) && gdr_near(od, Dv);
    if (a.dvp == 64) quick ? grads_of(std::integral_constant<int, 64>{}, std::true_type{}) : grads_of(std::integral_constant<int, 64>{}, std::false_type{});
    else quick ? grads_of(std::integral_constant<int, 128>{}, std::true_type{}) : grads_of(std::integral_constant<int, 128>{}, std::false_type{});
    ARD_LAUNCH_CHECK("gdr_grads_kernel");
    return (int32_t)ARD_OK;
  });
}
