// Loss against a teacher's K largest logits, and the labels, of R rows of V logits z; T the temperature:
//   p = softmax(t / T) over the row's K entries,  qT = softmax(z / T),  q = softmax(z) over all V
//   loss = alpha T^2 sum_k p_k (log p_k - log qT[id_k]) - (1 - alpha) log q[y]
//   dz = g (alpha T (qT - sum_k p_k [id_k = j]) + (1 - alpha) (q - [y = j]))
//
// A workgroup takes a row.  It holds the row in registers as it was read, so that the largest logit, both sums of exponentials and the
// gradient come from one reading: the bytes of z and dz are what bounds it.  Rows longer than its registers hold are read again for each of
// the three (out of the caches, mostly).  Sums and statistics are fp32, a lane's of up to 128 values one after the other (more of rows that are read again), the lanes' in trees.
//
// Measured, bf16, 8192 x 32768, K = 64, T = 2 with labels, loss and gradient: 270 us, 4.0 TB/s of the 1.07 GB (a large copy: 5.1 TB/s); the loss alone 133, the gradient from its
// statistics 224; labels alone 87, 211 with the gradient, 207 from statistics.  Beside the bytes it has about 22 vector instructions an element, 2 of them exponentials; so two workgroups
// share a compute unit, one in its arithmetic while the other waits for memory.  That takes 64 registers a lane (one workgroup with 83: an eighth more).
// Rows that are read again, loss / with the gradient: fp32 1024 x 131072 159 / 332 us, bf16 2048 x 151936 186 / 363, 3.2 to 3.4 TB/s of z and dz once.

// The K entries change few elements: the gradient is stored first as if there were none, then again at the entries, computed anew
// rather than corrected, so that it is rounded once.  Entries that name one element twice each store the sum of all its p; the label, if no entry names it, is one more.
#include "rows.hpp"

namespace ard {

constexpr int kMaxTop = 1024;  // teacher's entries of a row

struct DistillArgs {
  int R, V, K;
  const void* z;
  int64_t ldz;
  const int32_t* ids;
  const void* t;
  const int32_t* labels;
  float tau, cold, alpha, soft, hard;  // log2(e) / T (log2(e) without the teacher), log2(e), alpha T^2 of the loss, alpha T of the gradient, 1 - alpha of the labels
  const float* dloss;
  float *loss, *stats;
  void* dz;
  int64_t lddz;
};

constexpr float kLn2 = 0.693147180559945309f;
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// log2 of an exponential's share.  The difference comes first: z scale - m scale in one instruction leaves the rounding of m scale at the largest
// logit itself, and that is past every exponent for rows whose logits are all a mask's lowest value.
__device__ __forceinline__ float above(float z, float top, float scale) { return (z - top) * scale; }

struct Shared {
  float part[3][16];
  float p[kMaxTop], z[kMaxTop];
  int32_t id[kMaxTop];
};

// the largest and the sums over a workgroup of up to 16 wavefronts, in all of its lanes; `slot` must not be in use
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
template <bool MAX> __device__ __forceinline__ float over_group(float x, float* slot) {
  x = MAX ? lanes_max(x) : wave_sum(x);
  const int waves = blockDim.x >> 6, lane = threadIdx.x & 63;
  if (waves == 1) return x;
  if (lane == 0) slot[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lane < waves ? slot[lane] : MAX ? -INFINITY : 0.0f;
  return MAX ? lanes_max(x) : wave_sum(x);
}

// MODE 1: the loss; 2: the gradient, from the statistics of an earlier call; 3: both.  TWO: the sums at T and at 1 are different ones and both
// are wanted: for T = 2 and 4 the exponential at 1 is the square, or its square, of that at T (one or two products for an instruction of four times a product's
// time; 8192 x 32768 bf16 270 us, with both made, as for T = 1.5, 287), with 1 it is made.  C runs of 16 bytes a lane hold the row; C = 0: it is read again where it is needed.
template <typename T, typename S, int MODE, int TWO, int C>
__global__ __launch_bounds__(1024, C <= 4 ? 8 : 4) void distill_kernel(DistillArgs a) {
  constexpr int N = 16 / sizeof(T), HELD = C ? C : 1;
  using Run16 = typename Run<T, N>::V;
  __shared__ Shared sh;
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.R) return;
  const T* z = (const T*)a.z + row * a.ldz;
  const int V = a.V, threads = blockDim.x, span = threads * N;
  Run16 held[HELD];
  const auto at = [&](int c) { return (c * threads + (int)threadIdx.x) * N; };
  // a run's values; behind the row's end -infinity, which has no share in anything
  const auto values = [&](int c, float (&x)[N]) {
    const int j = at(c);
    if (C) {
      if constexpr (C > 0 && C <= 4) asm volatile("" : "+v"(held[c]));  // taken apart again in each pass: what is kept of one is twice as many registers
      values_of<N, T>(held[C ? c : 0], x);
    } else if (j + N <= V) {
      load_run<N>(z + j, x);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = j + e < V ? ElemTraits<T>::to_f32(z[j + e]) : -INFINITY;
    }
  };
  const auto each = [&](auto&& f) {
    if constexpr (C > 0) {
#pragma unroll
      for (int c = 0; c < C; ++c) f(c);
    } else {
      for (int c = 0, runs = (V + span - 1) / span; c < runs; ++c) f(c);
    }
  };
  if (C) {
#pragma unroll
    for (int c = 0; c < HELD; ++c) {
      const int j = at(c);
      if (j + N <= V) {
        held[c] = *reinterpret_cast<const Run16*>(z + j);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {  // (bf16: two elements a register)
          if constexpr (sizeof(T) == 4) held[c][e] = j + e < V ? (float)z[j + e] : -INFINITY;
          else if (e % 2 == 0) held[c][e / 2] = (j + e < V ? (uint32_t)z[j + e] : 0xff80u) | (j + e + 1 < V ? (uint32_t)z[j + e + 1] : 0xff80u) << 16;
        }
      }
    }
  }
  const auto at_one = [&](float p, float x, float top) { return TWO == 1 ? exp2_of(above(x, top, a.cold)) : TWO == 2 ? p * p : (p * p) * (p * p); };
  // the teacher's entries, kept in LDS with the logits that they meet (which a gradient in z's place would take away)
  const int K = a.K;
  const S* t = (const S*)a.t + row * a.K;
  float tmax = -INFINITY;
  for (int k = threadIdx.x; k < K; k += threads) {
    const int id = a.ids[row * a.K + k];
    const bool there = id >= 0 && id < V;
    const float x = there ? ElemTraits<S>::to_f32(t[k]) : -INFINITY;
    sh.id[k] = there ? id : -1;
    sh.p[k] = x;
    sh.z[k] = there ? ElemTraits<T>::to_f32(z[id]) : 0.0f;
    tmax = x != x ? x : fmaxf(tmax, x);
  }
  const int y = a.labels ? a.labels[row] : -1;
  const bool labelled = y >= 0 && y < V;
  const float zy = labelled ? ElemTraits<T>::to_f32(z[y]) : 0.0f;
  float m, sT, s1;
  if (MODE & 1) {
    m = -INFINITY;
    each([&](int c) {
      float x[N];
      values(c, x);
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, x[e]);
    });
    m = over_group<true>(m, sh.part[0]);
    const float top = m == -INFINITY ? 0.0f : m;
    sT = s1 = 0.0f;
    each([&](int c) {
      float x[N];
      values(c, x);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float p = exp2_of(above(x[e], top, a.tau));
        sT += p;
        if (TWO) s1 += at_one(p, x[e], top);
      }
    });
    sT = over_group<false>(sT, sh.part[1]);
    s1 = TWO ? over_group<false>(s1, sh.part[2]) : sT;
    if (threadIdx.x == 0) a.stats[row * 3] = m, a.stats[row * 3 + 1] = sT, a.stats[row * 3 + 2] = s1;
  } else {
    m = a.stats[row * 3], sT = a.stats[row * 3 + 1], s1 = a.stats[row * 3 + 2];
  }
  const bool any = m != -INFINITY || sT != sT;  // some logit is not masked (NaN is none): otherwise the row has no part in anything
  // the teacher's shares
  float tsum = 0.0f;
  if (K) {
    __syncthreads();
    tmax = over_group<true>(tmax, sh.part[0]);
    const float off = tmax == -INFINITY ? 0.0f : tmax;
    for (int k = threadIdx.x; k < K; k += threads) tsum += exp2_of((sh.p[k] - off) * a.tau);
    __syncthreads();
    tsum = over_group<false>(tsum, sh.part[1]);
  }
  const bool taught = K && tsum != 0.0f && any;
  const float inv = 1.0f / tsum;
  float kl = 0.0f;
  if (taught) {
    const float lse = log2f(sT), tlse = log2f(tsum);
    for (int k = threadIdx.x; k < K; k += threads) {
      const float x = (sh.p[k] - tmax) * a.tau, p = exp2_of(x) * inv;
      if ((MODE & 1) && p != 0.0f) kl += p * ((x - tlse) - (above(sh.z[k], m, a.tau) - lse));
      sh.p[k] = p;
    }
  }
  if (MODE & 1) {
    if (K) {
      __syncthreads();
      kl = over_group<false>(kl, sh.part[2]);
    }
    if (threadIdx.x == 0) {
      float l = 0.0f;
      if (taught) l = a.alpha * kLn2 * kl;
      // (one sum: it is at the labels' temperature, T = 1 or without a teacher; squares: so is the logit's place)
      if (labelled && any) l += a.hard * kLn2 * (log2f(s1) - above(zy, m, TWO == 1 ? a.cold : TWO ? a.tau * TWO : a.tau));
      a.loss[row] = l;
    }
  }
  if (!(MODE & 2)) return;
  if (MODE == 2 && !K) __syncthreads();  // no lane's store in z's place comes before the last lane's read of the label's logit
  T* dz = (T*)a.dz + row * a.lddz;
  const float g = a.dloss ? a.dloss[row] : 1.0f, hard = labelled && any ? a.hard * g : 0.0f, soft = taught ? a.soft * g : 0.0f;
  const float fT = soft / sT, f1 = hard / s1, top = m == -INFINITY ? 0.0f : m;
  // of an element without the label's and the teacher's own terms
  const auto dense = [&](float x) {
    const float p = exp2_of(above(x, top, a.tau));
    return TWO ? fmaf(fT, p, f1 * at_one(p, x, top)) : (fT + f1) * p;
  };
  const bool shared = any && (taught || labelled);  // (nothing of a row that neither teaches: NaN and infinities of padding have no part either)
  if (shared) {
    each([&](int c) {
      const int j = at(c);
      if (j >= V) return;
      float x[N];
      values(c, x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = dense(x[e]);
      // (passes in a row 270 us, with stores that stay in the caches 279; with the two products that read dz behind it, bf16 rows of 32768: 8192 1080 and 1095 us, 2048 456 and 461, 1024,
      // whose dz the last cache would hold, 251 and 233; in z's place, whose lines are there, 222 both)
      if (V - j >= N) store_run_past(dz + j, x);
      else store_some<N>(dz + j, V - j, x);
    });
  } else {
    const float none[N] = {};
    each([&](int c) {
      if (at(c) < V) store_some<N>(dz + at(c), V - at(c), none);
    });
  }
  if (!shared) return;
  __syncthreads();
  for (int k = threadIdx.x; k < (taught ? K : 0); k += threads) {
    const int id = sh.id[k];
    if (id < 0) continue;
    float p = 0.0f;
    for (int i = 0; i < K; ++i) p += sh.id[i] == id ? sh.p[i] : 0.0f;
    float x = dense(sh.z[k]) - soft * p;
    if (id == y) x -= hard;
    dz[id] = ElemTraits<T>::from_f32(x);
  }
  if (labelled && threadIdx.x == threads - 1) {
    bool named = false;  // an entry names it: that one's lane has stored it
    for (int i = 0; i < (taught ? K : 0); ++i) named |= sh.id[i] == y;
    if (!named) dz[y] = ElemTraits<T>::from_f32(dense(zy) - hard);
  }
}

// ---- host ---------------------------------------------------------------------
static int32_t distill_check(int32_t dtype, int32_t tdtype, int32_t R, int32_t V, int32_t K, const void* Z, int64_t ldz, const int32_t* d_ids, const void* t,
                             const int32_t* d_labels, float temperature, float alpha) {
  if (dtype != ARD_F32 && dtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", dtype);
  if (tdtype != ARD_F32 && tdtype != dtype) return fail(ARD_EDTYPE, "the teacher's logits are fp32 or of the logits' dtype (got %d)", tdtype);
  if (R <= 0 || V <= 0 || K < 0) return fail(ARD_ESHAPE, "R and V must be positive, K not negative (got %d, %d, %d)", R, V, K);
  if (V > 1 << 30) return fail(ARD_ESHAPE, "V = %d is too large", V);
  if (K > kMaxTop) return fail(ARD_EUNSUPPORTED, "a row has at most %d teacher's logits (got %d)", kMaxTop, K);
  if (ldz < V) return fail(ARD_ESHAPE, "the logits' leading dimension must be at least V");
  if (!(temperature >= 0x1p-60f && temperature <= 0x1p60f)) return fail(ARD_EINVAL, "the temperature must be from 2^-60 to 2^60 (got %g)", temperature);
  if (!(alpha >= 0.0f && alpha <= 1.0f)) return fail(ARD_EINVAL, "alpha must be from 0 to 1 (got %g)", alpha);
  if (!Z) return fail(ARD_EINVAL, "null tensor pointer");
  if (alpha > 0.0f && K > 0 && (!d_ids || !t)) return fail(ARD_EINVAL, "a teacher's share needs its logits and their ids");
  const size_t es = dtype == ARD_F32 ? 4 : 2;
  if (misaligned(Z, es) || misaligned(t, tdtype == ARD_F32 ? 4 : 2) || misaligned(d_ids, 4) || misaligned(d_labels, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  return ARD_OK;
}

template <typename T, typename S, int MODE, int TWO, int C> static int32_t distill_launch(const DistillArgs& a, int threads, hipStream_t st) {
  const int x = imin(a.R, 1 << 20), y = (int)(((int64_t)a.R + x - 1) / x);  // (a sum of R and x may pass 32 bits)
  ARD_LAUNCH_NAMED(launch_instance("distill_kernel", x, y, threads), (distill_kernel<T, S, MODE, TWO, C>), dim3(x, y), dim3(threads), 0, st, a);
  ARD_LAUNCH_CHECK("distill_kernel");
  return ARD_OK;
}
// As many lanes as hold the row in 4 runs each, so that there are loads in flight and little is held behind the row's end; 8 or 16 runs
// where 1024 lanes do not, and from there on the row is read again.
template <typename T, typename S, int MODE, int TWO> static int32_t distill_sized(const DistillArgs& a, hipStream_t st) {
  const int runs = ceil_div(a.V, 16 / (int)sizeof(T));
  const auto lanes = [&](int c) { return (ceil_div(runs, c) + 63) / 64 * 64; };
  if (lanes(4) <= 1024) return distill_launch<T, S, MODE, TWO, 4>(a, lanes(4), st);
  if constexpr (MODE & 1) {
    if (lanes(8) <= 1024) return distill_launch<T, S, MODE, TWO, 8>(a, lanes(8), st);
    if (lanes(16) <= 1024) return distill_launch<T, S, MODE, TWO, 16>(a, lanes(16), st);
  }
  return distill_launch<T, S, MODE, TWO, 0>(a, 1024, st);
}
template <int MODE> static int32_t distill_run(int32_t dtype, int32_t tdtype, DistillArgs a, float temperature, float alpha, hipStream_t st) {
  const bool taught = alpha > 0.0f && a.K > 0, labelled = alpha < 1.0f && a.labels;
  if (!taught) a.K = 0;
  if (!labelled) a.labels = nullptr;
  constexpr double log2e = 1.4426950408889634074;
  a.tau = (float)(taught ? log2e / temperature : log2e), a.cold = (float)log2e, a.alpha = alpha * temperature * temperature, a.soft = alpha * temperature, a.hard = 1.0f - alpha;
  const bool two = taught && labelled && temperature != 1.0f;
  const auto with = [&](auto z, auto t) {
    using T = decltype(z);
    using S = decltype(t);
    if (!two) return distill_sized<T, S, MODE, 0>(a, st);
    return temperature == 2.0f ? distill_sized<T, S, MODE, 2>(a, st) : temperature == 4.0f ? distill_sized<T, S, MODE, 4>(a, st) : distill_sized<T, S, MODE, 1>(a, st);
  };
  if (dtype == ARD_F32) return with(0.0f, 0.0f);
  return tdtype == ARD_F32 ? with((uint16_t)0, 0.0f) : with((uint16_t)0, (uint16_t)0);
}

}  // namespace ard

using namespace ard;

extern "C" int32_t ard_distill_fwd(int32_t dtype, int32_t tdtype, int32_t R, int32_t V, int32_t K, const void* Z, int64_t ldz, const int32_t* d_ids,
                                   const void* t, const int32_t* d_labels, float temperature, float alpha, const float* d_dloss, float* loss, float* stats,
                                   void* dZ, int64_t lddz, void* stream) {
  if (int32_t st = distill_check(dtype, tdtype, R, V, K, Z, ldz, d_ids, t, d_labels, temperature, alpha)) return st;
  if (!loss || !stats) return fail(ARD_EINVAL, "null tensor pointer");
  if (misaligned(loss, 4) || misaligned(stats, 4) || misaligned(d_dloss, 4) || misaligned(dZ, dtype == ARD_F32 ? 4 : 2))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  if (dZ && lddz < V) return fail(ARD_ESHAPE, "the gradient's leading dimension must be at least V");
  if (dZ == Z && lddz != ldz && R > 1) return fail(ARD_EINVAL, "a gradient in the logits' place has their leading dimension");
  const DistillArgs a{R, V, K, Z, ldz, d_ids, t, d_labels, 0, 0, 0, 0, 0, d_dloss, loss, stats, dZ, lddz};
  return dZ ? distill_run<3>(dtype, tdtype, a, temperature, alpha, (hipStream_t)stream) : distill_run<1>(dtype, tdtype, a, temperature, alpha, (hipStream_t)stream);
}

extern "C" int32_t ard_distill_bwd(int32_t dtype, int32_t tdtype, int32_t R, int32_t V, int32_t K, const void* Z, int64_t ldz, const int32_t* d_ids,
                                   const void* t, const int32_t* d_labels, float temperature, float alpha, const float* stats, const float* d_dloss, void* dZ,
                                   int64_t lddz, void* stream) {
  if (int32_t st = distill_check(dtype, tdtype, R, V, K, Z, ldz, d_ids, t, d_labels, temperature, alpha)) return st;
  if (!stats || !dZ) return fail(ARD_EINVAL, "null tensor pointer");
  if (misaligned(stats, 4) || misaligned(d_dloss, 4) || misaligned(dZ, dtype == ARD_F32 ? 4 : 2)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  if (lddz < V) return fail(ARD_ESHAPE, "the gradient's leading dimension must be at least V");
  if (dZ == Z && lddz != ldz && R > 1) return fail(ARD_EINVAL, "a gradient in the logits' place has their leading dimension");
  const DistillArgs a{R, V, K, Z, ldz, d_ids, t, d_labels, 0, 0, 0, 0, 0, d_dloss, nullptr, const_cast<float*>(stats), dZ, lddz};
  return distill_run<2>(dtype, tdtype, a, temperature, alpha, (hipStream_t)stream);
}
