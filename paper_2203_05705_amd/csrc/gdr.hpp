// What the passes of the gated delta rule share: products of fp32 values on the bf16 matrix instructions, and the workspace.
//
// An fp32 value is the sum of three bf16 values (8 bits of its 24 each), so a product of two is the sum of the six products of parts that
// reach its 24 bits, each exact, added in fp32: as good as fp32's own, at 2.7 times the rate of the fp32 matrix instructions.
// What is bf16 already is one part, and its product with an fp32 value takes three.  A result that is rounded to bf16 needs its factors' 24 bits too: with two parts
// (16 bits) of them 3e-4 to 1e-3 of all results are rounded to bf16's other neighbour, with three under 7e-5.
//
// v_mfma_f32_16x16x32_bf16, lane = 16 g + c: A[row c][8 g + j], B[8 g + j][column c], j = 0..7; result[row 4 g + r][column c], r = 0..3.
// A contraction may take its indices in any order that both operands share: with index 4 g + (j & 3) + 16 (j >> 2) in the place of
// 8 g + j, the results of two row tiles are the B operand of the next product as they lie in their lane's registers.  So a chain of products
// with a state, held by columns, stays inside a wavefront, without LDS or barriers.
#pragma once
#include <type_traits>

#include "rows.hpp"

namespace ard {

constexpr int kChunk = ARD_GDR_CHUNK;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// N parts of 8 values of a lane
template <int N> struct Parts {
  u32x4 p[N];
};
template <int N> __device__ __forceinline__ Parts<N> parts_of(const float (&x)[8]) {
  Parts<N> s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t hi = bf16_pair(a, b);
      s.p[n][i] = hi;
      a -= __uint_as_float(hi << 16), b -= __uint_as_float(hi & 0xffff0000u);
    }
  }
  return s;
}
template <int N> __device__ __forceinline__ Parts<N> parts_of(const f32x4& lo, const f32x4& hi) {
  const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return parts_of<N>(x);
}
// acc += a b, of all products of parts those that reach the larger operand's last part; the small ones first
template <int NA, int NB> __device__ __forceinline__ void mul_add(const Parts<NA>& a, const Parts<NB>& b, f32x4& acc) {
  constexpr int L = NA > NB ? NA : NB;
#pragma unroll
  for (int s = L - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.p[i]), __builtin_bit_cast(bf16x8, b.p[s - i]), acc, 0, 0, 0);
}
// The same of several tiles of rows, in turn: a product waits for the one before it in its own sum, not for the others.
template <int TILES, int NA, int NB> __device__ __forceinline__ void mul_add(const Parts<NA> (&a)[TILES], const Parts<NB>& b, f32x4 (&acc)[TILES]) {
  constexpr int L = NA > NB ? NA : NB;
#pragma unroll
  for (int s = L - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[t].p[i]), __builtin_bit_cast(bf16x8, b.p[s - i]), acc[t], 0, 0, 0);
      }
}
// Operands in the workspace or in LDS, 64 lanes x 16 bytes a part as a lane takes them; base: the lane's place in the first.
template <int N> __device__ __forceinline__ Parts<N> load_parts(const u32x4* base, int frag) {
  Parts<N> s;
#pragma unroll
  for (int n = 0; n < N; ++n) s.p[n] = base[(frag * N + n) * 64];
  return s;
}
// of TILES tiles of rows, `step` operands from one to the next
template <int TILES, int N> __device__ __forceinline__ void load_parts(const u32x4* base, int first, int step, Parts<N> (&s)[TILES]) {
#pragma unroll
  for (int t = 0; t < TILES; ++t) s[t] = load_parts<N>(base, first + t * step);
}
template <int N> __device__ __forceinline__ void store_parts(u32x4* base, int frag, const Parts<N>& s) {
#pragma unroll
  for (int n = 0; n < N; ++n) base[(frag * N + n) * 64] = s.p[n];
}
// Operands of fp32 values: their three parts, or, in two thirds of the room, the values (FLOATS), which become parts where they are used.
template <bool FLOATS> struct Operands {
  static constexpr int PER = FLOATS ? 2 : 3;  // KB of an operand
  static __device__ __forceinline__ void store(u32x4* base, int frag, const f32x4& lo, const f32x4& hi) {
    if constexpr (FLOATS) base[frag * 2 * 64] = __builtin_bit_cast(u32x4, lo), base[(frag * 2 + 1) * 64] = __builtin_bit_cast(u32x4, hi);
    else store_parts<3>(base, frag, parts_of<3>(lo, hi));
  }
  static __device__ __forceinline__ void store(u32x4* base, int frag, const float (&x)[8]) { store(base, frag, f32x4{x[0], x[1], x[2], x[3]}, f32x4{x[4], x[5], x[6], x[7]}); }
  static __device__ __forceinline__ Parts<3> load(const u32x4* base, int frag) {
    if constexpr (FLOATS) return parts_of<3>(__builtin_bit_cast(f32x4, base[frag * 2 * 64]), __builtin_bit_cast(f32x4, base[(frag * 2 + 1) * 64]));
    else return load_parts<3>(base, frag);
  }
  template <int TILES> static __device__ __forceinline__ void load(const u32x4* base, int first, int step, Parts<3> (&s)[TILES]) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) s[t] = load(base, first + t * step);
  }
};
// FRAGS x 1 KB from global memory to the same order in LDS, without a register in between: each of a workgroup's four wavefronts its share of
// neighbours, four to an address.
// (The last wavefront's share may reach behind the end: it takes the last operand again, so that every wavefront makes as many accesses.)
template <int FRAGS> __device__ __forceinline__ void stage(const u32x4* from, u32x4* lds, int wave) {
  constexpr int PER = (FRAGS + 3) / 4;
  if constexpr (FRAGS % 4 != 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = imin(wave * PER + i, FRAGS - 1);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(from + j * 64 + (threadIdx.x & 63)), (__attribute__((address_space(3))) uint32_t*)(lds + j * 64),
                                       16, 0, 0);
    }
    return;
  }
  const u32x4* src = from + wave * PER * 64 + (threadIdx.x & 63);
  u32x4* dst = lds + wave * PER * 64;
#define ARD_GDR_STAGE(i, offset)                                                                                                   \
  if ((i) < PER)                                                                                                                     \
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(src + ((i) - offset) * 64),                   \
                                   (__attribute__((address_space(3))) uint32_t*)(dst + ((i) - offset) * 64), 16, offset * 1024, 0)
#pragma unroll
  for (int i = 0; i < PER; i += 4) {
    ARD_GDR_STAGE(i, 0);
    ARD_GDR_STAGE(i + 1, 1);
    ARD_GDR_STAGE(i + 2, 2);
    ARD_GDR_STAGE(i + 3, 3);
  }
#undef ARD_GDR_STAGE
}
// All of this wavefront's loads have ended but what came behind its last `later` accesses (a wavefront's accesses end in their order; the stores of a
// half chunk take longer than what was staged before them), and every wavefront's.
template <int LATER> __device__ __forceinline__ void all_landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LATER & 15) | (LATER >> 4) << 14 | 0x70);  // vmcnt(LATER) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// nothing moves past this: accesses are counted from here on
__device__ __forceinline__ void staged() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// Operands of a lower triangular 64 x 64 matrix: six tiles of 16 rows x 32 columns are not all zeros; of its transpose likewise.
__host__ __device__ constexpr int lower_frag(int rt, int kb) { return rt < 2 ? rt : 2 * rt - 2 + kb; }
__host__ __device__ constexpr int upper_frag(int rt, int kb) { return rt < 2 ? 2 * rt + kb : rt + 2; }

// What a chunk's steps are weighed by (0 behind the sequence's end, where keys, queries and write strengths are taken for 0).
struct Steps64 {
  double G[kChunk];     // sums of log(a) from the chunk's first step on
  float since[kChunk];  // exp(G_i)
  float still[kChunk];  // exp(G_last - G_i)
  float rk[kChunk], rq[kChunk];
  float w[kChunk], ka[kChunk], qa[kChunk], ke[kChunk];  // w, rk since, scale rq since, rk still: what the passes over the states read, 1 KB
  float whole;          // exp(G_last)
  float pad[127];
};
static_assert(sizeof(Steps64) == 3 * 1024, "it goes to LDS in whole KB");

struct GdrArgs {
  int T, B, Hk, H, Dk, Dv, group, chunks;
  ard_steps q, k, v, f, b;
  float scale, eps;
  const int32_t* len;
  // workspace: operands by (chunk, sequence, key head) and by (chunk, sequence, head)
  u32x4 *rows, *cols, *tri;  // K and Q; their transposes (Q's for the backward pass); M and P, or M and the transposes of M and P
  Steps64* steps;
  float *u, *dx, *ds;  // [64][dvp], [64][dvp], [dkp][dvp] of a chunk
  int dvp;
  int span, segments;   // chunks of a segment, and their number
  float *sums, *starts; // of a segment [DK][dvp + DK]: what it leaves of a state of zeros, and its transition; [DK][dvp]: the state before it
};
__device__ __forceinline__ int live_steps(const GdrArgs& a, int n) { return a.len ? imin(imax(a.len[n], 0), a.T) : a.T; }

template <typename T> constexpr int kInput = sizeof(T) == 2 ? 1 : 3;  // parts of an input

// KB of LDS that the operands of a walk over the chunks take, of keys of DK with IN parts: of both halves of a chunk, in which forward has K, Q, the columns of K, M and P (for
// sums no Q and no P), backward K, the columns of K and Q, and the transposes of M and P.  0: LDS does not hold them, they are read from the caches.
constexpr int walk_operands(bool backward, bool sum, int DK, int IN) {
  const int keys = DK / 8 * IN, m = 6 * 3, p = 6 * Operands<true>::PER, all = backward ? 3 * keys + 2 * m : 3 * keys + m + p;
  return all > 150 ? 0 : sum && !backward ? 2 * keys + m : all;
}

// exp(x), x <= 0: the argument's rounding costs |x| 2^-24 of it, and |x| < 104 where it is not 0
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float logistic(float x) {
  const float e = expf(-fabsf(x));
  return x >= 0.0f ? 1.0f / (1.0f + e) : e / (1.0f + e);
}

}  // namespace ard
