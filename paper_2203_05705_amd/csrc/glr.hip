// Gated linear recurrence: the cell of an LSTM without its recurrent products, so that time can be cut.
//
//   F = sigma(f), c_t = F_t c_{t-1} + (1 - F_t) v_t, h_t = sigma(o_t) c_t          (without o: h = c)
//   dc_t = sigma(o_t) dh_t + e_t, e_{t-1} = F_t dc_t, e_T = dcT
//   dv = dc (1 - F), df = dc (c_{t-1} - v) F (1 - F), do = dh c sigma(o) (1 - sigma(o)), dc0 = e_0
//
// Each step is affine in the state, so a stretch of steps is a pair (P, S): it takes c to P c + S, and stretches
// compose.  A wavefront takes 8 steps of 64 lanes' channels into registers, makes their pair there, and the wavefronts
// of a workgroup, which have neighbouring stretches, exchange pairs through LDS: every input is read once and every
// output written once, and that traffic is what bounds these passes.  8 steps, not 16: half the registers, twice the
// wavefronts whose loads are in flight (64 x 128 x 1024 bf16 with a gate: forward 16.6 us against 21.7); the forward pass asks for
// the next turn's steps while it works on one (14.7; the backward pass has no registers for it: 30 -> 33).
// Where batch and channels alone give too few wavefronts, time is cut into segments for several workgroups; a first pass
// then makes the segments' pairs (reading f and v, or f, o and dh, once more; a wavefront takes stretches that follow each other and
// meets the others only at the end), and the main pass composes those before its segment.  (One pass would have workgroups wait for others; the second reading comes partly out of the last cache.)
// A state in flight and the pairs that move it over 8 steps and more are fp64, everything inside a stretch fp32.  F of a long memory is so near 1
// that what rounding takes, from F or from a state that hardly moves, is the same at every step of a steady gate and adds up (in fp32
// what is left of a state after 32768 steps at f = 12 came out 1.8e-3 of itself off, 1e-7 so): P comes from 1 - P, a sum of positive terms with
// digits of its own.  The card's fp64 multiply-add takes no longer than its fp32 one; the reads from LDS cost 0 to 4 % of a pass.  The backward pass starts from the states that the forward pass left
// before every 8th step, so it needs no second scan for them.
// Lanes are counted through the sequences, so few channels a sequence fill wavefronts too: 4000 x 48 x 24 forward 23 us and backward 44
// against 47 and 64 with whole wavefronts for each sequence, 4000 x 47 x 192 82 and 130 against 93 and 156; where nothing is
// saved, sequences and addresses by lane cost the backward pass 1 to 5 % (64 x 128 x 1024).
//
// Measured, bf16 with a gate: 64 x 128 x 1024 forward 14.7 us, backward 26 behind it and 32 from memory (4.6, 3.7 TB/s; a large
// copy 4.9), fp32 32 and 55 from memory (4.1, 4.3 TB/s); 32768 x 1 x 1024 forward 25 + 51 us; 8192 x 4 x 1024 without one forward 27 + 42, backward
// 25 + 58; a single step of 128 sequences 2.8 us.
#include <type_traits>

#include "rows.hpp"

namespace ard {

constexpr int kSteps = ARD_GLR_CHUNK;  // steps of a wavefront's stretch, and between the states kept for the backward pass
constexpr int kMaxWaves = 8;           // stretches a workgroup has at a time

struct Strides {
  int64_t t, b;
};
struct GlrArgs {
  int T, B, H;      // H: channels that take part
  int wide;         // channels stored in f, v, o, h and their gradients: H, or pad8(H), zeros behind H
  int per_seq;      // lanes of a sequence
  int lanes;        // of all sequences
  int groups;       // wavefronts of 64 lanes that hold them
  int seg_steps;    // steps of a segment
  int segs;
  const int32_t* len;
};

// F = sigma(x), I = 1 - F from e = exp(-x), without cancellation: for x >= 0 as e F, where 1 - F would lose the digits of a long memory.
__device__ __forceinline__ float shut(float x) { return __builtin_amdgcn_exp2f(x * -1.44269504088896341f); }
__device__ __forceinline__ void gate_pair(float e, float& F, float& I) {
  F = __builtin_amdgcn_rcpf(1.0f + e);
  I = e <= 1.0f ? e * F : 1.0f - F;
}
__device__ __forceinline__ float gate(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504088896341f)); }

// Loads stay in front of this, in flight together: left to itself the compiler moves them next to their uses.
__device__ __forceinline__ void all_issued() { __builtin_amdgcn_sched_barrier(0); }

// What a workgroup works on.  Its wavefronts all have the same 64 lanes' channels, counted through the sequences (few channels
// a sequence still fill the lanes), at different steps.
struct GlrPlace {
  int seg;
  int b, ch;        // the lane's sequence and first channel; lanes behind the last one read what that reads and write nothing
  bool on;
  int n;            // of the lane's channels, those that states are kept of (H may end inside a lane's pair)
  int t0, t1;       // its steps
  int live, lo, hi; // steps before the sequence's end, up to T: the lane's, the least and the most of the wavefront
};
template <int VEC> __device__ __forceinline__ GlrPlace glr_place(const GlrArgs& a) {
  GlrPlace p;
  p.seg = blockIdx.x / a.groups;
  const int at = (blockIdx.x - p.seg * a.groups) * 64 + (threadIdx.x & 63), lane = imin(at, a.lanes - 1);
  p.on = at < a.lanes;
  p.b = (int)((unsigned)lane / (unsigned)a.per_seq);
  p.ch = (lane - p.b * a.per_seq) * VEC;
  p.n = p.on ? a.H - p.ch : 0;
  p.t0 = p.seg * a.seg_steps, p.t1 = imin(a.T - p.t0, a.seg_steps) + p.t0;
  p.live = p.lo = p.hi = a.T;
  if (a.len) {
    p.live = imin(imax(a.len[p.b], 0), a.T);
    p.lo = p.hi = __builtin_amdgcn_readfirstlane(p.live);
    if (__builtin_amdgcn_readlane(p.b, 0) != __builtin_amdgcn_readlane(p.b, 63))
      p.lo = a.T - (int)wave_max((uint32_t)(a.T - p.live)), p.hi = (int)wave_max((uint32_t)p.live);
  }
  return p;
}
// Steps of a stretch that begins at t before the ends of its sequences: the lane's own, and the least and the most of the
// wavefront's, the same for all of it (below 0 and above a stretch's steps as they come).
struct Steps {
  int mine, lo, hi;
  __device__ __forceinline__ Steps(const GlrPlace& p, int t) : mine(imin(p.t1, p.live) - t), lo(imin(p.t1, p.lo) - t), hi(imin(p.t1, p.hi) - t) {}
};

// A stretch (or segment) of steps: takes c to P c + S.
template <int VEC> struct Pair {
  double P[VEC], S[VEC];
};
// The same as it is made from the steps of a stretch, in fp32: Q = 1 - P beside P, each with its own digits.  (S is the caller's.)
template <int VEC> struct Steps8 {
  float P[VEC], Q[VEC], S[VEC];
  __device__ __forceinline__ Steps8() {
#pragma unroll
    for (int j = 0; j < VEC; ++j) P[j] = 1.0f, Q[j] = S[j] = 0.0f;
  }
  // one more step of gate F, I = 1 - F, before those that it has or behind them
  __device__ __forceinline__ void times(int j, float F, float I) {
    Q[j] = fmaf(I, P[j], Q[j]);
    P[j] *= F;
  }
  __device__ __forceinline__ double whole(int j) const { return P[j] >= 0.5f ? 1.0 - (double)Q[j] : (double)P[j]; }
};

// pairs of the wavefronts' stretches of a turn, in LDS
template <int VEC> struct Pairs {
  double v[2][kMaxWaves][2][VEC][64];  // [turn's parity][stretch][P, S]
  double c[2][VEC][64];                // [turn's parity]: the state behind the turn before it
};
// One wavefront moves the state over a whole turn and leaves it for the others' next one: written behind a turn's barrier, read behind the next one's, in
// the place that was read behind the barrier before.  (Where each did it for itself, 1000 x 16 x 1024 took 36.2 + 64.0 us, 34.9 + 62.0 so.)
template <int VEC> __device__ __forceinline__ void hand_on(Pairs<VEC>& s, int turn, const double (&c)[VEC]) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) s.c[turn][j][threadIdx.x & 63] = c[j];
}
template <int VEC> __device__ __forceinline__ void take(const Pairs<VEC>& s, int turn, double (&c)[VEC]) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) c[j] = s.c[turn][j][threadIdx.x & 63];
}

template <int VEC> __device__ __forceinline__ void apply(const Pairs<VEC>& s, int turn, int w, double (&c)[VEC]) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) c[j] = fma(s.v[turn][w][0][j][threadIdx.x & 63], c[j], s.v[turn][w][1][j][threadIdx.x & 63]);
}
template <int VEC> __device__ __forceinline__ void leave(Pairs<VEC>& s, int turn, int w, const Steps8<VEC>& m) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) s.v[turn][w][0][j][threadIdx.x & 63] = m.whole(j), s.v[turn][w][1][j][threadIdx.x & 63] = m.S[j];
}
// Pairs of many stretches, as a first pass makes them: a wavefront joins its own, which follow each other, and the first one the wavefronts'.
template <int VEC> __device__ __forceinline__ void join(Pair<VEC>& all, int j, double P, double S) {
  all.P[j] *= P, all.S[j] = fma(P, all.S[j], S);
}
template <int VEC> __device__ __forceinline__ void none(Pair<VEC>& all) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) all.P[j] = 1.0, all.S[j] = 0.0;
}
// Segment pairs in the workspace, fp32: [segment][A, S][B][H], A = P, or -(1 - P) with its sign set where P is 1/2 or more.  `all`: the
// wavefront's own; the workgroup's are joined from wavefront `from` on in steps of 1 or -1.
template <int VEC>
__device__ __forceinline__ void leave_segment(const GlrArgs& a, const GlrPlace& p, float* seg_pairs, Pair<VEC>& all, int from, int step, Pairs<VEC>& lds) {
  const int waves = blockDim.x >> 6, w = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < VEC; ++j) lds.v[0][w][0][j][threadIdx.x & 63] = all.P[j], lds.v[0][w][1][j][threadIdx.x & 63] = all.S[j];
  __syncthreads();
  if (w) return;
  none(all);
  for (int k = 0; k < waves; ++k)
#pragma unroll
    for (int j = 0; j < VEC; ++j) join(all, j, lds.v[0][from + step * k][0][j][threadIdx.x & 63], lds.v[0][from + step * k][1][j][threadIdx.x & 63]);
  float A[VEC], S[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) A[j] = all.P[j] >= 0.5 ? -(float)(1.0 - all.P[j]) : (float)all.P[j], S[j] = (float)all.S[j];
  float* out = seg_pairs + ((int64_t)p.seg * 2 * a.B + p.b) * a.H + p.ch;
  store_some<VEC>(out, p.n, A);
  store_some<VEC>(out + (int64_t)a.B * a.H, p.n, S);
}
// Composes those of segments [from, from + step * count) in order, dealt to the workgroup's wavefronts in neighbouring shares, and
// applies them to c (uses parity 0 of the pairs).
template <int VEC>
__device__ __forceinline__ void apply_segments(const GlrArgs& a, const GlrPlace& p, const float* seg_pairs, int from, int step, int count,
                                               Pairs<VEC>& lds, double (&c)[VEC]) {
  const int waves = blockDim.x >> 6, w = threadIdx.x >> 6;
  const int lo = (int)((int64_t)count * w / waves), hi = (int)((int64_t)count * (w + 1) / waves);
  const int64_t plane = (int64_t)a.B * a.H;
  Pair<VEC> m;
  none(m);
  for (int i0 = lo; i0 < hi; i0 += 4) {  // (four segments' pairs in flight)
    float q[4][VEC], r[4][VEC];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* at = seg_pairs + (int64_t)(from + step * imin(i0 + i, hi - 1)) * 2 * plane + (int64_t)p.b * a.H + p.ch;
      load_some<VEC>(at, p.n, q[i]);
      load_some<VEC>(at + plane, p.n, r[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i0 + i < hi) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const double P = (__float_as_int(q[i][j]) < 0 ? 1.0 : 0.0) + (double)q[i][j];
          join(m, j, P, (double)r[i][j]);
        }
      }
  }
#pragma unroll
  for (int j = 0; j < VEC; ++j) lds.v[0][w][0][j][threadIdx.x & 63] = m.P[j], lds.v[0][w][1][j][threadIdx.x & 63] = m.S[j];
  __syncthreads();
  if (w == 0) {
    for (int k = 0; k < waves; ++k) apply<VEC>(lds, 0, k, c);
    hand_on<VEC>(lds, 0, c);
  }
  __syncthreads();
  take<VEC>(lds, 0, c);
}

// Results.  CUT: of a launch whose inputs are read a second time, by way of the caches; results are kept from taking their room.
template <bool CUT, int VEC, typename T> __device__ __forceinline__ void put(T* p, const float (&x)[VEC]) {
  if constexpr (CUT) store_run_past<VEC>(p, x);
  else store_run<VEC>(p, x);
}

// ---- forward ------------------------------------------------------------------
// A stretch's values as they lie in memory; in the place of steps from `steps` (1 at least) on, which nobody looks at, those of the
// last one before (every register is written on every path, so loads stay in flight behind the branch).
template <typename T, int VEC> __device__ __forceinline__ void ask(const T* p, int64_t st, int steps, Raw<T, VEC> (&r)[kSteps]) {
  if (steps >= kSteps) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = load_raw<T, VEC>(p + i * st);
  } else {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = load_raw<T, VEC>(p + (int64_t)imin(i, steps - 1) * st);
  }
}

// F and (1 - F) v of a stretch's steps, and its pair.  WHOLE: all of its steps are live in all lanes; else those behind a
// lane's end leave the state as it is (selected, not multiplied: nothing that lies there takes part).
template <bool WHOLE, typename T, int VEC>
__device__ __forceinline__ void stretch_fwd(const Raw<T, VEC> (&rf)[kSteps], const Raw<T, VEC> (&rv)[kSteps], const Steps& n, float (&F)[kSteps][VEC],
                                            float (&b)[kSteps][VEC], Steps8<VEC>& m) {
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (WHOLE || i < n.hi) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float I;
        gate_pair(shut(part_of(rf[i], j)), F[i][j], I);
        b[i][j] = I * part_of(rv[i], j);
        if (!WHOLE) F[i][j] = i < n.mine ? F[i][j] : 1.0f, b[i][j] = i < n.mine ? b[i][j] : 0.0f, I = i < n.mine ? I : 0.0f;
        m.times(j, F[i][j], I);
        m.S[j] = fmaf(F[i][j], m.S[j], b[i][j]);
      }
    }
}

template <typename T, int VEC>
__global__ __launch_bounds__(64 * kMaxWaves) void glr_fwd_pairs_kernel(GlrArgs a, const T* f, const T* v, Strides z, float* seg_pairs) {
  __shared__ Pairs<VEC> lds;
  const GlrPlace p = glr_place<VEC>(a);
  const int waves = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t base = p.b * z.b + p.ch;
  Pair<VEC> all;
  none(all);
  Raw<T, VEC> rf[kSteps], rv[kSteps];
  auto ask_all = [&](int tw) {
    // (a stretch behind the end takes a step that is stored)
    const int from = imin(tw, a.T - 1), steps = imax(Steps(p, tw).hi, 1);
    const int64_t at = base + from * z.t;
    ask<T, VEC>(f + at, z.t, steps, rf), ask<T, VEC>(v + at, z.t, steps, rv);
    all_issued();
  };
  const int turns = (p.t1 - p.t0 + waves * kSteps - 1) / (waves * kSteps), first = p.t0 + w * turns * kSteps;
  ask_all(first);
  for (int i = 0; i < turns; ++i) {
    const int tw = first + i * kSteps;
    const Steps n(p, tw);
    float F[kSteps][VEC], b[kSteps][VEC];
    Steps8<VEC> m;
    if (n.lo >= kSteps) stretch_fwd<true, T, VEC>(rf, rv, n, F, b, m);
    else stretch_fwd<false, T, VEC>(rf, rv, n, F, b, m);
    if (i + 1 < turns) ask_all(tw + kSteps);  // (the next stretch's, in flight meanwhile)
#pragma unroll
    for (int j = 0; j < VEC; ++j) join(all, j, m.whole(j), (double)m.S[j]);
  }
  leave_segment<VEC>(a, p, seg_pairs, all, 0, 1, lds);
}

// results of a stretch whose state before it is s; zeros for those of its `stored` steps that lie behind a lane's end
template <bool WHOLE, typename T, int VEC, bool GATE, bool CUT>
__device__ __forceinline__ void stretch_out(T* h, int64_t st, bool on, const Steps& n, int stored, const float (&F)[kSteps][VEC], const float (&b)[kSteps][VEC],
                                            const Raw<T, VEC> (&g)[kSteps], float (&s)[VEC]) {
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (!WHOLE && i >= stored) break;
    float y[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) y[j] = 0.0f;
    if (WHOLE || i < n.hi) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = fmaf(F[i][j], s[j], b[i][j]);
        y[j] = GATE ? gate(part_of(g[i], j)) * s[j] : s[j];
        if (!WHOLE) y[j] = i < n.mine ? y[j] : 0.0f;
      }
    }
    if (on) put<CUT, VEC>(h + i * st, y);
  }
}

template <typename T, int VEC, bool GATE, bool CUT>
__global__ __launch_bounds__(64 * kMaxWaves) void glr_fwd_kernel(GlrArgs a, const T* f, const T* v, const T* o, Strides z, const float* c0, T* h,
                                                                 Strides hs, float* cT, float* ckpt, const float* seg_pairs) {
  __shared__ Pairs<VEC> lds;
  const GlrPlace p = glr_place<VEC>(a);
  const int waves = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t plane = (int64_t)a.B * a.H, state = (int64_t)p.b * a.H + p.ch;
  double c[VEC];
  {
    float start[VEC] = {};
    if (c0) load_some<VEC>(c0 + state, p.n, start);
#pragma unroll
    for (int j = 0; j < VEC; ++j) c[j] = start[j];
  }
  if (CUT && p.seg) apply_segments<VEC>(a, p, seg_pairs, 0, 1, p.seg, lds, c);
  const int64_t base = p.b * z.b + p.ch;
  Raw<T, VEC> rf[kSteps], rv[kSteps], rg[kSteps], g[kSteps];
  auto ask_all = [&](int tw) {
    // (a stretch behind the end takes a step that is stored)
    const int from = imin(tw, a.T - 1), steps = imax(Steps(p, tw).hi, 1);
    const int64_t at = base + from * z.t;
    ask<T, VEC>(f + at, z.t, steps, rf), ask<T, VEC>(v + at, z.t, steps, rv);
    if (GATE) ask<T, VEC>(o + at, z.t, steps, rg);
    all_issued();
  };
  int turn = 0;
  ask_all(p.t0 + w * kSteps);
  for (int t = p.t0; t < p.t1; t += waves * kSteps, turn ^= 1) {
    const int tw = t + w * kSteps;
    const Steps n(p, tw);
    float F[kSteps][VEC], b[kSteps][VEC], s[VEC];
    Steps8<VEC> m;
    if (n.lo >= kSteps) stretch_fwd<true, T, VEC>(rf, rv, n, F, b, m);
    else stretch_fwd<false, T, VEC>(rf, rv, n, F, b, m);
    if (GATE) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) g[i] = rg[i];
    }
    if (t + waves * kSteps < p.t1) ask_all(tw + waves * kSteps);  // (the next turn's, in flight meanwhile)
    if (waves > 1) {
      leave<VEC>(lds, turn, w, m);
      __syncthreads();
      if (w && t > p.t0) take<VEC>(lds, turn, c);
#pragma unroll 2
      for (int k = 0; k < w; ++k) apply<VEC>(lds, turn, k, c);
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = (float)c[j];
      if (w == 0) {
#pragma unroll 2
        for (int k = 0; k < waves; ++k) apply<VEC>(lds, turn, k, c);
        hand_on<VEC>(lds, turn ^ 1, c);
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = (float)c[j], c[j] = fma(m.whole(j), c[j], (double)m.S[j]);
    }
    if (tw < p.t1) {
      if (ckpt) store_some<VEC>(ckpt + (int64_t)(tw / kSteps) * plane + state, p.n, s);
      T* out = h + tw * hs.t + p.b * hs.b + p.ch;
      if (n.lo >= kSteps) stretch_out<true, T, VEC, GATE, CUT>(out, hs.t, p.on, n, kSteps, F, b, g, s);
      else stretch_out<false, T, VEC, GATE, CUT>(out, hs.t, p.on, n, p.t1 - tw, F, b, g, s);
    }
  }
  if (cT && w == 0 && p.seg == a.segs - 1) {
    float end[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) end[j] = (float)c[j];
    store_some<VEC>(cT + state, p.n, end);
  }
}

// One step, as generation calls it: a lane's channels of one sequence.  cT may be c0.
template <typename T, int VEC, bool GATE>
__global__ __launch_bounds__(64) void glr_step_kernel(GlrArgs a, const T* f, const T* v, const T* o, Strides z, const float* c0, T* h, Strides hs,
                                                      float* cT, float* ckpt) {
  const GlrPlace p = glr_place<VEC>(a);
  if (!p.on) return;
  const int64_t at = p.b * z.b + p.ch, state = (int64_t)p.b * a.H + p.ch;
  float c[VEC], x[VEC], u[VEC], g[VEC], y[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) c[j] = y[j] = 0.0f;
  if (c0) load_some<VEC>(c0 + state, p.n, c);
  if (ckpt) store_some<VEC>(ckpt + state, p.n, c);
  if (p.live > 0) {
    load_run<VEC>(f + at, x);
    load_run<VEC>(v + at, u);
    if (GATE) load_run<VEC>(o + at, g);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float F, I;
      const float e = shut(x[j]);
      gate_pair(e, F, I);
      c[j] = (float)fma(e <= 1.0f ? 1.0 - (double)I : (double)F, (double)c[j], (double)I * u[j]);
      y[j] = GATE ? gate(g[j]) * c[j] : c[j];
    }
  }
  store_run<VEC>(h + p.b * hs.b + p.ch, y);
  if (cT) store_some<VEC>(cT + state, p.n, c);
}

// ---- backward -----------------------------------------------------------------
// The adjoint's pair of a stretch takes e behind its last step to e behind the step before its first.
template <bool WHOLE, typename T, int VEC, bool GATE>
__device__ __forceinline__ void stretch_adjoint(const T* f, const T* o, const T* dh, int64_t st, int64_t dst, const Steps& n, Steps8<VEC>& m) {
  Raw<T, VEC> F[kSteps], q[kSteps], g[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (WHOLE || i < n.hi) {
      F[i] = load_raw<T, VEC>(f + i * st);
      q[i] = load_raw<T, VEC>(dh + i * dst);
      if (GATE) g[i] = load_raw<T, VEC>(o + i * st);
    }
  all_issued();
  float E[VEC] = {};  // 1 / P - 1, the (1 + e) multiplied less 1 (nobody looks at one past 1)
#pragma unroll
  for (int i = kSteps - 1; i >= 0; --i)
    if (WHOLE || i < n.hi) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float e = shut(part_of(F[i], j)), d = part_of(q[i], j);
        if (GATE) d *= gate(part_of(g[i], j));
        if (!WHOLE) e = i < n.mine ? e : 0.0f, d = i < n.mine ? d : 0.0f;
        const float x = __builtin_amdgcn_rcpf(1.0f + e);
        m.S[j] = x * (m.S[j] + d);
        m.P[j] *= x;
        E[j] = fmaf(e, E[j], e + E[j]);
      }
    }
#pragma unroll
  for (int j = 0; j < VEC; ++j) m.Q[j] = E[j] * __builtin_amdgcn_rcpf(1.0f + E[j]);
}

template <typename T, int VEC, bool GATE>
__global__ __launch_bounds__(64 * kMaxWaves) void glr_bwd_pairs_kernel(GlrArgs a, const T* f, const T* o, Strides z, const T* dh, Strides ds,
                                                                       const float* dcT, float* seg_pairs) {
  __shared__ Pairs<VEC> lds;
  const GlrPlace p = glr_place<VEC>(a);
  if (p.seg == 0) {  // nothing lies before it: its pair is not needed, and its place keeps a gradient that dc0 will be stored over
    if (dcT && threadIdx.x < 64) {
      float e[VEC];
      const int64_t state = (int64_t)p.b * a.H + p.ch;
      load_some<VEC>(dcT + state, p.n, e);
      store_some<VEC>(seg_pairs + state, p.n, e);
    }
    // Of many segments it is read all the same, for the last cache: alone without its inputs there it would be what the main launch waits for
    // (8192 x 4 x 1024 without a gate, 16 segments, 24 + 65 us in place of 24 + 57; 4608 x 24 x 256, 10, 31 + 81 and 32 + 71).  Of few that costs more than it
    // gives (1000 x 16 x 1000, 4, 21 + 51 us in place of 17 + 51; with 7 or 8 both take as long).
    if (a.segs < 8) return;
  }
  const int waves = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Pair<VEC> all;
  none(all);
  const int turns = (p.t1 - p.t0 + waves * kSteps - 1) / (waves * kSteps), first = p.t0 + w * turns * kSteps;
  for (int i = turns - 1; i >= 0; --i) {
    const int tw = first + i * kSteps;
    const Steps n(p, tw);
    const int64_t at = tw * z.t + p.b * z.b + p.ch, dat = tw * ds.t + p.b * ds.b + p.ch;
    Steps8<VEC> m;
    if (n.lo >= kSteps) stretch_adjoint<true, T, VEC, GATE>(f + at, o + at, dh + dat, z.t, ds.t, n, m);
    else stretch_adjoint<false, T, VEC, GATE>(f + at, o + at, dh + dat, z.t, ds.t, n, m);
#pragma unroll
    for (int j = 0; j < VEC; ++j) join(all, j, m.whole(j), (double)m.S[j]);
  }
  if (p.seg) leave_segment<VEC>(a, p, seg_pairs, all, waves - 1, -1, lds);
}

// Loads of a stretch, its states again from the one before it, and its adjoint's pair; do is stored on the way (it needs
// no gradient from later steps).  Leaves ex = exp(-f) (F and 1 - F are made from it again where they are wanted, as holding them would cost a
// workgroup of the two that a CU has registers for), u = c_{t-1} - v, and q = sigma(o) dh.
template <bool WHOLE, typename T, int VEC, bool GATE, bool CUT>
__device__ __forceinline__ void stretch_back(const T* f, const T* v, const T* o, const T* dh, T* dg, int64_t st, int64_t dst, int64_t gst, bool on, const Steps& n,
                                             float (&c)[VEC], float (&ex)[kSteps][VEC], float (&u)[kSteps][VEC], float (&q)[kSteps][VEC], Steps8<VEC>& m) {
  Raw<T, VEC> rf[kSteps], rv[kSteps], g[kSteps], rd[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (WHOLE || i < n.hi) {
      rf[i] = load_raw<T, VEC>(f + i * st);
      rv[i] = load_raw<T, VEC>(v + i * st);
      if (GATE) g[i] = load_raw<T, VEC>(o + i * st);
      rd[i] = load_raw<T, VEC>(dh + i * dst);
    }
  all_issued();
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (WHOLE || i < n.hi) {
      float y[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const bool live = WHOLE || i < n.mine;
        float F, I;
        ex[i][j] = shut(part_of(rf[i], j));
        if (!live) ex[i][j] = 0.0f;
        gate_pair(ex[i][j], F, I);
        const float x = part_of(rv[i], j);
        u[i][j] = c[j] - x;
        const float next = fmaf(F, c[j], I * x);
        c[j] = live ? next : c[j];
        q[i][j] = part_of(rd[i], j);
        if (GATE) {
          float O, N;
          gate_pair(shut(part_of(g[i], j)), O, N);
          q[i][j] *= O;
          y[j] = live ? q[i][j] * c[j] * N : 0.0f;
        }
        if (!live) q[i][j] = 0.0f;
        m.times(j, F, I);
        m.S[j] = fmaf(m.P[j], q[i][j], m.S[j]);
      }
      if (GATE && on) put<CUT, VEC>(dg + i * gst, y);
    }
}
// df and dv of a stretch, e behind its last step in s; zeros (do's too) for those of its `stored` steps behind a lane's end
template <bool WHOLE, typename T, int VEC, bool GATE, bool CUT>
__device__ __forceinline__ void stretch_grads(T* df, T* dv, T* dg, int64_t gst, bool on, const Steps& n, int stored, const float (&ex)[kSteps][VEC],
                                              const float (&u)[kSteps][VEC], const float (&q)[kSteps][VEC],
                                              float (&s)[VEC]) {
#pragma unroll
  for (int i = kSteps - 1; i >= 0; --i) {
    if (!WHOLE && i >= stored) continue;
    float x[VEC], y[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = y[j] = 0.0f;
    if (WHOLE || i < n.hi) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float dc = q[i][j] + s[j];
        float F, I;
        gate_pair(ex[i][j], F, I);
        s[j] = F * dc;
        y[j] = dc * I;
        x[j] = y[j] * F * u[i][j];
        if (!WHOLE) x[j] = i < n.mine ? x[j] : 0.0f, y[j] = i < n.mine ? y[j] : 0.0f;
      }
    } else if (GATE) {
      if (on) put<CUT, VEC>(dg + i * gst, x);
    }
    if (on) put<CUT, VEC>(df + i * gst, x), put<CUT, VEC>(dv + i * gst, y);
  }
}

template <typename T, int VEC, bool GATE, bool CUT>
__global__ __launch_bounds__(64 * kMaxWaves, 4) void glr_bwd_kernel(GlrArgs a, const T* f, const T* v, const T* o, Strides z, const float* ckpt, const T* dh,
                                                                 Strides ds, const float* dcT, T* df, T* dv, T* dg, Strides gs, float* dc0,
                                                                 const float* seg_pairs) {
  __shared__ Pairs<VEC> lds;
  const GlrPlace p = glr_place<VEC>(a);
  const int waves = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t plane = (int64_t)a.B * a.H, state = (int64_t)p.b * a.H + p.ch;
  double e[VEC];
  {
    float end[VEC] = {};
    if (dcT) load_some<VEC>(dcT + state, p.n, end);
#pragma unroll
    for (int j = 0; j < VEC; ++j) e[j] = end[j];
  }
  if (CUT && p.seg < a.segs - 1) apply_segments<VEC>(a, p, seg_pairs, a.segs - 1, -1, a.segs - 1 - p.seg, lds, e);
  const int span = waves * kSteps, turns = (p.t1 - p.t0 + span - 1) / span;
  int turn = 0;
  for (int t = p.t0 + (turns - 1) * span; t >= p.t0; t -= span, turn ^= 1) {
    const int tw = t + w * kSteps;
    const Steps n(p, tw);
    float ex[kSteps][VEC], u[kSteps][VEC], q[kSteps][VEC], c[VEC], s[VEC];
    Steps8<VEC> m;
    const int64_t at = tw * z.t + p.b * z.b + p.ch, dat = tw * ds.t + p.b * ds.b + p.ch, gat = tw * gs.t + p.b * gs.b + p.ch;
    if (n.hi > 0) load_some<VEC>(ckpt + (int64_t)(tw / kSteps) * plane + state, p.n, c);
    if (n.lo >= kSteps) stretch_back<true, T, VEC, GATE, CUT>(f + at, v + at, o + at, dh + dat, dg + gat, z.t, ds.t, gs.t, p.on, n, c, ex, u, q, m);
    else stretch_back<false, T, VEC, GATE, CUT>(f + at, v + at, o + at, dh + dat, dg + gat, z.t, ds.t, gs.t, p.on, n, c, ex, u, q, m);
    if (waves > 1) {
      leave<VEC>(lds, turn, w, m);
      __syncthreads();
      const bool last = w == waves - 1;
      if (!last && t + span < p.t1) take<VEC>(lds, turn, e);
#pragma unroll 2
      for (int k = waves - 1; k > w; --k) apply<VEC>(lds, turn, k, e);
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = (float)e[j];
      if (last) {
#pragma unroll 2
        for (int k = waves - 1; k >= 0; --k) apply<VEC>(lds, turn, k, e);
        hand_on<VEC>(lds, turn ^ 1, e);
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = (float)e[j], e[j] = fma(m.whole(j), e[j], (double)m.S[j]);
    }
    if (n.lo >= kSteps) stretch_grads<true, T, VEC, GATE, CUT>(df + gat, dv + gat, dg + gat, gs.t, p.on, n, kSteps, ex, u, q, s);
    else stretch_grads<false, T, VEC, GATE, CUT>(df + gat, dv + gat, dg + gat, gs.t, p.on, n, p.t1 - tw, ex, u, q, s);
  }
  if (dc0 && w == waves - 1 && p.seg == 0) {
    float start[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) start[j] = (float)e[j];
    store_some<VEC>(dc0 + state, p.n, start);
  }
}

// ---- host ---------------------------------------------------------------------
struct GlrPlan {
  GlrArgs a;
  int waves, vec;
};
static GlrPlan glr_plan(int32_t dtype, int T, int B, int H, int32_t flags, const int32_t* len) {
  const int wide = flags ? pad8(H) : H, pieces = T / kSteps + (T % kSteps != 0), waves = imin(pieces, kMaxWaves);
  const auto groups_of = [&](int vec) { return ((int64_t)B * (wide / vec) + 63) / 64; };
  GlrPlan g{};
  g.vec = 1;
  if (dtype == ARD_BF16 && wide % 2 == 0) {
    // Two channels a lane, 256 bytes a wavefront's row, as one's 128 fetch less well (64 x 128 x 1024 forward and backward 14.8 + 31.8 us,
    // 14.8 + 36.7 with one; 4000 x 47 x 192 82 + 130, 92 + 146).  One where that leaves fewer than 8 stretches a CU, as a lane's two come one
    // after the other (130 x 8 x 512 8.4 + 11.3, 6.9 + 8.8 with one; 1000 x 8 x 512, which has 16, takes as long either way), and
    // where one fills the CUs with wavefronts and two would not (224 x 16 x 1024 12.6 + 19.1, 9.7 + 15.4; 4000: 149 + 244, 128 + 230).
    const int64_t two = groups_of(2);
    g.vec = two * pieces <= 2048 || (two * waves < 2048 && groups_of(1) * waves >= 2048) ? 1 : 2;
  }
  const int64_t lanes = (int64_t)B * (wide / g.vec);
  g.a.T = T, g.a.B = B, g.a.H = H, g.a.wide = wide, g.a.len = len;
  if (lanes > INT32_MAX - 64) return g;  // (refused: no wavefronts)
  g.waves = waves;
  g.a.per_seq = wide / g.vec, g.a.lanes = (int)lanes, g.a.groups = (int)groups_of(g.vec);
  const int64_t have = (int64_t)g.a.groups * g.waves;  // wavefronts without cutting time
  const int turns = ceil_div(pieces, g.waves);
  int segs = 1;
  // Time is cut below 8 wavefronts a CU, into 16 a CU: with half as many 32768 x 1 x 1024 takes 87 us (81), 8192 x 4 x 1024 without a gate 77 + 102 (73 + 96);
  // with twice as many 87 and 75 + 99, as more pairs are read.  (Where there are few bytes, half as many would do: 4000 x 48 x 24 20 + 38, 23 + 44 so.)
  // The second launch is worth four turns of 64 steps where there is little work (bf16 192 x 8 x 512 forward and backward 7.5 + 10.4 us in
  // one launch, 9.4 + 10.3 in two; 256: 8.6 + 13.5, 8.9 + 10.5), the second reading eight where there is more (320 x 16 x 1000 16.2 + 25.7,
  // 17.1 + 25.4; 1000: 50 + 93, 48 + 80).
  if (have < 2048 && turns >= (have <= 512 ? 4 : 8)) segs = imin(turns, (int)(4096 / have));
  const int per = ceil_div(turns, segs);
  g.a.segs = ceil_div(turns, per);
  g.a.seg_steps = per * g.waves * kSteps;
  return g;
}
static size_t glr_ws_bytes(const GlrArgs& a) { return a.segs > 1 ? (size_t)a.segs * 2 * a.B * a.H * sizeof(float) : 0; }

struct GlrCall {
  GlrPlan g;
  const void *f, *v, *o;
  Strides z;
};

static int32_t glr_check(int32_t dtype, int32_t T, int32_t B, int32_t H, int32_t flags) {
  if (dtype != ARD_F32 && dtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", dtype);
  if (T <= 0 || B <= 0 || H <= 0) return fail(ARD_ESHAPE, "T, B and H must be positive (got %d, %d, %d)", T, B, H);
  if (T > 1 << 30 || H > 1 << 24) return fail(ARD_ESHAPE, "T = %d or H = %d is too large", T, H);
  if (flags != 0 && flags != (ARD_IN_COMPACT | ARD_OUT_COMPACT)) return fail(ARD_EINVAL, "flags are 0 or ARD_IN_COMPACT | ARD_OUT_COMPACT (got 0x%x)", flags);
  return ARD_OK;
}
static int32_t glr_check_grid(const GlrPlan& g) {  // (HIP counts a grid's threads in 32 bits)
  if (!g.waves || (int64_t)g.a.groups * g.a.segs * g.waves >= 1 << 26) return fail(ARD_ESHAPE, "B * H is too large (%d, %d)", g.a.B, g.a.H);
  return ARD_OK;
}

// The one shape of all these launches: every wavefront's worth of lanes, segment by segment (what glr_place takes apart; a
// workgroup of a segment that does not exist would read behind the segments' pairs).
static dim3 glr_grid(const GlrArgs& a, int segs) { return dim3((unsigned)a.groups * (unsigned)segs); }

// (a dry run's log says the grid, the lanes' wavefronts and the segments)
#define ARD_GLR_LAUNCH(name, kernel, grid, ...) ARD_LAUNCH_NAMED(launch_instance(name, (int)(grid).x, a.groups, a.segs), kernel, grid, __VA_ARGS__)

template <typename T, int VEC, bool GATE>
static int32_t glr_fwd_t(const GlrCall& c, const float* c0, void* h, Strides hs, float* cT, float* ckpt, float* ws, hipStream_t st) {
  const GlrArgs& a = c.g.a;
  const T *f = (const T*)c.f, *v = (const T*)c.v, *o = (const T*)c.o;
  if (a.T == 1) {
    ARD_GLR_LAUNCH("glr_step_kernel", (glr_step_kernel<T, VEC, GATE>), glr_grid(a, 1), dim3(64), 0, st, a, f, v, o, c.z, c0, (T*)h, hs, cT, ckpt);
    ARD_LAUNCH_CHECK("glr_step_kernel");
    return ARD_OK;
  }
  const dim3 block(64 * c.g.waves);
  if (a.segs > 1) {  // (the last segment's pair is not needed)
    ARD_GLR_LAUNCH("glr_fwd_pairs_kernel", (glr_fwd_pairs_kernel<T, VEC>), glr_grid(a, a.segs - 1), block, 0, st, a, f, v, c.z, ws);
    ARD_LAUNCH_CHECK("glr_fwd_pairs_kernel");
  }
  const dim3 grid = glr_grid(a, a.segs);
  if (a.segs > 1) ARD_GLR_LAUNCH("glr_fwd_kernel", (glr_fwd_kernel<T, VEC, GATE, true>), grid, block, 0, st, a, f, v, o, c.z, c0, (T*)h, hs, cT, ckpt, ws);
  else ARD_GLR_LAUNCH("glr_fwd_kernel", (glr_fwd_kernel<T, VEC, GATE, false>), grid, block, 0, st, a, f, v, o, c.z, c0, (T*)h, hs, cT, ckpt, nullptr);
  ARD_LAUNCH_CHECK("glr_fwd_kernel");
  return ARD_OK;
}

template <typename T, int VEC, bool GATE>
static int32_t glr_bwd_t(const GlrCall& c, const float* ckpt, const void* dh, Strides ds, const float* dcT, void* df, void* dv, void* dg, Strides gs,
                         float* dc0, float* ws, hipStream_t st) {
  const GlrArgs& a = c.g.a;
  const T *f = (const T*)c.f, *v = (const T*)c.v, *o = (const T*)c.o;
  const dim3 block(64 * c.g.waves);
  if (a.segs > 1) {
    // Every segment's workgroups of the main launch begin with dcT; the first segment's store dc0.  Where the two are one, dcT is kept for them by the
    // first segment's workgroups of this launch, which make no pair.
    const float* keep = dcT && dcT == dc0 ? dcT : nullptr;
    ARD_GLR_LAUNCH("glr_bwd_pairs_kernel", (glr_bwd_pairs_kernel<T, VEC, GATE>), glr_grid(a, a.segs), block, 0, st, a, f, o, c.z, (const T*)dh, ds, keep, ws);
    ARD_LAUNCH_CHECK("glr_bwd_pairs_kernel");
    if (keep) dcT = ws;
  }
  const dim3 grid = glr_grid(a, a.segs);
  if (a.segs > 1)
    ARD_GLR_LAUNCH("glr_bwd_kernel", (glr_bwd_kernel<T, VEC, GATE, true>), grid, block, 0, st, a, f, v, o, c.z, ckpt, (const T*)dh, ds, dcT, (T*)df, (T*)dv,
                   (T*)dg, gs, dc0, ws);
  else
    ARD_GLR_LAUNCH("glr_bwd_kernel", (glr_bwd_kernel<T, VEC, GATE, false>), grid, block, 0, st, a, f, v, o, c.z, ckpt, (const T*)dh, ds, dcT, (T*)df, (T*)dv,
                   (T*)dg, gs, dc0, nullptr);
  ARD_LAUNCH_CHECK("glr_bwd_kernel");
  return ARD_OK;
}

template <class F> static int32_t glr_instance(int32_t dtype, int vec, F&& with) {
  using One = std::integral_constant<int, 1>;
  if (dtype == ARD_F32) return with(0.0f, One{});
  return vec == 1 ? with((uint16_t)0, One{}) : with((uint16_t)0, std::integral_constant<int, 2>{});
}

}  // namespace ard

using namespace ard;

extern "C" int32_t ard_glr_chunk(void) { return kSteps; }

extern "C" size_t ard_glr_workspace_bytes(int32_t dtype, int32_t T, int32_t B, int32_t H) {
  if (dtype < 0 || dtype > ARD_BF16 || T <= 0 || B <= 0 || H <= 0 || T > 1 << 30 || H > 1 << 24) return 0;
  // (channels may be stored in H or in pad8(H) columns, dealt to different numbers of workgroups)
  const size_t n = glr_ws_bytes(glr_plan(dtype, T, B, H, 0, nullptr).a), m = glr_ws_bytes(glr_plan(dtype, T, B, H, ARD_IN_COMPACT | ARD_OUT_COMPACT, nullptr).a);
  return n > m ? n : m;
}

extern "C" int32_t ard_glr_fwd(int32_t dtype, int32_t T, int32_t B, int32_t H, const void* f, const void* v, const void* o, int64_t z_t, int64_t z_b,
                               const float* c0, const int32_t* d_lengths, void* h, int64_t h_t, int64_t h_b, float* cT, float* ckpt, int32_t flags,
                               void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = glr_check(dtype, T, B, H, flags)) return st;
  if (!f || !v || !h) return fail(ARD_EINVAL, "null tensor pointer");
  if (c0 && cT == c0 && T > 1) return fail(ARD_EINVAL, "cT may take the place of c0 for a single step only");
  const size_t es = dtype == ARD_F32 ? 4 : 2;
  if (misaligned(f, es) || misaligned(v, es) || misaligned(o, es) || misaligned(h, es) || misaligned(c0, 4) || misaligned(cT, 4) || misaligned(ckpt, 4) ||
      misaligned(d_lengths, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const GlrCall c{glr_plan(dtype, T, B, H, flags, d_lengths), f, v, o, {z_t, z_b}};
  if (int32_t st = glr_check_grid(c.g)) return st;
  const size_t need = glr_ws_bytes(c.g.a);
  if (need && (!ws || ws_bytes < need || misaligned(ws, 4))) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws ? ws_bytes : 0);
  const Strides hs{h_t, h_b};
  hipStream_t st = (hipStream_t)stream;
  auto with = [&](auto t, auto vec) {
    using E = decltype(t);
    constexpr int N = decltype(vec)::value;
    return o ? glr_fwd_t<E, N, true>(c, c0, h, hs, cT, ckpt, (float*)ws, st) : glr_fwd_t<E, N, false>(c, c0, h, hs, cT, ckpt, (float*)ws, st);
  };
  return glr_instance(dtype, c.g.vec, with);
}

extern "C" int32_t ard_glr_bwd(int32_t dtype, int32_t T, int32_t B, int32_t H, const void* f, const void* v, const void* o, int64_t z_t, int64_t z_b,
                               const int32_t* d_lengths, const float* ckpt, const void* dh, int64_t dh_t, int64_t dh_b, const float* dcT, void* df,
                               void* dv, void* dout, int64_t dz_t, int64_t dz_b, float* dc0, int32_t flags, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = glr_check(dtype, T, B, H, flags)) return st;
  if (!f || !v || !ckpt || !dh || !df || !dv || (o && !dout)) return fail(ARD_EINVAL, "null tensor pointer");
  if (!o && dout) return fail(ARD_EINVAL, "a gradient of o is asked for, but there is no o");
  const size_t es = dtype == ARD_F32 ? 4 : 2;
  if (misaligned(f, es) || misaligned(v, es) || misaligned(o, es) || misaligned(dh, es) || misaligned(df, es) || misaligned(dv, es) || misaligned(dout, es) ||
      misaligned(ckpt, 4) || misaligned(dcT, 4) || misaligned(dc0, 4) || misaligned(d_lengths, 4))
    return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const GlrCall c{glr_plan(dtype, T, B, H, flags, d_lengths), f, v, o, {z_t, z_b}};
  if (int32_t st = glr_check_grid(c.g)) return st;
  const size_t need = glr_ws_bytes(c.g.a);
  if (need && (!ws || ws_bytes < need || misaligned(ws, 4))) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws ? ws_bytes : 0);
  const Strides ds{dh_t, dh_b}, gs{dz_t, dz_b};
  hipStream_t st = (hipStream_t)stream;
  auto with = [&](auto t, auto vec) {
    using E = decltype(t);
    constexpr int N = decltype(vec)::value;
    return o ? glr_bwd_t<E, N, true>(c, ckpt, dh, ds, dcT, df, dv, dout, gs, dc0, (float*)ws, st)
             : glr_bwd_t<E, N, false>(c, ckpt, dh, ds, dcT, df, dv, dout, gs, dc0, (float*)ws, st);
  };
  return glr_instance(dtype, c.g.vec, with);
}
