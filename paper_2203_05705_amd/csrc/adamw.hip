// AdamW over many tensors in one launch, states in 32 bits or in 8.
//
//   g' = scale g, m = b1 m + (1 - b1) g', v = b2 v + (1 - b2) g'^2, p = (1 - lr wd) p - lr' m / (sqrt(v) r2 + eps)
//   with lr' = lr / (1 - b1^t) and r2 = 1 / sqrt(1 - b2^t)
//
// Bound by memory: a parameter costs 28 bytes with 32-bit states and fp32 gradients, 14 with 8-bit states and bf16
// gradients (16 with a bf16 copy): 67M parameters of the latter kind take 208 us, 5.2 TB/s, and 16.8M of the former 93 us, 5.0 TB/s.  A wavefront takes a block of 256 neighbouring elements, four a lane in 16-byte accesses; that is also
// the block that shares the scales of an 8-bit state, so its largest m and v are maxima over a wavefront's registers and
// the state is read, updated and written in one pass.  The tensors' table travels in the kernel's arguments.
#include <math.h>

#include <type_traits>

#include "rows.hpp"

namespace ard {

constexpr int kBlock = ARD_ADAMW_BLOCK;
static_assert(kBlock == 256, "a wavefront's four elements a lane");
constexpr int chunk_of(int blocks) { return 4 * blocks * kBlock; }         // elements of a workgroup of four wavefronts
constexpr int kMaxTensors = 48;                                           // of a launch: 64 bytes each, in 4 KB of arguments

struct AdamTable {
  int count;
  int chunk0[kMaxTensors + 1];  // first workgroup of each tensor
  ard_adamw_tensor t[kMaxTensors];
};
struct AdamConsts {
  float b1, b2, omb1, omb2;  // 1 - b1, 1 - b2, rounded from the doubles' differences
  float keep, lr, r2, eps;   // 1 - lr wd, lr', r2
  const float* scale;
};

// the tensor that a workgroup belongs to
__device__ __forceinline__ int tensor_at(const int* chunk0, int count, int chunk) {
  int lo = 0, hi = count;  // chunk0[lo] <= chunk < chunk0[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chunk0[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// One element's step, each operation rounded (no fused multiply-add): the new m and v decide 8-bit codes, which are to be
// the same for everybody who computes the stated formula in fp32.
__device__ __forceinline__ void adam_states(const AdamConsts& k, float g, float& m, float& v) {
#pragma clang fp contract(off)
  m = m * k.b1 + g * k.omb1;
  v = v * k.b2 + (g * g) * k.omb2;
}
__device__ __forceinline__ float adam_param(const AdamConsts& k, float p, float m, float v) {
  // (the root's instruction takes what is below the smallest normal number for 0: such a v is scaled up before it)
  const bool tiny = v < 0x1p-100f;
  const float root = fmaf(__builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v), tiny ? k.r2 * 0x1p-32f : k.r2, k.eps);
  return fmaf(-k.lr * m, __builtin_amdgcn_rcpf(root), p * k.keep);
}

// ---- 8-bit states --------------------------------------------------------------
// value = (c/127) |c/127| top;  value = (c/255)^4 top
__device__ __forceinline__ float decode_m(int c, float top) {
#pragma clang fp contract(off)
  const float t = (float)c * (float)(1.0 / 127.0);
  return t * fabsf(t) * top;
}
__device__ __forceinline__ float decode_v(uint32_t c, float top) {
#pragma clang fp contract(off)
  float t = (float)c * (float)(1.0 / 255.0);
  t = t * t;
  return t * t * top;
}
// (a top below the smallest normal number has no reciprocal to scale by: its block is held as zeros; codes of a block whose top is
// no number are zeros, which its top makes NaN)
__device__ __forceinline__ float share_of(float top) { return top >= 1.17549435e-38f && top <= 3.4028234e38f ? 1.0f / top : 0.0f; }
// sqrt(x) of 0 < x <= 1 rounded to nearest, as sqrtf gives it: a reciprocal root of 1 ulp, then the root's residual (exact in one
// fused multiply-add) times half of it.  A fifth of sqrtf's instructions, which scales for the smallest numbers and sorts out
// the others; the same bits for every x from 1e-24 to 1.
__device__ __forceinline__ float root_of_share(float x) {
  const float y = __builtin_amdgcn_rsqf(x), s = x * y;
  return fmaf(fmaf(-s, s, x), 0.5f * y, s);
}
constexpr float kLeast = 1e-24f;    // shares below it have code 0 (and need no root): 127 sqrt(x) and 255 x^(1/4) are below 1/2
constexpr float kRound = 12582912;  // 1.5 * 2^23: a sum with it is a whole number, ties to even, in its low bits (two's complement)
__device__ __forceinline__ uint32_t low_bytes(const float (&z)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(z[1]), __float_as_uint(z[0]), 0x0c0c0400u);
  const uint32_t b = __builtin_amdgcn_perm(__float_as_uint(z[3]), __float_as_uint(z[2]), 0x04000c0cu);
  return a | b;
}
// Four codes, bytes from low to high.  (Whatever a NaN or infinity leaves in the bytes is dropped: its block has no inv.)
__device__ __forceinline__ uint32_t encode_m(const float (&m)[4], float inv) {
#pragma clang fp contract(off)
  float z[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) z[j] = root_of_share(fmaxf(fabsf(m[j]) * inv, kLeast)) * copysignf(127.0f, m[j]) + kRound;
  return inv > 0.0f ? low_bytes(z) : 0u;
}
__device__ __forceinline__ uint32_t encode_v(const float (&v)[4], float inv) {
#pragma clang fp contract(off)
  float z[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float r = root_of_share(root_of_share(fmaxf(v[j] * inv, kLeast))) * 255.0f;
    z[j] = (v[j] > 0.0f ? fmaxf(r, 1.0f) : r) + kRound;
  }
  return inv > 0.0f ? low_bytes(z) : 0u;
}
// Four codes of a lane (bytes from low to high); a lane with fewer elements takes and leaves its bytes one by one.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
  typedef uint32_t u32 __attribute__((aligned(1)));
  if (n >= 4) return *reinterpret_cast<const u32*>(p);
  uint32_t c = 0;
  for (int j = 0; j < n; ++j) c |= (uint32_t)p[j] << (8 * j);
  return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, uint32_t c) {
  typedef uint32_t u32 __attribute__((aligned(1)));
  if (n >= 4) {
    *reinterpret_cast<u32*>(p) = c;
    return;
  }
  for (int j = 0; j < n; ++j) p[j] = (uint8_t)(c >> (8 * j));
}

// BLOCKS of a wavefront, one after another.
template <typename G, bool EIGHT, int BLOCKS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamTable tab, AdamConsts k) {
  float scale = 1.0f;
  if (k.scale) {
    scale = *k.scale;
    if (!(fabsf(scale) <= 3.4028234e38f)) return;  // (the step is skipped)
  }
  const int i = tensor_at(tab.chunk0, tab.count, blockIdx.x);
  const ard_adamw_tensor t = tab.t[i];
  const int64_t first = (int64_t)((int)blockIdx.x - tab.chunk0[i]) * chunk_of(BLOCKS);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < BLOCKS; ++r) {
    const int64_t block = first + (w * BLOCKS + r) * kBlock;
    if (block >= t.n) return;
    const int64_t at = block + lane * 4;
    const int n = t.n - at >= 4 ? 4 : (int)(t.n - at);  // (may be negative)
    float p[4], g[4], m[4], v[4];
    load_some<4>(t.p + at, n, p);
    load_some<4>((const G*)t.g + at, n, g);
    if constexpr (EIGHT) {
      const uint32_t mc = load_codes((const uint8_t*)t.m + at, n), vc = load_codes((const uint8_t*)t.v + at, n);
      const float mt = t.m_scale[block / kBlock], vt = t.v_scale[block / kBlock];
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = decode_m((int)(int8_t)(mc >> (8 * j)), mt), v[j] = decode_v(vc >> (8 * j) & 255u, vt);
    } else {
      load_some<4>((const float*)t.m + at, n, m);
      load_some<4>((const float*)t.v + at, n, v);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      adam_states(k, g[j] * scale, m[j], v[j]);
      p[j] = adam_param(k, p[j], m[j], v[j]);
    }
    store_some<4>(t.p + at, n, p);
    if (t.w) store_some<4>((uint16_t*)t.w + at, n, p);
    if constexpr (EIGHT) {
      // maxima of magnitudes as bit patterns, among which a NaN is larger than every number and so is not lost; lanes
      // without elements have decoded zeros (codes 0) and gradients 0: with a NaN scale they are NaN as their block is
      uint32_t mb = 0, vb = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t a = __float_as_uint(m[j]) & 0x7fffffffu, b = __float_as_uint(v[j]) & 0x7fffffffu;
        mb = a > mb ? a : mb, vb = b > vb ? b : vb;
      }
      const float mt = __uint_as_float(wave_max(mb)), vt = __uint_as_float(wave_max(vb));
      store_codes((uint8_t*)t.m + at, n, encode_m(m, share_of(mt)));
      store_codes((uint8_t*)t.v + at, n, encode_v(v, share_of(vt)));
      if (lane == 0) t.m_scale[block / kBlock] = mt, t.v_scale[block / kBlock] = vt;
    } else {
      store_some<4>((float*)t.m + at, n, m);
      store_some<4>((float*)t.v + at, n, v);
    }
  }
}

// the values of 8-bit states; the table's p and w hold the places for those of m and v
__global__ __launch_bounds__(256) void adamw_values_kernel(AdamTable tab) {
  const int i = tensor_at(tab.chunk0, tab.count, blockIdx.x);
  const ard_adamw_tensor t = tab.t[i];
  const int64_t first = (int64_t)((int)blockIdx.x - tab.chunk0[i]) * chunk_of(1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t block = first + w * kBlock;
  if (block >= t.n) return;
  const int64_t at = block + lane * 4;
  const int n = t.n - at >= 4 ? 4 : (int)(t.n - at);
  const uint32_t mc = load_codes((const uint8_t*)t.m + at, n), vc = load_codes((const uint8_t*)t.v + at, n);
  const float mt = t.m_scale[block / kBlock], vt = t.v_scale[block / kBlock];
  float m[4], v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = decode_m((int)(int8_t)(mc >> (8 * j)), mt), v[j] = decode_v(vc >> (8 * j) & 255u, vt);
  store_some<4>(t.p + at, n, m);
  store_some<4>((float*)t.w + at, n, v);
}

// Deals the tensors that have elements over launches of up to kMaxTensors; `launch` issues one, `advance` moves a tensor's
// pointers behind a part of it.
template <class A, class F> static int32_t adam_launches(int32_t count, const ard_adamw_tensor* tensors, int chunk, A&& advance, F&& launch) {
  AdamTable tab{};
  int64_t chunks = 0;
  auto flush = [&]() -> int32_t {
    if (!tab.count) return ARD_OK;
    tab.chunk0[tab.count] = (int)chunks;
    const int32_t st = launch(tab, (int)chunks);
    tab.count = 0, chunks = 0;
    return st;
  };
  for (int i = 0; i < count; ++i) {
    ard_adamw_tensor t = tensors[i];
    while (t.n > 0) {
      // (a launch holds up to 2^23 workgroups: HIP counts a grid's threads in 32 bits; a longer tensor is dealt to several)
      const int64_t room = (1 << 23) - chunks, need = (t.n + chunk - 1) / chunk, take = need < room ? need : room;
      if (tab.count == kMaxTensors || take == 0) {
        if (int32_t st = flush()) return st;
        continue;
      }
      tab.chunk0[tab.count] = (int)chunks;
      tab.t[tab.count] = t;
      const int64_t part = take < need ? take * chunk : t.n;
      tab.t[tab.count++].n = part;
      chunks += take;
      t.n -= part;
      if (t.n) advance(t, part);
    }
  }
  return flush();
}

static int32_t adam_tensor_check(const ard_adamw_tensor& t, int i, bool eight, size_t gs) {
  if (t.n < 0) return fail(ARD_ESHAPE, "tensor %d has %lld elements", i, (long long)t.n);
  if (t.n == 0) return ARD_OK;
  if (!t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return fail(ARD_EINVAL, "tensor %d: null state pointer", i);
  if (!eight && (t.m_scale || t.v_scale)) return fail(ARD_EINVAL, "tensor %d: 32-bit states have no scales", i);
  if (gs && (!t.p || !t.g)) return fail(ARD_EINVAL, "tensor %d: null tensor pointer", i);
  if (misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4) || (!eight && (misaligned(t.m, 4) || misaligned(t.v, 4))) ||
      (gs && (misaligned(t.p, 4) || misaligned(t.g, gs) || misaligned(t.w, 2))))
    return fail(ARD_EINVAL, "tensor %d does not start at a whole element", i);
  return ARD_OK;
}

}  // namespace ard

using namespace ard;

extern "C" int32_t ard_adamw_step(int32_t bits, int32_t gdtype, int32_t count, const ard_adamw_tensor* tensors, double lr, double beta1, double beta2,
                                  double eps, double weight_decay, int64_t step, const float* d_grad_scale, void* stream) {
  if (bits != 32 && bits != 8) return fail(ARD_EINVAL, "states have 32 or 8 bits (got %d)", bits);
  if (gdtype != ARD_F32 && gdtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", gdtype);
  if (count < 0) return fail(ARD_ESHAPE, "negative number of tensors");
  if (count && !tensors) return fail(ARD_EINVAL, "null tensor table");
  if (!(lr >= 0.0 && lr <= 1e30) || !(weight_decay >= 0.0 && weight_decay <= 1e30)) return fail(ARD_EINVAL, "lr and weight_decay must not be negative (got %g, %g)", lr, weight_decay);
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return fail(ARD_EINVAL, "betas must lie in [0, 1) (got %g, %g)", beta1, beta2);
  if (!(eps >= 1e-37 && eps <= 1e30)) return fail(ARD_EINVAL, "eps must be positive (got %g)", eps);
  if (step < 1) return fail(ARD_EINVAL, "steps count from 1 (got %lld)", (long long)step);
  if (misaligned(d_grad_scale, 4)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  for (int i = 0; i < count; ++i)
    if (int32_t st = adam_tensor_check(tensors[i], i, bits == 8, gdtype == ARD_F32 ? 4 : 2)) return st;
  const AdamConsts k{(float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2), (float)(1.0 - lr * weight_decay),
                     (float)(lr / (1.0 - pow(beta1, (double)step))), (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step))), (float)eps, d_grad_scale};
  hipStream_t st = (hipStream_t)stream;
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += tensors[i].n;
  // Four blocks a wavefront cost one look at the table for four, but leave CUs without work where there is little: 868k parameters
  // 7.6 us against 6.9 with one, 1M with 8-bit states 9.6 against 6.9; from 4M on the two are within 1 %.
  const bool few = total < (1 << 22);
  return adam_launches(
      count, tensors, chunk_of(few ? 1 : 4),
      [&](ard_adamw_tensor& t, int64_t part) {
        t.p += part, t.g = (const char*)t.g + part * (gdtype == ARD_F32 ? 4 : 2);
        t.m = (char*)t.m + part * (bits / 8), t.v = (char*)t.v + part * (bits / 8);
        if (bits == 8) t.m_scale += part / kBlock, t.v_scale += part / kBlock;
        if (t.w) t.w = (char*)t.w + part * 2;
      },
      [&](const AdamTable& tab, int chunks) -> int32_t {
        auto with = [&](auto g, auto eight) {
          using G = decltype(g);
          if (few) ARD_LAUNCH((adamw_kernel<G, eight.value, 1>), dim3(chunks), dim3(256), 0, st, tab, k);
          else ARD_LAUNCH((adamw_kernel<G, eight.value, 4>), dim3(chunks), dim3(256), 0, st, tab, k);
        };
        if (gdtype == ARD_F32) bits == 8 ? with(0.0f, std::true_type()) : with(0.0f, std::false_type());
        else bits == 8 ? with((uint16_t)0, std::true_type()) : with((uint16_t)0, std::false_type());
        ARD_LAUNCH_CHECK("adamw_kernel");
        return ARD_OK;
      });
}

extern "C" int32_t ard_adamw_values(int32_t count, const ard_adamw_tensor* tensors, float* const* m_out, float* const* v_out, void* stream) {
  if (count < 0) return fail(ARD_ESHAPE, "negative number of tensors");
  if (count && (!tensors || !m_out || !v_out)) return fail(ARD_EINVAL, "null tensor table");
  for (int i = 0; i < count; ++i) {
    if (int32_t st = adam_tensor_check(tensors[i], i, true, 0)) return st;
    if (tensors[i].n && (!m_out[i] || !v_out[i])) return fail(ARD_EINVAL, "tensor %d: null tensor pointer", i);
    if (misaligned(m_out[i], 4) || misaligned(v_out[i], 4)) return fail(ARD_EINVAL, "tensor %d does not start at a whole element", i);
  }
  hipStream_t st = (hipStream_t)stream;
  // a table of at most kMaxTensors at a time, m_out and v_out in the places of p and w
  for (int at = 0; at < count; at += kMaxTensors) {
    ard_adamw_tensor some[kMaxTensors];
    const int n = imin(kMaxTensors, count - at);
    for (int i = 0; i < n; ++i) some[i] = tensors[at + i], some[i].p = m_out[at + i], some[i].w = v_out[at + i];
    const int32_t rc = adam_launches(
        n, some, chunk_of(1),
        [&](ard_adamw_tensor& t, int64_t part) {
          t.p += part, t.w = (float*)t.w + part, t.m = (char*)t.m + part, t.v = (char*)t.v + part;
          t.m_scale += part / kBlock, t.v_scale += part / kBlock;
        },
        [&](const AdamTable& tab, int chunks) -> int32_t {
          ARD_LAUNCH(adamw_values_kernel, dim3(chunks), dim3(256), 0, st, tab);
          ARD_LAUNCH_CHECK("adamw_values_kernel");
          return ARD_OK;
        });
    if (rc) return rc;
  }
  return ARD_OK;
}
