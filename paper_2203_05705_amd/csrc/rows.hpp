// What the kernels over rows, sequences and parameters share: loads of a few neighbouring elements at any
// alignment, and sums and maxima over a wavefront.
#pragma once
#include "common.hpp"

namespace ard {

// N neighbouring elements as fp32.  The vector types carry the alignment of one element: gfx950 takes 16-byte global
// accesses from any element boundary, so rows of odd length need no path of their own.
template <typename T, int N> struct Run;
template <> struct Run<uint16_t, 8> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Run<uint16_t, 4> { typedef uint32_t V __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Run<uint16_t, 2> { typedef uint32_t V __attribute__((aligned(2))); };
template <> struct Run<float, 8> { typedef float V __attribute__((ext_vector_type(8), aligned(4))); };
template <> struct Run<float, 4> { typedef float V __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Run<float, 2> { typedef float V __attribute__((ext_vector_type(2), aligned(4))); };

// two fp32 values as a pair of bf16, each to nearest even (the first in the low half)
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

template <int N> __device__ __forceinline__ void load_run(const float* p, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = *p;
  } else {
    const typename Run<float, N>::V v = *reinterpret_cast<const typename Run<float, N>::V*>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = v[j];
  }
}
template <int N> __device__ __forceinline__ void load_run(const uint16_t* p, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = bf16_bits_to_f32(*p);
  } else if constexpr (N == 2) {
    const uint32_t v = *reinterpret_cast<const typename Run<uint16_t, 2>::V*>(p);
    x[0] = __uint_as_float(v << 16), x[1] = __uint_as_float(v & 0xffff0000u);
  } else {
    const typename Run<uint16_t, N>::V v = *reinterpret_cast<const typename Run<uint16_t, N>::V*>(p);
#pragma unroll
    for (int j = 0; j < N / 2; ++j) x[2 * j] = __uint_as_float(v[j] << 16), x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
  }
}
template <int N> __device__ __forceinline__ void store_run(float* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    *p = x[0];
  } else {
    typename Run<float, N>::V v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = x[j];
    *reinterpret_cast<typename Run<float, N>::V*>(p) = v;
  }
}
template <int N> __device__ __forceinline__ void store_run(uint16_t* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    *p = (uint16_t)bf16_pair(x[0], 0.0f);
  } else if constexpr (N == 2) {
    *reinterpret_cast<typename Run<uint16_t, 2>::V*>(p) = bf16_pair(x[0], x[1]);
  } else {
    typename Run<uint16_t, N>::V v;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) v[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
    *reinterpret_cast<typename Run<uint16_t, N>::V*>(p) = v;
  }
}
// the same past the caches' order of use: for what is written once and does better so with what reads it next, as measured where it is used
template <int N> __device__ __forceinline__ void store_run_past(float* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    __builtin_nontemporal_store(x[0], p);
  } else {
    using V = typename Run<float, 4>::V;
#pragma unroll
    for (int j = 0; j < N; j += 4) __builtin_nontemporal_store(V{x[j], x[j + 1], x[j + 2], x[j + 3]}, reinterpret_cast<V*>(p + j));
  }
}
template <int N> __device__ __forceinline__ void store_run_past(uint16_t* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    __builtin_nontemporal_store((uint16_t)bf16_pair(x[0], 0.0f), p);
  } else {
    typename Run<uint16_t, N>::V v;
    if constexpr (N == 2) {
      v = bf16_pair(x[0], x[1]);
    } else {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) v[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
    }
    __builtin_nontemporal_store(v, reinterpret_cast<typename Run<uint16_t, N>::V*>(p));
  }
}

// A run of a lane as it lies in memory, to be taken apart where it is used (two bf16 stay one register until then).
template <typename T, int N> struct Raw;
template <> struct Raw<float, 1> { float v; };
template <> struct Raw<uint16_t, 1> { uint16_t v; };
template <> struct Raw<uint16_t, 2> { uint32_t v; };
template <typename T, int N> __device__ __forceinline__ Raw<T, N> load_raw(const T* p) {
  if constexpr (N == 1) return Raw<T, N>{*p};
  else return Raw<T, N>{*reinterpret_cast<const typename Run<T, N>::V*>(p)};
}
__device__ __forceinline__ float part_of(const Raw<float, 1>& r, int) { return r.v; }
__device__ __forceinline__ float part_of(const Raw<uint16_t, 1>& r, int) { return bf16_bits_to_f32(r.v); }
__device__ __forceinline__ float part_of(const Raw<uint16_t, 2>& r, int j) { return __uint_as_float(j ? r.v & 0xffff0000u : r.v << 16); }

// the first n of N elements (n >= N: all, one access), the others 0
template <int N, typename T> __device__ __forceinline__ void load_some(const T* p, int n, float (&x)[N]) {
  if (n >= N) {
    load_run<N>(p, x);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = j < n ? ElemTraits<T>::to_f32(p[j]) : 0.0f;
}
template <int N, typename T> __device__ __forceinline__ void store_some(T* p, int n, const float (&x)[N]) {
  if (n >= N) {
    store_run<N>(p, x);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < n) p[j] = ElemTraits<T>::from_f32(x[j]);
}

// A run of N elements as it lies in memory, and its values.
template <typename T> struct Run<T, 1> { typedef T V; };
template <int N, typename T> __device__ __forceinline__ typename Run<T, N>::V load_whole(const T* p) {
  return *reinterpret_cast<const typename Run<T, N>::V*>(p);
}
template <int N, typename T> __device__ __forceinline__ void values_of(const typename Run<T, N>::V& v, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = ElemTraits<T>::to_f32(v);
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < N / 2; ++j) x[2 * j] = __uint_as_float(v[j] << 16), x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = v[j];
  }
}

// ---- over a wavefront -----------------------------------------------------------
// Cross-lane moves in the vector pipe (swaps inside quads, mirrors inside rows of 16, broadcasts of a row's last lane):
// a sum of 64 lanes in seven instructions, without LDS.  Lane 63 ends with the whole; all lanes get it.
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_or_zero(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float half_row_sum(float v) {  // over 8 neighbouring lanes, in all of them
  v += dpp_or_zero<0xB1, 0xf>(v);
  v += dpp_or_zero<0x4E, 0xf>(v);
  v += dpp_or_zero<0x141, 0xf>(v);
  return v;
}
__device__ __forceinline__ float row_sum(float v) {  // over 16
  v = half_row_sum(v);
  v += dpp_or_zero<0x140, 0xf>(v);
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum(v);
  v += dpp_or_zero<0x142, 0xa>(v);
  v += dpp_or_zero<0x143, 0xc>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = dpp_max<0xB1, 0xf>(v);
  v = dpp_max<0x4E, 0xf>(v);
  v = dpp_max<0x141, 0xf>(v);
  v = dpp_max<0x140, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

static inline bool misaligned(const void* p, size_t to) { return ((uintptr_t)p % to) != 0; }

}  // namespace ard
