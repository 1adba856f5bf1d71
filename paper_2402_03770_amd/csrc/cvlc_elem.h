// Element types of the local step's operators (fp32, bfloat16, fp16), held in 32 bits while they are worked on, and
// what their kernels share: 16-byte accesses at any element's address, sums over wavefronts and workgroups.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cvlc_common.h"

namespace cvlc {

using bf16_t = __bf16;
using f16_t = _Float16;

inline bool type_known(uint32_t type) { return type == CVLC_F32 || type == CVLC_BF16 || type == CVLC_F16; }
inline uint32_t type_bytes(uint32_t type) { return type == CVLC_F32 ? 4u : 2u; }

// A device buffer that a call reads or writes: there, and at a multiple of its elements' size.
inline bool buffer_ok(const void* p, uint32_t bytes) { return p && reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Values that one 16-byte access of the wider of two types holds.
template <class A, class B = A>
constexpr uint32_t kPerAccess = 16u / (sizeof(A) > sizeof(B) ? sizeof(A) : sizeof(B));

// N consecutive elements.  Rows start wherever the caller's stride puts them, so the address is a multiple of the
// element's size only; global memory takes 16 bytes at any such address in one access.
template <class T, uint32_t N>
struct __attribute__((packed, aligned(sizeof(T)))) Packed {
  T v[N];
};

template <uint32_t N, class T>
__device__ __forceinline__ void load_values(const T* p, float (&x)[N]) {
  const Packed<T, N> raw = *reinterpret_cast<const Packed<T, N>*>(p);
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) x[i] = (float)raw.v[i];
}
// The first `count` of them, `fill` in the place of the others.
template <uint32_t N, class T>
__device__ __forceinline__ void load_some(const T* p, uint32_t count, float fill, float (&x)[N]) {
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) x[i] = i < count ? (float)p[i] : fill;
}
// Rounded to the nearest value of the type, once: the only rounding an output sees.
template <uint32_t N, class T>
__device__ __forceinline__ void store_values(T* p, const float (&x)[N]) {
  Packed<T, N> raw;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) raw.v[i] = (T)x[i];
  *reinterpret_cast<Packed<T, N>*>(p) = raw;
}
template <uint32_t N, class T>
__device__ __forceinline__ void store_some(T* p, uint32_t count, const float (&x)[N]) {
#pragma unroll
  for (uint32_t i = 0; i < N; ++i)
    if (i < count) p[i] = (T)x[i];
}
// Values [at, at + N) of a row of `width`, as far as it goes.
template <uint32_t N, class T>
__device__ __forceinline__ void load_row(const T* row, uint32_t at, uint32_t width, float fill, float (&x)[N]) {
  if (at + N <= width)
    load_values<N>(row + at, x);
  else
    load_some<N>(row + at, at < width ? width - at : 0u, fill, x);
}
template <uint32_t N, class T>
__device__ __forceinline__ void store_row(T* row, uint32_t at, uint32_t width, const float (&x)[N]) {
  if (at + N <= width)
    store_values<N>(row + at, x);
  else if (at < width)
    store_some<N>(row + at, width - at, x);
}

// What a wavefront's lanes wrote to LDS before is seen by its other lanes after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Sums of two values over a workgroup of NW wavefronts, the same in every thread.  `scratch` holds 2 * NW floats.
template <uint32_t NW>
__device__ __forceinline__ void block_sum2(float& a, float& b, float* scratch) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (NW > 1) {
    __syncthreads();
    if (lane_id() == 0) {
      scratch[2 * wave_id()] = a;
      scratch[2 * wave_id() + 1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < NW; ++w) {
      a += scratch[2 * w];
      b += scratch[2 * w + 1];
    }
  }
}

// Calls f with a value of the element type that `type` names.
template <class F>
auto by_type(uint32_t type, F f) {
  if (type == CVLC_BF16) return f(bf16_t{});
  if (type == CVLC_F16) return f(f16_t{});
  return f(0.0f);
}
// Two types, of which the second is the first or, beside fp32, any.
template <class F>
auto by_types(uint32_t wide, uint32_t narrow, F f) {
  if (wide != CVLC_F32) return by_type(wide, [&](auto t) { return f(t, t); });
  return by_type(narrow, [&](auto t) { return f(0.0f, t); });
}
inline bool types_go(uint32_t wide, uint32_t narrow) {
  return type_known(wide) && type_known(narrow) && (wide == narrow || wide == CVLC_F32);
}

}  // namespace cvlc
