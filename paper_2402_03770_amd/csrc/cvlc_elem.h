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

// Rows start wherever the caller's stride puts them, so an access's address is a multiple of the element's size only;
// global memory takes 16 bytes at any such address in one access.  Said with vectors of words: of a struct of elements the
// compiler makes accesses of 2, 4 and 8 bytes.
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
typedef uint32_t Pair __attribute__((ext_vector_type(2)));
typedef Quad UnalignedQuad __attribute__((aligned(2)));
typedef Pair UnalignedPair __attribute__((aligned(2)));

// N consecutive elements as they lie in memory, to be worked on later.  Kept as words: taken apart into elements the
// compiler would want them at once, and wait for the load where it was issued.
template <class T, uint32_t N>
struct Raw {
  static constexpr uint32_t kWords = N * sizeof(T) / 4;
  static_assert(kWords == 2 || kWords == 4, "an access of 8 or 16 bytes");
  uint32_t w[kWords];

  // ONCE: past the caches' replacement order, for what is larger than the caches.
  template <bool ONCE>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kWords == 4) {
      const UnalignedQuad* q = reinterpret_cast<const UnalignedQuad*>(p);
      const Quad v = ONCE ? (Quad)__builtin_nontemporal_load(q) : (Quad)*q;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) w[i] = v[i];
    } else {
      const UnalignedPair* q = reinterpret_cast<const UnalignedPair*>(p);
      const Pair v = ONCE ? (Pair)__builtin_nontemporal_load(q) : (Pair)*q;
      w[0] = v[0];
      w[1] = v[1];
    }
  }
  __device__ __forceinline__ void values(float (&x)[N]) const {
#pragma unroll
    for (uint32_t i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        x[2 * i] = (float)__builtin_bit_cast(T, (uint16_t)(w[i] & 0xFFFFu));
        x[2 * i + 1] = (float)__builtin_bit_cast(T, (uint16_t)(w[i] >> 16));
      }
    }
  }
};

// Elements [at, at + N) of a row of `width`, as far as it goes; zero bits beyond.
template <bool ONCE = false, class T, uint32_t N>
__device__ __forceinline__ void load_raw(Raw<T, N>& raw, const T* row, uint32_t at, uint32_t width) {
  if (at + N <= width) {
    raw.template load<ONCE>(row + at);
  } else {
    constexpr uint32_t kEach = 4 / sizeof(T);
#pragma unroll
    for (uint32_t i = 0; i < Raw<T, N>::kWords; ++i) {
      raw.w[i] = 0;
#pragma unroll
      for (uint32_t k = 0; k < kEach; ++k)
        if (at + i * kEach + k < width) {
          if constexpr (sizeof(T) == 4)
            raw.w[i] = __float_as_uint(row[at + i]);
          else
            raw.w[i] |= (uint32_t)__builtin_bit_cast(uint16_t, row[at + i * kEach + k]) << (16 * k);
        }
    }
  }
}

// Rounds N values to the type, once, and writes them in accesses of 16 bytes (or one of 8).
template <bool ONCE, uint32_t N, class T>
__device__ __forceinline__ void store_whole(T* p, const float (&x)[N]) {
  static_assert(N * sizeof(T) == 8 || N * sizeof(T) % 16 == 0, "accesses of 8 or 16 bytes");
  uint32_t w[N * sizeof(T) / 4];
#pragma unroll
  for (uint32_t i = 0; i < N * sizeof(T) / 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(x[i]);
    } else {
      w[i] = __builtin_bit_cast(uint16_t, (T)x[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i + 1]) << 16;
    }
  }
  if constexpr (N * sizeof(T) >= 16) {
#pragma unroll
    for (uint32_t i = 0; i < N * sizeof(T) / 16; ++i) {
      const Quad v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
      UnalignedQuad* q = reinterpret_cast<UnalignedQuad*>(p) + i;
      if constexpr (ONCE)
        __builtin_nontemporal_store(v, q);
      else
        *q = v;
    }
  } else {
    const Pair v = {w[0], w[1]};
    UnalignedPair* q = reinterpret_cast<UnalignedPair*>(p);
    if constexpr (ONCE)
      __builtin_nontemporal_store(v, q);
    else
      *q = v;
  }
}

// Where a thread's N elements of a row of `width` >= N lie.  The row's last access, where it is not a whole one, is moved
// back to end with the row, and the thread's own elements are those from `skip` on: its load is one access like any
// other, that can be under way while something else is worked on.  skip = N: none.
template <uint32_t N>
struct Place {
  uint32_t at, skip;
  __device__ __forceinline__ Place() {}
  __device__ __forceinline__ Place(uint32_t first, uint32_t width) {
    at = min(first, width - N);
    skip = min(first - at, N);
  }
  __device__ __forceinline__ bool any() const { return skip < N; }
  // x with `fill` in the place of what is not the thread's
  __device__ __forceinline__ void mask(float (&x)[N], float fill) const {
    if (skip == 0) return;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) x[i] = i < skip ? fill : x[i];
  }
  template <bool ONCE, class T>
  __device__ __forceinline__ void store(T* row, const float (&x)[N]) const {
    if (skip == 0) {
      store_whole<ONCE, N>(row + at, x);
    } else if (skip < N) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i)
        if (i >= skip) row[at + i] = (T)x[i];
    }
  }
};

template <uint32_t N, class T>
__device__ __forceinline__ void load_values(const T* p, float (&x)[N]) {
  constexpr uint32_t kEach = N * sizeof(T) > 16 ? 16 / sizeof(T) : N;
#pragma unroll
  for (uint32_t k = 0; k < N; k += kEach) {
    Raw<T, kEach> raw;
    float part[kEach];
    raw.template load<false>(p + k);
    raw.values(part);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) x[k + i] = part[i];
  }
}
// The first `count` of them, `fill` in the place of the others.
template <uint32_t N, class T>
__device__ __forceinline__ void load_some(const T* p, uint32_t count, float fill, float (&x)[N]) {
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) x[i] = i < count ? (float)p[i] : fill;
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
template <uint32_t N, bool ONCE = false, class T>
__device__ __forceinline__ void store_row(T* row, uint32_t at, uint32_t width, const float (&x)[N]) {
  if (at + N <= width)
    store_whole<ONCE, N>(row + at, x);
  else if (at < width)
    store_some<N>(row + at, width - at, x);
}

// What a wavefront's lanes wrote to LDS before is seen by its other lanes after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// v of the lane that DPP control CTRL names; 0 outside the rows of 16 lanes that ROWS selects.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xF, false));
}
// Sum over the wavefront's lanes, in every lane: rotations inside rows of 16, then row to row, in the vector ALU
// alone (a shuffle goes through LDS, six of them one after the other take ten times as long).
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0x128, 0xF>(v);  // row_ror:8
  v += dpp<0x124, 0xF>(v);  // row_ror:4
  v += dpp<0x122, 0xF>(v);  // row_ror:2
  v += dpp<0x121, 0xF>(v);  // row_ror:1
  v += dpp<0x142, 0xA>(v);  // row_bcast:15, rows 1 and 3
  v += dpp<0x143, 0xC>(v);  // row_bcast:31, rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ __forceinline__ float wave_max(float v) {
  auto other = [&](auto ctrl, auto rows) {
    const int w = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(w, w, ctrl.value, rows.value, 0xF, false));
  };
  using std::integral_constant;
  v = fmaxf(v, other(integral_constant<int, 0x128>{}, integral_constant<int, 0xF>{}));
  v = fmaxf(v, other(integral_constant<int, 0x124>{}, integral_constant<int, 0xF>{}));
  v = fmaxf(v, other(integral_constant<int, 0x122>{}, integral_constant<int, 0xF>{}));
  v = fmaxf(v, other(integral_constant<int, 0x121>{}, integral_constant<int, 0xF>{}));
  v = fmaxf(v, other(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{}));
  v = fmaxf(v, other(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{}));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// The sum of a value over a workgroup of NW wavefronts, the same in every thread.  `scratch` holds NW floats.
template <uint32_t NW>
__device__ __forceinline__ float block_sum(float a, float* scratch) {
  a = wave_sum(a);
  if constexpr (NW > 1) {
    __syncthreads();
    if (lane_id() == 0) scratch[wave_id()] = a;
    __syncthreads();
    a = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < NW; ++w) a += scratch[w];
  }
  return a;
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
