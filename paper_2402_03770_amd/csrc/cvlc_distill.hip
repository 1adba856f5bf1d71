// cvlc_distill.hip -- distillation from a teacher's top logits: the loss of every
// row and the gradient of the student's logits.
//
// A workgroup per row.  It first turns the teacher's list into probabilities in
// LDS (the list is short), then passes over the row with a running maximum m and
// sum S of exp((z - m) / T), and, where the gradient is wanted, passes over it
// again and writes w T P q everywhere; the few listed places are then written
// again with their own gradient, every one by the thread of its entry.
//
// m starts at the type's lowest finite value, so that a row of masked logits
// (-inf) ends with S = 0, which stands for q = 0, and a row of logits that are all
// at the lowest value ends like any other.  Differences to m are taken before
// they are scaled: a scaled logit may overflow, a difference of exactly 0 may not.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include <algorithm>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kDistillBlock = 256, kDistillWaves = kDistillBlock / kWave;
constexpr uint32_t kMaxK = CVLC_DISTILL_MAX_K;

struct DistillArgs {
  uint32_t n, vocab, k;
  uint64_t stride, dstride;
  const void *ids, *values;
  uint32_t id_bytes, value_type;
  float T, c;  // c = log2(e) / T
  uint32_t logprobs;
  const float* weights;
  float *loss, *stats;  // stats: written by the loss, read by the gradient alone
  uint32_t* status;
};

// exp((z - m) / T).  The instruction flushes results below 2^-126, which a sum of at least 1 does not notice.
__device__ __forceinline__ float exp_part(float z, float m, float c) { return __builtin_amdgcn_exp2f((z - m) * c); }
// exp((z - m) / T) * scale, where `scaled` is scale * 2^-kLift: lifted into the normal range until the one product that
// may leave it, so that the smallest gradients are rounded once.
constexpr float kLift = 32.0f, kUnlift = 0x1p-32f;
__device__ __forceinline__ float exp_scaled(float z, float m, float c, float scaled) {
  return scaled * __builtin_amdgcn_exp2f(fmaf(z - m, c, kLift));
}

struct MaxSum {
  float m, s;
};

__device__ __forceinline__ int64_t load_id(const void* ids, uint32_t id_bytes, uint64_t i) {
  return id_bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}
__device__ __forceinline__ float load_as_float(const void* p, uint32_t type, uint64_t i) {
  if (type == CVLC_F32) return static_cast<const float*>(p)[i];
  return type == CVLC_BF16 ? (float)static_cast<const bf16_t*>(p)[i] : (float)static_cast<const f16_t*>(p)[i];
}

// The maximum, ignoring NaN, of one value per thread, and the sum of another, in every thread.
template <uint32_t NW>
__device__ __forceinline__ float block_max(float v, float* scratch) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if (lane_id() == 0) scratch[wave_id()] = v;
  __syncthreads();
  v = scratch[0];
#pragma unroll
  for (uint32_t w = 1; w < NW; ++w) v = fmaxf(v, scratch[w]);
  return v;
}

// The teacher's list of a row, in LDS: entries that are not there have id -1 and p = 0.
struct List {
  int32_t id[kMaxK];
  float p[kMaxK], tlogp[kMaxK], z[kMaxK];  // tlogp: T ln p, which stays finite where ln p does not
  float scratch[2 * kDistillWaves];
};

// Fills the list but for z; returns P (0: the list is empty).
__device__ float load_list(const DistillArgs& a, uint32_t row, List& l) {
  const uint64_t at = (uint64_t)row * a.k;
  float top = -INFINITY;
  for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) {
    const int64_t id = load_id(a.ids, a.id_bytes, at + j);
    const float t = load_as_float(a.values, a.value_type, at + j);
    const bool there = id >= 0 && id < (int64_t)a.vocab && t != -INFINITY;
    if (id >= (int64_t)a.vocab && a.status) atomicOr(a.status, CVLC_DEV_INDEX);
    l.id[j] = there ? (int32_t)id : -1;
    l.tlogp[j] = t;
    if (there) top = fmaxf(top, t);
  }
  top = a.logprobs ? 0.0f : block_max<kDistillWaves>(top, l.scratch);
  const float c = a.logprobs ? (float)M_LOG2E : a.c;
  float sum = 0.0f, unused = 0.0f;
  for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) {
    l.p[j] = l.id[j] >= 0 ? exp2f((l.tlogp[j] - top) * c) : 0.0f;
    sum += l.p[j];
  }
  block_sum2<kDistillWaves>(sum, unused, l.scratch);
  if (!a.logprobs && sum != 0.0f) {
    const float inv = 1.0f / sum, tlog_sum = a.T * logf(sum);
    for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) {
      l.p[j] *= inv;
      l.tlogp[j] = (l.tlogp[j] - top) - tlog_sum;
    }
    sum = sum == sum ? 1.0f : sum;
  } else if (a.logprobs) {
    for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) l.tlogp[j] *= a.T;
  }
  __syncthreads();
  return sum;
}

// w T^2 times the sum over the list of p (ln p - ln q), q from the row's m and S.
__device__ float list_loss(const DistillArgs& a, List& l, float m, float S, float wT) {
  const float tlog_S = a.T * logf(S);
  float loss = 0.0f, unused = 0.0f;
  for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) {
    if (l.id[j] < 0 || l.p[j] == 0.0f) continue;
    const float tlogq = S == 0.0f ? -INFINITY : (l.z[j] - m) - tlog_S;
    loss += wT * l.p[j] * (l.tlogp[j] - tlogq);
  }
  block_sum2<kDistillWaves>(loss, unused, l.scratch);
  return loss;
}

// The listed places of a row's gradient.
template <class T>
__device__ void write_listed(const DistillArgs& a, const List& l, T* drow, float m, float inv, float P, float wT) {
  for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) {
    const int32_t id = l.id[j];
    if (id < 0) continue;
    float p = 0.0f;
    for (uint32_t i = 0; i < a.k; ++i) p += l.id[i] == id ? l.p[i] : 0.0f;
    drow[id] = (T)(wT * (exp_scaled(l.z[j], m, a.c, P * inv * kUnlift) - p));
  }
}

template <class T, bool LOSS, bool GRAD>
__global__ __launch_bounds__(kDistillBlock) void distill_kernel(DistillArgs a, const T* logits, T* dlogits) {
  constexpr uint32_t N = kPerAccess<T>;
  __shared__ List l;
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* zr = logits + row * a.stride;
    T* dr = GRAD ? dlogits + row * a.dstride : nullptr;
    const float w = a.weights ? a.weights[row] : 1.0f;
    __syncthreads();
    const float P = w == 0.0f ? 0.0f : load_list(a, row, l);
    if (P == 0.0f) {  // nothing to learn here
      if (LOSS && threadIdx.x == 0) {
        if (a.loss) a.loss[row] = 0.0f;
        if (a.stats) a.stats[2 * (uint64_t)row] = a.stats[2 * (uint64_t)row + 1] = 0.0f;
      }
      if (GRAD)
        for (uint32_t at = threadIdx.x * N; at < a.vocab; at += kDistillBlock * N) {
          const float zero[N] = {};
          store_row<N>(dr, at, a.vocab, zero);
        }
      continue;
    }
    for (uint32_t j = threadIdx.x; j < a.k; j += kDistillBlock) l.z[j] = l.id[j] >= 0 ? (float)zr[l.id[j]] : 0.0f;
    MaxSum t{-FLT_MAX, 0.0f};
    if (LOSS) {
      for (uint32_t at = threadIdx.x * N; at < a.vocab; at += kDistillBlock * N) {
        float v[N];
        load_row<N>(zr, at, a.vocab, -INFINITY, v);
        float m = t.m;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) m = fmaxf(m, v[i]);
        t.s *= exp_part(t.m, m, a.c);
        t.m = m;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) t.s += exp_part(v[i], m, a.c);
      }
      const float m = block_max<kDistillWaves>(t.m, l.scratch);
      float unused = 0.0f;
      t.s *= exp_part(t.m, m, a.c);
      t.m = m;
      block_sum2<kDistillWaves>(t.s, unused, l.scratch);
      const float loss = a.loss ? list_loss(a, l, t.m, t.s, w * a.T) : 0.0f;
      if (threadIdx.x == 0) {
        if (a.loss) a.loss[row] = loss;
        if (a.stats) {
          a.stats[2 * (uint64_t)row] = t.m;
          a.stats[2 * (uint64_t)row + 1] = t.s;
        }
      }
    } else {
      t = {a.stats[2 * (uint64_t)row], a.stats[2 * (uint64_t)row + 1]};
    }
    if (GRAD) {
      const float inv = t.s == 0.0f ? 0.0f : 1.0f / t.s, wT = w * a.T, scale = wT * P * inv * kUnlift;
      __syncthreads();  // every listed logit has been read: the gradient may take the logits' place
      for (uint32_t at = threadIdx.x * N; at < a.vocab; at += kDistillBlock * N) {
        float v[N];
        load_row<N>(zr, at, a.vocab, 0.0f, v);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] = exp_scaled(v[i], t.m, a.c, scale);
        store_row<N>(dr, at, a.vocab, v);
      }
      __syncthreads();
      write_listed(a, l, dr, t.m, inv, P, wT);
    }
  }
}

int check(uint32_t n, uint32_t vocab, const void* logits, uint32_t type, uint64_t stride, uint32_t k, const void* ids,
          uint32_t id_bytes, const void* values, uint32_t value_type, float T, uint32_t flags, const float* weights,
          const float* stats, const void* dlogits, uint64_t dstride, const uint32_t* status) {
  if (vocab < 1 || vocab > 0x7FFFFFFFu || n > 0x7FFFFFFFu || k < 1 || k > kMaxK) return CVLC_ERR_ARG;
  if (!type_known(type) || !type_known(value_type) || stride < vocab) return CVLC_ERR_ARG;
  if ((id_bytes != 4 && id_bytes != 8) || (flags & ~CVLC_DISTILL_LOGPROBS)) return CVLC_ERR_ARG;
  // 1 / T and T^2 are finite and not 0
  if (!(T >= 1e-18f && T <= 1e18f)) return CVLC_ERR_ARG;
  if (weights && !buffer_ok(weights, 4)) return CVLC_ERR_ARG;
  if (stats && !buffer_ok(stats, 4)) return CVLC_ERR_ARG;
  if (status && !buffer_ok(status, 4)) return CVLC_ERR_ARG;
  if (dlogits && (dstride < vocab || !buffer_ok(dlogits, type_bytes(type)))) return CVLC_ERR_ARG;
  if (n == 0) return CVLC_OK;
  if (!buffer_ok(logits, type_bytes(type)) || !buffer_ok(ids, id_bytes) || !buffer_ok(values, type_bytes(value_type))) return CVLC_ERR_ARG;
  if (dlogits == logits && dstride != stride) return CVLC_ERR_ARG;
  return CVLC_OK;
}

template <bool LOSS, bool GRAD>
int launch(const DistillArgs& a, uint32_t type, const void* logits, void* dlogits, void* hip_stream) {
  by_type(type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((distill_kernel<T, LOSS, GRAD>), dim3(std::min(a.n, 1u << 20)), dim3(kDistillBlock), 0,
                       static_cast<hipStream_t>(hip_stream), a, static_cast<const T*>(logits), static_cast<T*>(dlogits));
  });
  return hip_check(hipGetLastError());
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_distill_workspace_bytes(uint32_t n, uint32_t vocab) {
  (void)n;
  (void)vocab;
  return 256u;
}

int cvlc_distill(uint32_t n, uint32_t vocab, const void* d_logits, uint32_t type, uint64_t stride, uint32_t k, const void* d_ids,
                 uint32_t id_bytes, const void* d_values, uint32_t value_type, float temperature, uint32_t flags,
                 const float* d_weights, float* d_loss, float* d_stats, void* d_dlogits, uint64_t dlogits_stride,
                 void* d_workspace, size_t ws_bytes, uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  const int rc = check(n, vocab, d_logits, type, stride, k, d_ids, id_bytes, d_values, value_type, temperature, flags, d_weights,
                       d_stats, d_dlogits, dlogits_stride, d_status);
  if (rc) return rc;
  if (d_loss && !buffer_ok(d_loss, 4)) return CVLC_ERR_ARG;
  if (n && !d_loss && !d_stats && !d_dlogits) return CVLC_ERR_ARG;
  if (!buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  if (ws_bytes < cvlc_distill_workspace_bytes(n, vocab)) return CVLC_ERR_CAPACITY;
  if (n == 0) return CVLC_OK;
  const DistillArgs a{n, vocab, k, stride, dlogits_stride, d_ids, d_values, id_bytes, value_type, temperature,
                      (float)(M_LOG2E / temperature), flags & CVLC_DISTILL_LOGPROBS, d_weights, d_loss, d_stats, d_status};
  return d_dlogits ? launch<true, true>(a, type, d_logits, d_dlogits, hip_stream)
                   : launch<true, false>(a, type, d_logits, nullptr, hip_stream);
}

int cvlc_distill_grad(uint32_t n, uint32_t vocab, const void* d_logits, uint32_t type, uint64_t stride, uint32_t k,
                      const void* d_ids, uint32_t id_bytes, const void* d_values, uint32_t value_type, float temperature,
                      uint32_t flags, const float* d_weights, const float* d_stats, void* d_dlogits, uint64_t dlogits_stride,
                      uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  const int rc = check(n, vocab, d_logits, type, stride, k, d_ids, id_bytes, d_values, value_type, temperature, flags, d_weights,
                       d_stats, d_dlogits, dlogits_stride, d_status);
  if (rc) return rc;
  if (n == 0) return CVLC_OK;
  if (!d_stats || !d_dlogits) return CVLC_ERR_ARG;
  const DistillArgs a{n, vocab, k, stride, dlogits_stride, d_ids, d_values, id_bytes, value_type, temperature,
                      (float)(M_LOG2E / temperature), flags & CVLC_DISTILL_LOGPROBS, d_weights, nullptr,
                      const_cast<float*>(d_stats), d_status};
  return launch<false, true>(a, type, d_logits, d_dlogits, hip_stream);
}

}  // extern "C"
