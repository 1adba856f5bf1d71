// cvlc_adamw.hip -- one AdamW step over all tensors of a model, its averages in 32 bits or in 8.
//
// With g the gradient times its scale and t the step's number,
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// Averages in 8 bits are held as codes of m and of r = sqrt(v) with one scale for
// each per 256 values of a tensor.  r is halfway between the powers that v spans,
// and what the step divides by.  A step changes r by a fraction of a code, so
// rounding to nearest would hold it where it is for good: it goes up or down by 16
// random bits, right on average; the codes' relative step of 1/8 at most then is
// noise, not drift.  It never goes down to zero, where the next step would divide by eps.
// The same holds for m: to nearest, codes of 1 to 4 never decay at b1 = 0.9 and none does at
// 0.99, while r does, so a weight whose gradient has ended moves by the same amount
// at every step.  CVLC_ADAMW_M_BY_CHANCE rounds m as r is, by bits of its own, and down to zero too.
//
// Everything is read and written once and nothing is shared between workgroups but
// the tensors' table: bound by HBM (28 bytes a weight with fp32 gradients and
// averages, 16 with averages in 8 bits).  One launch, whatever the number of
// tensors: the plan has laid out which tensor every workgroup's chunk lies in.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kAdamBlock = 256;
constexpr uint32_t kEach = 8;                    // values of a thread at a time: what one Philox counter serves
constexpr uint32_t kHeld = CVLC_ADAMW_BLOCK;     // values that share a scale: half a wavefront's
constexpr uint32_t kChunk = 8192;                // values of a workgroup
static_assert(kHeld == 32 * kEach && kChunk % (kAdamBlock * kEach) == 0, "blocks do not span wavefronts or chunks");
constexpr float kTop = 448.0f;                   // largest e4m3 value
constexpr float kTiny = 0x1p-100f;               // a block that lies below is zeros: its scale's inverse would overflow

// A tensor as the workgroups read it.
struct Entry {
  uint64_t n;
  float* param;
  const void* grad;
  void *m, *v;
  float* scales;
  void* copy;
  uint32_t first_chunk;
  uint8_t grad_type, copy_type, bits, flags;
  float decay;
};
static_assert(sizeof(Entry) % 8 == 0, "entries are 8-byte granular");

constexpr uint32_t kPerUpload = 32;
struct Upload {
  Entry entry[kPerUpload];
  uint32_t first, count;
};
static_assert(sizeof(Upload) <= 3584, "kernel arguments");

uint64_t chunks_of(uint64_t n) { return (n + kChunk - 1) / kChunk; }

// Tensors' entries as kernel arguments (the one way from the host that needs neither pinned memory nor a wait), and for
// every chunk the number of its tensor.
__global__ __launch_bounds__(kAdamBlock) void adamw_table_kernel(Upload u, Entry* entries, uint32_t* tensor_of) {
  const Entry& e = u.entry[blockIdx.y];
  if (blockIdx.x == 0 && threadIdx.x == 0) entries[u.first + blockIdx.y] = e;
  const uint32_t chunks = (uint32_t)((e.n + kChunk - 1) / kChunk);
  for (uint32_t c = blockIdx.x * kAdamBlock + threadIdx.x; c < chunks; c += gridDim.x * kAdamBlock)
    tensor_of[e.first_chunk + c] = u.first + blockIdx.y;
}

struct Rates {
  float b1, rest1, b2, rest2, eps, grad_scale;
  float lr, rate, root;       // rate = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
  double log_b1, log_b2;      // for rates that are read on the device
  uint32_t step, k0, k1;
};

__host__ __device__ inline void with_step(Rates& r, float lr, double step) {
  step = fmax(step, 1.0);
  r.lr = lr;
  r.rate = (float)(lr / -expm1(step * r.log_b1));
  r.root = (float)(1.0 / sqrt(-expm1(step * r.log_b2)));
  r.step = (uint32_t)step;
}

// The eight 16-bit halves of Philox4x32-10's words (Salmon et al., 2011), low ones first.
__device__ __forceinline__ void chances(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1,
                                        uint32_t (&out)[kEach]) {
#pragma unroll
  for (uint32_t round = 0; round < 10; ++round) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) out[i] = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
}

// Eight codes, at any byte's address.
typedef Pair BytePair __attribute__((aligned(1)));

template <bool ONCE>
__device__ __forceinline__ Pair load_codes(const uint8_t* p) {
  const BytePair* q = reinterpret_cast<const BytePair*>(p);
  return ONCE ? (Pair)__builtin_nontemporal_load(q) : (Pair)*q;
}
__device__ __forceinline__ void decode(Pair c, float scale, float (&x)[kEach]) {
  typedef float Two __attribute__((ext_vector_type(2)));
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
    const Two a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
    x[4 * i] = a[0] * scale;
    x[4 * i + 1] = a[1] * scale;
    x[4 * i + 2] = b[0] * scale;
    x[4 * i + 3] = b[1] * scale;
  }
}
// Codes of values within +-448, to nearest.
__device__ __forceinline__ Pair encode(const float (&y)[kEach]) {
  Pair c;
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], low, true);
  }
  return c;
}

// y >= 0 to one of the two codes around it: up with the probability of its distance from the lower one, in steps of 2^-16,
// and never below `least` unless it is zero.  From 2^-6 on eight codes to an octave, steps of 2^-9 below.
__device__ __forceinline__ float by_chance(float y, uint32_t chance, float least) {
  const float normal = __uint_as_float((__float_as_uint(y) + (chance << 4)) & 0xFFF00000u);
  const float small = fmaxf(floorf(y * 512.0f + (float)chance * 0x1p-16f) * 0x1p-9f, least);
  const float z = y >= 0x1p-6f ? normal : small;
  return y > 0.0f ? fminf(z, kTop) : 0.0f;
}

__device__ __forceinline__ float half_wave_max(float v) {
  auto other = [&](auto ctrl) {
    const int w = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(w, w, ctrl.value, 0xF, 0xF, false));
  };
  using std::integral_constant;
  v = fmaxf(v, other(integral_constant<int, 0x128>{}));  // row_ror
  v = fmaxf(v, other(integral_constant<int, 0x124>{}));
  v = fmaxf(v, other(integral_constant<int, 0x122>{}));
  v = fmaxf(v, other(integral_constant<int, 0x121>{}));
  return fmaxf(v, __shfl_xor(v, 16, 64));
}

// kEach values from p on, of which `count` are there; zeros for the others.
template <bool ONCE, class T>
__device__ __forceinline__ void load_each(const T* p, uint32_t count, float (&x)[kEach]) {
  if (count == kEach) {
    constexpr uint32_t kWhole = 16 / sizeof(T);
#pragma unroll
    for (uint32_t k = 0; k < kEach; k += kWhole) {
      Raw<T, kWhole> raw;
      float part[kWhole];
      raw.template load<ONCE>(p + k);
      raw.values(part);
#pragma unroll
      for (uint32_t i = 0; i < kWhole; ++i) x[k + i] = part[i];
    }
  } else {
    load_some<kEach>(p, count, 0.0f, x);
  }
}
template <bool ONCE, class T>
__device__ __forceinline__ void store_each(T* p, uint32_t count, const float (&x)[kEach]) {
  if (count == kEach)
    store_whole<ONCE, kEach>(p, x);
  else
    store_some<kEach>(p, count, x);
}

template <uint32_t BITS, bool ONCE>
__device__ __forceinline__ void step_each(const Entry& e, uint32_t tensor, const Rates& r, uint64_t at, uint32_t count, bool& bad) {
  float p[kEach], g[kEach], m[kEach], v[kEach], q[kEach];
  if (e.grad_type == CVLC_F32)
    load_each<ONCE>(static_cast<const float*>(e.grad) + at, count, g);
  else if (e.grad_type == CVLC_BF16)
    load_each<ONCE>(static_cast<const bf16_t*>(e.grad) + at, count, g);
  else
    load_each<ONCE>(static_cast<const f16_t*>(e.grad) + at, count, g);
  load_each<ONCE>(e.param + at, count, p);
  uint8_t *mc = static_cast<uint8_t*>(e.m) + at, *vc = static_cast<uint8_t*>(e.v) + at;
  if constexpr (BITS == 32) {
    load_each<ONCE>(static_cast<const float*>(e.m) + at, count, m);
    load_each<ONCE>(static_cast<const float*>(e.v) + at, count, v);
  } else {
    Pair cm = {0, 0}, cv = {0, 0};
    if (count == kEach) {
      cm = load_codes<ONCE>(mc);
      cv = load_codes<ONCE>(vc);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i)
        if (i < count) {
          cm[i / 4] |= (uint32_t)mc[i] << (8 * (i % 4));
          cv[i / 4] |= (uint32_t)vc[i] << (8 * (i % 4));
        }
    }
    float2 scale = {0.0f, 0.0f};
    if (count) scale = reinterpret_cast<const float2*>(e.scales)[at / kHeld];
    decode(cm, scale.x, m);
    decode(cv, scale.y, v);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) v[i] *= v[i];
  }
  const float keep = 1.0f - r.lr * e.decay;
  bool some = false;
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) {
    const float gi = g[i] * r.grad_scale;
    const float mi = m[i] * r.b1 + gi * r.rest1, vi = v[i] * r.b2 + gi * gi * r.rest2;
    q[i] = sqrtf(vi);
    const float to = p[i] * keep - r.rate * (mi / (q[i] * r.root + r.eps));
    const bool fine = fabsf(to) + vi < INFINITY;  // and neither they nor m is a NaN
    some |= !fine;
    m[i] = fine ? mi : m[i];
    v[i] = fine ? vi : v[i];
    p[i] = fine ? to : p[i];
  }
  if (some) {
    bad = true;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) q[i] = sqrtf(v[i]);
  }
  store_each<ONCE>(e.param + at, count, p);
  if (e.copy) {
    if (e.copy_type == CVLC_BF16)
      store_each<ONCE>(static_cast<bf16_t*>(e.copy) + at, count, p);
    else
      store_each<ONCE>(static_cast<f16_t*>(e.copy) + at, count, p);
  }
  if constexpr (BITS == 32) {
    store_each<ONCE>(static_cast<float*>(e.m) + at, count, m);
    store_each<ONCE>(static_cast<float*>(e.v) + at, count, v);
  } else {
    float top_m = 0.0f, top_q = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
      m[i] = i < count ? m[i] : 0.0f;
      q[i] = i < count ? q[i] : 0.0f;
      top_m = fmaxf(top_m, fabsf(m[i]));
      top_q = fmaxf(top_q, q[i]);
    }
    top_m = half_wave_max(top_m);
    top_q = half_wave_max(top_q);
    top_m = top_m >= kTiny ? top_m : 0.0f;
    top_q = top_q >= kTiny ? top_q : 0.0f;
    const float inv_m = top_m > 0.0f ? 1.0f / top_m * kTop : 0.0f, inv_q = top_q > 0.0f ? 1.0f / top_q * kTop : 0.0f;
    uint32_t chance[kEach];
    chances((uint32_t)(at / kEach), 0, r.step, tensor, r.k0, r.k1, chance);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
      m[i] = fminf(fmaxf(m[i] * inv_m, -kTop), kTop);
      q[i] = by_chance(fminf(q[i] * inv_q, kTop), chance[i], 0x1p-9f);
    }
    if (e.flags & CVLC_ADAMW_M_BY_CHANCE) {
      chances((uint32_t)(at / kEach), 1, r.step, tensor, r.k0, r.k1, chance);
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i) m[i] = copysignf(by_chance(fabsf(m[i]), chance[i], 0.0f), m[i]);
    }
    const Pair cm = encode(m), cv = encode(q);
    if (count == kEach) {
      *reinterpret_cast<BytePair*>(mc) = cm;
      *reinterpret_cast<BytePair*>(vc) = cv;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i)
        if (i < count) {
          mc[i] = (uint8_t)(cm[i / 4] >> (8 * (i % 4)));
          vc[i] = (uint8_t)(cv[i / 4] >> (8 * (i % 4)));
        }
    }
    if (count && at % kHeld == 0) reinterpret_cast<float2*>(e.scales)[at / kHeld] = float2{top_m * (1.0f / kTop), top_q * (1.0f / kTop)};
  }
}

template <bool ONCE>
__global__ __launch_bounds__(kAdamBlock) void adamw_kernel(const Entry* entries, const uint32_t* tensor_of, Rates r, const float* now,
                                                           uint32_t* status) {
  const uint32_t tensor = tensor_of[blockIdx.x];
  const Entry e = entries[tensor];
  if (now) {
    r.grad_scale = now[2];
    with_step(r, now[1], now[0]);
  }
  const uint64_t first = (uint64_t)(blockIdx.x - e.first_chunk) * kChunk;
  bool bad = false;
  for (uint32_t k = threadIdx.x * kEach; k < kChunk; k += kAdamBlock * kEach) {
    const uint64_t at = first + k;
    if (at / (kWave * kEach) * (kWave * kEach) >= e.n) break;  // the whole wavefront
    const uint32_t count = at >= e.n ? 0u : (uint32_t)min(e.n - at, (uint64_t)kEach);
    if (e.bits == 8)
      step_each<8, ONCE>(e, tensor, r, at, count, bad);
    else
      step_each<32, ONCE>(e, tensor, r, at, count, bad);
  }
  if (status && __ballot(bad) && lane_id() == 0) atomicOr(status, CVLC_DEV_NONFINITE);
}

// Whether some tensors' buffers share bytes that a step writes.  All buffers by their addresses: one that is written must
// begin behind all before it, one that is read behind those that are written.
bool buffers_meet(uint32_t count, const cvlc_adamw_tensor_t* tensors) {
  struct Span {
    uintptr_t first, end;
    bool written;
  };
  std::vector<Span> spans;
  spans.reserve(6 * (size_t)count);
  auto add = [&](const void* p, uint64_t bytes, bool written) {
    if (p && bytes) spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
  };
  for (uint32_t i = 0; i < count; ++i) {
    const cvlc_adamw_tensor_t& t = tensors[i];
    const uint64_t held = t.n * (t.state_bits / 8);
    add(t.d_param, 4 * t.n, true);
    add(t.d_grad, type_bytes(t.grad_type) * t.n, false);
    add(t.d_m, held, true);
    add(t.d_v, held, true);
    if (t.state_bits == 8) add(t.d_scales, (t.n + kHeld - 1) / kHeld * 8, true);
    add(t.d_copy, 2 * t.n, true);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.first < b.first; });
  uintptr_t any = 0, written = 0;
  for (const Span& s : spans) {
    if (s.first < written || (s.written && s.first < any)) return true;
    any = std::max(any, s.end);
    if (s.written) written = std::max(written, s.end);
  }
  return false;
}

bool tensor_ok(const cvlc_adamw_tensor_t& t) {
  if (t.state_bits != 8 && t.state_bits != 32) return false;
  if (!type_known(t.grad_type) || !std::isfinite(t.weight_decay) || (t.flags & ~CVLC_ADAMW_M_BY_CHANCE)) return false;
  if (t.d_copy && t.copy_type != CVLC_BF16 && t.copy_type != CVLC_F16) return false;
  if (t.n == 0) return true;
  if (t.n > 1ull << 35) return false;  // its eighths are counted in 32 bits
  if (!buffer_ok(t.d_param, 4) || !buffer_ok(t.d_grad, type_bytes(t.grad_type))) return false;
  if (t.d_copy && !buffer_ok(t.d_copy, 2)) return false;
  const uint32_t e = t.state_bits == 32 ? 4 : 1;
  if (!buffer_ok(t.d_m, e) || !buffer_ok(t.d_v, e)) return false;
  return t.state_bits == 32 || buffer_ok(t.d_scales, 8);
}

constexpr uint64_t kMostChunks = 1u << 23;  // a launch of fewer than 2^32 threads

// All chunks of a model; 0 where it has too many, or a tensor that does not go.
bool count_chunks(uint32_t count, const cvlc_adamw_tensor_t* t, uint64_t* chunks) {
  *chunks = 0;
  for (uint32_t i = 0; i < count; ++i) {
    if (!tensor_ok(t[i])) return false;
    *chunks += chunks_of(t[i].n);
  }
  return *chunks <= kMostChunks;
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_adamw_workspace_bytes(uint32_t count, const cvlc_adamw_tensor_t* tensors) {
  uint64_t chunks = 0;
  if (tensors)
    for (uint32_t i = 0; i < count; ++i) chunks += cvlc::chunks_of(tensors[i].n);
  return 256u + (size_t)count * sizeof(cvlc::Entry) + (size_t)chunks * 4u;
}

int cvlc_adamw_plan(uint32_t count, const cvlc_adamw_tensor_t* tensors, void* d_workspace, size_t ws_bytes,
                    cvlc_adamw_plan_t* plan_out, void* hip_stream) {
  using namespace cvlc;
  if (!plan_out || (count && !tensors) || !buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  uint64_t chunks;
  if (!count_chunks(count, tensors, &chunks)) return CVLC_ERR_ARG;
  if (ws_bytes < cvlc_adamw_workspace_bytes(count, tensors)) return CVLC_ERR_CAPACITY;
  try {
    if (buffers_meet(count, tensors)) return CVLC_ERR_ARG;
  } catch (const std::bad_alloc&) {
    return CVLC_ERR_CAPACITY;
  }
  Entry* entries = static_cast<Entry*>(d_workspace);
  uint32_t* tensor_of = reinterpret_cast<uint32_t*>(entries + count);
  uint64_t moved = 0;
  uint32_t at = 0;
  for (uint32_t first = 0; first < count; first += kPerUpload) {
    Upload u{};
    u.first = first;
    u.count = std::min(kPerUpload, count - first);
    uint64_t most = 1;
    for (uint32_t i = 0; i < u.count; ++i) {
      const cvlc_adamw_tensor_t& t = tensors[first + i];
      u.entry[i] = Entry{t.n, t.d_param, t.d_grad, t.d_m, t.d_v, t.d_scales, t.d_copy, at, (uint8_t)t.grad_type,
                         (uint8_t)t.copy_type, (uint8_t)t.state_bits, (uint8_t)t.flags, t.weight_decay};
      at += (uint32_t)chunks_of(t.n);
      most = std::max(most, chunks_of(t.n));
      moved += t.n * (4u + type_bytes(t.grad_type) + (t.d_copy ? 2u : 0u) + (t.state_bits == 32 ? 8u : 2u));
    }
    hipLaunchKernelGGL(adamw_table_kernel, dim3((uint32_t)std::min<uint64_t>((most + kAdamBlock - 1) / kAdamBlock, 256), u.count),
                       dim3(kAdamBlock), 0, static_cast<hipStream_t>(hip_stream), u, entries, tensor_of);
  }
  *plan_out = cvlc_adamw_plan_t{d_workspace, count, (uint32_t)chunks, moved};
  if (count == 0) return CVLC_OK;
  return hip_check(hipGetLastError());
}

int cvlc_adamw(const cvlc_adamw_plan_t* plan, const cvlc_adamw_rates_t* rates, const float* d_now, uint64_t seed,
               uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  if (!plan || !rates || !buffer_ok(plan->d_workspace, 256) || plan->chunks > kMostChunks) return CVLC_ERR_ARG;
  if (!(rates->beta1 >= 0.0 && rates->beta1 < 1.0 && rates->beta2 >= 0.0 && rates->beta2 < 1.0)) return CVLC_ERR_ARG;
  if (!((float)rates->eps > 0.0f && rates->eps <= 1e30)) return CVLC_ERR_ARG;
  if (d_now && !buffer_ok(d_now, 4)) return CVLC_ERR_ARG;
  if (!d_now && (rates->step < 1 || !std::isfinite(rates->lr) || !std::isfinite(rates->grad_scale))) return CVLC_ERR_ARG;
  if (d_status && !buffer_ok(d_status, 4)) return CVLC_ERR_ARG;
  if (plan->chunks == 0) return CVLC_OK;
  Rates r{};
  r.b1 = (float)rates->beta1;
  r.rest1 = (float)(1.0 - rates->beta1);
  r.b2 = (float)rates->beta2;
  r.rest2 = (float)(1.0 - rates->beta2);
  r.eps = (float)rates->eps;
  r.grad_scale = (float)rates->grad_scale;
  r.log_b1 = std::log(rates->beta1);
  r.log_b2 = std::log(rates->beta2);
  r.k0 = (uint32_t)seed;
  r.k1 = (uint32_t)(seed >> 32);
  if (!d_now) with_step(r, (float)rates->lr, rates->step);
  const Entry* entries = static_cast<const Entry*>(plan->d_workspace);
  const uint32_t* tensor_of = reinterpret_cast<const uint32_t*>(entries + plan->count);
  // past the caches' order where the caches do not hold it
  auto* kernel = plan->moved > 256ull * 1000000 ? adamw_kernel<true> : adamw_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(plan->chunks), dim3(kAdamBlock), 0, static_cast<hipStream_t>(hip_stream), entries, tensor_of, r,
                     d_now, d_status);
  return hip_check(hipGetLastError());
}

}  // extern "C"
