// cvlc_distill.hip -- distillation from a teacher's top logits: the loss of every
// row and the gradient of the student's logits.
//
// A row's logits give a maximum m and a sum S of exp((z - m) / T), kept as a
// running pair: a value above the maximum scales the sum so far.  Its list gives
// such a pair too.  Then every place of the gradient is w T P q, and the few
// listed ones are written again with their own gradient.
//
//   rows     a row in the registers of W wavefronts between the sum and the
//            gradient: one read, one write.  Workgroups go from row to row, and
//            every access that has been turned into gradient is loaded again
//            from the next row at once.
//            Rows of which only the loss or only the gradient is wanted too, as
//            long as they are one wavefront's.
//   long     longer rows: in passes of four accesses per thread.
//   part_sum, part_finish   few rows: parts of a row per workgroup, their pairs
//            joined by every workgroup that goes on with a part.
//
// Differences to m are taken before they are scaled: a scaled logit may overflow,
// a difference of exactly 0 may not.  m starts at the type's lowest finite value, so
// that a row of masked logits (-inf) ends with S = 0, which stands for q = 0, and a
// row of logits that are all at the lowest value ends like any other.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include <algorithm>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

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
  // few rows: the parts' pairs, [n][parts], and the listed logits, [n][k], read before any gradient may take their place
  uint32_t parts;
  float2* pairs;
  float* logits;
};

// exp((z - m) / T).  The instruction flushes results below 2^-126, which a sum of at least 1 does not notice.
__device__ __forceinline__ float exp_part(float z, float m, float c) { return __builtin_amdgcn_exp2f((z - m) * c); }
// What a row's exponentials are multiplied by.  Far below the maximum an exponential is lifted by 2^kLift into the
// normal range until the one product that may leave it, so that the smallest gradients are rounded once.  Next to the
// maximum that would cost bits (an exponent of 32 and more has a step of 2^-19, 11 roundings of fp32 in the result), so
// fp32 lifts beyond kFar alone, where the exponent's own step is no finer; 16-bit results do not notice and are spared the
// choice.  They do not lift a scale below kTiny: it would become subnormal and lose its bits, and what it makes of an
// exponential that needs a lift is 0.  Exponentials below 2^-158 become 0: no result of a scale up to 2^8 notices, and of a
// larger one what is that far below the row's largest.
constexpr float kLift = 32.0f, kUnlift = 0x1p-32f, kFar = -64.0f, kTiny = 0x1p-24f;
template <class T>
struct GradScale {
  float plain, lift, lifted;
  __device__ __forceinline__ explicit GradScale(float scale) : plain(scale), lift(kLift), lifted(scale * kUnlift) {
    if (sizeof(T) < 4 && fabsf(scale) < kTiny) {
      lift = 0.0f;
      lifted = scale;
    }
  }
};
// v becomes exp((v - m) / T) * scale, for results of type T
template <class T, uint32_t N>
__device__ __forceinline__ void exp_scaled(float (&v)[N], float m, float c, GradScale<T> s) {
  if constexpr (sizeof(T) == 4) {
    float least = INFINITY;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      v[i] = (v[i] - m) * c;
      least = fminf(least, v[i]);
    }
    if (least < kFar) {  // asked once for all of them: a choice for each took 2 % of the call
#pragma unroll
      for (uint32_t i = 0; i < N; ++i)
        v[i] = (v[i] < kFar ? s.lifted : s.plain) * __builtin_amdgcn_exp2f(v[i] < kFar ? v[i] + s.lift : v[i]);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[i] = s.plain * __builtin_amdgcn_exp2f(v[i]);
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = s.lifted * __builtin_amdgcn_exp2f(fmaf(v[i] - m, c, s.lift));
  }
}

// A maximum and the sum of exponentials relative to it.
struct MaxSum {
  float m, s;
};
constexpr MaxSum kNothing{-FLT_MAX, 0.0f};

template <uint32_t N>
__device__ __forceinline__ void take(MaxSum& t, const float (&v)[N], float c) {
  float m = t.m;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) m = fmaxf(m, v[i]);
  t.s *= exp_part(t.m, m, c);
  t.m = m;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) t.s += exp_part(v[i], m, c);
}
__device__ __forceinline__ MaxSum wave_join(MaxSum t, float c) {
  const float m = wave_max(t.m);
  return {m, wave_sum(t.s * exp_part(t.m, m, c))};
}

// ----------------------------------------------------------------------------- the teacher's list
__device__ __forceinline__ int64_t load_id(const void* ids, uint32_t id_bytes, uint64_t i) {
  return id_bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}
__device__ __forceinline__ float load_as_float(const void* p, uint32_t type, uint64_t i) {
  if (type == CVLC_F32) return static_cast<const float*>(p)[i];
  return type == CVLC_BF16 ? (float)static_cast<const bf16_t*>(p)[i] : (float)static_cast<const f16_t*>(p)[i];
}

// An entry of a list: its place in the row (-1: it is not there), its value and the student's logit, as it lies in memory.
template <class T>
struct Entry {
  int32_t id;
  float t;
  T z;
};
// As it lies in memory, to be looked at later.
struct RawEntry {
  int64_t id;
  float t;
  __device__ __forceinline__ void load(const DistillArgs& a, uint32_t row, uint32_t j) {
    const uint64_t at = (uint64_t)row * a.k + j;
    id = load_id(a.ids, a.id_bytes, at);
    t = load_as_float(a.values, a.value_type, at);
  }
};
template <class T>
__device__ __forceinline__ Entry<T> entry_of(const DistillArgs& a, RawEntry r, const T* zr, bool with_logit = true) {
  const bool inside = r.id >= 0 && r.id < (int64_t)a.vocab;
  if (r.id >= (int64_t)a.vocab && a.status) atomicOr(a.status, CVLC_DEV_INDEX);
  Entry<T> e{-1, r.t, (T)0.0f};
  if (inside && r.t != -INFINITY) {
    e.id = (int32_t)r.id;
    if (with_logit) e.z = zr[e.id];
  }
  return e;
}

// What a list's pair says: the scale that turns exp((t - m) c) into p, T ln p up to t, and P (0: the list is empty).
// T ln p and T ln q stay finite where ln p and ln q do not.
struct ListSums {
  float m, c, inv, tlog, slope, P;
  __device__ __forceinline__ ListSums(const DistillArgs& a, MaxSum t) {
    if (a.logprobs) {
      m = 0.0f;
      c = (float)M_LOG2E;
      inv = 1.0f;
      tlog = 0.0f;
      slope = a.T;
      P = t.s == 0.0f ? 0.0f : t.s * exp2f(t.m * c);
    } else {
      m = t.m;
      c = a.c;
      inv = 1.0f / t.s;
      tlog = a.T * logf(t.s);
      slope = 1.0f;
      P = t.s == 0.0f ? 0.0f : t.s == t.s ? 1.0f : t.s;
    }
  }
  __device__ __forceinline__ float p(float t) const { return exp2f((t - m) * c) * inv; }
  // p (T ln p - T ln q)
  __device__ __forceinline__ float loss(float t, float tlogq) const {
    const float pt = p(t);
    return pt == 0.0f ? 0.0f : pt * ((t - m) * slope - tlog - tlogq);
  }
};
// c of a list's pair while it is made
__device__ __forceinline__ float list_c(const DistillArgs& a) { return a.logprobs ? (float)M_LOG2E : a.c; }
__device__ __forceinline__ void take_entry(MaxSum& t, int32_t id, float value, float c) {
  if (id < 0) return;
  const float v[1] = {value};
  take<1>(t, v, c);
}
// T ln q of a logit
__device__ __forceinline__ float tlogq_of(const DistillArgs& a, float z, MaxSum t) {
  return t.s == 0.0f ? -INFINITY : (z - t.m) - a.T * logf(t.s);
}

// Lists in LDS, while a row is worked on: ids, p and logits, each of k entries and up to three without an id, so that four
// at a time can be read.
__host__ __device__ constexpr uint32_t list_room(uint32_t k) { return (k + 3u) & ~3u; }
struct ListLds {
  int32_t* id;
  float *p, *z;
  __device__ __forceinline__ ListLds(float* base, uint32_t k)
      : id(reinterpret_cast<int32_t*>(base)), p(base + list_room(k)), z(base + 2 * list_room(k)) {}
  // by any four threads
  __device__ __forceinline__ void end(uint32_t thread, uint32_t k) const {
    if (k + thread < list_room(k)) id[k + thread] = -1;
  }
};
constexpr uint32_t kListWords = 3;

// Entry j's place of a row's gradient.  Entries of one id share it, and each writes the whole sum: k^2 comparisons, four to
// a read of LDS and DEEP reads under way (one entry to a read, 3000 rows of 8000 bf16 with lists of 200: 65 us, now 41).
// DEEP is 1 where the next row fills the registers meanwhile (4096 rows of 131072: 498 us, 583 with four).
template <uint32_t DEEP, class T>
__device__ __forceinline__ void write_listed(const DistillArgs& a, const ListLds& l, uint32_t j, T* drow, MaxSum t, float P, float wT) {
  const int32_t id = l.id[j];
  if (id < 0) return;
  float p = 0.0f;
#pragma unroll DEEP
  for (uint32_t i = 0; i < a.k; i += 4) {
    const int4 ids = *reinterpret_cast<const int4*>(l.id + i);
    const float4 ps = *reinterpret_cast<const float4*>(l.p + i);
    p += ids.x == id ? ps.x : 0.0f;
    p += ids.y == id ? ps.y : 0.0f;
    p += ids.z == id ? ps.z : 0.0f;
    p += ids.w == id ? ps.w : 0.0f;
  }
  const float inv = t.s == 0.0f ? 0.0f : 1.0f / t.s;
  float q[1] = {l.z[j]};
  exp_scaled<T>(q, t.m, a.c, GradScale<T>(P * inv));
  drow[id] = (T)(wT * (q[0] - p));
}

template <uint32_t W>
__device__ __forceinline__ void group_sync() {
  if constexpr (W == 1)
    wave_sync();
  else
    __syncthreads();
}

// ----------------------------------------------------------------------------- rows in registers
// N elements of a row of `width` >= N from `first` on; see Place, whose values are worked out again where they are needed.
template <bool ONCE, class T, uint32_t N>
__device__ __forceinline__ void load_place(Raw<T, N>& raw, const T* row, uint32_t first, uint32_t width) {
  if (first < width) raw.template load<ONCE>(row + min(first, width - N));
}

// A place that is worked out where the row ends and nowhere else: known before the loop over the rows, the masks of 16 of
// them would be held all along, and there are not that many registers.
template <uint32_t N>
__device__ __forceinline__ Place<N> place_here(uint32_t first, uint32_t width) {
  asm volatile("" : "+v"(first));
  return Place<N>(first, width);
}

// W wavefronts to a row, V accesses per thread; workgroups of at least four wavefronts, which are then rows of their own.
template <class T, bool LOSS, bool GRAD, bool ONCE, uint32_t W, uint32_t V, uint32_t O>
__global__ __launch_bounds__((W == 1 ? 4 : W) * kWave, O) void distill_rows_kernel(DistillArgs a, const T* logits, T* dlogits) {
  constexpr uint32_t N = kPerAccess<T>, L = W * kWave, ROWS = W == 1 ? 4 : 1;
  extern __shared__ float4 list_space[];  // [ROWS][2][kListWords][list_room(k)]
  float* lists = reinterpret_cast<float*>(list_space);
  __shared__ float4 pairs[2][ROWS][W];
  __shared__ float losses[2][ROWS][W];
  // a row is the same in all of a wavefront's lanes: said so, its addresses are in scalar registers
  const uint32_t mine = ROWS == 1 ? 0u : __builtin_amdgcn_readfirstlane(threadIdx.x / L), step = gridDim.x * ROWS;
  const uint32_t lane = threadIdx.x % L, wave = __builtin_amdgcn_readfirstlane(lane / kWave);
  uint32_t row = blockIdx.x * ROWS + mine, turn = 0;
  Raw<T, N> raw[V];
  RawEntry entry{-1, 0.0f};
#pragma unroll
  for (uint32_t j = 0; j < V; ++j)
#pragma unroll
    for (uint32_t i = 0; i < Raw<T, N>::kWords; ++i) raw[j].w[i] = 0;
  const bool has_entry = lane < a.k;
  float w = 0.0f;
  if (row < a.n) {
    w = a.weights ? a.weights[row] : 1.0f;
    if (w != 0.0f) {
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) load_place<ONCE>(raw[j], logits + row * a.stride, (j * L + lane) * N, a.vocab);
      if (has_entry) entry.load(a, row, lane);
    }
  }
  for (; row < a.n; row += step) {
    const T* zr = logits + row * a.stride;
    const uint32_t next = row + step;
    const bool more = next < a.n;
    const float w_next = !more ? 0.0f : a.weights ? a.weights[next] : 1.0f;
    const bool load_next = w_next != 0.0f;
    const T* zn = logits + (uint64_t)(more ? next : row) * a.stride;
    const ListLds l(lists + (2 * mine + turn) * kListWords * list_room(a.k), a.k);
    MaxSum t = kNothing;
    float P = 0.0f;
    if (w != 0.0f) {
      // the list: every thread its entries
      Entry<T> e{-1, 0.0f, (T)0.0f};
      MaxSum q = kNothing;
      const float lc = list_c(a);
      if (has_entry) e = entry_of(a, entry, zr);
      for (uint32_t j = lane + L; j < a.k; j += L) {
        RawEntry r;
        r.load(a, row, j);
        const Entry<T> f = entry_of(a, r, zr);
        take_entry(q, f.id, f.t, lc);
        l.id[j] = f.id;
        l.p[j] = f.t;
        l.z[j] = (float)f.z;
      }
      take_entry(q, e.id, e.t, lc);
      if (LOSS) {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
          const uint32_t first = (j * L + lane) * N;
          if (first >= a.vocab) break;
          float v[N];
          raw[j].values(v);
          if (first + N > a.vocab) place_here<N>(first, a.vocab).mask(v, -INFINITY);
          take(t, v, a.c);
          if (!GRAD && load_next) load_place<ONCE>(raw[j], zn, first, a.vocab);
        }
        t = wave_join(t, a.c);
      }
      q = wave_join(q, lc);
      l.end(lane, a.k);
      if (has_entry) {
        l.id[lane] = e.id;
        l.p[lane] = e.t;
        l.z[lane] = (float)e.z;
      }
      if (W > 1) {
        if (lane_id() == 0) pairs[turn][mine][wave] = make_float4(t.m, t.s, q.m, q.s);
        __syncthreads();
        const float4 x = lane_id() < W ? pairs[turn][mine][lane_id()] : make_float4(-FLT_MAX, 0.0f, -FLT_MAX, 0.0f);
        if (LOSS) t = wave_join({x.x, x.y}, a.c);
        q = wave_join({x.z, x.w}, lc);
      } else {
        wave_sync();
      }
      if (!LOSS) t = {a.stats[2 * (uint64_t)row], a.stats[2 * (uint64_t)row + 1]};
      const ListSums s(a, q);
      P = s.P;
      // p of every entry, and the loss
      float loss = 0.0f;
      for (uint32_t j = lane; j < a.k; j += L) {
        if (l.id[j] < 0) continue;
        const float value = l.p[j];
        if (LOSS) loss += w * a.T * s.loss(value, tlogq_of(a, l.z[j], t));
        l.p[j] = s.p(value);
      }
      if (LOSS) {
        loss = wave_sum(loss);
        if (W > 1 && lane_id() == 0) losses[turn][mine][wave] = loss;
        if (W == 1 && lane == 0 && a.loss) a.loss[row] = loss;
        if (lane == 0 && a.stats) {
          a.stats[2 * (uint64_t)row] = P == 0.0f ? 0.0f : t.m;
          a.stats[2 * (uint64_t)row + 1] = P == 0.0f ? 0.0f : t.s;
        }
      }
    } else if (LOSS && lane == 0) {
      if (a.loss) a.loss[row] = 0.0f;
      if (a.stats) a.stats[2 * (uint64_t)row] = a.stats[2 * (uint64_t)row + 1] = 0.0f;
    }
    if (load_next && has_entry) entry.load(a, next, lane);
    if (GRAD || w == 0.0f) {
      T* dr = GRAD ? dlogits + row * a.dstride : nullptr;
      const GradScale<T> scale(P == 0.0f || t.s == 0.0f ? 0.0f : w * a.T * P * (1.0f / t.s));
      const bool nothing = P == 0.0f;
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) {
        const uint32_t first = (j * L + lane) * N;
        if (first >= a.vocab) break;
        if constexpr (GRAD) {
          float v[N];
          raw[j].values(v);
          exp_scaled<T>(v, t.m, a.c, scale);
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) v[i] = nothing ? 0.0f : v[i];
          if (first + N <= a.vocab)
            store_whole<ONCE, N>(dr + first, v);
          else
            place_here<N>(first, a.vocab).template store<ONCE>(dr, v);
        }
        if (load_next) load_place<ONCE>(raw[j], zn, first, a.vocab);
      }
    }
    if (w != 0.0f) {
      group_sync<W>();  // every place is written, every p known
      if (LOSS && W > 1 && lane == 0 && a.loss) {
        float sum = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < W; ++i) sum += losses[turn][mine][i];
        a.loss[row] = sum;
      }
      if (GRAD && P != 0.0f)
        for (uint32_t j = lane; j < a.k; j += L) write_listed<(V < 16 ? 4 : 1)>(a, l, j, dlogits + row * a.dstride, t, P, w * a.T);
      turn ^= 1;  // the other half of LDS: this one may still be read
    }
    w = w_next;
  }
}

// ----------------------------------------------------------------------------- long rows, parts of rows
constexpr uint32_t kLongBlock = 512, kLongWaves = kLongBlock / kWave;
constexpr uint32_t kDeep = 4;  // accesses under way per thread

// f(first, values) over elements [from, to) of a row, four accesses per thread at a time.  Elements beyond `to` read -inf.
template <bool ONCE, class T, class F>
__device__ __forceinline__ void over_row(const T* zr, uint32_t from, uint32_t to, F f) {
  constexpr uint32_t N = kPerAccess<T>;
  for (uint64_t base = from + threadIdx.x * N; base < to; base += kDeep * kLongBlock * N) {
    Raw<T, N> raw[kDeep];
#pragma unroll
    for (uint32_t u = 0; u < kDeep; ++u) {
      const uint64_t first = base + u * kLongBlock * N;
      if (first + N <= to) raw[u].template load<ONCE>(zr + first);
    }
#pragma unroll
    for (uint32_t u = 0; u < kDeep; ++u) {
      const uint64_t first = base + u * kLongBlock * N;
      float v[N];
      if (first + N <= to)
        raw[u].values(v);
      else if (first < to)
        load_some<N>(zr + first, (uint32_t)(to - first), -INFINITY, v);
      else
        break;
      f((uint32_t)first, v);
    }
  }
}
template <bool ONCE, uint32_t N, class T>
__device__ __forceinline__ void store_part(T* row, uint32_t first, uint32_t to, const float (&v)[N]) {
  if (first + N <= to)
    store_whole<ONCE, N>(row + first, v);
  else
    store_some<N>(row + first, to - first, v);
}

// The pair of a workgroup from its threads'.
__device__ __forceinline__ MaxSum block_join(MaxSum t, float c, float2* scratch) {
  t = wave_join(t, c);
  __syncthreads();
  if (lane_id() == 0) scratch[wave_id()] = make_float2(t.m, t.s);
  __syncthreads();
  const float2 x = lane_id() < kLongWaves ? scratch[lane_id()] : make_float2(-FLT_MAX, 0.0f);
  return wave_join({x.x, x.y}, c);
}

// A row's list into LDS, with values in the place of p.  Its sums; all threads.  `saved`: the listed logits, or NULL.
template <class T>
__device__ __forceinline__ ListSums load_list(const DistillArgs& a, uint32_t row, const T* zr, const float* saved, const ListLds& l,
                                              float2* scratch) {
  MaxSum q = kNothing;
  const float c = list_c(a);
  l.end(threadIdx.x, a.k);
  for (uint32_t j = threadIdx.x; j < a.k; j += kLongBlock) {
    RawEntry r;
    r.load(a, row, j);
    const Entry<T> e = entry_of(a, r, zr, !saved);
    take_entry(q, e.id, e.t, c);
    l.id[j] = e.id;
    l.p[j] = e.t;
    l.z[j] = saved ? saved[j] : (float)e.z;
  }
  return ListSums(a, block_join(q, c, scratch));
}
// Turns the values into p; the loss (a thread's share of it).
__device__ __forceinline__ float finish_list(const DistillArgs& a, const ListLds& l, const ListSums& s, MaxSum t, float wT) {
  float loss = 0.0f;
  for (uint32_t j = threadIdx.x; j < a.k; j += kLongBlock) {
    if (l.id[j] < 0) continue;
    const float value = l.p[j];
    loss += wT * s.loss(value, tlogq_of(a, l.z[j], t));
    l.p[j] = s.p(value);
  }
  return loss;
}

// Elements [from, to) of a row's gradient.
template <bool ONCE, class T>
__device__ __forceinline__ void write_gradient(const DistillArgs& a, const T* zr, T* dr, uint32_t from, uint32_t to, MaxSum t, float P,
                                               float wT) {
  constexpr uint32_t N = kPerAccess<T>;
  if (P == 0.0f) {
    const float zero[N] = {};
    for (uint64_t first = from + threadIdx.x * N; first < to; first += kLongBlock * N) store_part<ONCE, N>(dr, (uint32_t)first, to, zero);
    return;
  }
  const GradScale<T> scale(t.s == 0.0f ? 0.0f : wT * P * (1.0f / t.s));
  over_row<ONCE>(zr, from, to, [&](uint32_t first, float (&v)[N]) {
    exp_scaled<T>(v, t.m, a.c, scale);
    store_part<ONCE, N>(dr, first, to, v);
  });
}

// A workgroup per row (LOSS, PARTS = false) or per part of a row, whose pairs or statistics are known then.
template <class T, bool LOSS, bool GRAD, bool ONCE, bool PARTS>
__global__ __launch_bounds__(kLongBlock) void distill_long_kernel(DistillArgs a, const T* logits, T* dlogits) {
  constexpr uint32_t N = kPerAccess<T>;
  extern __shared__ float4 list_space[];
  __shared__ float2 scratch[kLongWaves];
  __shared__ float sums[kLongWaves];
  const ListLds l(reinterpret_cast<float*>(list_space), a.k);
  const uint32_t part = PARTS ? blockIdx.y : 0u;
  const uint32_t each = PARTS ? ((a.vocab + a.parts - 1) / a.parts + N - 1) / N * N : a.vocab;
  const uint32_t from = min((uint64_t)part * each, (uint64_t)a.vocab), to = min((uint64_t)from + each, (uint64_t)a.vocab);
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* zr = logits + row * a.stride;
    T* dr = GRAD ? dlogits + row * a.dstride : nullptr;
    const float w = a.weights ? a.weights[row] : 1.0f, wT = w * a.T;
    MaxSum t = kNothing;
    float P = 0.0f;
    __syncthreads();
    if (w != 0.0f) {
      const ListSums s = load_list(a, row, zr, PARTS && LOSS ? a.logits + (uint64_t)row * a.k : nullptr, l, scratch);
      P = s.P;
      if (P != 0.0f) {
        if (!LOSS) {
          t = {a.stats[2 * (uint64_t)row], a.stats[2 * (uint64_t)row + 1]};
        } else if (PARTS) {
          for (uint32_t i = lane_id(); i < a.parts; i += kWave) {
            const float2 x = a.pairs[(uint64_t)row * a.parts + i];
            const float m = fmaxf(t.m, x.x);
            t = {m, t.s * exp_part(t.m, m, a.c) + x.y * exp_part(x.x, m, a.c)};
          }
          t = wave_join(t, a.c);
        } else {
          over_row<false>(zr, from, to, [&](uint32_t, float (&v)[N]) { take(t, v, a.c); });
          t = block_join(t, a.c, scratch);
        }
        const float loss = finish_list(a, l, s, t, wT);
        if (LOSS && part == 0) {
          const float sum = block_sum<kLongWaves>(loss, sums);
          if (threadIdx.x == 0) {
            if (a.loss) a.loss[row] = sum;
            if (a.stats) {
              a.stats[2 * (uint64_t)row] = t.m;
              a.stats[2 * (uint64_t)row + 1] = t.s;
            }
          }
        }
      }
    }
    if (LOSS && P == 0.0f && part == 0 && threadIdx.x == 0) {
      if (a.loss) a.loss[row] = 0.0f;
      if (a.stats) a.stats[2 * (uint64_t)row] = a.stats[2 * (uint64_t)row + 1] = 0.0f;
    }
    if (GRAD) {
      __syncthreads();  // every listed logit has been read: the gradient may take the logits' place
      write_gradient<ONCE>(a, zr, dr, from, to, t, P, wT);
      __syncthreads();
      if (P != 0.0f)
        for (uint32_t j = threadIdx.x; j < a.k; j += kLongBlock)
          if (l.id[j] >= (int32_t)from && l.id[j] < (int32_t)to) write_listed<4>(a, l, j, dr, t, P, wT);
    }
  }
}

// The pair of a part of a row.
template <class T>
__global__ __launch_bounds__(kLongBlock) void part_sum_kernel(DistillArgs a, const T* logits) {
  constexpr uint32_t N = kPerAccess<T>;
  __shared__ float2 scratch[kLongWaves];
  const uint32_t row = blockIdx.x, part = blockIdx.y, each = ((a.vocab + a.parts - 1) / a.parts + N - 1) / N * N;
  const uint32_t from = min((uint64_t)part * each, (uint64_t)a.vocab), to = min((uint64_t)from + each, (uint64_t)a.vocab);
  if (a.weights && a.weights[row] == 0.0f) return;
  if (part == 0)
    for (uint32_t j = threadIdx.x; j < a.k; j += kLongBlock) {
      RawEntry r;
      r.load(a, row, j);
      if (r.id >= 0 && r.id < (int64_t)a.vocab) a.logits[(uint64_t)row * a.k + j] = (float)logits[row * a.stride + r.id];
    }
  MaxSum t = kNothing;
  over_row<false>(logits + row * a.stride, from, to, [&](uint32_t, float (&v)[N]) { take(t, v, a.c); });
  t = block_join(t, a.c, scratch);
  if (threadIdx.x == 0) a.pairs[(uint64_t)row * a.parts + part] = make_float2(t.m, t.s);
}

// ----------------------------------------------------------------------------- host
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

template <uint32_t W_, uint32_t V_, uint32_t O_>
struct RowShape {
  static constexpr uint32_t W = W_, V = V_, O = O_, kRows = W == 1 ? 4 : 1, kWaves = W * kRows;
  static constexpr uint32_t kPerCu = 4 * O > kWaves ? 4 * O / kWaves : 1;
};
// Registers hold the row (16 bytes an access), and a thread's 128 hold up to 16 of them at four wavefronts a SIMD, so a CU has
// one row of 131072 bf16 at a time: 4096 of them 490 us, 4.1 TB/s (two passes over each row, from HBM and then from the
// caches, 692).  8192 rows of 32000 bf16 215 us, 4.9 TB/s.
// Calls f with the shape that holds a row of `accesses`; false: none does, or there is none for rows that are only read or
// only written.
template <bool BOTH, class F>
bool by_row_shape(uint32_t accesses, F f) {
  if (accesses <= 64) return f(RowShape<1, 1, 8>{});
  if (accesses <= 128) return f(RowShape<1, 2, 6>{});
  if (accesses <= 256) return f(RowShape<1, 4, 4>{});
  if constexpr (BOTH) {
    if (accesses <= 512) return f(RowShape<4, 2, 6>{});
    if (accesses <= 1024) return f(RowShape<4, 4, 4>{});
    if (accesses <= 2048) return f(RowShape<8, 4, 4>{});
    if (accesses <= 4096) return f(RowShape<8, 8, 4>{});
    if (accesses <= 8192) return f(RowShape<16, 8, 4>{});
    if (accesses <= 16384) return f(RowShape<16, 16, 4>{});
  }
  return false;
}

// Parts that few rows are cut into, by elements alone, so that the workspace does not depend on their type: 1 = none.
// 24 rows of 200003 fp16, the loss: 11 us, 36 with a workgroup per row.
constexpr uint32_t kPartRows = 512, kPartElements = 8192;
uint32_t parts_for(uint32_t n, uint32_t vocab) {
  if (n == 0 || n >= kPartRows) return 1;
  return std::max(1u, std::min(vocab / kPartElements, (2 * kPartRows + n - 1) / n));
}

bool once(uint32_t n, uint32_t vocab, uint32_t bytes) { return (uint64_t)n * vocab * bytes > 256ull * 1000000; }

template <bool LOSS, bool GRAD>
int launch(DistillArgs a, uint32_t type, const void* logits, void* dlogits, hipStream_t stream) {
  by_type(type, [&](auto t) {
    using T = decltype(t);
    constexpr uint32_t N = kPerAccess<T>;
    const T* z = static_cast<const T*>(logits);
    T* d = static_cast<T*>(dlogits);
    const bool past = once(a.n, a.vocab, (GRAD ? 2 : 1) * sizeof(T));
    if (a.parts > 1) {
      const uint32_t lds = kListWords * list_room(a.k) * sizeof(float);
      if (LOSS) hipLaunchKernelGGL(part_sum_kernel<T>, dim3(a.n, a.parts), dim3(kLongBlock), 0, stream, a, z);
      hipLaunchKernelGGL((distill_long_kernel<T, LOSS, GRAD, false, true>), dim3(a.n, GRAD ? a.parts : 1), dim3(kLongBlock), lds, stream,
                         a, z, d);
      return;
    }
    if (a.vocab >= N && by_row_shape<LOSS && GRAD>((a.vocab + N - 1) / N, [&](auto shape) {
          using S = decltype(shape);
          const uint32_t lds = S::kRows * 2 * kListWords * list_room(a.k) * sizeof(float);
          const uint32_t grid = std::min((a.n + S::kRows - 1) / S::kRows, 256u * S::kPerCu);
          auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(S::kWaves * kWave), lds, stream, a, z, d); };
          if (past)
            go(distill_rows_kernel<T, LOSS, GRAD, true, S::W, S::V, S::O>);
          else
            go(distill_rows_kernel<T, LOSS, GRAD, false, S::W, S::V, S::O>);
          return true;
        }))
      return;
    const uint32_t lds = kListWords * list_room(a.k) * sizeof(float);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(std::min(a.n, 1u << 20)), dim3(kLongBlock), lds, stream, a, z, d); };
    if (past)
      go(distill_long_kernel<T, LOSS, GRAD, true, false>);
    else
      go(distill_long_kernel<T, LOSS, GRAD, false, false>);
  });
  return hip_check(hipGetLastError());
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_distill_workspace_bytes(uint32_t n, uint32_t vocab) {
  using namespace cvlc;
  (void)vocab;
  // the most that fewer rows need, and rows that are not cut need nothing: never less for more rows or longer ones
  const uint64_t rows = std::min(n, kPartRows);
  return 256u + (size_t)((rows * kMaxK * sizeof(float)) + (2 * kPartRows + 2 * rows) * sizeof(float2));
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
  const uint32_t parts = parts_for(n, vocab);
  float2* pairs = static_cast<float2*>(d_workspace);
  const DistillArgs a{n, vocab, k, stride, dlogits_stride, d_ids, d_values, id_bytes, value_type, temperature,
                      (float)(M_LOG2E / temperature), flags & CVLC_DISTILL_LOGPROBS, d_weights, d_loss, d_stats, d_status,
                      parts, pairs, reinterpret_cast<float*>(pairs + (uint64_t)n * parts)};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return d_dlogits ? launch<true, true>(a, type, d_logits, d_dlogits, stream) : launch<true, false>(a, type, d_logits, nullptr, stream);
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
  // in place a part's gradient might take a listed logit's place before another part's workgroup has read it
  const uint32_t parts = d_dlogits == d_logits ? 1u : parts_for(n, vocab);
  const DistillArgs a{n, vocab, k, stride, dlogits_stride, d_ids, d_values, id_bytes, value_type, temperature,
                      (float)(M_LOG2E / temperature), flags & CVLC_DISTILL_LOGPROBS, d_weights, nullptr,
                      const_cast<float*>(d_stats), d_status, parts, nullptr, nullptr};
  return launch<false, true>(a, type, d_logits, d_dlogits, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
