// cvlc_scan.hip -- a gated linear recurrence over sequences, channel by channel, and its backward pass.
//
// Forward, with f = sigmoid(gate):   h_t = f_t h_(t-1) + (1 - f_t) x_t.
// Backward, with c_t = f_t D_t what a token hands to the one before it:
//   D_t = dy_t + c_(t+1),   c_t = f_t (dy_t + c_(t+1)),
//   dx_t = (1 - f_t) D_t,   dgate_t = D_t (h_(t-1) - x_t) f_t (1 - f_t).
// Both are one walk, u <- a u + b, that way and back: steps chain as (A, B), u <- A u + B,
// so rows are cut into pieces whose (A, B) are found side by side and joined.
//
// A workgroup has a block of channels and goes over its rows some hundred at a time:
// every thread has `L` rows of 16 bytes' worth of channels in registers, the threads'
// (A, B) meet in LDS, and each thread walks its rows again from what comes before
// them.  Rows are read once that way, bound by HBM: the arithmetic (an exponential
// and a reciprocal a value) is less than half of the time that the bytes take.  Where sequences and
// channels are too few to fill the device, each is cut into ranges: one launch finds
// the ranges' (A, B), which reads the walk's two inputs once more, the next joins
// those before its own and writes.  No workgroup waits for another.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kScanBlock = 512;
constexpr uint32_t kGroupsMost = 16;    // threads side by side on a row: 256 bytes of it
constexpr uint32_t kSteps = 8;          // L: rows of a thread

struct ScanArgs {
  uint32_t n, dim, n_seq, start_bytes;
  const void* starts;                   // null: sequences of `each` rows
  uint32_t each;
  uint32_t flat, walks, len;            // what is walked: every sequence, or (flat) once all rows of all sequences
  uint32_t ranges, range_len;           // parts of a walk, of whole iterations
  uint32_t groups_log2, blocks;         // threads on a row, blocks of channels
  uint64_t v_stride, gate_stride, x_stride, h_stride, out_stride, dgate_stride;
  const float* first;                   // what walks start from: h0, or the last state's gradient
  const float* h0;                      // backward: the state before a sequence's first row
  float* last;                          // what they end with: the last state, or the first one's gradient
  uint32_t main_grid;                   // workgroups that walk; those behind them see to sequences without rows
  float2* partial;                      // (A, B) of every range and channel
  uint32_t* status;
};

// Sequence j's first row; j = n_seq: the end of all.
__device__ __forceinline__ int64_t start_as_given(const ScanArgs& a, uint32_t j) {
  if (!a.starts) return (int64_t)j * a.each;
  return a.start_bytes == 8 ? static_cast<const int64_t*>(a.starts)[j] : (int64_t)static_cast<const int32_t*>(a.starts)[j];
}
__device__ __forceinline__ uint32_t start_of(const ScanArgs& a, uint32_t j) {
  return (uint32_t)min(max(start_as_given(a, j), (int64_t)0), (int64_t)a.n);
}

// f = sigmoid(z) and 1 - f, each with its own last bits.  The product with log2 e is taken apart: its rounding would
// grow with |z|.
__device__ __forceinline__ void gates(float z, float& f, float& rest) {
  constexpr float kLog2E = 0x1.715476p+0f, kLow = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
  float x = fabsf(z);
  x = x > 120.0f ? 120.0f : x;          // a NaN stays one
  const float t = -x * kLog2E;
  const float low = fmaf(-x, kLog2E, -t) - x * kLow;
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, low * kLn2, e);
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  f = z >= 0.0f ? r : e * r;
  rest = z >= 0.0f ? e * r : r;
}

// Marks of an iteration's rows, by their place in it: the sequence that begins, or ends, with a row; -1: none.
template <uint32_t W>
struct Marks {
  int32_t begins[W], ends[W];
  uint32_t any;
};

// Rows [low, high) of an iteration.  Where sequences are few everybody looks at one or two boundaries, else the first that
// matters is searched for.
template <uint32_t W>
__device__ __forceinline__ void fill_marks(const ScanArgs& a, uint32_t low, uint32_t high, uint32_t most, Marks<W>& marks) {
  __syncthreads();                      // the iteration before is done with them
  for (uint32_t i = threadIdx.x; i < most; i += kScanBlock) marks.begins[i] = marks.ends[i] = -1;
  if (threadIdx.x == 0) marks.any = 0;
  __syncthreads();
  uint32_t from = 0;
  if (a.n_seq >= kScanBlock) {          // the first boundary at or behind `low`
    uint32_t end = a.n_seq + 1;
    while (from < end) {
      const uint32_t mid = (from + end) / 2;
      if (start_of(a, mid) < low)
        from = mid + 1;
      else
        end = mid;
    }
  }
  for (uint32_t j = from + threadIdx.x; j <= a.n_seq; j += kScanBlock) {
    const uint32_t at = start_of(a, j);
    if (at > high && a.n_seq >= kScanBlock) break;
    if (at < low || at > high) continue;
    if (j < a.n_seq && at < high && start_of(a, j + 1) > at) {
      marks.begins[at - low] = (int32_t)j;
      marks.any = 1;
    }
    if (j > 0 && at > low && start_of(a, j - 1) < at) {
      marks.ends[at - 1 - low] = (int32_t)j - 1;
      marks.any = 1;
    }
  }
  __syncthreads();
}

// N channels of a row: 16 bytes, or as many as there are where rows are narrower.
template <class T, uint32_t N>
__device__ __forceinline__ void load_channels(Raw<T, N>& raw, const T* row, uint32_t at, uint32_t dim) {
  if (dim >= N)
    raw.template load<false>(row + at);
  else
    load_raw(raw, row, at, dim);
}
template <uint32_t N>
__device__ __forceinline__ void load_state(const float* p, uint64_t seq, uint32_t at, uint32_t dim, float (&u)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) u[k] = p && at + k < dim ? p[seq * dim + at + k] : 0.0f;
}
template <uint32_t N>
__device__ __forceinline__ void store_state(float* p, uint64_t seq, uint32_t at, uint32_t dim, const float (&u)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k)
    if (p && at + k < dim) p[seq * dim + at + k] = u[k];
}

// Where a thread and its workgroup are.
template <uint32_t N>
struct Spot {
  uint32_t group, row, rows;            // of the workgroup's threads
  uint32_t at;                          // first channel
  uint32_t walk, range;
  __device__ __forceinline__ Spot(const ScanArgs& a, uint32_t block) {
    const uint32_t groups = 1u << a.groups_log2;
    group = threadIdx.x & (groups - 1);
    row = threadIdx.x >> a.groups_log2;
    rows = kScanBlock >> a.groups_log2;
    const uint32_t c = block % a.blocks;
    // the last threads of a row move back to end with it: channels that two threads have come out the same from both
    const uint32_t want = (c * groups + group) * N;
    at = a.dim >= N ? min(want, a.dim - N) : 0u;
    walk = block / a.blocks / a.ranges;
    range = block / a.blocks % a.ranges;
  }
};

// The workgroup's joined steps: after it `in` is what comes before the thread's rows.  carry[ch]: what comes before all rows,
// then what comes after them; FACTOR: factor[ch] is multiplied by their A.
template <uint32_t N, bool FACTOR>
__device__ __forceinline__ void join(const Spot<N>& s, uint32_t groups, float (&A)[N], float (&B)[N], float* sa, float* sb, float* carry,
                                     float* factor, float (&in)[N]) {
  const uint32_t width = groups * N, mine = s.row * width + s.group * N;
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    sa[mine + k] = A[k];
    sb[mine + k] = B[k];
  }
  __syncthreads();
  if (threadIdx.x < width) {
    float u = carry[threadIdx.x], f = FACTOR ? factor[threadIdx.x] : 0.0f;
#pragma unroll 8
    for (uint32_t r = 0; r < s.rows; ++r) {
      const float x = sa[r * width + threadIdx.x], y = sb[r * width + threadIdx.x];
      sb[r * width + threadIdx.x] = u;
      u = fmaf(x, u, y);
      if (FACTOR) f *= x;
    }
    carry[threadIdx.x] = u;
    if (FACTOR) factor[threadIdx.x] = f;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) in[k] = sb[mine + k];
}

// FORWARD or back.  WRITE: the walk's results are written; else the range's (A, B) are found.
template <class T, bool FORWARD, bool WRITE>
__global__ __launch_bounds__(kScanBlock) void scan_kernel(ScanArgs a, const T* v, const T* gate, const T* x, const T* h, T* out, T* dgate) {
  constexpr uint32_t N = kPerAccess<T>, L = kSteps;
  constexpr uint32_t kMarks = kScanBlock * L;
  __shared__ float sa[kScanBlock * N], sb[kScanBlock * N], carry[kGroupsMost * N], factor[kGroupsMost * N];
  __shared__ Marks<kMarks> marks;
  if (WRITE && blockIdx.x >= a.main_grid) {
    // sequences without rows hand on what they start from; offsets that are out of order or out of the rows are told of
    for (uint32_t j = (blockIdx.x - a.main_grid) * kScanBlock + threadIdx.x; j < a.n_seq; j += (gridDim.x - a.main_grid) * kScanBlock) {
      const int64_t from = start_as_given(a, j), to = start_as_given(a, j + 1);
      if (a.status && (from < 0 || to < from || to > (int64_t)a.n)) atomicOr(a.status, CVLC_DEV_INDEX);
      if (a.last && start_of(a, j + 1) <= start_of(a, j))
        for (uint32_t c = 0; c < a.dim; ++c) a.last[(uint64_t)j * a.dim + c] = a.first ? a.first[(uint64_t)j * a.dim + c] : 0.0f;
    }
    return;
  }
  const uint32_t main_blocks = a.walks * a.ranges * a.blocks;
  for (uint32_t block = blockIdx.x; block < main_blocks; block += a.main_grid) {
  // the launch that writes goes the other way round: what the one before read last may still be in the last-level cache
  const Spot<N> s(a, WRITE && a.ranges > 1 ? main_blocks - 1 - block : block);
  const uint32_t groups = 1u << a.groups_log2, width = groups * N, W = s.rows * L;
  const uint32_t base = s.walk * a.len;
  uint32_t live_low = base, live_high = base + a.len;     // rows that belong to a sequence
  if (a.flat) {
    live_low = start_of(a, 0);
    live_high = start_of(a, a.n_seq);
  }
  const bool ends_here = !a.flat && s.range + 1 == a.ranges;
  float in[N], A[N], B[N];
  // what comes before the range: the walk's start through all ranges before
  if (threadIdx.x < width) {
    carry[threadIdx.x] = 0.0f;
    factor[threadIdx.x] = 1.0f;
  }
  __syncthreads();
  if (WRITE && !a.flat && s.row == 0) {
    load_state<N>(a.first, s.walk, s.at, a.dim, in);
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) carry[s.group * N + k] = in[k];
  }
  __syncthreads();
  if (WRITE && s.range > 0) {
    const uint32_t per = (s.range + s.rows - 1) / s.rows;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) A[k] = 1.0f, B[k] = 0.0f;
    for (uint32_t q = s.row * per; q < min((s.row + 1) * per, s.range); ++q) {
      const float2* p = a.partial + ((uint64_t)s.walk * a.ranges + q) * a.dim + s.at;
#pragma unroll
      for (uint32_t k = 0; k < N; ++k)
        if (s.at + k < a.dim) {
          const float2 ab = p[k];
          A[k] *= ab.x;
          B[k] = fmaf(ab.x, B[k], ab.y);
        }
    }
    join<N, false>(s, groups, A, B, sa, sb, carry, nullptr, in);
    __syncthreads();
  }
  const uint32_t first_p = s.range * a.range_len, end_p = min(first_p + a.range_len, a.len);
  for (uint32_t p0 = first_p; p0 < end_p; p0 += W) {
    const uint32_t count = min(W, end_p - p0);            // rows of this iteration
    const uint32_t low = FORWARD ? base + p0 : base + a.len - p0 - count;
    auto row_of = [&](uint32_t i) { return FORWARD ? low + s.row * L + i : low + count - 1 - s.row * L - i; };
    auto there = [&](uint32_t i) {
      const uint32_t t = row_of(i);
      return s.row * L + i < count && t >= live_low && t < live_high;
    };
    Raw<T, N> rv[L], rg[L], rx[L], rh[L];
#pragma unroll
    for (uint32_t i = 0; i < L; ++i)
      if (there(i)) {
        load_channels<T, N>(rg[i], gate + row_of(i) * a.gate_stride, s.at, a.dim);
        load_channels<T, N>(rv[i], v + row_of(i) * a.v_stride, s.at, a.dim);
      }
    if (WRITE && !FORWARD) {
#pragma unroll
      for (uint32_t i = 0; i < L; ++i)
        if (there(i)) {
          load_channels<T, N>(rx[i], x + row_of(i) * a.x_stride, s.at, a.dim);
          if (row_of(i) > live_low) load_channels<T, N>(rh[i], h + (row_of(i) - 1) * a.h_stride, s.at, a.dim);
        }
    }
    bool marked = false;
    if (a.flat) {
      fill_marks<kMarks>(a, low, low + count, count, marks);
      marked = marks.any;
    }
    auto mark = [&](const int32_t* m, uint32_t i) { return marked ? m[row_of(i) - low] : -1; };
    const int32_t *enters = FORWARD ? marks.begins : marks.ends, *leaves = FORWARD ? marks.ends : marks.begins;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) A[k] = 1.0f, B[k] = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < L; ++i)
      if (there(i)) {
        const int32_t seq = mark(enters, i);
        if (seq >= 0) {
          load_state<N>(a.first, (uint32_t)seq, s.at, a.dim, B);
#pragma unroll
          for (uint32_t k = 0; k < N; ++k) A[k] = 0.0f;
        }
        float z[N], y[N];
        rg[i].values(z);
        rv[i].values(y);
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) {
          float f, rest;
          gates(z[k], f, rest);
          A[k] *= f;
          B[k] = FORWARD ? fmaf(f, B[k], rest * y[k]) : f * (y[k] + B[k]);
        }
      }
    join<N, !WRITE>(s, groups, A, B, sa, sb, carry, factor, in);
    if (WRITE) {
#pragma unroll
      for (uint32_t i = 0; i < L; ++i)
        if (there(i)) {
          const uint32_t t = row_of(i);
          int32_t seq = mark(enters, i);
          if (seq >= 0) load_state<N>(a.first, (uint32_t)seq, s.at, a.dim, in);
          float z[N], y[N], o[N];
          rg[i].values(z);
          rv[i].values(y);
          if (FORWARD) {
#pragma unroll
            for (uint32_t k = 0; k < N; ++k) {
              float f, rest;
              gates(z[k], f, rest);
              o[k] = in[k] = fmaf(f, in[k], rest * y[k]);
            }
          } else {
            float xs[N], before[N], dg[N];
            rx[i].values(xs);
            seq = a.flat ? mark(leaves, i) : t == live_low ? (int32_t)s.walk : -1;
            if (seq >= 0)
              load_state<N>(a.h0, (uint32_t)seq, s.at, a.dim, before);
            else
              rh[i].values(before);
#pragma unroll
            for (uint32_t k = 0; k < N; ++k) {
              float f, rest;
              gates(z[k], f, rest);
              const float d = y[k] + in[k];
              in[k] = f * d;
              o[k] = rest * d;
              dg[k] = d * (before[k] - xs[k]) * (f * rest);
            }
            store_row<N>(dgate + t * a.dgate_stride, s.at, a.dim, dg);
          }
          store_row<N>(out + t * a.out_stride, s.at, a.dim, o);
          seq = a.flat ? mark(leaves, i) : ends_here && p0 + s.row * L + i + 1 == a.len ? (int32_t)s.walk : -1;
          if (seq >= 0) store_state<N>(a.last, (uint32_t)seq, s.at, a.dim, in);
        }
    }
    __syncthreads();                    // sb is read
  }
  if (!WRITE && s.row == 0) {
    float2* p = a.partial + ((uint64_t)s.walk * a.ranges + s.range) * a.dim + s.at;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k)
      if (s.at + k < a.dim) p[k] = float2{factor[s.group * N + k], carry[s.group * N + k]};
  }
  __syncthreads();                      // carry is read
  }
}

constexpr uint32_t kFull = 512;         // workgroups that fill the device
constexpr uint32_t kMostGrid = 1u << 21;  // launches stay below 2^32 threads

struct Cut {
  uint32_t groups_log2, blocks, ranges, range_len;
};
uint32_t groups_log2_for(uint32_t dim, uint32_t each) {
  uint32_t log2 = 0;
  while ((1u << log2) < std::min((dim + each - 1) / each, kGroupsMost)) ++log2;
  return log2;
}
uint32_t rows_at_once(uint32_t dim, uint32_t each) { return (kScanBlock >> groups_log2_for(dim, each)) * kSteps; }
// How rows and channels are dealt out.
Cut cut_for(uint32_t dim, uint32_t each, uint32_t walks, uint32_t len) {
  Cut c{};
  c.groups_log2 = groups_log2_for(dim, each);
  c.blocks = ((dim + each - 1) / each + (1u << c.groups_log2) - 1) >> c.groups_log2;
  const uint32_t W = rows_at_once(dim, each), iterations = std::max(1u, (len + W - 1) / W);
  const uint64_t pairs = (uint64_t)walks * c.blocks;
  uint32_t ranges = 1;
  if (pairs && pairs < kFull / 2 && iterations > 2) ranges = (uint32_t)std::min<uint64_t>(kFull / pairs, iterations);
  c.range_len = (iterations + ranges - 1) / ranges * W;  // iterations * W < 2^31 + 2^13
  c.ranges = std::max(1u, (uint32_t)(((uint64_t)len + c.range_len - 1) / c.range_len));
  return c;
}

// What both directions ask of their arguments.
int check(uint32_t n, uint32_t dim, uint32_t type, uint32_t n_seq, const void* d_starts, uint32_t start_bytes, const void* d_workspace,
          size_t ws_bytes, const uint32_t* d_status) {
  if (dim < 1 || dim > 0x7FFFFFFFu || n > 0x7FFFFFFFu || n_seq > 0x7FFFFFFFu || !type_known(type)) return CVLC_ERR_ARG;
  if (d_starts) {
    if ((start_bytes != 4 && start_bytes != 8) || !buffer_ok(d_starts, start_bytes)) return CVLC_ERR_ARG;
  } else if (n_seq ? n % n_seq != 0 : n != 0) {
    return CVLC_ERR_ARG;
  }
  if (d_status && !buffer_ok(d_status, 4)) return CVLC_ERR_ARG;
  if (!buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  if (ws_bytes < cvlc_gated_scan_workspace_bytes(n, dim, n_seq)) return CVLC_ERR_CAPACITY;
  return CVLC_OK;
}
bool state_ok(const float* p) { return !p || buffer_ok(p, 4); }
template <class... P>
bool matrices_ok(uint32_t type, P... p) {
  return (buffer_ok(p, type_bytes(type)) && ...);
}

template <bool FORWARD>
int launch(ScanArgs a, uint32_t type, const void* v, const void* gate, const void* x, const void* h, void* out, void* dgate,
           void* d_workspace, hipStream_t stream) {
  const uint32_t per = 16 / type_bytes(type);
  a.each = a.n_seq ? a.n / a.n_seq : 0u;
  // sequences that leave most of a workgroup's threads without rows are walked together
  a.flat = a.starts || a.each < rows_at_once(a.dim, per) / 2;
  a.walks = a.n == 0 ? 0u : a.flat ? 1u : a.n_seq;
  a.len = a.flat ? a.n : a.each;
  a.partial = static_cast<float2*>(d_workspace);
  const Cut c = cut_for(a.dim, per, a.walks, a.len);
  a.groups_log2 = c.groups_log2;
  a.blocks = c.blocks;
  a.ranges = c.ranges;
  a.range_len = c.range_len;
  const uint64_t main_blocks = (uint64_t)a.walks * a.ranges * a.blocks;
  if (main_blocks > 0xFFFFFFFFull) return CVLC_ERR_ARG;
  a.main_grid = (uint32_t)std::min<uint64_t>(main_blocks, kMostGrid);
  const uint32_t more =
      (a.starts || a.n == 0) && (a.last || a.status) ? std::min((a.n_seq + kScanBlock - 1) / kScanBlock, kMostGrid) : 0u;
  if (a.main_grid + more == 0) return CVLC_OK;
  by_type(type, [&](auto t) {
    using T = decltype(t);
    auto as = [](const void* p) { return static_cast<const T*>(p); };
    if (a.ranges > 1)
      hipLaunchKernelGGL((scan_kernel<T, FORWARD, false>), dim3(a.main_grid), dim3(kScanBlock), 0, stream, a, as(v), as(gate),
                         as(x), as(h), static_cast<T*>(out), static_cast<T*>(dgate));
    hipLaunchKernelGGL((scan_kernel<T, FORWARD, true>), dim3(a.main_grid + more), dim3(kScanBlock), 0, stream, a, as(v),
                       as(gate), as(x), as(h), static_cast<T*>(out), static_cast<T*>(dgate));
  });
  return hip_check(hipGetLastError());
}

// ------------------------------------------------------------------------------ one token of many sequences
constexpr uint32_t kStepBlock = 256;

struct StepArgs {
  uint32_t n, dim, n_slots, slot_bytes;
  const void* slots;
  uint64_t x_stride, gate_stride, h_stride;
  float* states;
  uint32_t* status;
};

__device__ __forceinline__ int64_t slot_of(const StepArgs& a, uint32_t i) {
  if (!a.slots) return i;
  return a.slot_bytes == 8 ? static_cast<const int64_t*>(a.slots)[i] : (int64_t)static_cast<const int32_t*>(a.slots)[i];
}

template <class T>
__global__ __launch_bounds__(kStepBlock) void scan_step_kernel(StepArgs a, const T* x, const T* gate, T* h) {
  constexpr uint32_t N = kPerAccess<T>;
  for (uint32_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int64_t slot = slot_of(a, i);
    bool live = slot >= 0 && slot < (int64_t)a.n_slots;
    bool wrong = slot >= (int64_t)a.n_slots;
    if (a.slots && live) {
      // a slot is the first token's that names it
      bool taken = false;
      for (uint32_t j = threadIdx.x; j < i; j += kStepBlock) taken |= slot_of(a, j) == slot;
      if (__syncthreads_or(taken)) {
        live = false;
        wrong = true;
      }
    }
    if (wrong && a.status && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(a.status, CVLC_DEV_INDEX);
    for (uint32_t at = (blockIdx.y * kStepBlock + threadIdx.x) * N; at < a.dim; at += gridDim.y * kStepBlock * N) {
      float u[N] = {};
      if (live) {
        float xs[N], z[N];
        float* state = a.states + (uint64_t)slot * a.dim;
        load_row<N>(x + i * a.x_stride, at, a.dim, 0.0f, xs);
        load_row<N>(gate + i * a.gate_stride, at, a.dim, 0.0f, z);
        load_row<N>(state, at, a.dim, 0.0f, u);
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) {
          float f, rest;
          gates(z[k], f, rest);
          u[k] = fmaf(f, u[k], rest * xs[k]);
        }
        store_row<N>(state, at, a.dim, u);
      }
      store_row<N>(h + i * a.h_stride, at, a.dim, u);
    }
  }
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_gated_scan_workspace_bytes(uint32_t n, uint32_t dim, uint32_t n_seq) {
  using namespace cvlc;
  (void)n, (void)dim, (void)n_seq;
  // workgroups that have ranges are kFull at most, with 16 bytes' worth of channels for each of kGroupsMost threads
  return 256u + (size_t)kFull * kGroupsMost * 8u * sizeof(float2);
}

int cvlc_gated_scan(uint32_t n, uint32_t dim, const void* d_x, uint64_t x_stride, const void* d_gate, uint64_t gate_stride, uint32_t type,
                    uint32_t n_seq, const void* d_starts, uint32_t start_bytes, const float* d_h0, void* d_h, uint64_t h_stride,
                    float* d_last, void* d_workspace, size_t ws_bytes, uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  if (const int rc = check(n, dim, type, n_seq, d_starts, start_bytes, d_workspace, ws_bytes, d_status)) return rc;
  if (x_stride < dim || gate_stride < dim || h_stride < dim || !state_ok(d_h0) || !state_ok(d_last)) return CVLC_ERR_ARG;
  if (n && !matrices_ok(type, d_x, d_gate, d_h)) return CVLC_ERR_ARG;
  ScanArgs a{};
  a.n = n, a.dim = dim, a.n_seq = n_seq, a.start_bytes = start_bytes, a.starts = d_starts;
  a.v_stride = x_stride, a.gate_stride = gate_stride, a.out_stride = h_stride;
  a.first = d_h0, a.last = d_last, a.status = d_status;
  return launch<true>(a, type, d_x, d_gate, nullptr, nullptr, d_h, nullptr, d_workspace, static_cast<hipStream_t>(hip_stream));
}

int cvlc_gated_scan_grad(uint32_t n, uint32_t dim, const void* d_dy, uint64_t dy_stride, const void* d_x, uint64_t x_stride,
                         const void* d_gate, uint64_t gate_stride, const void* d_h, uint64_t h_stride, uint32_t type, uint32_t n_seq,
                         const void* d_starts, uint32_t start_bytes, const float* d_h0, const float* d_dlast, void* d_dx,
                         uint64_t dx_stride, void* d_dgate, uint64_t dgate_stride, float* d_dh0, void* d_workspace, size_t ws_bytes,
                         uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  if (const int rc = check(n, dim, type, n_seq, d_starts, start_bytes, d_workspace, ws_bytes, d_status)) return rc;
  if (dy_stride < dim || x_stride < dim || gate_stride < dim || h_stride < dim || dx_stride < dim || dgate_stride < dim) return CVLC_ERR_ARG;
  if (!state_ok(d_h0) || !state_ok(d_dlast) || !state_ok(d_dh0)) return CVLC_ERR_ARG;
  if (n && !matrices_ok(type, d_dy, d_x, d_gate, d_h, d_dx, d_dgate)) return CVLC_ERR_ARG;
  ScanArgs a{};
  a.n = n, a.dim = dim, a.n_seq = n_seq, a.start_bytes = start_bytes, a.starts = d_starts;
  a.v_stride = dy_stride, a.gate_stride = gate_stride, a.x_stride = x_stride, a.h_stride = h_stride;
  a.out_stride = dx_stride, a.dgate_stride = dgate_stride;
  a.first = d_dlast, a.h0 = d_h0, a.last = d_dh0, a.status = d_status;
  return launch<false>(a, type, d_dy, d_gate, d_x, d_h, d_dx, d_dgate, d_workspace, static_cast<hipStream_t>(hip_stream));
}

int cvlc_gated_scan_step(uint32_t n, uint32_t dim, const void* d_x, uint64_t x_stride, const void* d_gate, uint64_t gate_stride,
                         uint32_t type, const void* d_slots, uint32_t slot_bytes, uint32_t n_slots, float* d_states, void* d_h,
                         uint64_t h_stride, uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  if (dim < 1 || dim > 0x7FFFFFFFu || n > 0x7FFFFFFFu || n_slots > 0x7FFFFFFFu || !type_known(type)) return CVLC_ERR_ARG;
  if (x_stride < dim || gate_stride < dim || h_stride < dim) return CVLC_ERR_ARG;
  if (d_slots && ((slot_bytes != 4 && slot_bytes != 8) || !buffer_ok(d_slots, slot_bytes))) return CVLC_ERR_ARG;
  if (!d_slots && n_slots < n) return CVLC_ERR_ARG;
  if (d_status && !buffer_ok(d_status, 4)) return CVLC_ERR_ARG;
  if (n == 0) return CVLC_OK;
  if (!matrices_ok(type, d_x, d_gate, d_h) || (n_slots && !buffer_ok(d_states, 4))) return CVLC_ERR_ARG;
  const StepArgs a{n, dim, n_slots, slot_bytes, d_slots, x_stride, gate_stride, h_stride, d_states, d_status};
  by_type(type, [&](auto t) {
    using T = decltype(t);
    const uint32_t pieces = (dim + kStepBlock * kPerAccess<T> - 1) / (kStepBlock * kPerAccess<T>);
    hipLaunchKernelGGL(scan_step_kernel<T>, dim3(std::min(n, 1u << 16), std::min(pieces, 64u)), dim3(kStepBlock), 0,
                       static_cast<hipStream_t>(hip_stream), a, static_cast<const T*>(d_x), static_cast<const T*>(d_gate),
                       static_cast<T*>(d_h));
  });
  return hip_check(hipGetLastError());
}

}  // extern "C"
