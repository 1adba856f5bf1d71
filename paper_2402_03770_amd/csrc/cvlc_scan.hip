// cvlc_scan.hip -- a gated linear recurrence over sequences, channel by channel, and its backward pass.
//
// Forward, with f = sigmoid(gate):   h_t = f_t h_(t-1) + (1 - f_t) x_t.
// Backward, with c_t = f_t D_t what a token hands to the one before it:
//   D_t = dy_t + c_(t+1),   c_t = f_t (dy_t + c_(t+1)),
//   dx_t = (1 - f_t) D_t,   dgate_t = D_t (h_(t-1) - x_t) f_t (1 - f_t).
// Both are one walk, u <- a u + b, that way and back: steps chain as (A, B), u <- A u + B,
// so rows are cut into pieces whose (A, B) are found side by side and joined.  A piece in which a sequence begins
// forgets what comes before it: its A is kAnew, not 0, which would hand a NaN or an infinity on to the next sequence.
//
// Where sequences and channels fill the device (scan_rows), a workgroup has a block of channels of one
// sequence and goes over its rows some hundred at a time: every thread has `L` rows of 16 bytes' worth of
// channels in registers, the threads' (A, B) meet in LDS, and each thread walks its rows again from what
// comes before them.  Every byte is read once: bound by HBM, with the arithmetic (an exponential and a
// reciprocal a value) close behind.  Sequences by offsets are walked together, as one, which a width beyond 16 320
// (fp32 8160) makes enough work of.  Otherwise, or where sequences are few, rows are cut into ranges, one thread's each:
// one launch finds the ranges' (A, B) (scan_range), one joins them (scan_carry), one walks again and writes
// (scan_range, APPLY); the walk's two inputs are read twice.  No workgroup waits for another.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kScanBlock = 512;
constexpr uint32_t kGroupsMost = 8;     // scan_rows: threads side by side on a row, 128 bytes of it
// L, rows of a thread: more take registers from the wavefronts that have their loads under way, fewer meet more often.
// 65 536 x 2048 bf16 in 16 sequences, us: forward 231 with one row, 182 with two, 195 with four; backward 344, 372 and 384;
// backward of 32 x 512 x 1024 fp32 98, 83 and 89.
template <class T, bool FORWARD>
constexpr uint32_t kSteps = !FORWARD && sizeof(T) == 2 ? 1 : 2;

struct ScanArgs {
  uint32_t n, dim, n_seq, start_bytes;
  const void* starts;                   // null: sequences of `each` rows
  uint32_t each;
  uint32_t flat, walks, len;            // what is walked: every sequence, or (flat) once all rows of all sequences
  uint32_t ranges, range_len;           // parts of a walk
  uint32_t groups_log2, blocks;         // threads on a row, blocks of channels
  uint64_t v_stride, gate_stride, x_stride, h_stride, out_stride, dgate_stride;
  const float* first;                   // what walks start from: h0, or the last state's gradient
  const float* h0;                      // backward: the state before a sequence's first row
  float* last;                          // what they end with: the last state, or the first one's gradient
  uint32_t main_grid;                   // workgroups that walk; those behind them see to sequences without rows
  float2* partial;                      // (A, B) of every range and channel
  float* enter;                         // what every range starts from
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

// The smaller of f = sigmoid(z) and 1 - f with its own last bits, negative where it is 1 - f: u f = u + g u then, and
// u f = g u where g is positive.  EXACT: the product with log2 e is taken apart, whose rounding grows with |z| (16-bit results
// do not show it, and it costs a third of the instructions).
template <bool EXACT>
__device__ __forceinline__ float gate_of(float z) {
  constexpr float kLog2E = 0x1.715476p+0f, kLow = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
  float e;
  if (EXACT) {
    float x = fabsf(z);
    x = x > 120.0f ? 120.0f : x;        // a NaN stays one
    const float t = -x * kLog2E;
    e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, (fmaf(-x, kLog2E, -t) - x * kLow) * kLn2, e);
  } else {
    e = __builtin_amdgcn_exp2f(fabsf(z) * -kLog2E);
  }
  const float s = e * __builtin_amdgcn_rcpf(1.0f + e);
  return z >= 0.0f ? -s : s;
}
__device__ __forceinline__ bool keeps(float g) { return __float_as_int(g) < 0; }   // f >= 1/2; -0 too
// f u
__device__ __forceinline__ float through(float g, float u) { return fmaf(g, u, keeps(g) ? u : 0.0f); }
// f u + (1 - f) x: from the one that counts more towards the other
__device__ __forceinline__ float blend(float g, float u, float x) {
  const float near = keeps(g) ? u : x, far = keeps(g) ? x : u;
  return fmaf(fabsf(g), far - near, near);
}

constexpr float kAnew = -1.0f;          // other A are products of gates: never negative, and 0 where they are too small
__device__ __forceinline__ float chain(float A, float B, float u) { return A < 0.0f ? B : fmaf(A, u, B); }

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
template <class T, uint32_t N, bool ONCE = false>
__device__ __forceinline__ void load_channels(Raw<T, N>& raw, const T* row, uint32_t at, uint32_t dim) {
  if (dim >= N)
    raw.template load<ONCE>(row + at);
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

// The first of a thread's N channels: the last threads of a row move back to end with it, and channels that two threads
// have come out the same from both.
template <uint32_t N>
__device__ __forceinline__ uint32_t channel_of(uint32_t group, uint32_t dim) {
  return dim >= N ? min(group * N, dim - N) : 0u;
}

// Sequences without rows hand on what they start from; offsets that are out of order or out of the rows are told of.  A wavefront
// has some sequences and kSeeWide channels of their states, which its lanes copy side by side.
constexpr uint32_t kSeeEach = 8, kSeeWide = kWave * kSeeEach, kSeeFew = 1u << 12;
__host__ __device__ inline uint32_t see_per(uint32_t n_seq) { return n_seq <= kSeeFew ? 1 : kWave; }   // sequences of a wavefront
__host__ __device__ inline uint64_t see_items(uint32_t n_seq, uint32_t dim) {
  return ((uint64_t)n_seq + see_per(n_seq) - 1) / see_per(n_seq) * (((uint64_t)dim + kSeeWide - 1) / kSeeWide);
}
__device__ __forceinline__ void see_to_empty(const ScanArgs& a, uint32_t wave, uint32_t waves) {
  const uint32_t dim = a.last ? a.dim : 1, per = see_per(a.n_seq), parts = (dim + kSeeWide - 1) / kSeeWide, lane = lane_id();
  const uint64_t all = see_items(a.n_seq, dim);
  for (uint64_t item = wave; item < all; item += waves) {
    const uint32_t first = (uint32_t)(item / parts) * per, part = (uint32_t)(item % parts), low = part * kSeeWide, high = min(dim - low, kSeeWide) + low;
    const uint32_t j = first + lane;
    bool empty = false;
    if (lane < per && j < a.n_seq) {
      const int64_t from = start_as_given(a, j), to = start_as_given(a, j + 1);
      if (part == 0 && a.status && (from < 0 || to < from || to > (int64_t)a.n)) atomicOr(a.status, CVLC_DEV_INDEX);
      empty = a.last && start_of(a, j + 1) <= start_of(a, j);
    }
    const uint64_t which = __ballot(empty);
    if (which == 0) continue;
    uint32_t wide = kWave;              // lanes that share a state: fewer where it is narrower
    while (wide > 1 && wide / 2 >= high - low) wide /= 2;
    for (uint32_t k = lane / wide; k < per; k += kWave / wide) {
      if (!(which >> k & 1)) continue;
      const uint64_t row = (uint64_t)(first + k) * a.dim;
      float u[kSeeEach];
#pragma unroll
      for (uint32_t i = 0; i < kSeeEach; ++i) {
        const uint32_t c = low + lane % wide + i * wide;
        u[i] = a.first && c < high ? a.first[row + c] : 0.0f;
      }
#pragma unroll
      for (uint32_t i = 0; i < kSeeEach; ++i) {
        const uint32_t c = low + lane % wide + i * wide;
        if (c < high) a.last[row + c] = u[i];
      }
    }
  }
}

// A row's gates, and what one step of the walk makes of them.  With 16-bit matrices the forward walk holds f and
// (1 - f) x, each rounded to fp32, and a step is one instruction; else it holds the gate as gate_of gives it, which keeps the
// last bits of both f and 1 - f.
template <class T, bool FORWARD>
constexpr bool kPlainSteps = FORWARD && sizeof(T) == 2;

template <class T, bool FORWARD, uint32_t N>
__device__ __forceinline__ void first_walk(float (&g)[N], float (&y)[N], float (&A)[N], float (&B)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    const float s = gate_of<sizeof(T) == 4>(g[k]);
    if constexpr (kPlainSteps<T, FORWARD>) {
      const float low = fabsf(s), high = 1.0f - low;
      g[k] = keeps(s) ? high : low;
      y[k] *= keeps(s) ? low : high;
      A[k] *= g[k];
      B[k] = fmaf(g[k], B[k], y[k]);
    } else {
      g[k] = s;
      A[k] = through(s, A[k]);
      B[k] = FORWARD ? blend(s, B[k], y[k]) : through(s, y[k] + B[k]);
    }
  }
}
template <class T, uint32_t N>
__device__ __forceinline__ void step_forward(const float (&g)[N], const float (&y)[N], float (&u)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) u[k] = kPlainSteps<T, true> ? fmaf(g[k], u[k], y[k]) : blend(g[k], u[k], y[k]);
}
template <uint32_t N>
__device__ __forceinline__ void step_back(const float (&g)[N], const float (&dy)[N], const float (&x)[N], const float (&before)[N],
                                          float (&u)[N], float (&dx)[N], float (&dg)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    const float d = dy[k] + u[k], s = fabsf(g[k]);
    u[k] = through(g[k], d);
    dx[k] = through(-g[k], d);
    dg[k] = d * (before[k] - x[k]) * fmaf(-s, s, s);
  }
}

// ------------------------------------------------------------------------------ every byte once
// A workgroup's joined steps: `in` is what comes before the thread's rows then.  carry[ch]: what comes before all rows, then
// what comes after them.  `anew`: whether some A may be kAnew; asking each lengthens the chain
// (1728 x 142 bf16 in 9 sequences 10.4 us, 9.9 without).
template <uint32_t N>
__device__ __forceinline__ void join(uint32_t mine, uint32_t width, uint32_t rows, bool anew, const float (&A)[N], const float (&B)[N], float* sa,
                                     float* sb, float* carry, float (&in)[N]) {
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    sa[mine + k] = A[k];
    sb[mine + k] = B[k];
  }
  __syncthreads();
  if (threadIdx.x < width) {
    float u = carry[threadIdx.x];
    auto walk = [&](auto asks) {
#pragma unroll 8
      for (uint32_t r = 0; r < rows; ++r) {
        const float x = sa[r * width + threadIdx.x], y = sb[r * width + threadIdx.x];
        sb[r * width + threadIdx.x] = u;
        u = decltype(asks)::value ? chain(x, y, u) : fmaf(x, u, y);
      }
    };
    if (anew)
      walk(std::true_type{});
    else
      walk(std::false_type{});
    carry[threadIdx.x] = u;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) in[k] = sb[mine + k];
}

// ONCE: past the caches' order.
template <class T, bool FORWARD, bool ONCE>
__global__ __launch_bounds__(kScanBlock, 4) void scan_rows_kernel(ScanArgs a, const T* v, const T* gate, const T* x, const T* h, T* out,
                                                                  T* dgate) {
  constexpr uint32_t N = kPerAccess<T>, L = kSteps<T, FORWARD>;
  constexpr uint32_t kMarks = kScanBlock * L;
  __shared__ float sa[kScanBlock * N], sb[kScanBlock * N], carry[kGroupsMost * N];
  __shared__ Marks<kMarks> marks;
  if (__builtin_expect(blockIdx.x >= a.main_grid, 0)) {
    see_to_empty(a, (blockIdx.x - a.main_grid) * (kScanBlock / kWave) + wave_id(), (gridDim.x - a.main_grid) * (kScanBlock / kWave));
    return;
  }
  const uint32_t groups = 1u << a.groups_log2, width = groups * N, rows = kScanBlock >> a.groups_log2, W = rows * L;
  const uint32_t group = threadIdx.x & (groups - 1), row = threadIdx.x >> a.groups_log2, mine = row * width + group * N;
  for (uint32_t block = blockIdx.x; block < a.walks * a.blocks; block += a.main_grid) {
    const uint32_t walk = block / a.blocks, at = channel_of<N>(block % a.blocks * groups + group, a.dim);
    const uint32_t base = walk * a.len;
    uint32_t live_low = base, live_high = base + a.len;   // rows that belong to a sequence
    if (a.flat) {
      live_low = start_of(a, 0);
      live_high = start_of(a, a.n_seq);
    }
    float in[N], A[N], B[N];
    if (row == 0) {
      load_state<N>(a.flat ? nullptr : a.first, walk, at, a.dim, in);
#pragma unroll
      for (uint32_t k = 0; k < N; ++k) carry[group * N + k] = in[k];
    }
    for (uint32_t p0 = 0; p0 < a.len; p0 += W) {
      const uint32_t count = min(W, a.len - p0);          // rows of this iteration
      const uint32_t low = FORWARD ? base + p0 : base + a.len - p0 - count;
      auto row_of = [&](uint32_t i) { return FORWARD ? low + row * L + i : low + count - 1 - row * L - i; };
      auto there = [&](uint32_t i) {
        const uint32_t t = row_of(i);
        return row * L + i < count && t >= live_low && t < live_high;
      };
      bool marked = false;
      if (a.flat) {
        fill_marks<kMarks>(a, low, low + count, count, marks);
        marked = marks.any;
      }
      auto mark = [&](const int32_t* m, uint32_t i) { return marked ? m[row_of(i) - low] : -1; };
      const int32_t *enters = FORWARD ? marks.begins : marks.ends, *leaves = FORWARD ? marks.ends : marks.begins;
      // WHOLE: rows that all belong to one sequence and do not begin or end it
      auto go = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        Raw<T, N> rv[L], rg[L], rx[L], rh[L];
#pragma unroll
        for (uint32_t i = 0; i < L; ++i)
          if (WHOLE || there(i)) {
            load_channels<T, N, ONCE>(rg[i], gate + row_of(i) * a.gate_stride, at, a.dim);
            load_channels<T, N, ONCE>(rv[i], v + row_of(i) * a.v_stride, at, a.dim);
          }
        if (!FORWARD) {
#pragma unroll
          for (uint32_t i = 0; i < L; ++i)
            if (WHOLE || there(i)) {
              load_channels<T, N, ONCE>(rx[i], x + row_of(i) * a.x_stride, at, a.dim);
              if (WHOLE || row_of(i) > live_low) load_channels<T, N, ONCE>(rh[i], h + (row_of(i) - 1) * a.h_stride, at, a.dim);
            }
        }
        float g[L][N], y[L][N];
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) A[k] = 1.0f, B[k] = 0.0f;
        bool anew = false;
#pragma unroll
        for (uint32_t i = 0; i < L; ++i)
          if (WHOLE || there(i)) {
            const int32_t seq = WHOLE ? -1 : mark(enters, i);
            if (seq >= 0) {
              load_state<N>(a.first, (uint32_t)seq, at, a.dim, B);
              anew = true;
            }
            rg[i].values(g[i]);
            rv[i].values(y[i]);
            first_walk<T, FORWARD>(g[i], y[i], A, B);
          }
        if (!WHOLE && anew)
#pragma unroll
          for (uint32_t k = 0; k < N; ++k) A[k] = kAnew;
        join<N>(mine, width, rows, !WHOLE && marked, A, B, sa, sb, carry, in);
#pragma unroll
        for (uint32_t i = 0; i < L; ++i)
          if (WHOLE || there(i)) {
            const uint32_t t = row_of(i);
            int32_t seq = WHOLE ? -1 : mark(enters, i);
            if (seq >= 0) load_state<N>(a.first, (uint32_t)seq, at, a.dim, in);
            if (FORWARD) {
              step_forward<T>(g[i], y[i], in);
              store_row<N, ONCE>(out + t * a.out_stride, at, a.dim, in);
            } else {
              float xs[N], before[N], o[N], dg[N];
              rx[i].values(xs);
              seq = WHOLE ? -1 : a.flat ? mark(leaves, i) : t == live_low ? (int32_t)walk : -1;
              if (seq >= 0)
                load_state<N>(a.h0, (uint32_t)seq, at, a.dim, before);
              else
                rh[i].values(before);
              step_back(g[i], y[i], xs, before, in, o, dg);
              store_row<N, ONCE>(dgate + t * a.dgate_stride, at, a.dim, dg);
              store_row<N, ONCE>(out + t * a.out_stride, at, a.dim, o);
            }
            if (!WHOLE) {
              seq = a.flat ? mark(leaves, i) : p0 + row * L + i + 1 == a.len ? (int32_t)walk : -1;
              if (seq >= 0) store_state<N>(a.last, (uint32_t)seq, at, a.dim, in);
            }
          }
      };
      if (a.dim >= N && count == W && low > live_low && low + count < live_high && !marked)
        go(std::true_type{});
      else
        go(std::false_type{});
      __syncthreads();                  // sb and carry are read
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------ ranges
constexpr uint32_t kRangeBlock = 256;
template <bool FORWARD, bool APPLY>
constexpr uint32_t kBatch = APPLY && !FORWARD ? 2 : 4;   // rows that a thread has under way

// The sequence that row t of a flat walk lies in; its first row and the one behind its last.
__device__ __forceinline__ void locate(const ScanArgs& a, uint32_t t, uint32_t& seq, uint32_t& begin, uint32_t& end) {
  uint32_t low = 1, high = a.n_seq;     // the first boundary behind t
  while (low < high) {
    const uint32_t mid = (low + high) / 2;
    if (start_of(a, mid) > t)
      high = mid;
    else
      low = mid + 1;
  }
  seq = low - 1;
  begin = start_of(a, seq);
  end = start_of(a, seq + 1);
}

// A thread's rows: 16 bytes' worth of channels of one range.  APPLY: walked from a.enter on and written; else its (A, B).
template <class T, bool FORWARD, bool APPLY, bool ONCE>
__global__ __launch_bounds__(kRangeBlock, 4) void scan_range_kernel(ScanArgs a, const T* v, const T* gate, const T* x, const T* h, T* out,
                                                                    T* dgate) {
  constexpr uint32_t N = kPerAccess<T>, P = kBatch<FORWARD, APPLY>;
  if (APPLY && __builtin_expect(blockIdx.x >= a.main_grid, 0)) {
    see_to_empty(a, (blockIdx.x - a.main_grid) * (kRangeBlock / kWave) + wave_id(), (gridDim.x - a.main_grid) * (kRangeBlock / kWave));
    return;
  }
  const uint32_t pieces = (a.dim + N - 1) / N;
  // the launch that writes goes the other way round: what the first one read last may still be in the last-level cache
  const uint32_t block = APPLY ? a.main_grid - 1 - blockIdx.x : blockIdx.x;
  const uint64_t id = (uint64_t)block * kRangeBlock + threadIdx.x;
  const uint32_t piece = (uint32_t)(id % pieces), part = (uint32_t)(id / pieces);
  if (part >= a.walks * a.ranges) return;
  const uint32_t walk = part / a.ranges, range = part % a.ranges, at = channel_of<N>(piece, a.dim);
  const uint32_t base = walk * a.len, first_p = range * a.range_len, count = min(a.range_len, a.len - first_p);
  // rows [from, to), walked that way or back
  uint32_t from = FORWARD ? base + first_p : base + a.len - first_p - count, to = from + count;
  uint32_t seq = walk, begin = base, end = base + a.len, lowest = base;
  if (a.flat) {
    lowest = start_of(a, 0);
    from = max(from, lowest);
    to = min(to, start_of(a, a.n_seq));
    if (from < to) locate(a, FORWARD ? from : to - 1, seq, begin, end);
  }
  float A[N], u[N];
  bool anew = false;
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) A[k] = 1.0f, u[k] = 0.0f;
  if (APPLY) {
    const float* p = a.enter + (uint64_t)part * a.dim + at;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k)
      if (at + k < a.dim) u[k] = p[k];
  }
  auto some = [&](uint32_t first, uint32_t rows, auto whole) {     // `rows` rows from `first` on, in the walk's order
    constexpr bool WHOLE = decltype(whole)::value;                 // P rows within a sequence
    Raw<T, N> rv[P], rg[P], rx[P], rh[P];
    auto row_of = [&](uint32_t i) { return FORWARD ? first + i : first - i; };
#pragma unroll
    for (uint32_t i = 0; i < P; ++i)
      if (WHOLE || i < rows) {
        load_channels<T, N, ONCE>(rg[i], gate + row_of(i) * a.gate_stride, at, a.dim);
        load_channels<T, N, ONCE>(rv[i], v + row_of(i) * a.v_stride, at, a.dim);
        if (APPLY && !FORWARD) {
          load_channels<T, N, ONCE>(rx[i], x + row_of(i) * a.x_stride, at, a.dim);
          if (WHOLE || row_of(i) > lowest) load_channels<T, N, ONCE>(rh[i], h + (row_of(i) - 1) * a.h_stride, at, a.dim);
        }
      }
#pragma unroll
    for (uint32_t i = 0; i < P; ++i)
      if (WHOLE || i < rows) {
        const uint32_t t = row_of(i);
        if (!WHOLE) {
          if (a.flat && (t < begin || t >= end)) locate(a, t, seq, begin, end);
          if (t == (FORWARD ? begin : end - 1)) {
            load_state<N>(a.first, seq, at, a.dim, u);
            anew = true;
          }
        }
        float g[N], y[N], none[N] = {};
        rg[i].values(g);
        rv[i].values(y);
        if (!APPLY) {
          first_walk<T, FORWARD>(g, y, A, u);
          continue;
        }
        if (FORWARD) {
          first_walk<T, FORWARD>(g, y, none, u);
          store_row<N, ONCE>(out + t * a.out_stride, at, a.dim, u);
        } else {
          float xs[N], before[N], o[N], dg[N];
          rx[i].values(xs);
          if (!WHOLE && t == begin)
            load_state<N>(a.h0, seq, at, a.dim, before);
          else
            rh[i].values(before);
#pragma unroll
          for (uint32_t k = 0; k < N; ++k) g[k] = gate_of<sizeof(T) == 4>(g[k]);
          step_back(g, y, xs, before, u, o, dg);
          store_row<N, ONCE>(dgate + t * a.dgate_stride, at, a.dim, dg);
          store_row<N, ONCE>(out + t * a.out_stride, at, a.dim, o);
        }
        if (!WHOLE && t == (FORWARD ? end - 1 : begin)) store_state<N>(a.last, seq, at, a.dim, u);
      }
  };
  for (uint32_t done = 0; from + done < to; done += P) {
    const uint32_t first = FORWARD ? from + done : to - 1 - done, rows = min(P, to - from - done);
    const uint32_t low = FORWARD ? first : first + 1 - rows;
    if (rows == P && low > begin && low + P < end && a.dim >= N)
      some(first, P, std::true_type{});
    else
      some(first, rows, std::false_type{});
  }
  if (!APPLY) {
    const float mark = a.flat ? kAnew : 0.0f;   // before a sequence that is walked by itself there is nothing to forget
    float2* p = a.partial + (uint64_t)part * a.dim + at;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k)
      if (at + k < a.dim) p[k] = float2{anew ? mark : A[k], u[k]};
  }
}

// What every range starts from: a workgroup has 16 channels of a walk, its threads 64 pieces of the ranges each.
constexpr uint32_t kCarryWide = 16, kCarryRows = 64;
template <bool FLAT>
__global__ __launch_bounds__(kCarryWide * kCarryRows) void scan_carry_kernel(ScanArgs a) {
  __shared__ float2 steps[kCarryRows][kCarryWide];
  const uint32_t blocks = (a.dim + kCarryWide - 1) / kCarryWide, x = threadIdx.x % kCarryWide, y = threadIdx.x / kCarryWide;
  const uint32_t walk = blockIdx.x / blocks, c = blockIdx.x % blocks * kCarryWide + x;
  const uint32_t per = (a.ranges + kCarryRows - 1) / kCarryRows, from = min(y * per, a.ranges), to = min(from + per, a.ranges);
  const float2* p = a.partial + (uint64_t)walk * a.ranges * a.dim + c;
  float2 all = {1.0f, 0.0f};
  auto next = [](float2 s, float u) { return FLAT ? chain(s.x, s.y, u) : fmaf(s.x, u, s.y); };
  if (c < a.dim)
#pragma unroll 8
    for (uint32_t r = from; r < to; ++r) {
      const float2 s = p[(uint64_t)r * a.dim];
      all = float2{FLAT && fminf(all.x, s.x) < 0.0f ? kAnew : all.x * s.x, next(s, all.y)};
    }
  steps[y][x] = all;
  __syncthreads();
  if (c >= a.dim) return;
  float u = a.first && !a.flat ? a.first[(uint64_t)walk * a.dim + c] : 0.0f;
#pragma unroll 8
  for (uint32_t r = 0; r < y; ++r) u = next(steps[r][x], u);
  float* e = a.enter + (uint64_t)walk * a.ranges * a.dim + c;
#pragma unroll 8
  for (uint32_t r = from; r < to; ++r) {
    const float2 s = p[(uint64_t)r * a.dim];
    e[(uint64_t)r * a.dim] = u;
    u = next(s, u);
  }
}

constexpr uint32_t kMostGrid = 1u << 21;  // launches stay below 2^32 threads
constexpr uint32_t kSeeGrid = 1u << 12;   // workgroups that see to sequences without rows, at most
constexpr uint32_t kFull = 256;           // walks times blocks of channels from which on scan_rows fills the device
constexpr uint32_t kFewIterations = 3;    // ... or that are over so soon that three launches are not worth it
constexpr uint32_t kThreads = 1u << 18;   // threads that ranges are cut for: sixteen wavefronts to a CU
constexpr uint32_t kRangeMin = 8;         // rows of a range, at least

uint32_t groups_log2_for(uint32_t dim, uint32_t each) {
  uint32_t log2 = 0;
  while ((1u << log2) < std::min((dim + each - 1) / each, kGroupsMost)) ++log2;
  return log2;
}
uint32_t rows_at_once(uint32_t dim, uint32_t each) { return (kScanBlock >> groups_log2_for(dim, each)) * 2; }

// How rows and channels are dealt out.
void cut(ScanArgs& a, uint32_t each) {
  a.groups_log2 = groups_log2_for(a.dim, each);
  const uint32_t pieces = (a.dim + each - 1) / each, W = rows_at_once(a.dim, each);
  a.blocks = (pieces + (1u << a.groups_log2) - 1) >> a.groups_log2;
  a.ranges = 1;
  if ((uint64_t)a.walks * a.blocks >= kFull || a.len <= kFewIterations * W) return;
  const uint64_t wanted = std::max<uint64_t>(1, kThreads / ((uint64_t)a.walks * pieces));
  a.range_len = (uint32_t)std::max<uint64_t>(kRangeMin, (((uint64_t)a.len + wanted - 1) / wanted + 7) / 8 * 8);
  a.ranges = (uint32_t)(((uint64_t)a.len + a.range_len - 1) / a.range_len);
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
  cut(a, per);
  a.enter = reinterpret_cast<float*>(a.partial + (uint64_t)a.walks * a.ranges * a.dim);
  const uint64_t pieces = (a.dim + per - 1) / per;
  const uint64_t main_blocks =
      a.ranges > 1 ? ((uint64_t)a.walks * a.ranges * pieces + kRangeBlock - 1) / kRangeBlock : (uint64_t)a.walks * a.blocks;
  if (main_blocks > 0xFFFFFFFFull) return CVLC_ERR_ARG;
  a.main_grid = (uint32_t)std::min<uint64_t>(main_blocks, kMostGrid);
  const uint64_t seen = (a.starts || a.n == 0) && (a.last || a.status) ? see_items(a.n_seq, a.last ? a.dim : 1) : 0;
  const uint32_t more = (uint32_t)std::min<uint64_t>((seen + kRangeBlock / kWave - 1) / (kRangeBlock / kWave), kSeeGrid);
  if (a.main_grid + more == 0) return CVLC_OK;
  by_type(type, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto kernel, uint32_t grid, uint32_t block) {
      hipLaunchKernelGGL(kernel, dim3(grid), dim3(block), 0, stream, a, static_cast<const T*>(v), static_cast<const T*>(gate),
                         static_cast<const T*>(x), static_cast<const T*>(h), static_cast<T*>(out), static_cast<T*>(dgate));
    };
    // what the last-level cache (256 MB) does not hold anyway goes past the caches' order, but for the first reading of what
    // is read twice: 100 003 x 1000 bf16 in 7 sequences, backward 403 -> 361 us, forward 265 -> 236
    const bool past = (uint64_t)a.n * a.dim * sizeof(T) * (FORWARD ? 3 : 6) > 256ull * 1000000;
    if (a.ranges == 1) {
      go(past ? scan_rows_kernel<T, FORWARD, true> : scan_rows_kernel<T, FORWARD, false>, a.main_grid + more, kScanBlock);
    } else {
      go(scan_range_kernel<T, FORWARD, false, false>, a.main_grid, kRangeBlock);
      hipLaunchKernelGGL(a.flat ? scan_carry_kernel<true> : scan_carry_kernel<false>, dim3(a.walks * ((a.dim + kCarryWide - 1) / kCarryWide)), dim3(kCarryWide * kCarryRows), 0,
                         stream, a);
      go(past ? scan_range_kernel<T, FORWARD, true, true> : scan_range_kernel<T, FORWARD, true, false>, a.main_grid + more, kRangeBlock);
    }
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

// ROWS rows of a workgroup.  Every slot is compared with those of all rows before, which takes as long as the rows themselves from
// some 4000 of them on; there the slots before are read once for 16 rows: 16 384 x 256 bf16 85 -> 39 us, 65 536 x 1024 1027 -> 265
// (without slots 163).  With few rows one to a workgroup fills the chip sooner.
constexpr uint32_t kStepRows = 16, kStepMany = 4096;

template <class T, uint32_t ROWS>
__global__ __launch_bounds__(kStepBlock) void scan_step_kernel(StepArgs a, const T* x, const T* gate, T* h) {
  constexpr uint32_t N = kPerAccess<T>;
  __shared__ uint32_t taken;
  const uint32_t columns = (a.dim + N - 1) / N;
  for (uint32_t first = blockIdx.x * ROWS; first < a.n; first += gridDim.x * ROWS) {
    const uint32_t rows = min(ROWS, a.n - first);
    int32_t slot[ROWS];                 // -1: none that is there
    uint32_t live = 0, wrong = 0;       // bits of rows
#pragma unroll
    for (uint32_t r = 0; r < ROWS; ++r) {
      const int64_t given = r < rows ? slot_of(a, first + r) : -1;
      const bool there = given >= 0 && given < (int64_t)a.n_slots;
      slot[r] = there ? (int32_t)given : -1;
      live |= (uint32_t)there << r;
      wrong |= (uint32_t)(given >= (int64_t)a.n_slots) << r;
    }
    if (a.slots && live) {
      // a slot is the first token's that names it
      bool found[ROWS] = {};
      auto look = [&](auto* slots) {
        constexpr uint32_t kAtOnce = ROWS == 1 ? 2 : 8;
        for (uint32_t at = threadIdx.x; at < first; at += kAtOnce * kStepBlock) {
          int64_t other[kAtOnce];
#pragma unroll
          for (uint32_t c = 0; c < kAtOnce; ++c) other[c] = slots[min(at + c * kStepBlock, first - 1)];
#pragma unroll
          for (uint32_t c = 0; c < kAtOnce; ++c) {
            const int32_t key = other[c] >= 0 && other[c] < (int64_t)a.n_slots ? (int32_t)other[c] : -2;
#pragma unroll
            for (uint32_t r = 0; r < ROWS; ++r) found[r] |= key == slot[r];
          }
        }
      };
      if (a.slot_bytes == 8)
        look(static_cast<const int64_t*>(a.slots));
      else
        look(static_cast<const int32_t*>(a.slots));
      uint32_t mine = 0;
#pragma unroll
      for (uint32_t r = 0; r < ROWS; ++r) {
#pragma unroll
        for (uint32_t q = 0; q < r; ++q) found[r] |= slot[q] == slot[r];
        mine |= (uint32_t)found[r] << r;
      }
      if (threadIdx.x == 0) taken = 0;
      __syncthreads();
      if (mine) atomicOr(&taken, mine);
      __syncthreads();
      const uint32_t again = taken & live;
      __syncthreads();                  // before it is cleared for the next rows
      live &= ~again;
      wrong |= again;
    }
    if (wrong && a.status && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(a.status, CVLC_DEV_INDEX);
    const uint64_t all = (uint64_t)rows * columns;
    for (uint64_t e = blockIdx.y * kStepBlock + threadIdx.x; e < all; e += gridDim.y * kStepBlock) {
      const uint32_t r = ROWS == 1 ? 0 : (uint32_t)(e / columns), i = first + r, at = (uint32_t)(e - (uint64_t)r * columns) * N;
      float u[N] = {};
      if (live >> r & 1) {
        float xs[N], z[N];
        float* state = a.states + (uint64_t)(a.slots ? slot_of(a, i) : i) * a.dim;
        load_row<N>(x + i * a.x_stride, at, a.dim, 0.0f, xs);
        load_row<N>(gate + i * a.gate_stride, at, a.dim, 0.0f, z);
        load_row<N>(state, at, a.dim, 0.0f, u);
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) u[k] = blend(gate_of<sizeof(T) == 4>(z[k]), u[k], xs[k]);
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
  // the (A, B) and the start of every range, whichever way the call is cut
  uint64_t most = 0;
  for (uint32_t each : {4u, 8u})
    for (uint32_t flat : {0u, 1u}) {
      if (n == 0 || dim == 0 || (!flat && (n_seq == 0 || n % n_seq))) continue;
      ScanArgs a{};
      a.dim = dim;
      a.walks = flat ? 1 : n_seq;
      a.len = flat ? n : n / n_seq;
      cut(a, each);
      if (a.ranges > 1) most = std::max(most, (uint64_t)a.walks * a.ranges * a.dim);
    }
  return 256u + (size_t)(most * (sizeof(float2) + sizeof(float)));
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
    auto go = [&](auto many) {
      constexpr uint32_t R = decltype(many)::value;
      const uint32_t blocks = std::min((n + R - 1) / R, 1u << 16);
      const uint64_t accesses = ((uint64_t)dim + kPerAccess<T> - 1) / kPerAccess<T> * R, pieces = (accesses + kStepBlock - 1) / kStepBlock;
      const uint32_t side = (uint32_t)std::min<uint64_t>(pieces, R == 1 ? 64 : std::max(1u, 2048 / blocks));
      hipLaunchKernelGGL((scan_step_kernel<T, R>), dim3(blocks, side), dim3(kStepBlock), 0, static_cast<hipStream_t>(hip_stream), a,
                         static_cast<const T*>(d_x), static_cast<const T*>(d_gate), static_cast<T*>(d_h));
    };
    if (d_slots && n > kStepMany)
      go(std::integral_constant<uint32_t, kStepRows>{});
    else
      go(std::integral_constant<uint32_t, 1>{});
  });
  return hip_check(hipGetLastError());
}

}  // extern "C"
