// cvlc_norm.hip -- layer norm of rows and its backward pass.
//
// Forward: the mean, then the mean square of what is left of it (not the
// difference of two large sums), then y.  Backward: two sums, of g and of g * h,
// then dx.  dgamma and dbeta are sums over all rows: every workgroup keeps its
// share while it goes over its rows and leaves it as partial sums, a second
// launch adds those up in order.  All of it is bound by HBM: the arithmetic is
// a fifth of the time that the bytes take, as long as the next row is on its way
// while one is worked on.
//
// Rows of up to 16384 elements lie in registers between the sums and the output
// (norm_rows, norm_grad_rows): one read, one write.  Longer rows, and rows
// shorter than one access, are read again for every step (norm, norm_dx,
// norm_columns).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kNormBlock = 256, kNormWaves = kNormBlock / kWave;

struct NormArgs {
  uint32_t n, dim;
  uint64_t x_stride, y_stride, dx_stride;  // y: forward's output, backward's dy
  const float *gamma, *beta;
  float eps;
  float* stats;
};

template <class TX, class TY>
__global__ __launch_bounds__(kNormBlock) void norm_kernel(NormArgs a, const TX* x, TY* y) {
  constexpr uint32_t N = kPerAccess<TX, TY>;
  __shared__ float scratch[kNormWaves];
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const TX* xr = x + row * a.x_stride;
    float sum = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N];
      load_row<N>(xr, at, a.dim, 0.0f, v);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sum += v[i];
    }
    const float mean = block_sum<kNormWaves>(sum, scratch) / (float)a.dim;
    float sq = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N];
      load_row<N>(xr, at, a.dim, mean, v);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sq = fmaf(v[i] - mean, v[i] - mean, sq);
    }
    const float r = 1.0f / sqrtf(block_sum<kNormWaves>(sq, scratch) / (float)a.dim + a.eps);
    if (a.stats && threadIdx.x == 0) {
      a.stats[2 * (uint64_t)row] = mean;
      a.stats[2 * (uint64_t)row + 1] = r;
    }
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N], g[N], b[N];
      load_row<N>(xr, at, a.dim, 0.0f, v);
      if (a.gamma) load_row<N>(a.gamma, at, a.dim, 1.0f, g);
      if (a.beta) load_row<N>(a.beta, at, a.dim, 0.0f, b);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[i] = fmaf((v[i] - mean) * r, a.gamma ? g[i] : 1.0f, a.beta ? b[i] : 0.0f);
      store_row<N>(y + row * a.y_stride, at, a.dim, v);
    }
  }
}

template <class TX, class TY>
__global__ __launch_bounds__(kNormBlock) void norm_dx_kernel(NormArgs a, const TX* x, const TY* dy, TX* dx) {
  constexpr uint32_t N = kPerAccess<TX, TY>;
  __shared__ float scratch[2 * kNormWaves];
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const TX* xr = x + row * a.x_stride;
    const TY* dyr = dy + row * a.y_stride;
    const float mean = a.stats[2 * (uint64_t)row], r = a.stats[2 * (uint64_t)row + 1];
    float sg = 0.0f, sgh = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N], d[N], g[N];
      load_row<N>(xr, at, a.dim, 0.0f, v);
      load_row<N>(dyr, at, a.dim, 0.0f, d);
      if (a.gamma) load_row<N>(a.gamma, at, a.dim, 0.0f, g);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float t = a.gamma ? d[i] * g[i] : d[i];
        sg += t;
        sgh = fmaf(t, (v[i] - mean) * r, sgh);
      }
    }
    block_sum2<kNormWaves>(sg, sgh, scratch);
    sg /= (float)a.dim;
    sgh /= (float)a.dim;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N], d[N], g[N];
      load_row<N>(xr, at, a.dim, 0.0f, v);
      load_row<N>(dyr, at, a.dim, 0.0f, d);
      if (a.gamma) load_row<N>(a.gamma, at, a.dim, 0.0f, g);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float t = a.gamma ? d[i] * g[i] : d[i];
        v[i] = r * (t - sg - (v[i] - mean) * r * sgh);
      }
      store_row<N>(dx + row * a.dx_stride, at, a.dim, v);
    }
  }
}

// Partial sums of dy * h and dy over a block of rows, for kNormBlock columns: part[block][0 or 1][dim].
template <class TX, class TY>
__global__ __launch_bounds__(kNormBlock) void norm_columns_kernel(NormArgs a, const TX* x, const TY* dy, uint32_t block_rows,
                                                                  float* part) {
  const uint32_t row0 = blockIdx.y * block_rows, rows = min(block_rows, a.n - row0);
  for (uint32_t c = blockIdx.x * kNormBlock + threadIdx.x; c < a.dim; c += gridDim.x * kNormBlock) {
    float dg = 0.0f, db = 0.0f;
    for (uint32_t i = 0; i < rows; ++i) {
      const uint64_t row = row0 + i;
      const float d = (float)dy[row * a.y_stride + c];
      dg = fmaf(d, ((float)x[row * a.x_stride + c] - a.stats[2 * row]) * a.stats[2 * row + 1], dg);
      db += d;
    }
    part[(2 * (uint64_t)blockIdx.y) * a.dim + c] = dg;
    part[(2 * (uint64_t)blockIdx.y + 1) * a.dim + c] = db;
  }
}

// ----------------------------------------------------------------------------- rows in registers
// W wavefronts to a row, V accesses per thread, O wavefronts on a SIMD at a time.  Workgroups (of four rows where a row is
// one wavefront's) stay and go from row to row, so that gamma and beta are read once, and ask for the next row before
// they work on this one.  The grid is what the device holds at once: with more workgroups than that the last ones run
// after the others (three of eight wavefronts on a CU that held two: 215 us for 180).
template <uint32_t W_, uint32_t V_, uint32_t O_, bool LDS_ = false>
struct RowShape {
  static constexpr uint32_t W = W_, V = V_, O = O_;
  static constexpr bool LDS = LDS_;  // the sums over the rows are kept in LDS
  static constexpr uint32_t kRows = W == 1 ? 4 : 1, kWaves = W * kRows, kThreads = kWaves * kWave;
  static constexpr uint32_t kPerCu = 4 * O > kWaves ? 4 * O / kWaves : 1;
};

// A thread's part of a row; what is not its own stays zero bits.
template <class T, uint32_t N, class S, bool ONCE>
struct RawRow {
  Raw<T, N> v[S::V];
  __device__ __forceinline__ RawRow() {
#pragma unroll
    for (uint32_t j = 0; j < S::V; ++j)
#pragma unroll
      for (uint32_t i = 0; i < Raw<T, N>::kWords; ++i) v[j].w[i] = 0;
  }
  __device__ __forceinline__ void load(const T* row, const Place<N> (&place)[S::V]) {
#pragma unroll
    for (uint32_t j = 0; j < S::V; ++j)
      if (place[j].any()) v[j].template load<ONCE>(row + place[j].at);
  }
};

template <class TX, class TY, class S, bool ONCE>
__global__ __launch_bounds__(S::kThreads, S::O) void norm_rows_kernel(NormArgs a, const TX* x, TY* y) {
  constexpr uint32_t N = kPerAccess<TX, TY>, L = S::W * kWave, V = S::V;
  __shared__ float scratch[2 * S::W];
  const uint32_t lane = threadIdx.x % L, step = gridDim.x * S::kRows;
  float g[V][N], b[V][N];
  Place<N> place[V];
#pragma unroll
  for (uint32_t j = 0; j < V; ++j) {
    place[j] = Place<N>((j * L + lane) * N, a.dim);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      g[j][i] = 1.0f;
      b[j][i] = 0.0f;
    }
    if (a.gamma) load_values<N>(a.gamma + place[j].at, g[j]);
    if (a.beta) load_values<N>(a.beta + place[j].at, b[j]);
  }
  const float dim = (float)a.dim;
  uint32_t row = blockIdx.x * S::kRows + threadIdx.x / L;
  RawRow<TX, N, S, ONCE> raw;
  if (row < a.n) raw.load(x + row * a.x_stride, place);
  for (; row < a.n; row += step) {
    float v[V][N], sum = 0.0f, sq = 0.0f;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
      raw.v[j].values(v[j]);
      place[j].mask(v[j], 0.0f);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sum += v[j][i];
    }
    if (row + step < a.n) raw.load(x + (row + step) * a.x_stride, place);
    const float mean = block_sum<S::W>(sum, scratch) / dim;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[j][i] -= mean;
      place[j].mask(v[j], 0.0f);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sq = fmaf(v[j][i], v[j][i], sq);
    }
    const float r = 1.0f / sqrtf(block_sum<S::W>(sq, scratch) / dim + a.eps);
    if (a.stats && lane == 0) {
      a.stats[2 * (uint64_t)row] = mean;
      a.stats[2 * (uint64_t)row + 1] = r;
    }
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[j][i] = fmaf(v[j][i] * r, g[j][i], b[j][i]);
      place[j].template store<ONCE>(y + row * a.y_stride, v[j]);
    }
  }
}

// The backward pass of rows, and the thread's share of the sums over the rows.
template <class TX, class TY, class S, bool ONCE>
__global__ __launch_bounds__(S::kThreads, S::O) void norm_grad_rows_kernel(NormArgs a, const TX* x, const TY* dy, TX* dx, float* part) {
  constexpr uint32_t N = kPerAccess<TX, TY>, L = S::W * kWave, V = S::V;
  __shared__ float scratch[2 * S::W];
  const uint32_t lane = threadIdx.x % L, step = gridDim.x * S::kRows;
  // the sums over the rows: in registers, or in LDS where a thread has too many columns for that
  constexpr uint32_t R = S::LDS ? 1 : V;
  float g[R][N], dg[R][N], db[R][N];
  extern __shared__ float4 sums[];  // [2][V * N / 4][L]
  auto sum_at = [&](uint32_t which, uint32_t j, uint32_t q) -> float4& { return sums[((which * V + j) * (N / 4) + q) * L + lane]; };
  Place<N> place[V];
#pragma unroll
  for (uint32_t j = 0; j < V; ++j) {
    place[j] = Place<N>((j * L + lane) * N, a.dim);
    if constexpr (S::LDS) {
#pragma unroll
      for (uint32_t q = 0; q < N / 4; ++q) sum_at(0, j, q) = sum_at(1, j, q) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        g[j][i] = 1.0f;
        dg[j][i] = db[j][i] = 0.0f;
      }
      if (a.gamma) load_values<N>(a.gamma + place[j].at, g[j]);
    }
  }
  const float dim = (float)a.dim;
  uint32_t row = blockIdx.x * S::kRows + threadIdx.x / L;
  RawRow<TX, N, S, ONCE> rx;
  RawRow<TY, N, S, ONCE> ry;
  float mean = 0.0f, r = 0.0f;
  auto ask = [&](uint32_t at) {
    rx.load(x + at * a.x_stride, place);
    ry.load(dy + at * a.y_stride, place);
    mean = a.stats[2 * (uint64_t)at];
    r = a.stats[2 * (uint64_t)at + 1];
  };
  if (row < a.n) ask(row);
  for (; row < a.n; row += step) {
    float h[V][N], t[V][N], sg = 0.0f, sgh = 0.0f;
    const float r_now = r;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
      rx.v[j].values(h[j]);
      ry.v[j].values(t[j]);
      place[j].mask(h[j], mean);  // what is not the thread's adds nothing
      place[j].mask(t[j], 0.0f);
      float gj[N];
      if constexpr (S::LDS) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) gj[i] = 1.0f;
        if (a.gamma) load_values<N>(a.gamma + place[j].at, gj);
      }
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) h[j][i] = (h[j][i] - mean) * r_now;
      if constexpr (S::LDS) {
#pragma unroll
        for (uint32_t q = 0; q < N / 4; ++q) {
          float4 &sdg = sum_at(0, j, q), &sdb = sum_at(1, j, q);
          float* tq = t[j] + 4 * q;
          const float* hq = h[j] + 4 * q;
          sdg = make_float4(fmaf(tq[0], hq[0], sdg.x), fmaf(tq[1], hq[1], sdg.y), fmaf(tq[2], hq[2], sdg.z), fmaf(tq[3], hq[3], sdg.w));
          sdb = make_float4(sdb.x + tq[0], sdb.y + tq[1], sdb.z + tq[2], sdb.w + tq[3]);
        }
      } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
          dg[j][i] = fmaf(t[j][i], h[j][i], dg[j][i]);
          db[j][i] += t[j][i];
        }
      }
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        t[j][i] *= S::LDS ? gj[i] : g[S::LDS ? 0 : j][i];
        sg += t[j][i];
        sgh = fmaf(t[j][i], h[j][i], sgh);
      }
    }
    if (row + step < a.n) ask(row + step);
    if (!dx) continue;
    block_sum2<S::W>(sg, sgh, scratch);
    sg /= dim;
    sgh /= dim;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) t[j][i] = r_now * (t[j][i] - sg - h[j][i] * sgh);
      place[j].template store<ONCE>(dx + row * a.dx_stride, t[j]);
    }
  }
  if (!part) return;
  float* to = part + 2 * (uint64_t)blockIdx.x * a.dim;
  if constexpr (S::kRows > 1) {  // the workgroup's rows in turn
    for (uint32_t turn = 0; turn < S::kRows; ++turn) {
      if (threadIdx.x / L == turn)
#pragma unroll
        for (uint32_t j = 0; j < V; ++j)
#pragma unroll
          for (uint32_t q = 0; q < N / 4; ++q) {
            float4 &sdg = sum_at(0, j, q), &sdb = sum_at(1, j, q);
            float *dgq = dg[j] + 4 * q, *dbq = db[j] + 4 * q;
            if (turn) {
              dgq[0] += sdg.x, dgq[1] += sdg.y, dgq[2] += sdg.z, dgq[3] += sdg.w;
              dbq[0] += sdb.x, dbq[1] += sdb.y, dbq[2] += sdb.z, dbq[3] += sdb.w;
            }
            sdg = make_float4(dgq[0], dgq[1], dgq[2], dgq[3]);
            sdb = make_float4(dbq[0], dbq[1], dbq[2], dbq[3]);
          }
      __syncthreads();
    }
    if (threadIdx.x / L != S::kRows - 1) return;
  }
#pragma unroll
  for (uint32_t j = 0; j < V; ++j) {
    if constexpr (S::LDS) {
      float all[2][N];
#pragma unroll
      for (uint32_t q = 0; q < N / 4; ++q)
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
          const float4 s = sum_at(k, j, q);
          float* to_q = all[k] + 4 * q;
          to_q[0] = s.x, to_q[1] = s.y, to_q[2] = s.z, to_q[3] = s.w;
        }
      place[j].template store<false>(to, all[0]);
      place[j].template store<false>(to + a.dim, all[1]);
    } else {
      place[j].template store<false>(to, dg[j]);
      place[j].template store<false>(to + a.dim, db[j]);
    }
  }
}

// Few wavefronts with many bytes under way each do best: rows of one wavefront need no barrier (65536 x 4096 bf16: a
// wavefront with eight accesses per thread 183 us, four with two 201, eight with one 220).  With few rows that leaves
// CUs empty, so rows of more than 128 accesses are spread over two wavefronts below 8192 rows, rows of more than 256 over
// four below 16384.  By one wavefront and by the more, bf16: rows of 2048, 200 of them 4.3 and 3.2 us on the device, 2048 6.1
// and 5.7, 4096 8.9 both, 8192 12.6 and 12.8 a call; of 4096, 200 6.4 and 3.5 on the device, 4096 15.3 and 13.0 a call, 8192 27.9
// and 26.7, 16384 48.4 and 47.9, 32768 92.4 and 95.6; of 2500, which leave three of eight accesses idle, 8192 24.6 and 20.1,
// 16384 43.7 and 36.9.  fp32: 8192 x 1300 19.1 and 18.0, 16384 32.8 and 34.8.
// Calls f with the shape for rows of `dim` elements, `per` of them an access; false: too long for registers, or shorter than
// an access.
template <uint32_t per, class F>
bool by_norm_shape(uint32_t n, uint32_t dim, F f) {
  const uint32_t vectors = (dim + per - 1) / per;
  if (dim < per) return false;
  if (vectors <= 64) return f(RowShape<1, 1, 8>{});
  if (vectors <= 128) return f(RowShape<1, 2, 2>{});
  if (vectors <= 256) return n >= 8192 ? f(RowShape<1, 4, 2>{}) : f(RowShape<2, 2, 4>{});
  if (vectors <= 512) return n >= 16384 ? f(RowShape<1, 8, 1>{}) : f(RowShape<4, 2, 6>{});
  if (vectors <= 1024) return f(RowShape<8, 2, 4>{});
  if (vectors <= 2048) return f(RowShape<8, 4, 2>{});
  if constexpr (per == 4)
    if (vectors <= 4096) return f(RowShape<16, 4, 4>{});
  return false;
}
// Backward a thread holds five values per column (gamma, two sums, h, g), so one access per thread as far as a workgroup
// goes.  Beyond 8192 fp32 (1024 threads with 16 columns each) the sums over the rows lie in LDS (8192 x 16384 fp32: 281 us,
// 437 with them in registers that spill).  Two accesses of eight values, 16 columns as well, fit for bf16 (8192 x 16384: 148 us)
// and nearly for fp16, which spills 4 registers (185).
template <uint32_t per, class F>
bool by_norm_grad_shape(uint32_t dim, F f) {
  const uint32_t vectors = (dim + per - 1) / per;
  if (dim < per) return false;
  if (vectors <= 64) return f(RowShape<1, 1, 6>{});
  if (vectors <= 128) return f(RowShape<2, 1, 4>{});
  if (vectors <= 256) return f(RowShape<4, 1, 4>{});
  if (vectors <= 512) return f(RowShape<8, 1, 4>{});
  if (vectors <= 1024) return f(RowShape<16, 1, 4>{});
  if (vectors <= 2048) return f(RowShape<16, 2, 4>{});
  if constexpr (per == 4)
    if (vectors <= 4096) return f(RowShape<16, 4, 4, true>{});
  return false;
}

// Adds the blocks up: 64 columns a workgroup, a sixteenth of the blocks a wavefront.
constexpr uint32_t kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves * kWave) void norm_join_kernel(const float* part, uint32_t blocks, uint32_t dim,
                                                                       uint32_t add, float* dgamma, float* dbeta) {
  __shared__ float sums[kJoinWaves][kWave];
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const uint32_t each = (blocks + kJoinWaves - 1) / kJoinWaves;
  const uint32_t from = min(wave_id() * each, blocks), to = min(from + each, blocks);
  for (uint32_t first = blockIdx.x * kWave; first < dim; first += gridDim.x * kWave) {
    const uint32_t c = first + lane_id();
    float s = 0.0f;
    if (c < dim)
#pragma unroll 8
      for (uint32_t b = from; b < to; ++b) s += part[(2 * (uint64_t)b + blockIdx.y) * dim + c];
    sums[wave_id()][lane_id()] = s;
    __syncthreads();
    if (wave_id() == 0 && c < dim) {
      s = add ? out[c] : 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < kJoinWaves; ++w) s += sums[w][lane_id()];
      out[c] = s;
    }
    __syncthreads();
  }
}

constexpr uint32_t kRowBlocks = 2048;  // workgroups that leave partial sums, at most ...
constexpr uint32_t kRowsEach = 8;      // ... and rows that each goes over, at least, beyond 256 workgroups
uint32_t partials(uint32_t n) { return std::min(kRowBlocks, std::max(std::min(n, 256u), n / kRowsEach)); }

// Data that the last-level cache (256 MB) does not hold anyway are read and written past the caches' order (65536 x 4096
// bf16: 198 -> 183 us; 2007 x 1003 fp32, which it does hold, 14.5 -> 16.5).
bool once(uint32_t n, uint32_t dim, uint32_t bytes) { return (uint64_t)n * dim * bytes > 256ull * 1000000; }

uint32_t rows_per_block(uint32_t n) { return std::max(1u, (n + 255u) / 256u); }

int launched() { return hip_check(hipGetLastError()); }

}  // namespace
}  // namespace cvlc

extern "C" {

int cvlc_layer_norm(uint32_t n, uint32_t dim, const void* d_x, uint32_t x_type, uint64_t x_stride, const float* d_gamma,
                    const float* d_beta, float eps, void* d_y, uint32_t y_type, uint64_t y_stride, float* d_stats,
                    void* hip_stream) {
  using namespace cvlc;
  if (dim < 1 || dim > 0x7FFFFFFFu || n > 0x7FFFFFFFu || !types_go(x_type, y_type) || x_stride < dim || y_stride < dim)
    return CVLC_ERR_ARG;
  if (!(eps >= 0.0f) || std::isinf(eps)) return CVLC_ERR_ARG;
  if (d_gamma && !buffer_ok(d_gamma, 4)) return CVLC_ERR_ARG;
  if (d_beta && !buffer_ok(d_beta, 4)) return CVLC_ERR_ARG;
  if (d_stats && !buffer_ok(d_stats, 4)) return CVLC_ERR_ARG;
  if (n == 0) return CVLC_OK;
  if (!buffer_ok(d_x, type_bytes(x_type)) || !buffer_ok(d_y, type_bytes(y_type))) return CVLC_ERR_ARG;
  if (d_x == d_y && (x_type != y_type || x_stride != y_stride)) return CVLC_ERR_ARG;
  const NormArgs a{n, dim, x_stride, y_stride, 0, d_gamma, d_beta, eps, d_stats};
  const bool past = once(n, dim, type_bytes(x_type) + type_bytes(y_type));
  by_types(x_type, y_type, [&](auto tx, auto ty) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    if (by_norm_shape<kPerAccess<TX, TY>>(n, dim, [&](auto shape) {
          using S = decltype(shape);
          hipLaunchKernelGGL((past ? norm_rows_kernel<TX, TY, S, true> : norm_rows_kernel<TX, TY, S, false>),
                             dim3(std::min((n + S::kRows - 1) / S::kRows, 256u * S::kPerCu)), dim3(S::kThreads), 0,
                             static_cast<hipStream_t>(hip_stream), a, static_cast<const TX*>(d_x), static_cast<TY*>(d_y));
          return true;
        }))
      return;
    hipLaunchKernelGGL((norm_kernel<TX, TY>), dim3(std::min(n, 1u << 20)), dim3(kNormBlock), 0, static_cast<hipStream_t>(hip_stream),
                       a, static_cast<const TX*>(d_x), static_cast<TY*>(d_y));
  });
  return launched();
}

size_t cvlc_layer_norm_grad_workspace_bytes(uint32_t n, uint32_t dim) {
  const uint64_t blocks = cvlc::partials(n);
  return 256u + (size_t)(blocks * 2u * dim * sizeof(float));
}

int cvlc_layer_norm_grad(uint32_t n, uint32_t dim, const void* d_dy, uint32_t dy_type, uint64_t dy_stride, const void* d_x,
                         uint32_t x_type, uint64_t x_stride, const float* d_stats, const float* d_gamma, void* d_dx,
                         uint64_t dx_stride, float* d_dgamma, float* d_dbeta, uint32_t flags, void* d_workspace,
                         size_t ws_bytes, void* hip_stream) {
  using namespace cvlc;
  if (dim < 1 || dim > 0x7FFFFFFFu || n > 0x7FFFFFFFu || !types_go(x_type, dy_type) || x_stride < dim || dy_stride < dim)
    return CVLC_ERR_ARG;
  if (flags & ~CVLC_GRAD_ACCUMULATE) return CVLC_ERR_ARG;
  if (!d_dx && !d_dgamma && !d_dbeta && n) return CVLC_ERR_ARG;
  if (d_dx && dx_stride < dim) return CVLC_ERR_ARG;
  if (d_gamma && !buffer_ok(d_gamma, 4)) return CVLC_ERR_ARG;
  if (d_dgamma && !buffer_ok(d_dgamma, 4)) return CVLC_ERR_ARG;
  if (d_dbeta && !buffer_ok(d_dbeta, 4)) return CVLC_ERR_ARG;
  if (!buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  if (n) {
    if (!buffer_ok(d_x, type_bytes(x_type)) || !buffer_ok(d_dy, type_bytes(dy_type)) || !buffer_ok(d_stats, 4)) return CVLC_ERR_ARG;
    if (d_dx) {
      if (!buffer_ok(d_dx, type_bytes(x_type))) return CVLC_ERR_ARG;
      if (d_dx == d_x && dx_stride != x_stride) return CVLC_ERR_ARG;
      if (d_dx == d_dy && (dx_stride != dy_stride || x_type != dy_type)) return CVLC_ERR_ARG;
    }
  }
  if (ws_bytes < cvlc_layer_norm_grad_workspace_bytes(n, dim)) return CVLC_ERR_CAPACITY;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const NormArgs a{n, dim, x_stride, dy_stride, dx_stride, d_gamma, nullptr, 0.0f, const_cast<float*>(d_stats)};
  const bool past = once(n, dim, (d_dx ? 2u : 1u) * type_bytes(x_type) + type_bytes(dy_type));
  float* part = static_cast<float*>(d_workspace);
  const uint32_t block_rows = rows_per_block(n);
  uint32_t blocks = (n + block_rows - 1) / block_rows;
  if (n)
    by_types(x_type, dy_type, [&](auto tx, auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      const TX* x = static_cast<const TX*>(d_x);
      const TY* dy = static_cast<const TY*>(d_dy);
      if (by_norm_grad_shape<kPerAccess<TX, TY>>(dim, [&](auto shape) {
            using S = decltype(shape);
            blocks = std::min({(n + S::kRows - 1) / S::kRows, 256u * S::kPerCu, partials(n)});
            constexpr uint32_t lds = S::LDS || S::kRows > 1 ? 2 * S::V * kPerAccess<TX, TY> * S::W * kWave * sizeof(float) : 0;
            hipLaunchKernelGGL((past ? norm_grad_rows_kernel<TX, TY, S, true> : norm_grad_rows_kernel<TX, TY, S, false>), dim3(blocks),
                               dim3(S::kThreads), lds, stream, a, x, dy,
                               static_cast<TX*>(d_dx), d_dgamma || d_dbeta ? part : nullptr);
            return true;
          }))
        return;
      // the sums over the rows come first: dx may lie where dy or x does
      if (d_dgamma || d_dbeta)
        hipLaunchKernelGGL((norm_columns_kernel<TX, TY>), dim3(std::min((dim + kNormBlock - 1) / kNormBlock, 65536u), blocks),
                           dim3(kNormBlock), 0, stream, a, x, dy, block_rows, part);
      if (d_dx)
        hipLaunchKernelGGL((norm_dx_kernel<TX, TY>), dim3(std::min(n, 1u << 20)), dim3(kNormBlock), 0, stream, a, x, dy,
                           static_cast<TX*>(d_dx));
    });
  if (d_dgamma || d_dbeta)
    hipLaunchKernelGGL(norm_join_kernel, dim3(std::min((dim + kWave - 1) / kWave, 1u << 20), 2), dim3(kJoinWaves * kWave), 0, stream, part, blocks, dim,
                       flags & CVLC_GRAD_ACCUMULATE, d_dgamma, d_dbeta);
  return launched();
}

}  // extern "C"
