// cvlc_norm.hip -- layer norm of rows and its backward pass.
//
// Forward, a workgroup per row: the mean, then the mean square of what is left
// of it (not the difference of two large sums), then the row again for y.
// Backward, a workgroup per row for dx: two sums, of g and of g * h, then the
// row again.  dgamma and dbeta are sums over all rows: workgroups take blocks of
// rows and leave partial sums, a second launch adds the blocks up in order.
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
  __shared__ float scratch[2 * kNormWaves];
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const TX* xr = x + row * a.x_stride;
    float sum = 0.0f, unused = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N];
      load_row<N>(xr, at, a.dim, 0.0f, v);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sum += v[i];
    }
    block_sum2<kNormWaves>(sum, unused, scratch);
    const float mean = sum / (float)a.dim;
    float sq = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < a.dim; at += kNormBlock * N) {
      float v[N];
      load_row<N>(xr, at, a.dim, mean, v);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sq = fmaf(v[i] - mean, v[i] - mean, sq);
    }
    block_sum2<kNormWaves>(sq, unused, scratch);
    const float r = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
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

// Adds the blocks up: 64 columns a workgroup, a sixteenth of the blocks a wavefront.
constexpr uint32_t kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves * kWave) void norm_join_kernel(const float* part, uint32_t blocks, uint32_t dim,
                                                                       uint32_t add, float* dgamma, float* dbeta) {
  __shared__ float sums[kJoinWaves][kWave];
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const uint32_t c = blockIdx.x * kWave + lane_id();
  const uint32_t each = (blocks + kJoinWaves - 1) / kJoinWaves;
  const uint32_t from = wave_id() * each, to = min(from + each, blocks);
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
}

constexpr uint32_t kRowBlocks = 256;  // blocks of rows for the column sums, at most

uint32_t rows_per_block(uint32_t n) { return std::max(1u, (n + kRowBlocks - 1) / kRowBlocks); }

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
  by_types(x_type, y_type, [&](auto tx, auto ty) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    hipLaunchKernelGGL((norm_kernel<TX, TY>), dim3(std::min(n, 1u << 20)), dim3(kNormBlock), 0, static_cast<hipStream_t>(hip_stream),
                       a, static_cast<const TX*>(d_x), static_cast<TY*>(d_y));
  });
  return launched();
}

size_t cvlc_layer_norm_grad_workspace_bytes(uint32_t n, uint32_t dim) {
  const uint64_t blocks = std::min(n, cvlc::kRowBlocks);
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
  float* part = static_cast<float*>(d_workspace);
  const uint32_t block_rows = rows_per_block(n), blocks = (n + block_rows - 1) / block_rows;
  if (n)
    by_types(x_type, dy_type, [&](auto tx, auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      const TX* x = static_cast<const TX*>(d_x);
      const TY* dy = static_cast<const TY*>(d_dy);
      // the sums over the rows come first: dx may lie where dy or x does
      if (d_dgamma || d_dbeta)
        hipLaunchKernelGGL((norm_columns_kernel<TX, TY>), dim3(std::min((dim + kNormBlock - 1) / kNormBlock, 65536u), blocks),
                           dim3(kNormBlock), 0, stream, a, x, dy, block_rows, part);
      if (d_dx)
        hipLaunchKernelGGL((norm_dx_kernel<TX, TY>), dim3(std::min(n, 1u << 20)), dim3(kNormBlock), 0, stream, a, x, dy,
                           static_cast<TX*>(d_dx));
    });
  if (d_dgamma || d_dbeta)
    hipLaunchKernelGGL(norm_join_kernel, dim3((dim + kWave - 1) / kWave, 2), dim3(kJoinWaves * kWave), 0, stream, part, blocks, dim,
                       flags & CVLC_GRAD_ACCUMULATE, d_dgamma, d_dbeta);
  return launched();
}

}  // extern "C"
