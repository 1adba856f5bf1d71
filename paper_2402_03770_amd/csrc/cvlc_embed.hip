// cvlc_embed.hip -- embedding lookup and its gradient by sorted tokens.
//
// Gradient: dtable[v] = scale * sum of the dout rows whose token is v.  Texts'
// tokens are far from even (the commonest is a twentieth of all), so the work is
// cut by sorted place, not by token:
//   sort_hist, sort_scatter   stable radix sort of (token, place) pairs, up to 11
//                bits a pass, least significant digit first; a tile of 4096 pairs
//                per workgroup.  Tokens that are left out (negative or beyond the
//                vocabulary) sort behind all others, as token `vocab`.
//   sum          a chunk of kChunk consecutive sorted places and one vector of
//                columns per thread: adds rows up while the token stays, writes
//                the sum when it changes.  A token that reaches into other chunks
//                has one partial sum in each.  Marks the tokens that came.
//   finish       adds up the partial sums of such tokens, in order, and writes
//                zeros to the rows that no token named.
// The order of every sum is fixed by the places and the chunk length.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kEmbedBlock = 256;
constexpr uint32_t kSortBlock = 256, kSortWaves = kSortBlock / kWave;
constexpr uint32_t kTile = 4096;                           // pairs a workgroup sorts per pass
constexpr uint32_t kTileRounds = kTile / kSortBlock;       // of 64 consecutive pairs per wavefront
constexpr uint32_t kDigitBits = 11, kDigitsMax = 1u << kDigitBits;
constexpr uint32_t kInlineTiles = 64;                      // tiles whose counts every workgroup adds up for itself
constexpr uint32_t kChunk = 64;                            // sorted places that a thread adds up
constexpr uint32_t kDeep = 8;                              // rows in flight per thread

__device__ __forceinline__ int64_t load_token(const void* ids, uint32_t id_bytes, uint64_t i) {
  return id_bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}

// ----------------------------------------------------------------------------- lookup
// `lanes` threads (a power of two) to a row.
template <class TT, class TO>
__global__ __launch_bounds__(kEmbedBlock) void embed_kernel(uint32_t n, const void* ids, uint32_t id_bytes, const TT* table,
                                                            uint64_t table_stride, uint32_t vocab, uint32_t dim, float scale,
                                                            TO* out, uint64_t out_stride, uint32_t lanes_log, uint32_t* status) {
  constexpr uint32_t N = kPerAccess<TT, TO>;
  const uint32_t lanes = 1u << lanes_log, lane = threadIdx.x & (lanes - 1), rows = kEmbedBlock >> lanes_log;
  for (uint64_t row = (uint64_t)blockIdx.x * rows + (threadIdx.x >> lanes_log); row < n; row += (uint64_t)gridDim.x * rows) {
    const int64_t id = load_token(ids, id_bytes, row);
    const bool there = id >= 0 && id < (int64_t)vocab;
    if (id >= (int64_t)vocab && status && lane == 0) atomicOr(status, CVLC_DEV_INDEX);
    const TT* from = table + (there ? (uint64_t)id : 0u) * table_stride;
    TO* to = out + row * out_stride;
    for (uint32_t at = lane * N; at < dim; at += lanes * N) {
      float v[N] = {};
      if (there) {
        load_row<N>(from, at, dim, 0.0f, v);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] *= scale;
      }
      store_row<N>(to, at, dim, v);
    }
  }
}

// ----------------------------------------------------------------------------- sort
struct SortArgs {
  const void* ids;  // first pass: the tokens
  uint32_t id_bytes, vocab;
  const uint2* from;  // later passes: (token, place)
  uint2* to;
  uint32_t n, tiles, shift, bits;
  uint32_t* counts;  // [tiles][digits], then [digits] in all where a scan makes them running sums
  uint32_t* status;
};

template <bool FIRST>
__device__ __forceinline__ uint2 load_pair(const SortArgs& a, uint32_t i, uint32_t* bad) {
  if constexpr (!FIRST) {
    return a.from[i];
  } else {
    const int64_t id = load_token(a.ids, a.id_bytes, i);
    if (id >= (int64_t)a.vocab) *bad = 1;
    return make_uint2(id >= 0 && id < (int64_t)a.vocab ? (uint32_t)id : a.vocab, i);
  }
}

// Counts per digit of every tile; the first pass also clears the marks of tokens.
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void sort_hist_kernel(SortArgs a, uint32_t* marks, uint32_t mark_words) {
  __shared__ uint32_t hist[kDigitsMax];
  const uint32_t digits = 1u << a.bits;
  if (FIRST) {
    for (uint64_t i = (uint64_t)blockIdx.x * kSortBlock + threadIdx.x; i < mark_words; i += (uint64_t)gridDim.x * kSortBlock) marks[i] = 0;
  }
  for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock) hist[d] = 0;
  __syncthreads();
  uint32_t bad = 0;
#pragma unroll
  for (uint32_t u = 0; u < kTileRounds; ++u) {
    const uint64_t i = (uint64_t)blockIdx.x * kTile + u * kSortBlock + threadIdx.x;
    if (i < a.n) atomicAdd(&hist[(load_pair<FIRST>(a, (uint32_t)i, &bad).x >> a.shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock) a.counts[(uint64_t)blockIdx.x * digits + d] = hist[d];
}

// Many tiles: their counts become running sums over the tiles, the totals go behind them.  64 digits a workgroup.
constexpr uint32_t kScanWaves = 16;
__global__ __launch_bounds__(kScanWaves * kWave) void sort_scan_kernel(uint32_t* counts, uint32_t tiles, uint32_t digits) {
  __shared__ uint32_t sums[kScanWaves][kWave];
  const uint32_t d = blockIdx.x * kWave + lane_id(), each = (tiles + kScanWaves - 1) / kScanWaves;
  const uint32_t from = min(wave_id() * each, tiles), to = min(from + each, tiles);
  uint32_t s = 0;
  if (d < digits)
#pragma unroll 8
    for (uint32_t t = from; t < to; ++t) s += counts[(uint64_t)t * digits + d];
  sums[wave_id()][lane_id()] = s;
  __syncthreads();
  if (d >= digits) return;
  uint32_t before = 0, all = 0;
  for (uint32_t w = 0; w < kScanWaves; ++w) {
    if (w < wave_id()) before += sums[w][lane_id()];
    all += sums[w][lane_id()];
  }
#pragma unroll 8
  for (uint32_t t = from; t < to; ++t) {
    const uint32_t v = counts[(uint64_t)t * digits + d];
    counts[(uint64_t)t * digits + d] = before;
    before += v;
  }
  if (wave_id() == 0) counts[(uint64_t)tiles * digits + d] = all;
}

// Every pair to its place.  A wavefront takes kTile / kSortWaves consecutive pairs, 64 at a time, and numbers them within
// their digit: by ballot inside the 64, by a counter of its own per digit between them.
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void sort_scatter_kernel(SortArgs a) {
  __shared__ uint32_t place[kSortWaves][kDigitsMax];  // pairs of a digit in a wavefront's part, then where the first one goes
  __shared__ uint32_t scratch[kSortWaves];
  const uint32_t digits = 1u << a.bits, tile = blockIdx.x;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock)
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) place[w][d] = 0;
  __syncthreads();
  uint2 pair[kTileRounds];
  uint32_t rank[kTileRounds], bad = 0;
  const uint64_t first = (uint64_t)tile * kTile + wave_id() * (kTile / kSortWaves) + lane_id();
#pragma unroll
  for (uint32_t u = 0; u < kTileRounds; ++u) {
    const uint64_t i = first + u * kWave;
    if (i < a.n) pair[u] = load_pair<FIRST>(a, (uint32_t)i, &bad);
  }
  if (FIRST && bad && a.status) atomicOr(a.status, CVLC_DEV_INDEX);
#pragma unroll
  for (uint32_t u = 0; u < kTileRounds; ++u) {
    const bool there = first + u * kWave < a.n;
    const uint32_t d = there ? (pair[u].x >> a.shift) & (digits - 1) : 0u;
    uint64_t same = __ballot(there);
    for (uint32_t b = 0; b < a.bits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1u);
      same &= ((d >> b) & 1u) ? set : ~set;
    }
    const uint32_t before = place[wave_id()][d], in = lanes_below(same);
    rank[u] = before + in;
    wave_sync();
    if (there && in == 0) place[wave_id()][d] = before + (uint32_t)__popcll(same);
    wave_sync();
  }
  __syncthreads();
  // digits in turn, kSortBlock at a time: smaller digits, then earlier tiles, then earlier wavefronts
  uint32_t smaller = 0;
  for (uint32_t base = 0; base < digits; base += kSortBlock) {
    const uint32_t d = base + threadIdx.x;
    uint32_t earlier = 0, all = 0;
    if (d < digits) {
      if (a.tiles <= kInlineTiles) {
#pragma unroll 8
        for (uint32_t t = 0; t < a.tiles; ++t) {
          const uint32_t v = a.counts[(uint64_t)t * digits + d];
          earlier += t < tile ? v : 0u;
          all += v;
        }
      } else {
        earlier = a.counts[(uint64_t)tile * digits + d];
        all = a.counts[(uint64_t)a.tiles * digits + d];
      }
    }
    uint32_t total;
    uint32_t at = smaller + block_excl_scan<kSortWaves>(all, scratch, &total) + earlier;
    smaller += total;
    if (d < digits)
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) {
        const uint32_t v = place[w][d];
        place[w][d] = at;
        at += v;
      }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t u = 0; u < kTileRounds; ++u)
    if (first + u * kWave < a.n) a.to[place[wave_id()][(pair[u].x >> a.shift) & (digits - 1)] + rank[u]] = pair[u];
}

// ----------------------------------------------------------------------------- sums
struct SumArgs {
  const uint2* sorted;
  uint32_t n, chunks, vocab, dim, vectors;  // vectors of columns per row
  uint64_t dout_stride, dtable_stride;
  float scale;
  uint32_t add;
  float* dtable;
  float* part;      // [chunks][2][dim]: a token from the chunk before, and one that goes on in the chunk after
  uint8_t* marks;
};

template <uint32_t N>
__device__ __forceinline__ void write_sum(const SumArgs& a, uint32_t token, uint32_t at, float (&s)[N]) {
  float* to = a.dtable + token * a.dtable_stride;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) s[i] *= a.scale;
  if (a.add) {
    float old[N];
    load_row<N>(to, at, a.dim, 0.0f, old);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) s[i] += old[i];
  }
  store_row<N>(to, at, a.dim, s);
}

template <class T>
__global__ __launch_bounds__(kEmbedBlock) void sum_kernel(SumArgs a, const T* dout) {
  constexpr uint32_t N = kPerAccess<T>;
  const uint64_t items = (uint64_t)a.chunks * a.vectors;
  for (uint64_t item = (uint64_t)blockIdx.x * kEmbedBlock + threadIdx.x; item < items; item += (uint64_t)gridDim.x * kEmbedBlock) {
    const uint32_t chunk = (uint32_t)(item / a.vectors), at = (uint32_t)(item % a.vectors) * N;
    const uint32_t from = chunk * kChunk, to = min(from + kChunk, a.n);
    const uint32_t before = from ? a.sorted[from - 1].x : a.vocab, after = to < a.n ? a.sorted[to].x : a.vocab;
    float s[N] = {};
    uint32_t token = a.sorted[from].x;
    bool began = token != before || from == 0;  // the token's first place lies in this chunk
    if (token < a.vocab && began && at == 0) a.marks[token] = 1;
    for (uint32_t j = from; j < to && token < a.vocab; j += kDeep) {
      uint2 pair[kDeep];
      float v[kDeep][N];
#pragma unroll
      for (uint32_t u = 0; u < kDeep; ++u) {
        pair[u] = j + u < to ? a.sorted[j + u] : make_uint2(a.vocab, 0u);
        if (pair[u].x < a.vocab) load_row<N>(dout + pair[u].y * a.dout_stride, at, a.dim, 0.0f, v[u]);
      }
#pragma unroll
      for (uint32_t u = 0; u < kDeep; ++u) {
        if (j + u >= to) break;
        if (pair[u].x != token) {
          if (began) {
            write_sum<N>(a, token, at, s);
          } else {
            store_row<N>(a.part + (uint64_t)chunk * 2 * a.dim, at, a.dim, s);
          }
          token = pair[u].x;
          began = true;
          if (token >= a.vocab) break;
          if (at == 0) a.marks[token] = 1;
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) s[i] = 0.0f;
        }
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) s[i] += v[u][i];
      }
    }
    if (token >= a.vocab) continue;
    if (began && (after != token || to == a.n))
      write_sum<N>(a, token, at, s);
    else
      store_row<N>(a.part + ((uint64_t)chunk * 2 + (began ? 1 : 0)) * a.dim, at, a.dim, s);
  }
}

// Workgroups below `chunks`: the token that begins in this chunk and goes on in the next, if there is one.  The others:
// rows that no token named.
__global__ __launch_bounds__(kEmbedBlock) void finish_kernel(SumArgs a) {
  constexpr uint32_t N = kPerAccess<float>;
  for (uint64_t b = blockIdx.x; b < (uint64_t)a.chunks + (a.add ? 0u : a.vocab); b += gridDim.x) {
    if (b < a.chunks) {
      const uint32_t chunk = (uint32_t)b, from = chunk * kChunk, to = from + kChunk;
      if (to >= a.n) continue;
      const uint32_t token = a.sorted[to - 1].x;
      if (token >= a.vocab || a.sorted[to].x != token) continue;
      if (a.sorted[from].x == token && from && a.sorted[from - 1].x == token) continue;  // began earlier
      for (uint32_t at = threadIdx.x * N; at < a.dim; at += kEmbedBlock * N) {
        float s[N];
        load_row<N>(a.part + ((uint64_t)chunk * 2 + 1) * a.dim, at, a.dim, 0.0f, s);
        for (uint32_t c = chunk + 1; c < a.chunks && a.sorted[c * kChunk].x == token; ++c) {
          float v[N];
          load_row<N>(a.part + (uint64_t)c * 2 * a.dim, at, a.dim, 0.0f, v);
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) s[i] += v[i];
        }
        write_sum<N>(a, token, at, s);
      }
    } else {
      const uint32_t row = (uint32_t)(b - a.chunks);
      if (a.marks[row]) continue;
      const float zero[N] = {};
      for (uint32_t at = threadIdx.x * N; at < a.dim; at += kEmbedBlock * N) store_row<N>(a.dtable + row * a.dtable_stride, at, a.dim, zero);
    }
  }
}

__global__ void clear_kernel(uint32_t* status) { *status = 0; }

size_t align256(size_t v) { return (v + 255u) & ~(size_t)255u; }

// Digits of the sort: tokens 0 .. vocab in as few passes as kDigitBits allow, of like width.
struct Digits {
  uint32_t passes, bits;
};
Digits digits_for(uint32_t vocab) {
  const uint32_t all = 32u - (uint32_t)__builtin_clz(vocab);
  const uint32_t passes = (all + kDigitBits - 1) / kDigitBits;
  return {passes, (all + passes - 1) / passes};
}

struct Layout {
  size_t marks, counts, a, b, part, end;
};
Layout layout_for(uint32_t n, uint32_t vocab, uint32_t dim) {
  const uint64_t tiles = ((uint64_t)n + kTile - 1) / kTile, chunks = ((uint64_t)n + kChunk - 1) / kChunk;
  Layout l;
  l.marks = 256;
  l.counts = l.marks + align256(vocab);
  l.a = l.counts + align256((tiles + 1) * kDigitsMax * sizeof(uint32_t));
  l.b = l.a + align256((size_t)n * sizeof(uint2));
  l.part = l.b + align256((size_t)n * sizeof(uint2));
  l.end = l.part + align256(chunks * 2 * dim * sizeof(float));
  return l;
}

bool sizes_ok(uint32_t n, uint32_t vocab, uint32_t dim) {
  return n <= 0x7FFFFFFFu && vocab >= 1 && vocab <= 0x7FFFFFFFu && dim >= 1 && dim <= 0x7FFFFFFFu;
}

}  // namespace
}  // namespace cvlc

extern "C" {

int cvlc_embed(uint32_t n, const void* d_ids, uint32_t id_bytes, const void* d_table, uint32_t table_type, uint64_t table_stride,
               uint32_t vocab, uint32_t dim, float scale, void* d_out, uint32_t out_type, uint64_t out_stride,
               uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  if (!sizes_ok(n, vocab, dim) || !types_go(table_type, out_type) || table_stride < dim || out_stride < dim) return CVLC_ERR_ARG;
  if ((id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale)) return CVLC_ERR_ARG;
  if (d_status && !buffer_ok(d_status, 4)) return CVLC_ERR_ARG;
  if (n == 0) return CVLC_OK;
  if (!buffer_ok(d_ids, id_bytes) || !buffer_ok(d_table, type_bytes(table_type)) || !buffer_ok(d_out, type_bytes(out_type)))
    return CVLC_ERR_ARG;
  by_types(table_type, out_type, [&](auto tt, auto to) {
    using TT = decltype(tt);
    using TO = decltype(to);
    uint32_t lanes_log = 0;
    while (lanes_log < 8 && (kPerAccess<TT, TO> << lanes_log) < dim) ++lanes_log;
    const uint32_t rows = kEmbedBlock >> lanes_log;
    hipLaunchKernelGGL((embed_kernel<TT, TO>), dim3(std::min((n + rows - 1) / rows, 1u << 20)), dim3(kEmbedBlock), 0,
                       static_cast<hipStream_t>(hip_stream), n, d_ids, id_bytes, static_cast<const TT*>(d_table), table_stride,
                       vocab, dim, scale, static_cast<TO*>(d_out), out_stride, lanes_log, d_status);
  });
  return hip_check(hipGetLastError());
}

size_t cvlc_embed_grad_workspace_bytes(uint32_t n, uint32_t vocab, uint32_t dim) {
  return cvlc::sizes_ok(n, vocab, dim) ? cvlc::layout_for(n, vocab, dim).end : 0;
}

int cvlc_embed_grad(uint32_t n, const void* d_ids, uint32_t id_bytes, const void* d_dout, uint32_t dout_type,
                    uint64_t dout_stride, uint32_t vocab, uint32_t dim, float scale, float* d_dtable, uint64_t dtable_stride,
                    uint32_t flags, void* d_workspace, size_t ws_bytes, void* hip_stream) {
  using namespace cvlc;
  if (!sizes_ok(n, vocab, dim) || !type_known(dout_type) || dout_stride < dim || dtable_stride < dim) return CVLC_ERR_ARG;
  if ((id_bytes != 4 && id_bytes != 8) || !std::isfinite(scale) || (flags & ~CVLC_GRAD_ACCUMULATE)) return CVLC_ERR_ARG;
  if (!buffer_ok(d_dtable, 4) || !buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  if (n && (!buffer_ok(d_ids, id_bytes) || !buffer_ok(d_dout, type_bytes(dout_type)))) return CVLC_ERR_ARG;
  const Layout l = layout_for(n, vocab, dim);
  if (ws_bytes < l.end) return CVLC_ERR_CAPACITY;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(d_workspace);
  uint32_t* status = reinterpret_cast<uint32_t*>(ws);
  uint32_t* marks = reinterpret_cast<uint32_t*>(ws + l.marks);
  uint32_t* counts = reinterpret_cast<uint32_t*>(ws + l.counts);
  uint2* from = reinterpret_cast<uint2*>(ws + l.a);
  uint2* to = reinterpret_cast<uint2*>(ws + l.b);
  const uint32_t tiles = (uint32_t)(((uint64_t)n + kTile - 1) / kTile);
  const Digits dg = digits_for(vocab);
  hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(1), 0, stream, status);
  for (uint32_t pass = 0; pass < dg.passes; ++pass) {
    const SortArgs a{d_ids, id_bytes, vocab, from, to, n, tiles, pass * dg.bits, dg.bits, counts, status};
    const dim3 grid(std::max(tiles, 1u)), block(kSortBlock);
    const uint32_t mark_words = (uint32_t)(align256(vocab) / 4);
    if (pass == 0)
      hipLaunchKernelGGL(sort_hist_kernel<true>, grid, block, 0, stream, a, marks, mark_words);
    else if (n)
      hipLaunchKernelGGL(sort_hist_kernel<false>, grid, block, 0, stream, a, marks, mark_words);
    if (tiles > kInlineTiles)
      hipLaunchKernelGGL(sort_scan_kernel, dim3(((1u << dg.bits) + kWave - 1) / kWave), dim3(kScanWaves * kWave), 0, stream, counts,
                         tiles, 1u << dg.bits);
    if (n) {
      if (pass == 0)
        hipLaunchKernelGGL(sort_scatter_kernel<true>, grid, block, 0, stream, a);
      else
        hipLaunchKernelGGL(sort_scatter_kernel<false>, grid, block, 0, stream, a);
    }
    std::swap(from, to);
  }
  const uint32_t chunks = (uint32_t)(((uint64_t)n + kChunk - 1) / kChunk);
  by_type(dout_type, [&](auto t) {
    using T = decltype(t);
    const uint32_t vectors = (dim + kPerAccess<T> - 1) / kPerAccess<T>;
    const SumArgs a{from, n, chunks, vocab, dim, vectors, dout_stride, dtable_stride, scale, flags & CVLC_GRAD_ACCUMULATE,
                    d_dtable, reinterpret_cast<float*>(ws + l.part), reinterpret_cast<uint8_t*>(marks)};
    const uint64_t blocks = ((uint64_t)chunks * vectors + kEmbedBlock - 1) / kEmbedBlock;
    if (n)
      hipLaunchKernelGGL(sum_kernel<T>, dim3((uint32_t)std::min<uint64_t>(blocks, 1u << 20)), dim3(kEmbedBlock), 0, stream, a,
                         static_cast<const T*>(d_dout));
    hipLaunchKernelGGL(finish_kernel, dim3((uint32_t)std::min<uint64_t>((uint64_t)chunks + vocab, 1u << 20)), dim3(kEmbedBlock), 0,
                       stream, a);
  });
  return hip_check(hipGetLastError());
}

}  // extern "C"
