// cvlc_embed.hip -- embedding lookup and its gradient by sorted tokens.
//
// Gradient: dtable[v] = scale * sum of the dout rows whose token is v.  Texts'
// tokens are far from even (the commonest is a twentieth of all), so no token is
// one thread's, and every order of summation is fixed by places alone.  Few
// tokens: a row of the table is one workgroup's per block of columns, so a token
// that most places hold is what the call waits for.  Many: work is cut by places.
//
// Few tokens, in one launch:
//   direct       a workgroup owns every slices-th row of the table and a block of
//                columns, looks all tokens over, lists the places of its own in
//                LDS, by row and in order, and adds them up.
// Many:
//   sort_hist, sort_scatter   stable radix sort of (token, place) pairs, up to 11
//                bits a pass, least significant digit first; a tile of 4096 pairs
//                per workgroup.  Tokens that are left out (negative or beyond the
//                vocabulary) sort behind all others, as token `vocab`.  The first
//                pass marks the tokens that came; workgroups beyond the tiles'
//                write zeros to the rows of the others meanwhile.
//   sum          a chunk of kChunk consecutive sorted places and one vector of
//                columns per thread: adds rows up while the token stays, writes
//                the sum when it changes.  A token that reaches into other chunks
//                has one partial sum in each.
//   join         adds up the partial sums of such tokens, in order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

constexpr uint32_t kEmbedBlock = 256;
// Workgroups of one row per thread from which a thread takes four, past the caches' order.  Rows of 2048 bf16, one and four:
// 4096 of them 6.8 and 6.9 us, 8192 10.7 and 10.1, 16384 25.4 and 17.0; with a layer norm of the output behind them, which then finds
// less of it in the caches, 8192 26.9 and 27.9, 16384 50.7 and 49.1, 32768 83.1 and 78.5.
constexpr uint32_t kManyBlocks = 8192;
constexpr uint32_t kSortBlock = 256, kSortWaves = kSortBlock / kWave;
constexpr uint32_t kTile = 4096;                           // pairs a workgroup sorts per pass
constexpr uint32_t kTileRounds = kTile / kSortBlock;       // of 64 consecutive pairs per wavefront
constexpr uint32_t kDigitBits = 11, kDigitsMax = 1u << kDigitBits;
constexpr uint32_t kInlineTiles = 64;                      // tiles whose counts every workgroup adds up for itself
constexpr uint32_t kChunk = 32;                            // sorted places that a thread adds up
constexpr uint32_t kDeep = 8;                              // rows in flight per thread

__device__ __forceinline__ int64_t load_token(const void* ids, uint32_t id_bytes, uint64_t i) {
  return id_bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}

// ----------------------------------------------------------------------------- lookup
// `lanes` threads (a power of two) to a row, U rows under way per thread.  Many rows are written past the caches' order, which
// then hold the frequent tokens' rows of the table (65536 x 2048 bf16: 59 us; four rows in the caches' order 79, one 97).
template <class TT, class TO, uint32_t U>
__global__ __launch_bounds__(kEmbedBlock) void embed_kernel(uint32_t n, const void* ids, uint32_t id_bytes, const TT* table,
                                                            uint64_t table_stride, uint32_t vocab, uint32_t dim, float scale,
                                                            TO* out, uint64_t out_stride, uint32_t lanes_log, uint32_t* status) {
  constexpr uint32_t N = kPerAccess<TT, TO>;
  const uint32_t lanes = 1u << lanes_log, lane = threadIdx.x & (lanes - 1), rows = kEmbedBlock >> lanes_log;
  for (uint64_t first = (uint64_t)blockIdx.x * rows * U + (threadIdx.x >> lanes_log); first < n; first += (uint64_t)gridDim.x * rows * U) {
    int64_t id[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) id[u] = first + u * rows < n ? load_token(ids, id_bytes, first + u * rows) : -1;
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (id[u] >= (int64_t)vocab) {
        if (status && lane == 0) atomicOr(status, CVLC_DEV_INDEX);
        id[u] = -1;
      }
    for (uint32_t at = lane * N; at < dim; at += lanes * N) {
      Raw<TT, N> raw[U];
#pragma unroll
      for (uint32_t u = 0; u < U; ++u)
        if (id[u] >= 0) load_raw(raw[u], table + (uint64_t)id[u] * table_stride, at, dim);
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        if (first + u * rows >= n) break;
        float v[N];
        raw[u].values(v);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) v[i] = id[u] >= 0 ? v[i] * scale : 0.0f;
        store_row<N, (U > 1)>(out + (first + u * rows) * out_stride, at, dim, v);
      }
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
  // rows [zero_from, zero_to) of the table that are not marked become zeros, by the workgroups beyond the tiles'
  uint8_t* marks;
  float* dtable;
  uint64_t dtable_stride;
  uint32_t dim, lanes_log, zero_from, zero_to;
};

__device__ __forceinline__ void write_zeros(const SortArgs& a) {
  constexpr uint32_t N = kPerAccess<float>;
  const float zero[N] = {};
  const uint32_t lanes = 1u << a.lanes_log, lane = threadIdx.x & (lanes - 1), rows = kSortBlock >> a.lanes_log;
  const uint64_t step = (uint64_t)(gridDim.x - a.tiles) * rows;
  for (uint64_t first = a.zero_from + (uint64_t)(blockIdx.x - a.tiles) * rows + (threadIdx.x >> a.lanes_log); first < a.zero_to;
       first += kDeep * step) {
    uint8_t mark[kDeep];
#pragma unroll
    for (uint32_t u = 0; u < kDeep; ++u) mark[u] = first + u * step < a.zero_to ? a.marks[first + u * step] : 1;
#pragma unroll
    for (uint32_t u = 0; u < kDeep; ++u)
      if (!mark[u])
        for (uint32_t at = lane * N; at < a.dim; at += lanes * N) store_row<N, true>(a.dtable + (first + u * step) * a.dtable_stride, at, a.dim, zero);
  }
}

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

// Counts per digit of every tile; the first pass also marks the tokens.
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void sort_hist_kernel(SortArgs a) {
  __shared__ uint32_t hist[kDigitsMax];
  if (!FIRST && blockIdx.x >= a.tiles) return write_zeros(a);
  const uint32_t digits = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock) hist[d] = 0;
  __syncthreads();
  uint32_t bad = 0;
#pragma unroll
  for (uint32_t u = 0; u < kTileRounds; ++u) {
    const uint64_t i = (uint64_t)blockIdx.x * kTile + u * kSortBlock + threadIdx.x;
    if (i < a.n) {
      const uint32_t token = load_pair<FIRST>(a, (uint32_t)i, &bad).x;
      if (FIRST && a.marks && token < a.vocab) a.marks[token] = 1;
      atomicAdd(&hist[(token >> a.shift) & (digits - 1)], 1u);
    }
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
  if (blockIdx.x >= a.tiles) return write_zeros(a);
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
// Where the gradient goes.
struct TableArgs {
  float* dtable;
  uint64_t stride;
  uint32_t vocab, dim;
  float scale;
  uint32_t add;
};

template <uint32_t N, bool ONCE = false>
__device__ __forceinline__ void write_sum(const TableArgs& a, uint32_t token, uint32_t at, float (&s)[N]) {
  float* to = a.dtable + token * a.stride;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) s[i] *= a.scale;
  if (a.add) {
    float old[N];
    load_row<N>(to, at, a.dim, 0.0f, old);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) s[i] += old[i];
  }
  store_row<N, ONCE>(to, at, a.dim, s);
}

struct SumArgs {
  TableArgs table;
  const uint2* sorted;
  uint32_t n, chunks, vectors;  // vectors of columns per row
  uint64_t dout_stride;
  float* part;  // [chunks][2][dim]: a token from the chunk before, and one that goes on in the chunk after
};

// Bound by memory: 131072 tokens, as many rows of 2048 bf16, 186 us for 0.82 GB, 4.4 TB/s; with chunks of 64 and accesses in the
// caches' order 246, and 40000 tokens of 1000 fp32 346 us in all, now 295.
template <class T, bool ONCE>
__global__ __launch_bounds__(kEmbedBlock) void sum_kernel(SumArgs a, const T* dout) {
  constexpr uint32_t N = kPerAccess<T>;
  const uint64_t items = (uint64_t)a.chunks * a.vectors;
  for (uint64_t item = (uint64_t)blockIdx.x * kEmbedBlock + threadIdx.x; item < items; item += (uint64_t)gridDim.x * kEmbedBlock) {
    const uint32_t chunk = (uint32_t)(item / a.vectors), at = (uint32_t)(item % a.vectors) * N;
    const uint32_t from = chunk * kChunk, to = min(from + kChunk, a.n);
    const uint32_t before = from ? a.sorted[from - 1].x : a.table.vocab, after = to < a.n ? a.sorted[to].x : a.table.vocab;
    float s[N] = {};
    uint32_t token = a.sorted[from].x;
    bool began = token != before || from == 0;  // the token's first place lies in this chunk
    for (uint32_t j = from; j < to && token < a.table.vocab; j += kDeep) {
      uint2 pair[kDeep];
      Raw<T, N> raw[kDeep];
#pragma unroll
      for (uint32_t u = 0; u < kDeep; ++u) {
        pair[u] = j + u < to ? a.sorted[j + u] : make_uint2(a.table.vocab, 0u);
        if (pair[u].x < a.table.vocab) load_raw<ONCE>(raw[u], dout + pair[u].y * a.dout_stride, at, a.table.dim);
      }
#pragma unroll
      for (uint32_t u = 0; u < kDeep; ++u) {
        if (j + u >= to) break;
        if (pair[u].x != token) {
          if (began) {
            write_sum<N, true>(a.table, token, at, s);
          } else {
            store_row<N>(a.part + (uint64_t)chunk * 2 * a.table.dim, at, a.table.dim, s);
          }
          token = pair[u].x;
          began = true;
          if (token >= a.table.vocab) break;
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) s[i] = 0.0f;
        }
        float v[N];
        raw[u].values(v);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) s[i] += v[i];
      }
    }
    if (token >= a.table.vocab) continue;
    if (began && (after != token || to == a.n))
      write_sum<N, true>(a.table, token, at, s);
    else
      store_row<N>(a.part + ((uint64_t)chunk * 2 + (began ? 1 : 0)) * a.table.dim, at, a.table.dim, s);
  }
}

// The token that goes on from a chunk, where it began, to the next: its partial sums.  A workgroup per chunk and 64 vectors
// of columns; each wavefront adds up a part of the chain.
constexpr uint32_t kJoinWaves = kEmbedBlock / kWave;
__global__ __launch_bounds__(kEmbedBlock) void join_kernel(SumArgs a) {
  constexpr uint32_t N = kPerAccess<float>;
  __shared__ float sums[kJoinWaves][N][kWave];
  const uint32_t dim = a.table.dim;
  for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const uint32_t from = chunk * kChunk, to = from + kChunk;
    if (to >= a.n) return;
    const uint32_t token = a.sorted[to - 1].x;
    if (token >= a.table.vocab || a.sorted[to].x != token) continue;
    if (a.sorted[from].x == token && from && a.sorted[from - 1].x == token) continue;  // began earlier
    uint32_t more = 0;  // chunks it goes on in
    for (uint32_t base = chunk + 1; base < a.chunks; base += kWave) {
      const uint32_t c = base + lane_id();
      const uint64_t stays = __ballot(c < a.chunks && a.sorted[(uint64_t)min(c, a.chunks - 1) * kChunk].x == token);
      more += (uint32_t)__popcll(stays);
      if (stays != ~0ull) break;
    }
    const uint32_t first = (uint32_t)((uint64_t)more * wave_id() / kJoinWaves), last = (uint32_t)((uint64_t)more * (wave_id() + 1) / kJoinWaves);
    for (uint32_t base = blockIdx.y * kWave * N; base < dim; base += gridDim.y * kWave * N) {
      const uint32_t at = base + lane_id() * N;
      float s[N] = {};
      if (wave_id() == 0) load_row<N>(a.part + ((uint64_t)chunk * 2 + 1) * dim, at, dim, 0.0f, s);
      for (uint32_t c = first; c < last; c += kDeep) {
        Raw<float, N> raw[kDeep];
#pragma unroll
        for (uint32_t u = 0; u < kDeep; ++u)
          if (c + u < last) load_raw(raw[u], a.part + (uint64_t)(chunk + 1 + c + u) * 2 * dim, at, dim);
#pragma unroll
        for (uint32_t u = 0; u < kDeep; ++u) {
          if (c + u >= last) break;
          float v[N];
          raw[u].values(v);
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) s[i] += v[i];
        }
      }
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sums[wave_id()][i][lane_id()] = s[i];
      __syncthreads();
      if (wave_id() == 0) {
#pragma unroll
        for (uint32_t w = 1; w < kJoinWaves; ++w)
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) s[i] += sums[w][i][lane_id()];
        if (at < dim) write_sum<N>(a.table, token, at, s);
      }
      __syncthreads();
    }
  }
}

__global__ __launch_bounds__(kEmbedBlock) void clear_kernel(uint32_t* status, uint32_t* marks, uint32_t mark_words) {
  const uint32_t i = blockIdx.x * kEmbedBlock + threadIdx.x;
  if (i == 0) *status = 0;
  for (uint64_t w = i; w < mark_words; w += (uint64_t)gridDim.x * kEmbedBlock) marks[w] = 0;
}

// ----------------------------------------------------------------------------- few tokens
constexpr uint32_t kDirectBlock = 1024, kDirectWaves = kDirectBlock / kWave;
constexpr uint32_t kDirectTokens = 16384;  // places are kept in 16 bits of LDS each
constexpr uint32_t kSliceRows = 256;       // rows of the table that a workgroup owns, at most
constexpr uint32_t kScanDeep = 8;          // tokens under way per thread
constexpr uint32_t kSumDeep = 8;           // rows under way per thread
constexpr uint32_t kRowsDeep = 4;          // rows of the table under way per thread
constexpr uint32_t kFrequent = 16;         // a row of more places than this is added up by the whole workgroup

struct DirectArgs {
  TableArgs table;
  const void* ids;
  uint32_t id_bytes, n;
  uint64_t dout_stride;
  uint32_t slices_log, lanes_log;  // lanes: threads to a row's columns
  uint32_t* status;
};

// f(place, row) for the tokens of a wavefront's part that this slice owns, 64 consecutive places at a time, all lanes
// together; row = kSliceRows where a lane's token is another's.
template <class F>
__device__ __forceinline__ void over_tokens(const DirectArgs& a, uint32_t slice, uint32_t* bad, F f) {
  const uint32_t each = (a.n + kDirectBlock - 1) / kDirectBlock * kWave;
  const uint32_t from = min(wave_id() * each, a.n), to = min(from + each, a.n);
  for (uint32_t base = from; base < to; base += kScanDeep * kWave) {
    int64_t id[kScanDeep];
#pragma unroll
    for (uint32_t u = 0; u < kScanDeep; ++u) {
      const uint32_t i = base + u * kWave + lane_id();
      id[u] = i < to ? load_token(a.ids, a.id_bytes, i) : -1;
    }
#pragma unroll
    for (uint32_t u = 0; u < kScanDeep; ++u) {
      const bool there = id[u] >= 0 && id[u] < (int64_t)a.table.vocab;
      if (id[u] >= (int64_t)a.table.vocab) *bad = 1;
      const bool own = there && ((uint32_t)id[u] & ((1u << a.slices_log) - 1)) == slice;
      f(base + u * kWave + lane_id(), own ? (uint32_t)id[u] >> a.slices_log : kSliceRows);
    }
  }
}

// Sum of dout over places order[from .. to), from column `at` on.
template <uint32_t N, class T>
__device__ __forceinline__ void sum_places(const T* dout, uint64_t stride, uint32_t dim, const uint16_t* order, uint32_t from,
                                           uint32_t to, uint32_t at, float (&s)[N]) {
  for (uint32_t j = from; j < to; j += kSumDeep) {
    Raw<T, N> raw[kSumDeep];
#pragma unroll
    for (uint32_t u = 0; u < kSumDeep; ++u)
      if (j + u < to) load_raw(raw[u], dout + order[j + u] * stride, at, dim);
#pragma unroll
    for (uint32_t u = 0; u < kSumDeep; ++u) {
      if (j + u >= to) break;
      float v[N];
      raw[u].values(v);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) s[i] += v[i];
    }
  }
}

template <class T>
__global__ __launch_bounds__(kDirectBlock) void direct_kernel(DirectArgs a, const T* dout) {
  constexpr uint32_t N = kPerAccess<T>;
  extern __shared__ float dynamic[];  // a vector per thread, then the places
  float* sums = dynamic;
  uint16_t* order = reinterpret_cast<uint16_t*>(dynamic + kDirectBlock * N);
  __shared__ uint32_t place[kDirectWaves][kSliceRows];  // tokens of a row in a wavefront's part, then where the next one goes
  __shared__ uint32_t start[kSliceRows + 1], scratch[kDirectWaves], frequent;
  __shared__ uint16_t frequents[kSliceRows];
  __shared__ uint32_t any_bad;
  const uint32_t slice = blockIdx.x, rows = ((a.table.vocab - 1 - slice) >> a.slices_log) + 1;
  for (uint32_t d = threadIdx.x; d < kDirectWaves * kSliceRows; d += kDirectBlock) (&place[0][0])[d] = 0;
  if (threadIdx.x == 0) frequent = any_bad = 0;
  __syncthreads();
  uint32_t bad = 0;
  over_tokens(a, slice, &bad, [&](uint32_t, uint32_t row) {
    if (row < kSliceRows) atomicAdd(&place[wave_id()][row], 1u);
  });
  if (bad) any_bad = 1;
  __syncthreads();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status = any_bad ? CVLC_DEV_INDEX : 0u;
  {
    const uint32_t d = threadIdx.x;
    uint32_t all = 0, total;
    if (d < kSliceRows)
#pragma unroll
      for (uint32_t w = 0; w < kDirectWaves; ++w) all += place[w][d];
    uint32_t at = block_excl_scan<kDirectWaves>(all, scratch, &total);
    if (d <= kSliceRows) start[d] = at;
    if (d < kSliceRows) {
#pragma unroll
      for (uint32_t w = 0; w < kDirectWaves; ++w) {
        const uint32_t v = place[w][d];
        place[w][d] = at;
        at += v;
      }
      if (all > kFrequent) frequents[atomicAdd(&frequent, 1u)] = (uint16_t)d;
    }
  }
  __syncthreads();
  over_tokens(a, slice, &bad, [&](uint32_t i, uint32_t row) {
    for (uint64_t left = __ballot(row < kSliceRows); left;) {
      const uint32_t r = __builtin_amdgcn_readlane(row, __builtin_ctzll(left));
      const uint64_t same = __ballot(row == r);
      const uint32_t in = lanes_below(same), at = place[wave_id()][r];
      wave_sync();
      if (row == r) {
        order[at + in] = (uint16_t)i;
        if (in == 0) place[wave_id()][r] = at + (uint32_t)__popcll(same);
      }
      wave_sync();
      left &= ~same;
    }
  });
  __syncthreads();
  const uint32_t lanes = 1u << a.lanes_log, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log;
  const uint32_t groups = kDirectBlock >> a.lanes_log, at = (blockIdx.y * kWave + lane) * N, dim = a.table.dim;
  const uint32_t many = frequent;
  for (uint32_t f = 0; f < many; ++f) {
    const uint32_t row = frequents[f], from = start[row], count = start[row + 1] - from;
    float s[N] = {};
    if (at < dim) sum_places<N>(dout, a.dout_stride, dim, order, from + count * group / groups, from + count * (group + 1) / groups, at, s);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) sums[i * kDirectBlock + threadIdx.x] = s[i];
    __syncthreads();
    if (group == 0) {
      for (uint32_t g = 1; g < groups; ++g)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) s[i] += sums[i * kDirectBlock + g * lanes + lane];
      if (at < dim) write_sum<N>(a.table, (row << a.slices_log) + slice, at, s);
    }
    __syncthreads();
  }
  if (at >= dim) return;
  for (uint32_t first = group; first < rows; first += kRowsDeep * groups) {
    uint32_t from[kRowsDeep], to[kRowsDeep];
    Raw<T, N> raw[kRowsDeep];
#pragma unroll
    for (uint32_t u = 0; u < kRowsDeep; ++u) {
      const uint32_t row = min(first + u * groups, kSliceRows);
      from[u] = start[row];
      to[u] = start[min(row + 1, kSliceRows)];
      if (to[u] - from[u] - 1 < kFrequent) load_raw(raw[u], dout + order[from[u]] * a.dout_stride, at, dim);
    }
#pragma unroll
    for (uint32_t u = 0; u < kRowsDeep; ++u) {
      const uint32_t row = first + u * groups, count = to[u] - from[u];
      if (row >= rows) break;
      if (count > kFrequent || (a.table.add && count == 0)) continue;
      float s[N] = {};
      if (count) raw[u].values(s);
      if (count > 1) sum_places<N>(dout, a.dout_stride, dim, order, from[u] + 1, to[u], at, s);
      write_sum<N>(a.table, (row << a.slices_log) + slice, at, s);
    }
  }
}

// Slices (a power of two) that the table is cut into, if that is the way for so many tokens.  Every workgroup reads all the
// tokens, twice, so there is one, as large as they go, to a CU (12000 tokens, 2000 rows of 200 bf16: 16.6 us; two of 512
// threads each 20.7), except for a table of more rows than it keeps counts of.  Against the sort and its sums, with inputs
// that are not in the caches: 640 tokens of 96 fp32 6.7 us (35 sorted), 4096 of 768 bf16 into 32000 rows 40 (70), 12288 63 (72),
// 16384 70 (73), 24576 85 (76); 16384 of 512 fp32 58 (68), 24576 74 (71); 16384 of 512 bf16 into 8000 rows 29 (65), 24576 40
// (67); 1000 of 8192 bf16 into a table of 1 GB 217 (228).  The worst texts are those of one token: where it holds half of
// 16384 places and all of them, 256 bf16 65 (75) and 113 (77), 768 bf16 194 (81) and 322 (86); 4096 places of 2048 109 (88) and
// 140 (86).  More places than 16384 are sorted, also where the table is small, so that it stays at that.
constexpr uint32_t kDirectBlocks = 256;
constexpr uint64_t kDirectReads = 1u << 25;  // tokens read by all workgroups
bool direct_slices(uint32_t n, uint32_t vocab, uint32_t column_blocks, uint32_t* slices_log) {
  if (n > kDirectTokens) return false;
  uint32_t log = 0;
  while (log < 31 && (2ull << log) <= vocab && ((2ull << log) * column_blocks <= kDirectBlocks || ((uint64_t)kSliceRows << log) < vocab)) ++log;
  *slices_log = log;
  // (a launch of 2^32 threads and more would start only the rest of that division)
  return log <= 21 && ((uint64_t)kSliceRows << log) >= vocab && (1ull << log) * column_blocks * n <= kDirectReads;
}

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
    const auto go = [&](auto kernel, uint32_t each) {
      hipLaunchKernelGGL(kernel, dim3(std::min((n + rows * each - 1) / (rows * each), 1u << 20)), dim3(kEmbedBlock), 0,
                         static_cast<hipStream_t>(hip_stream), n, d_ids, id_bytes, static_cast<const TT*>(d_table), table_stride,
                         vocab, dim, scale, static_cast<TO*>(d_out), out_stride, lanes_log, d_status);
    };
    if ((n + rows - 1) / rows >= kManyBlocks)
      go(embed_kernel<TT, TO, 4>, 4);
    else
      go(embed_kernel<TT, TO, 1>, 1);
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
  const TableArgs table{d_dtable, dtable_stride, vocab, dim, scale, flags & CVLC_GRAD_ACCUMULATE};
  const uint32_t per = by_type(dout_type, [](auto t) { return kPerAccess<decltype(t)>; }), vectors = dim / per + (dim % per != 0);
  const uint32_t column_blocks = (vectors + kWave - 1) / kWave;
  uint32_t slices_log;
  if (column_blocks <= 65535 && direct_slices(n, vocab, column_blocks, &slices_log)) {
    uint32_t lanes_log = 3;  // at most kDirectBlock / 8 sums to join
    while (lanes_log < 6 && (1u << lanes_log) < vectors) ++lanes_log;
    by_type(dout_type, [&](auto t) {
      using T = decltype(t);
      const DirectArgs a{table, d_ids, id_bytes, n, dout_stride, slices_log, lanes_log, status};
      hipLaunchKernelGGL(direct_kernel<T>, dim3(1u << slices_log, column_blocks), dim3(kDirectBlock),
                         kDirectBlock * kPerAccess<T> * sizeof(float) + n * sizeof(uint16_t), stream, a, static_cast<const T*>(d_dout));
    });
    return hip_check(hipGetLastError());
  }
  const uint32_t tiles = (uint32_t)(((uint64_t)n + kTile - 1) / kTile);
  const Digits dg = digits_for(vocab);
  const uint32_t mark_words = table.add ? 0u : (uint32_t)(align256(vocab) / 4);
  hipLaunchKernelGGL(clear_kernel, dim3(std::min(mark_words / kEmbedBlock + 1, 1024u)), dim3(kEmbedBlock), 0, stream, status, marks,
                     mark_words);
  uint32_t lanes_log = 0;
  while (lanes_log < 8 && (kPerAccess<float> << lanes_log) < dim) ++lanes_log;
  uint32_t zeroed = 0, turn = 0;
  SortArgs a{d_ids, id_bytes, vocab, from, to, n, tiles, 0, dg.bits, counts, status, table.add ? nullptr : reinterpret_cast<uint8_t*>(marks),
             d_dtable, dtable_stride, dim, lanes_log, 0, 0};
  // The rows that no token named are dealt out evenly to the launches behind the first count.
  auto grid_with_zeros = [&] {
    ++turn;
    a.zero_from = zeroed;
    a.zero_to = zeroed = table.add ? 0u : (uint32_t)((uint64_t)vocab * turn / (2 * dg.passes - 1));
    const uint32_t rows = kSortBlock >> lanes_log;
    return dim3(tiles + std::min((a.zero_to - a.zero_from + rows - 1) / rows, 2048u));
  };
  const auto go = [&](auto kernel, dim3 grid) {
    if (grid.x) hipLaunchKernelGGL(kernel, grid, dim3(kSortBlock), 0, stream, a);
  };
  for (uint32_t pass = 0; pass < dg.passes; ++pass) {
    a.shift = pass * dg.bits;
    a.from = from;
    a.to = to;
    if (pass == 0)
      go(sort_hist_kernel<true>, dim3(tiles));
    else
      go(sort_hist_kernel<false>, grid_with_zeros());
    if (tiles > kInlineTiles)
      hipLaunchKernelGGL(sort_scan_kernel, dim3(((1u << dg.bits) + kWave - 1) / kWave), dim3(kScanWaves * kWave), 0, stream, counts,
                         tiles, 1u << dg.bits);
    if (pass == 0)
      go(sort_scatter_kernel<true>, grid_with_zeros());
    else
      go(sort_scatter_kernel<false>, grid_with_zeros());
    std::swap(from, to);
  }
  if (n == 0) return hip_check(hipGetLastError());
  const uint32_t chunks = (uint32_t)(((uint64_t)n + kChunk - 1) / kChunk);
  const SumArgs sa{table, from, n, chunks, vectors, dout_stride, reinterpret_cast<float*>(ws + l.part)};
  by_type(dout_type, [&](auto t) {
    using T = decltype(t);
    const uint64_t blocks = ((uint64_t)chunks * vectors + kEmbedBlock - 1) / kEmbedBlock;
    // rows of dout that the last-level cache (256 MB) does not hold anyway are read past the caches' order
    const bool once = (uint64_t)n * dim * sizeof(T) > 256ull * 1000000;
    hipLaunchKernelGGL((once ? sum_kernel<T, true> : sum_kernel<T, false>), dim3((uint32_t)std::min<uint64_t>(blocks, 1u << 20)),
                       dim3(kEmbedBlock), 0, stream, sa, static_cast<const T*>(d_dout));
  });
  const uint32_t join_columns = kWave * kPerAccess<float>;
  hipLaunchKernelGGL(join_kernel, dim3(std::min(chunks, 1u << 20), std::min(dim / join_columns + (dim % join_columns != 0), 65535u)), dim3(kEmbedBlock), 0,
                     stream, sa);
  return hip_check(hipGetLastError());
}

}  // extern "C"
