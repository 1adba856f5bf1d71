// cvlc_xent.hip -- softmax cross entropy of logits z = s h T^t over a large vocabulary, without the logits in memory.
//
// loss_i = w_i (ln sum_v exp z_iv - z_i,label),  G_iv = s w_i (softmax(z_i)_v - [v = label_i]),  dh = G T,  dT = G^t h.
//
// Products of matrices do nearly all the work: z once for the loss, once more for the gradients (a row's softmax needs its
// whole sum first, and keeping z is what this call is there to avoid), then dh and dT.  All run on the matrix units from
// 16-bit operands with K contiguous, sums in fp32:
//   - bfloat16 and fp16 matrices as they are;
//   - fp32 as three planes of bfloat16 (8 + 8 + 8 bits are its 24), of whose nine products the six largest are added: what is left
//     out is below 2^-24 of a term.  An fp32 matrix instruction has a sixteenth of the rate.
//   - G, in one plane where the result is of 16 bits (its rounding of 2^-9 or 2^-12 of a term is what the result's own is), in
//     two where an fp32 gradient of the table is asked of 16-bit matrices (2^-18), in three beside fp32 matrices.
// G is scaled by a power of two that brings the largest weight to about 2^13, so that neither tiny weights nor fp16 lose its
// small entries.
//
// The loss's product ends in every tile's (max, sum of exponentials) per row, joined in order by a second launch.  The
// gradients go over the vocabulary in pieces of a few thousand tokens whose G fits the last-level cache.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cvlc_elem.h"

namespace cvlc {
namespace {

typedef float Four __attribute__((ext_vector_type(4)));
typedef __bf16 EightB __attribute__((ext_vector_type(8)));
typedef _Float16 EightH __attribute__((ext_vector_type(8)));
typedef uint16_t Half;  // 16 bits of either type

constexpr uint32_t kDepth = 64;    // K of a tile: 128 bytes of a row
constexpr uint32_t kPadTo = 256;   // vocabulary pieces are whole tiles
constexpr float kLift = 0x1p13f;   // G's largest entries

uint64_t pad_to(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// ------------------------------------------------------------------------------ planes
// x as a sum of P values of a 16-bit type.  Three of bfloat16 cut bits off, which leaves the rest exact; one or two round.
template <class H, uint32_t P>
__device__ __forceinline__ void split(float x, Half (&out)[P]) {
#pragma unroll
  for (uint32_t p = 0; p < P; ++p) {
    const H h = P == 3 ? __builtin_bit_cast(H, (Half)(__float_as_uint(x) >> 16)) : (H)x;
    out[p] = __builtin_bit_cast(Half, h);
    x -= (float)h;
  }
}

// Which rows count: labels that are there, with a weight.
struct Rows {
  const void* labels;
  uint32_t id_bytes, vocab, n;
  const float* weights;
  __device__ __forceinline__ int64_t label(uint32_t i) const {
    return id_bytes == 8 ? static_cast<const int64_t*>(labels)[i] : (int64_t)static_cast<const int32_t*>(labels)[i];
  }
  __device__ __forceinline__ float weight(uint32_t i) const { return weights ? weights[i] : 1.0f; }
  __device__ __forceinline__ bool live(uint32_t i) const {
    const int64_t l = label(i);
    return l >= 0 && l < (int64_t)vocab && weight(i) != 0.0f;
  }
};

// A matrix's planes, its rows as they are and turned; zeros beyond it up to whole tiles of K.
constexpr uint32_t kPackSide = 64, kPackBlock = 256;
struct PackArgs {
  uint32_t rows, cols;
  uint64_t stride;
  Half *straight, *turned;          // either may be null
  uint64_t straight_stride, straight_plane, turned_stride, turned_plane;
  uint32_t masked;                  // rows that do not count become zeros
  Rows who;
};

template <class T, class H, uint32_t P>
__global__ __launch_bounds__(kPackBlock) void pack_kernel(PackArgs a, const T* src) {
  __shared__ Half tile[P][kPackSide][kPackSide + 2];   // [column][row]
  const uint32_t blocks = (a.cols + kPackSide - 1) / kPackSide;
  const uint32_t r0 = blockIdx.x / blocks * kPackSide, c0 = blockIdx.x % blocks * kPackSide;
  for (uint32_t k = threadIdx.x; k < kPackSide * kPackSide / 8; k += kPackBlock) {
    const uint32_t r = k / 8, c = k % 8 * 8, row = r0 + r;
    float x[8] = {};
    if (row < a.rows && !(a.masked && !a.who.live(row))) load_row<8>(src + row * a.stride, c0 + c, a.cols, 0.0f, x);
    Half h[P][8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      Half part[P];
      split<H, P>(x[i], part);
#pragma unroll
      for (uint32_t p = 0; p < P; ++p) {
        h[p][i] = part[p];
        tile[p][c + i][r] = part[p];
      }
    }
    if (a.straight && row < a.rows)
#pragma unroll
      for (uint32_t p = 0; p < P; ++p)
        *reinterpret_cast<Quad*>(a.straight + p * a.straight_plane + row * a.straight_stride + c0 + c) =
            Quad{h[p][0] | (uint32_t)h[p][1] << 16, h[p][2] | (uint32_t)h[p][3] << 16, h[p][4] | (uint32_t)h[p][5] << 16,
                 h[p][6] | (uint32_t)h[p][7] << 16};
  }
  if (!a.turned) return;
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < kPackSide * kPackSide / 8; k += kPackBlock) {
    const uint32_t c = k / 8, r = k % 8 * 8;
    if (c0 + c >= a.cols) continue;
#pragma unroll
    for (uint32_t p = 0; p < P; ++p) {
      Quad q;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) q[i] = tile[p][c][r + 2 * i] | (uint32_t)tile[p][c][r + 2 * i + 1] << 16;
      *reinterpret_cast<Quad*>(a.turned + p * a.turned_plane + (c0 + c) * a.turned_stride + r0 + r) = q;
    }
  }
}

// factors[0]: by which G is scaled, factors[1]: by which its products are; labels that are not there are told of.
__global__ __launch_bounds__(1024) void factors_kernel(Rows who, float scale, float* factors, uint32_t* status) {
  __shared__ float most[16];
  float m = 0.0f;
  bool wrong = false;
  for (uint32_t i = threadIdx.x; i < who.n; i += 1024) {
    wrong |= who.label(i) >= (int64_t)who.vocab;
    if (who.live(i)) m = fmaxf(m, fabsf(who.weight(i) * scale));
  }
  if (status && __ballot(wrong) && lane_id() == 0) atomicOr(status, CVLC_DEV_INDEX);
  m = wave_max(m);
  if (lane_id() == 0) most[wave_id()] = m;
  __syncthreads();
  if (threadIdx.x) return;
  for (uint32_t w = 1; w < 16; ++w) m = fmaxf(m, most[w]);
  const int e = m > 0.0f && m < INFINITY ? min(max(ilogbf(m), -100), 100) : 0;
  factors[0] = ldexpf(kLift, -e);
  factors[1] = ldexpf(1.0f / kLift, e);
}

// ------------------------------------------------------------------------------ the product
struct Operand {
  const Half* p;
  uint64_t stride, plane;   // elements from row to row, and from plane to plane
};
struct Product {
  Operand a, b;             // rows of both, K contiguous
  uint32_t m, n;            // their numbers
  uint32_t k_tiles;         // K in tiles of kDepth
  uint32_t pairs, a_planes, b_planes;  // which planes are multiplied: four bits a pair
  uint32_t slices;          // parts that all tiles of K are cut into
};

template <class H>
__device__ __forceinline__ Four mfma(Quad a, Quad b, Four c) {
  if constexpr (std::is_same_v<H, bf16_t>)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(EightB, a), __builtin_bit_cast(EightB, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(EightH, a), __builtin_bit_cast(EightH, b), c, 0, 0, 0);
}

// A tile's shape: WM x WN wavefronts of MT x NT matrix instructions (16 x 16) each.
template <uint32_t WM_, uint32_t WN_, uint32_t MT_, uint32_t NT_>
struct Shape {
  static constexpr uint32_t WM = WM_, WN = WN_, MT = MT_, NT = NT_, TM = WM * MT * 16, TN = WN * NT * 16, kThreads = WM * WN * kWave;
  static constexpr uint32_t kStage = (TM + TN) * kDepth * 2;   // bytes of both operands' tiles
};

// Where a wavefront's lane has its values: value r of acc[i][j] is row m + 16 i + r, column n + 16 j.
struct Spot {
  uint32_t tile_m, tile_n, slice;   // of the workgroup
  uint32_t m0, n0;                  // the workgroup's first row and column
  uint32_t wm, wn;                  // the wavefront's place
  uint32_t m, n;                    // the lane's first row and column
};

// A workgroup's tile: consecutive ones go to the eight dies in turn, so each die takes a run of tiles of its own, four tiles of
// rows by all columns at a time, which share their operands in its cache.
__device__ __forceinline__ void place(const Product& g, uint32_t tm, uint32_t tn, Spot& s) {
  const uint32_t tiles_m = (g.m + tm - 1) / tm, tiles_n = (g.n + tn - 1) / tn, all = tiles_m * tiles_n * g.slices;
  const uint32_t die = blockIdx.x % 8, each = all / 8, rest = all % 8;
  uint32_t id = die * each + min(die, rest) + blockIdx.x / 8;
  s.slice = id / (tiles_m * tiles_n);
  id %= tiles_m * tiles_n;
  constexpr uint32_t kTogether = 4;
  const uint32_t group = id / (kTogether * tiles_n), within = id % (kTogether * tiles_n), first = group * kTogether;
  const uint32_t rows = min(kTogether, tiles_m - first);
  s.tile_m = first + within % rows;
  s.tile_n = within / rows;
}

template <class H, class S, class E>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Product g, E epilogue) {
  __shared__ __attribute__((aligned(128))) uint8_t lds[2 * S::kStage];
  const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  Spot s;
  place(g, S::TM, S::TN, s);
  s.m0 = s.tile_m * S::TM;
  s.n0 = s.tile_n * S::TN;
  s.wm = wave / S::WN;
  s.wn = wave % S::WN;
  s.m = s.m0 + s.wm * S::MT * 16 + (lane >> 4) * 4;
  s.n = s.n0 + s.wn * S::NT * 16 + (lane & 15);
  const uint32_t all = g.pairs * g.k_tiles, per = (all + g.slices - 1) / g.slices;
  const uint32_t from = min(s.slice * per, all), to = min(from + per, all);
  // Tiles go straight to LDS, 16 bytes a lane in the order of the lanes.  A row's eight accesses lie there in an order that
  // depends on the row, so that the sixteen rows that a matrix instruction reads at one K are in sixteen different banks.
  constexpr uint32_t kLoadsA = S::TM * 8 / S::kThreads, kLoadsB = S::TN * 8 / S::kThreads;
  static_assert(kLoadsA * S::kThreads == S::TM * 8 && kLoadsB * S::kThreads == S::TN * 8, "whole loads");
  uint32_t off_a[kLoadsA], off_b[kLoadsB];
  {
    const uint32_t slot = threadIdx.x, at = ((slot & 7) ^ ((slot >> 4) & 7)) * 16;
    static_assert(S::kThreads % 128 == 0, "the order of accesses repeats every sixteen rows");
#pragma unroll
    for (uint32_t j = 0; j < kLoadsA; ++j)  // rows beyond the last one are read as the last one
      off_a[j] = min((j * S::kThreads + slot) / 8, g.m - 1 - s.m0) * (uint32_t)(g.a.stride * 2) + at;
#pragma unroll
    for (uint32_t j = 0; j < kLoadsB; ++j) off_b[j] = min((j * S::kThreads + slot) / 8, g.n - 1 - s.n0) * (uint32_t)(g.b.stride * 2) + at;
  }
  auto fetch = [&](uint32_t tile, uint32_t stage) {
    const uint32_t pair = tile / g.k_tiles, k = tile % g.k_tiles * kDepth;
    const uint8_t* a = reinterpret_cast<const uint8_t*>(g.a.p + (g.a_planes >> 4 * pair & 15) * g.a.plane + s.m0 * g.a.stride + k);
    const uint8_t* b = reinterpret_cast<const uint8_t*>(g.b.p + (g.b_planes >> 4 * pair & 15) * g.b.plane + s.n0 * g.b.stride + k);
    uint8_t* to = lds + stage * S::kStage + wave * kWave * 16;
    auto go = [&](const uint8_t* p, uint8_t* l) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, (__attribute__((address_space(3))) void*)l, 16,
                                       0, 0);
    };
#pragma unroll
    for (uint32_t j = 0; j < kLoadsA; ++j) go(a + off_a[j], to + j * S::kThreads * 16);
#pragma unroll
    for (uint32_t j = 0; j < kLoadsB; ++j) go(b + off_b[j], to + S::TM * kDepth * 2 + j * S::kThreads * 16);
  };
  Four acc[S::MT][S::NT];
#pragma unroll
  for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) acc[i][j] = Four{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t row = lane & 15, order = row >> 1;
  const uint32_t at_a = (s.wm * S::MT * 16 + row) * 128, at_b = S::TM * kDepth * 2 + (s.wn * S::NT * 16 + row) * 128;
  if (from < to) fetch(from, 0);
  for (uint32_t tile = from; tile < to; ++tile) {
    const uint32_t stage = (tile - from) & 1;
    __syncthreads();   // this tile has arrived, and the other stage's readers are done
    if (tile + 1 < to) fetch(tile + 1, stage ^ 1);
    const uint8_t* l = lds + stage * S::kStage;
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
      const uint32_t at = ((k * 4 + (lane >> 4)) ^ order) * 16;
      Quad a[S::MT], b[S::NT];
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i) a[i] = *reinterpret_cast<const Quad*>(l + at_a + at + i * 16 * 128);
#pragma unroll
      for (uint32_t j = 0; j < S::NT; ++j) b[j] = *reinterpret_cast<const Quad*>(l + at_b + at + j * 16 * 128);
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
        for (uint32_t j = 0; j < S::NT; ++j) acc[i][j] = mfma<H>(a[i], b[j], acc[i][j]);
    }
  }
  __syncthreads();
  epilogue.template operator()<S>(acc, s, lds);
}

// ------------------------------------------------------------------------------ what becomes of it
// Rows are the vocabulary's, columns are tokens.  Every tile's largest logit and sum of exponentials per token.
struct StatsEnd {
  Rows who;
  uint32_t first, tile;     // the piece's first token of the vocabulary, and its first tile's number
  float scale;
  float2* partial;          // [tile][token]
  float* answer;            // the logit of every token's label

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t* lds) const {
    float2* shared = reinterpret_cast<float2*>(lds);
    const uint32_t rest = who.vocab - first;   // rows that are there, counted from the piece's
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t token = s.n + j * 16;
      const int64_t label = token < who.n ? who.label(token) - first : -1;
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
          const uint32_t v = s.m + i * 16 + r;
          if (v < rest) {
            const float z = acc[i][j][r] * scale;
            top = fmaxf(top, z);
            if ((int64_t)v == label) answer[token] = z;
          }
        }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r)
          if (s.m + i * 16 + r < rest) sum += __expf(acc[i][j][r] * scale - top);
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      if (lane_id() < 16) shared[s.wm * S::TN + token - s.n0] = float2{top, sum};
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < S::TN; t += S::kThreads) {
      if (s.n0 + t >= who.n) continue;
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < S::WM; ++w) top = fmaxf(top, shared[w * S::TN + t].x);
#pragma unroll
      for (uint32_t w = 0; w < S::WM; ++w) {
        const float2 p = shared[w * S::TN + t];
        if (p.x > -INFINITY) sum += p.y * __expf(p.x - top);      // else nothing was there
        else sum += p.y;
      }
      partial[(uint64_t)(tile + s.tile_m) * who.n + s.n0 + t] = float2{top, sum};
    }
  }
};

// The tiles' statistics joined, and the losses.
constexpr uint32_t kJoinTokens = 16, kJoinRows = 16;
__global__ __launch_bounds__(kJoinTokens * kJoinRows) void loss_kernel(Rows who, uint32_t tiles, const float2* partial, const float* answer,
                                                                       float* loss, float2* stats, uint32_t* status) {
  __shared__ float2 shared[kJoinRows][kJoinTokens];
  const uint32_t x = threadIdx.x % kJoinTokens, y = threadIdx.x / kJoinTokens, token = blockIdx.x * kJoinTokens + x;
  float2 all = {-INFINITY, 0.0f};
  auto add = [](float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x);
    if (top == -INFINITY) return float2{top, a.y + b.y};
    return float2{top, a.y * expf(a.x - top) + b.y * expf(b.x - top)};
  };
  if (token < who.n)
    for (uint32_t t = y; t < tiles; t += kJoinRows) all = add(all, partial[(uint64_t)t * who.n + token]);
  shared[y][x] = all;
  __syncthreads();
  if (y || token >= who.n) return;
  for (uint32_t r = 1; r < kJoinRows; ++r) all = add(all, shared[r][x]);
  if (status && who.label(token) >= (int64_t)who.vocab) atomicOr(status, CVLC_DEV_INDEX);
  const bool live = who.live(token);
  if (loss) loss[token] = live ? who.weight(token) * (logf(all.y) + (all.x - answer[token])) : 0.0f;
  if (stats) stats[token] = live ? all : float2{0.0f, 0.0f};
}

// G in PY planes with the vocabulary contiguous, for dh, and in PT with the tokens contiguous, for dT.
template <class H, uint32_t PY, uint32_t PT>
struct GradEnd {
  Rows who;
  uint32_t first;
  float scale;
  const float2* stats;
  const float* factors;
  Half *g, *turned;
  uint64_t g_stride, g_plane, turned_stride, turned_plane;

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t*) const {
    const uint32_t rest = who.vocab - first;
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t token = s.n + j * 16;
      const bool live = token < who.n && who.live(token);
      const float2 st = live ? stats[token] : float2{0.0f, 1.0f};
      const float over = 1.0f / st.y, w = live ? who.weight(token) * scale * factors[0] : 0.0f;
      const int64_t label = live ? who.label(token) - first : -1;
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i) {
        Half y[PY][4], t[PT][4];
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
          const uint32_t v = s.m + i * 16 + r;
          float x = __expf(acc[i][j][r] * scale - st.x) * over;
          if ((int64_t)v == label) x -= 1.0f;
          x = live && v < rest ? x * w : 0.0f;
          Half part[PY > PT ? PY : PT];
          split<H, (PY > PT ? PY : PT)>(x, part);
#pragma unroll
          for (uint32_t p = 0; p < PY; ++p) y[p][r] = part[p];
#pragma unroll
          for (uint32_t p = 0; p < PT; ++p) t[p][r] = part[p];
        }
        const uint64_t v = s.m + i * 16;
        if (token < who.n)
#pragma unroll
          for (uint32_t p = 0; p < PY; ++p)
            *reinterpret_cast<Pair*>(g + p * g_plane + token * g_stride + v) = Pair{y[p][0] | (uint32_t)y[p][1] << 16, y[p][2] | (uint32_t)y[p][3] << 16};
        if (token < turned_stride)
#pragma unroll
          for (uint32_t p = 0; p < PT; ++p)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) turned[p * turned_plane + (v + r) * turned_stride + token] = t[p][r];
      }
    }
  }
};

// Rows are dh's columns, columns are tokens: fp32 sums, a matrix for every slice of K.
struct HiddenEnd {
  float* sums;
  uint64_t stride;          // of a token; whole fours
  uint32_t n, add;

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t*) const {
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t token = s.n + j * 16;
      if (token >= n) continue;
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i) {
        const uint32_t c = s.m + i * 16;
        if (c >= stride) continue;
        Four* p = reinterpret_cast<Four*>(sums + ((uint64_t)s.slice * n + token) * stride + c);
        *p = add ? *p + acc[i][j] : acc[i][j];
      }
    }
  }
};

// Rows are dT's columns, columns are the piece's tokens of the vocabulary.
template <class TO>
struct TableEnd {
  TO* out;
  uint64_t stride;
  uint32_t dim, count, add;   // count: the piece's
  const float* factors;

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t*) const {
    const float f = factors[1];
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t v = s.n + j * 16;
      if (v >= count) continue;
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i) {
        const uint32_t c = s.m + i * 16;
        if (c >= dim) continue;
        TO* p = out + v * stride + c;
        const uint32_t some = min(4u, dim - c);
        float x[4], old[4] = {};
        if (add) {
          if (some == 4)
            load_values<4>(p, old);
          else
            load_some<4>(p, some, 0.0f, old);
        }
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) x[r] = fmaf(acc[i][j][r], f, old[r]);
        if (some == 4)
          store_whole<false, 4>(p, x);
        else
          store_some<4>(p, some, x);
      }
    }
  }
};

// dh: the slices added up.
template <class T>
__global__ __launch_bounds__(256) void hidden_kernel(Rows who, uint32_t dim, const float* sums, uint64_t stride, uint32_t slices,
                                                     const float* factors, T* out, uint64_t out_stride) {
  const uint32_t blocks = (dim + 1023) / 1024;
  const uint32_t c = blockIdx.x % blocks * 1024 + threadIdx.x * 4;
  if (c >= dim) return;
  const float f = factors[1];
  for (uint32_t i = blockIdx.x / blocks; i < who.n; i += gridDim.x / blocks) {
    float x[4] = {};
    if (who.live(i))
      for (uint32_t k = 0; k < slices; ++k) {
        const Four p = *reinterpret_cast<const Four*>(sums + ((uint64_t)k * who.n + i) * stride + c);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) x[r] += p[r];
      }
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) x[r] *= f;
    store_row<4>(out + i * out_stride, c, dim, x);
  }
}

template <class TO>
__global__ __launch_bounds__(256) void zero_rows_kernel(uint64_t rows, uint32_t dim, TO* out, uint64_t stride) {
  for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (uint32_t c = threadIdx.x; c < dim; c += 256) out[r * stride + c] = (TO)0.0f;
}

// ------------------------------------------------------------------------------ host
using Large = Shape<2, 4, 8, 4>;   // 256 x 256
using Small = Shape<2, 2, 4, 4>;   // 128 x 128
using Thin = Shape<4, 1, 4, 2>;    // 256 x 32: few tokens

template <class T>
struct Kind {                      // how matrices of a type are multiplied
  using H = std::conditional_t<std::is_same_v<T, f16_t>, f16_t, bf16_t>;
  static constexpr uint32_t P = sizeof(T) == 4 ? 3 : 1;
};
// The pairs of planes of (pa, pb) that count, the smallest products first.
void set_pairs(Product& g, uint32_t pa, uint32_t pb) {
  const uint32_t most = std::max(pa, pb);
  g.pairs = g.a_planes = g.b_planes = 0;
  for (uint32_t order = most; order-- > 0;)
    for (uint32_t a = 0; a < pa; ++a)
      if (order >= a && order - a < pb) {
        g.a_planes |= a << 4 * g.pairs;
        g.b_planes |= (order - a) << 4 * g.pairs;
        ++g.pairs;
      }
}

template <class S>
uint64_t tiles_of(const Product& g) {
  return (uint64_t)((g.m + S::TM - 1) / S::TM) * ((g.n + S::TN - 1) / S::TN);
}
template <class H, class S, class E>
void run_as(const Product& g, const E& end, hipStream_t stream) {
  hipLaunchKernelGGL((product_kernel<H, S, E>), dim3((uint32_t)(tiles_of<S>(g) * g.slices)), dim3(S::kThreads), 0, stream, g, end);
}
constexpr uint32_t kCus = 256;
bool large_goes(const Product& g) { return tiles_of<Large>(g) * g.slices >= kCus * 3 / 4; }

struct Sizes {
  uint64_t depth, tokens, piece;      // dim and n in whole tiles of K; tokens of the vocabulary at a time
  uint32_t planes, py, pt, slices;
};
constexpr uint64_t kBudget = 256ull << 20;   // bytes of a piece's G and table
Sizes sizes_for(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type, uint32_t dtable_type, bool grad) {
  Sizes z{};
  z.depth = pad_to(dim, kDepth);
  z.tokens = pad_to(n, kDepth);
  z.planes = type == CVLC_F32 ? 3 : 1;
  z.py = type == CVLC_F32 ? 3 : 1;
  z.pt = type == CVLC_F32 ? 3 : dtable_type == CVLC_F32 ? 2 : 1;
  const uint64_t each = z.depth * z.planes * 2 * (grad ? 2 : 1) + (grad ? z.tokens * 2 * (z.py + z.pt) : 0);
  z.piece = std::min(pad_to(vocab, kPadTo), std::max<uint64_t>(kPadTo, kBudget / each / kPadTo * kPadTo));
  // dh has few tiles where tokens and columns are few: K, a piece of the vocabulary, is cut then
  const uint64_t tiles = ((z.depth + 127) / 128) * ((z.tokens + 127) / 128);
  z.slices = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(kCus / std::max<uint64_t>(tiles, 1), z.piece / 512));
  return z;
}

struct Room {                          // parts of a workspace
  uint8_t* base;
  uint64_t used = 256;                 // the factors lie first
  template <class P>
  P* take(uint64_t count) {
    P* p = reinterpret_cast<P*>(base + used);
    used = pad_to(used + count * sizeof(P), 256);
    return p;
  }
};

struct Call {
  uint32_t n, vocab, dim, type;
  const void *hidden, *table;
  uint64_t hidden_stride, table_stride;
  Rows who;
  float scale;
};

// Whether a matrix can be multiplied as it is: rows that begin at 16 bytes and end with a tile of K, near enough to each other
// for 32-bit offsets inside a tile.
bool as_it_is(const void* p, uint64_t stride, uint32_t dim, uint32_t type) {
  return type != CVLC_F32 && dim % kDepth == 0 && stride % 8 == 0 && stride < (1u << 22) && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <class T>
void pack(const T* src, const PackArgs& a, hipStream_t stream) {
  const uint64_t grid = ((a.rows + kPackSide - 1) / kPackSide) * (uint64_t)((a.cols + kPackSide - 1) / kPackSide);
  hipLaunchKernelGGL((pack_kernel<T, typename Kind<T>::H, Kind<T>::P>), dim3((uint32_t)grid), dim3(kPackBlock), 0, stream, a, src);
}

// The workspace of the loss; with base = null only its size.
struct LossRoom {
  uint64_t tiles;
  float2* partial;
  float* answer;
  Half *hidden, *table;
  uint64_t bytes;
  LossRoom(uint8_t* base, const Sizes& z, uint32_t n, uint32_t vocab) {
    Room r{base};
    tiles = vocab / 128 + vocab / z.piece + 2;
    partial = r.take<float2>(tiles * n);
    answer = r.take<float>(n);
    hidden = r.take<Half>(z.planes * n * z.depth);
    table = r.take<Half>(z.planes * z.piece * z.depth);
    bytes = r.used;
  }
};
struct GradRoom {
  Half *hidden, *hidden_turned, *table, *table_turned, *g, *g_turned;
  float* sums;
  uint64_t bytes;
  GradRoom(uint8_t* base, const Sizes& z, uint32_t n, uint32_t dim) {
    Room r{base};
    hidden = r.take<Half>(z.planes * n * z.depth);
    hidden_turned = r.take<Half>(z.planes * dim * z.tokens);
    table = r.take<Half>(z.planes * z.piece * z.depth);
    table_turned = r.take<Half>(z.planes * dim * z.piece);
    g = r.take<Half>(z.py * n * z.piece);
    g_turned = r.take<Half>(z.pt * z.piece * z.tokens);
    sums = r.take<float>(z.slices * n * z.depth);
    bytes = r.used;
  }
};

template <class T>
void loss_of(const Call& c, const Sizes& z, const LossRoom& room, float* loss, float2* stats, uint32_t* status, hipStream_t stream) {
  using H = typename Kind<T>::H;
  const T *hidden = static_cast<const T*>(c.hidden), *table = static_cast<const T*>(c.table);
  const bool hidden_goes = as_it_is(c.hidden, c.hidden_stride, c.dim, c.type), table_goes = as_it_is(c.table, c.table_stride, c.dim, c.type);
  if (!hidden_goes)
    pack<T>(hidden, PackArgs{c.n, c.dim, c.hidden_stride, room.hidden, nullptr, z.depth, c.n * z.depth, 0, 0, 0, c.who}, stream);
  Product g{};
  g.b = hidden_goes ? Operand{static_cast<const Half*>(c.hidden), c.hidden_stride, 0} : Operand{room.hidden, z.depth, c.n * z.depth};
  g.n = c.n;
  g.k_tiles = (uint32_t)(z.depth / kDepth);
  g.slices = 1;
  set_pairs(g, z.planes, z.planes);
  uint32_t tile = 0;
  const uint64_t step = table_goes ? pad_to(c.vocab, kPadTo) : z.piece;
  for (uint64_t first = 0; first < c.vocab; first += step) {
    g.m = (uint32_t)std::min<uint64_t>(step, c.vocab - first);
    if (table_goes) {
      g.a = Operand{static_cast<const Half*>(c.table) + first * c.table_stride, c.table_stride, 0};
    } else {
      pack<T>(table + first * c.table_stride, PackArgs{g.m, c.dim, c.table_stride, room.table, nullptr, z.depth, z.piece * z.depth, 0, 0, 0, c.who}, stream);
      g.a = Operand{room.table, z.depth, z.piece * z.depth};
    }
    const StatsEnd end{c.who, (uint32_t)first, tile, c.scale, room.partial, room.answer};
    if (c.n <= Thin::TN) {
      run_as<H, Thin>(g, end, stream);
      tile += (g.m + Thin::TM - 1) / Thin::TM;
    } else if (large_goes(g)) {
      run_as<H, Large>(g, end, stream);
      tile += (g.m + Large::TM - 1) / Large::TM;
    } else {
      run_as<H, Small>(g, end, stream);
      tile += (g.m + Small::TM - 1) / Small::TM;
    }
  }
  hipLaunchKernelGGL(loss_kernel, dim3((c.n + kJoinTokens - 1) / kJoinTokens), dim3(kJoinTokens * kJoinRows), 0, stream, c.who, tile,
                     room.partial, room.answer, loss, stats, status);
}

template <class T, class TO>
void grad_of(const Call& c, const Sizes& z, const GradRoom& room, float* factors, const float2* stats, T* dhidden, uint64_t dhidden_stride,
             TO* dtable, uint64_t dtable_stride, bool accumulate, uint32_t* status, hipStream_t stream) {
  using H = typename Kind<T>::H;
  constexpr uint32_t P = Kind<T>::P, PY = P, PT = P == 3 ? 3 : sizeof(TO) == 4 ? 2 : 1;
  const T *hidden = static_cast<const T*>(c.hidden), *table = static_cast<const T*>(c.table);
  const bool hidden_goes = as_it_is(c.hidden, c.hidden_stride, c.dim, c.type), table_goes = as_it_is(c.table, c.table_stride, c.dim, c.type);
  hipLaunchKernelGGL(factors_kernel, dim3(1), dim3(1024), 0, stream, c.who, c.scale, factors, status);
  // rows that do not count may hold anything, and G's zeros do not take a NaN away
  pack<T>(hidden, PackArgs{c.n, c.dim, c.hidden_stride, hidden_goes ? nullptr : room.hidden, dtable ? room.hidden_turned : nullptr, z.depth,
                           c.n * z.depth, z.tokens, c.dim * z.tokens, 1, c.who}, stream);
  auto go = [&](const Product& g, const auto& end) {
    if (large_goes(g))
      run_as<H, Large>(g, end, stream);
    else
      run_as<H, Small>(g, end, stream);
  };
  for (uint64_t first = 0; first < c.vocab; first += z.piece) {
    const uint32_t count = (uint32_t)std::min<uint64_t>(z.piece, c.vocab - first);
    if (!table_goes || dhidden)
      pack<T>(table + first * c.table_stride, PackArgs{count, c.dim, c.table_stride, table_goes ? nullptr : room.table, dhidden ? room.table_turned : nullptr,
                                                       z.depth, z.piece * z.depth, z.piece, c.dim * z.piece, 0, c.who}, stream);
    Product g{};
    g.slices = 1;
    g.a = table_goes ? Operand{static_cast<const Half*>(c.table) + first * c.table_stride, c.table_stride, 0} : Operand{room.table, z.depth, z.piece * z.depth};
    g.b = hidden_goes ? Operand{static_cast<const Half*>(c.hidden), c.hidden_stride, 0} : Operand{room.hidden, z.depth, c.n * z.depth};
    g.m = count;
    g.n = c.n;
    g.k_tiles = (uint32_t)(z.depth / kDepth);
    set_pairs(g, P, P);
    go(g, GradEnd<H, PY, PT>{c.who, (uint32_t)first, c.scale, stats, factors, room.g, room.g_turned, z.piece, c.n * z.piece, z.tokens,
                             z.piece * z.tokens});
    if (dhidden) {
      Product y{};
      y.a = Operand{room.table_turned, z.piece, c.dim * z.piece};
      y.b = Operand{room.g, z.piece, c.n * z.piece};
      y.m = c.dim;
      y.n = c.n;
      y.k_tiles = (uint32_t)(pad_to(count, kDepth) / kDepth);
      y.slices = z.slices;
      set_pairs(y, P, PY);
      go(y, HiddenEnd{room.sums, z.depth, c.n, first > 0});
    }
    if (dtable) {
      Product t{};
      t.a = Operand{room.hidden_turned, z.tokens, c.dim * z.tokens};
      t.b = Operand{room.g_turned, z.tokens, z.piece * z.tokens};
      t.m = c.dim;
      t.n = count;
      t.k_tiles = (uint32_t)(z.tokens / kDepth);
      t.slices = 1;
      set_pairs(t, P, PT);
      go(t, TableEnd<TO>{dtable + first * dtable_stride, dtable_stride, c.dim, count, accumulate, factors});
    }
  }
  if (dhidden) {
    const uint32_t blocks = (c.dim + 1023) / 1024;
    hipLaunchKernelGGL(hidden_kernel<T>, dim3(std::min(c.n, std::max(1u, 8192u / blocks)) * blocks), dim3(256), 0, stream, c.who, c.dim, room.sums,
                       z.depth, z.slices, factors, dhidden, dhidden_stride);
  }
}

constexpr uint32_t kMostRows = 1u << 22;   // offsets inside a tile of tokens' columns have 32 bits

// What both ask of their arguments.
int check(const Call& c, const float* d_stats, const void* d_workspace, const uint32_t* d_status) {
  const uint32_t e = type_known(c.type) ? type_bytes(c.type) : 1;
  if (c.vocab < 1 || c.dim < 1 || c.n > kMostRows || c.vocab > 0x7FFFFFFFu || c.dim > 1u << 20 || !type_known(c.type)) return CVLC_ERR_ARG;
  if (c.hidden_stride < c.dim || c.table_stride < c.dim || (c.who.id_bytes != 4 && c.who.id_bytes != 8)) return CVLC_ERR_ARG;
  if (!std::isfinite(c.scale)) return CVLC_ERR_ARG;
  if (!buffer_ok(d_workspace, 256)) return CVLC_ERR_ARG;
  if (d_status && !buffer_ok(d_status, 4)) return CVLC_ERR_ARG;
  if (c.n == 0) return CVLC_OK;
  if (!buffer_ok(c.hidden, e) || !buffer_ok(c.table, e) || !buffer_ok(c.who.labels, c.who.id_bytes)) return CVLC_ERR_ARG;
  if (c.who.weights && !buffer_ok(c.who.weights, 4)) return CVLC_ERR_ARG;
  if (d_stats && !buffer_ok(d_stats, 8)) return CVLC_ERR_ARG;
  // tiles of a launch, and threads of one: fewer than 2^32
  const uint64_t tiles = ((uint64_t)c.n / 32 + 1) * (pad_to(c.vocab, kPadTo) / 128), packs = ((uint64_t)std::max(c.n, c.vocab) / 64 + 1) * (c.dim / 64 + 1);
  if (tiles >= 1ull << 23 || packs >= 1ull << 24) return CVLC_ERR_ARG;
  return CVLC_OK;
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_linear_xent_workspace_bytes(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type) {
  using namespace cvlc;
  if (!n || !vocab || !dim) return 256;
  return (size_t)LossRoom(nullptr, sizes_for(n, vocab, dim, type, type, false), n, vocab).bytes;
}

int cvlc_linear_xent(uint32_t n, uint32_t vocab, uint32_t dim, const void* d_hidden, uint64_t hidden_stride, const void* d_table,
                     uint64_t table_stride, uint32_t type, const void* d_labels, uint32_t id_bytes, float scale, const float* d_weights,
                     float* d_loss, float* d_stats, void* d_workspace, size_t ws_bytes, uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  const Call c{n, vocab, dim, type, d_hidden, d_table, hidden_stride, table_stride, Rows{d_labels, id_bytes, vocab, n, d_weights}, scale};
  if (const int rc = check(c, d_stats, d_workspace, d_status)) return rc;
  if (d_loss && !buffer_ok(d_loss, 4)) return CVLC_ERR_ARG;
  if (n && !d_loss && !d_stats) return CVLC_ERR_ARG;
  if (ws_bytes < cvlc_linear_xent_workspace_bytes(n, vocab, dim, type)) return CVLC_ERR_CAPACITY;
  if (n == 0) return CVLC_OK;
  const Sizes z = sizes_for(n, vocab, dim, type, type, false);
  const LossRoom room(static_cast<uint8_t*>(d_workspace), z, n, vocab);
  by_type(type, [&](auto t) {
    loss_of<decltype(t)>(c, z, room, d_loss, reinterpret_cast<float2*>(d_stats), d_status, static_cast<hipStream_t>(hip_stream));
  });
  return hip_check(hipGetLastError());
}

size_t cvlc_linear_xent_grad_workspace_bytes(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type, uint32_t dtable_type) {
  using namespace cvlc;
  if (!n || !vocab || !dim) return 256;
  return (size_t)GradRoom(nullptr, sizes_for(n, vocab, dim, type, dtable_type, true), n, dim).bytes;
}

int cvlc_linear_xent_grad(uint32_t n, uint32_t vocab, uint32_t dim, const void* d_hidden, uint64_t hidden_stride, const void* d_table,
                          uint64_t table_stride, uint32_t type, const void* d_labels, uint32_t id_bytes, float scale, const float* d_weights,
                          const float* d_stats, void* d_dhidden, uint64_t dhidden_stride, void* d_dtable, uint32_t dtable_type,
                          uint64_t dtable_stride, uint32_t flags, void* d_workspace, size_t ws_bytes, uint32_t* d_status, void* hip_stream) {
  using namespace cvlc;
  const Call c{n, vocab, dim, type, d_hidden, d_table, hidden_stride, table_stride, Rows{d_labels, id_bytes, vocab, n, d_weights}, scale};
  if (const int rc = check(c, d_stats, d_workspace, d_status)) return rc;
  if (flags & ~CVLC_GRAD_ACCUMULATE) return CVLC_ERR_ARG;
  if (n && !d_stats) return CVLC_ERR_ARG;
  if (!d_dhidden && !d_dtable && n) return CVLC_ERR_ARG;
  if (d_dhidden && (dhidden_stride < dim || !buffer_ok(d_dhidden, type_bytes(type)))) return CVLC_ERR_ARG;
  if (d_dtable && (dtable_stride < dim || (dtable_type != type && dtable_type != CVLC_F32) || !buffer_ok(d_dtable, type_bytes(dtable_type))))
    return CVLC_ERR_ARG;
  const uint32_t out_type = d_dtable ? dtable_type : type;
  if (ws_bytes < cvlc_linear_xent_grad_workspace_bytes(n, vocab, dim, type, out_type)) return CVLC_ERR_CAPACITY;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool accumulate = flags & CVLC_GRAD_ACCUMULATE;
  if (n == 0) {
    if (!d_dtable || accumulate) return CVLC_OK;
    by_type(dtable_type, [&](auto t) {
      using TO = decltype(t);
      hipLaunchKernelGGL(zero_rows_kernel<TO>, dim3(std::min(vocab, 1u << 16)), dim3(256), 0, stream, vocab, dim, static_cast<TO*>(d_dtable), dtable_stride);
    });
    return hip_check(hipGetLastError());
  }
  const Sizes z = sizes_for(n, vocab, dim, type, out_type, true);
  const GradRoom room(static_cast<uint8_t*>(d_workspace), z, n, dim);
  float* factors = static_cast<float*>(d_workspace);
  by_type(type, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto to) {
      using TO = decltype(to);
      grad_of<T, TO>(c, z, room, factors, reinterpret_cast<const float2*>(d_stats), static_cast<T*>(d_dhidden), dhidden_stride,
                     static_cast<TO*>(d_dtable), dtable_stride, accumulate, d_status, stream);
    };
    if (out_type == type)
      go(T{});
    else
      go(0.0f);
  });
  return hip_check(hipGetLastError());
}

}  // extern "C"
