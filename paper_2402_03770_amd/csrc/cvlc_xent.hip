// cvlc_xent.hip -- softmax cross entropy of logits z = s h T^t over a large vocabulary, without the logits in memory.
//
// loss_i = w_i (ln sum_v exp z_iv - z_i,label),  G_iv = s w_i (softmax(z_i)_v - [v = label_i]),  dh = G T,  dT = G^t h.
//
// Products of matrices do nearly all the work: z once for the loss, once more for the gradients (a row's softmax needs its
// whole sum first, and keeping z is what this call is there to avoid), then dh and dT.  All run on the matrix units from
// 16-bit operands, sums in fp32:
//   - bfloat16 and fp16 matrices as they are;
//   - fp32 as two planes of fp16 (11 + 11 bits) of the matrix times a power of two that brings its largest element to about 2^14;
//     three of the four products of planes are added.  What is left out is below 2^-22 of a term, and an element is held to
//     2^-23 of itself or 2^-39 of the largest.  An fp32 matrix instruction has a sixteenth of the rate.
//   - G for dh of 16 bits in one plane of its type, whose rounding, but for the label's entry, is what the result's own is; what it
//     leaves of the label's entry is added (join_kernel).
//   - G for dT in two planes (2^-17 of an entry in bfloat16, 2^-23 in fp16).  dT adds up labels' entries of about -1 and others'
//     shares of them, which may nearly cancel: in one plane, half the product, values of 263 x 128 x 99 137 bf16 were 12 % off that
//     now are rounded.  Three for fp32 dT of bfloat16 matrices of fewer than kManyTokens rows: 2-norms of the error of 1, 24, 600,
//     2000 and 4096 tokens are 3.4e-6, 1.9e-6, 1.4e-6, 1.2e-6 and 1.1e-6 with two, where sums in fp32 alone have 4e-8, 2e-7, 4e-7,
//     8e-7 and 1.1e-6.
// G is scaled so that the largest weight becomes 2^13, by 2^126 at most: then neither tiny weights nor fp16 lose its small
// entries, and the label's entry, softmax - 1, is next to a value that every type has.
//
// The loss's product ends in every tile's (max, sum of exponentials) per row, joined in order by a second launch.  The
// gradients go over the vocabulary in pieces, G's and a copied table's part of which take kBudget at most: a workspace that does not
// grow with the vocabulary, and much of it still in the last-level cache (256 MB) when it is read.
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

constexpr uint32_t kDepth = 64;    // K is padded to whole ones of the deepest tiles
constexpr uint32_t kStep = 32;     // K of a matrix instruction
constexpr uint32_t kPadTo = 256;   // vocabulary pieces are whole tiles
constexpr float kLift = 0x1p13f;   // G's largest entries ...
constexpr float kMostLift = 0x1p126f;   // ... where they do not take more than this; its inverse is a normal value

uint64_t pad_to(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// ------------------------------------------------------------------------------ planes
// x as a sum of P values of a 16-bit type, each rounded or (CUT) with the bits behind it cut off; the rest is exact both ways.
template <class H, uint32_t P, bool CUT = false>
__device__ __forceinline__ void split(float x, Half (&out)[P]) {
#pragma unroll
  for (uint32_t p = 0; p < P; ++p) {
    const H h = CUT ? __builtin_bit_cast(H, (Half)(__float_as_uint(x) >> 16)) : (H)x;
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

// What a call's launches share, at the workspace's start.
struct Factors {
  float grad;               // by which G is multiplied ...
  float back;               // ... and by which its products are then
  float up[2], down[2];     // the same of hidden rows and table, powers of two
};

// What takes a product of G and one of the scaled matrices back; not infinite, which 0 times it would show.
__device__ __forceinline__ float back_of(const Factors& f, uint32_t side) { return fminf(f.back * f.down[side], 0x1.fffffep127f); }

constexpr uint32_t kSurveyBlock = 256, kSurveyGrid = 1024, kSurveyEach = 4096, kSurveyAlone = 1u << 14;
struct Matrix {
  const void* p;
  uint64_t stride;
  uint32_t rows;
};

// The largest magnitude of every workgroup's share of a matrix; rows that do not count are left out of the hidden ones.
template <uint32_t THREADS>
__device__ __forceinline__ float largest(const Matrix& m, uint32_t dim, const Rows* who, uint32_t part, uint32_t parts) {
  const float* p = static_cast<const float*>(m.p);
  const uint32_t across = (dim + 3) / 4;
  const uint64_t all = (uint64_t)m.rows * across;
  float top = 0.0f;
  for (uint64_t k = (uint64_t)part * THREADS + threadIdx.x; k < all; k += (uint64_t)parts * THREADS) {
    const uint32_t row = (uint32_t)(k / across), c = (uint32_t)(k % across) * 4;
    if (who && !who->live(row)) continue;
    float x[4];
    load_row<4>(p + row * m.stride, c, dim, 0.0f, x);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) top = fmaxf(top, fabsf(x[i]));
  }
  return wave_max(top);
}
__global__ __launch_bounds__(kSurveyBlock) void survey_kernel(Matrix hidden, Matrix table, uint32_t dim, Rows who, float* tops) {
  __shared__ float most[kSurveyBlock / kWave];
  float top = blockIdx.y ? largest<kSurveyBlock>(table, dim, nullptr, blockIdx.x, gridDim.x)
                         : largest<kSurveyBlock>(hidden, dim, &who, blockIdx.x, gridDim.x);
  if (lane_id() == 0) most[wave_id()] = top;
  __syncthreads();
  for (uint32_t w = 0; w < kSurveyBlock / kWave; ++w) top = fmaxf(top, most[w]);
  if (threadIdx.x == 0) tops[blockIdx.y * gridDim.x + blockIdx.x] = top;
}

// The factors, and labels that are not there told of.  tops: what survey_kernel found (`parts` a matrix); null: small matrices,
// looked over here, where they are given.
__global__ __launch_bounds__(1024) void factors_kernel(Rows who, float scale, const float* tops, uint32_t parts, Matrix hidden, Matrix table,
                                                       uint32_t dim, Factors* factors, uint32_t* status) {
  __shared__ float most[3][16];
  float m[3] = {0.0f, 0.0f, 0.0f};
  bool wrong = false;
  for (uint32_t i = threadIdx.x; i < who.n; i += 1024) {
    wrong |= who.label(i) >= (int64_t)who.vocab;
    if (who.live(i)) m[0] = fmaxf(m[0], fabsf(who.weight(i) * scale));
  }
  if (status && __ballot(wrong) && lane_id() == 0) atomicOr(status, CVLC_DEV_INDEX);
  if (tops) {
    for (uint32_t i = threadIdx.x; i < parts; i += 1024) {
      m[1] = fmaxf(m[1], tops[i]);
      m[2] = fmaxf(m[2], tops[parts + i]);
    }
  } else if (hidden.p) {
    m[1] = largest<1024>(hidden, dim, &who, 0, 1);
    m[2] = largest<1024>(table, dim, nullptr, 0, 1);
  }
#pragma unroll
  for (uint32_t k = 0; k < 3; ++k) {
    m[k] = wave_max(m[k]);
    if (lane_id() == 0) most[k][wave_id()] = m[k];
  }
  __syncthreads();
  if (threadIdx.x) return;
  for (uint32_t k = 0; k < 3; ++k)
    for (uint32_t w = 1; w < 16; ++w) m[k] = fmaxf(m[k], most[k][w]);
  const bool some = m[0] > 0.0f && m[0] < INFINITY, tiny = !(kLift / m[0] < kMostLift);
  factors->grad = !some ? 1.0f : tiny ? kMostLift : kLift / m[0];
  factors->back = !some ? 1.0f : tiny ? 1.0f / kMostLift : m[0] / kLift;
  for (uint32_t k = 0; k < 2; ++k) {
    const float top = m[k + 1];
    const int e = top > 0.0f && top < INFINITY ? min(max(14 - ilogbf(top), -100), 100) : 0;
    factors->up[k] = ldexpf(1.0f, e);
    factors->down[k] = ldexpf(1.0f, -e);
  }
}

// A matrix's planes with whole tiles of K in a row; zeros beyond it.
constexpr uint32_t kPackBlock = 256;
struct PackArgs {
  Matrix from;
  uint32_t cols, rows_to;           // rows that are written: those beyond the matrix's are zeros
  Half* to;
  uint64_t stride, plane;
  const float* up;
  uint32_t masked;                  // rows that do not count become zeros: they may hold anything, and G's zeros would not take a NaN away
};
template <class T, class H, uint32_t P>
__global__ __launch_bounds__(kPackBlock) void pack_kernel(PackArgs first, PackArgs second, uint32_t grid, Rows who) {
  const PackArgs& a = blockIdx.x < grid ? first : second;
  const uint32_t block = blockIdx.x < grid ? blockIdx.x : blockIdx.x - grid, blocks = blockIdx.x < grid ? grid : gridDim.x - grid;
  const uint32_t across = (uint32_t)(a.stride / 8);
  const uint64_t all = (uint64_t)a.rows_to * across;
  const float up = P == 2 ? *a.up : 1.0f;
  for (uint64_t k = (uint64_t)block * kPackBlock + threadIdx.x; k < all; k += (uint64_t)blocks * kPackBlock) {
    const uint32_t row = (uint32_t)(k / across), c = (uint32_t)(k % across) * 8;
    float x[8] = {};
    if (row < a.from.rows && !(a.masked && !who.live(row))) load_row<8>(static_cast<const T*>(a.from.p) + row * a.from.stride, c, a.cols, 0.0f, x);
    Half h[8][P];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) split<H, P, P == 3>(P == 2 ? x[i] * up : x[i], h[i]);
#pragma unroll
    for (uint32_t p = 0; p < P; ++p) {
      Quad q;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) q[i] = h[2 * i][p] | (uint32_t)h[2 * i + 1][p] << 16;
      *reinterpret_cast<Quad*>(a.to + p * a.plane + row * a.stride + c) = q;
    }
  }
}

// ------------------------------------------------------------------------------ the product
// An operand is wide, its rows in memory those of the product and K along them, or tall, K from row to row.
struct Operand {
  const Half* p;
  uint64_t stride, plane;   // elements from row to row, and from plane to plane
  uint32_t along;           // tall: elements of a row that may be read, whole eights
  uint32_t rows;            // rows that may be read; others are read as the last one, and count for nothing
};
struct Product {
  Operand a, b;
  uint32_t m, n;            // rows of a and of b
  uint32_t k;               // K, whole kDepths
  uint32_t pairs, a_planes, b_planes;  // which planes are multiplied: four bits a pair
  uint32_t slices;          // parts that all planes' K is cut into
};

template <class H>
__device__ __forceinline__ Four mfma(Quad a, Quad b, Four c) {
  if constexpr (std::is_same_v<H, bf16_t>)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(EightB, a), __builtin_bit_cast(EightB, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(EightH, a), __builtin_bit_cast(EightH, b), c, 0, 0, 0);
}

// A tile's shape: WM x WN wavefronts of MT x NT matrix instructions (16 x 16) each.  Two wavefronts share a SIMD (kPairs), and
// operands' tiles of kDepth are in LDS, or they do not, and there are STAGES of both operands' tiles of kStep.
template <uint32_t WM_, uint32_t WN_, uint32_t MT_, uint32_t NT_, uint32_t STAGES>
struct Shape {
  static constexpr uint32_t WM = WM_, WN = WN_, MT = MT_, NT = NT_, TM = WM * MT * 16, TN = WN * NT * 16, kThreads = WM * WN * kWave;
  static constexpr bool kPairs = WM * WN == 8;
  static constexpr uint32_t kK = kPairs ? kDepth : kStep, kStages = STAGES;
  static constexpr uint32_t kStage = (kPairs ? TM : TM + TN) * kK * 2;   // bytes of an operand's tile, or of both
  static_assert(!kPairs || TM == TN, "operands' tiles in one ring");
};
// Where a lane's rows are that belong to the i-th matrix instruction: eight neighbouring ones to two of them.
constexpr __host__ __device__ uint32_t run_of(uint32_t i) { return i / 2 * 32 + i % 2 * 4; }

// What lanes take to N matrix instructions, each from two reads of LDS that turn four rows of sixteen elements, FOUR bytes apart.
// One block of assembly with its wait: the builtin's read is taken for one that needs all that is on its way into LDS, and waits
// for it.
template <uint32_t FOUR, uint32_t N>
__device__ __forceinline__ void turned(const uint32_t (&at)[N], Quad (&out)[N]) {
  static_assert(N == 4 || N == 8 || N == 12, "blocks by size");
  Pair x[2 * N];
  if constexpr (N == 4) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\tds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\tds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(FOUR)
        : "memory");
  } else if constexpr (N == 8) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:%24\n\tds_read_b64_tr_b16 %2, %17\n\tds_read_b64_tr_b16 %3, %17 offset:%24\n\t"
        "ds_read_b64_tr_b16 %4, %18\n\tds_read_b64_tr_b16 %5, %18 offset:%24\n\tds_read_b64_tr_b16 %6, %19\n\tds_read_b64_tr_b16 %7, %19 offset:%24\n\t"
        "ds_read_b64_tr_b16 %8, %20\n\tds_read_b64_tr_b16 %9, %20 offset:%24\n\tds_read_b64_tr_b16 %10, %21\n\tds_read_b64_tr_b16 %11, %21 offset:%24\n\t"
        "ds_read_b64_tr_b16 %12, %22\n\tds_read_b64_tr_b16 %13, %22 offset:%24\n\tds_read_b64_tr_b16 %14, %23\n\tds_read_b64_tr_b16 %15, %23 offset:%24\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]),
          "=&v"(x[9]), "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7]), "n"(FOUR)
        : "memory");
  } else {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %24\n\tds_read_b64_tr_b16 %1, %24 offset:%36\n\tds_read_b64_tr_b16 %2, %25\n\tds_read_b64_tr_b16 %3, %25 offset:%36\n\t"
        "ds_read_b64_tr_b16 %4, %26\n\tds_read_b64_tr_b16 %5, %26 offset:%36\n\tds_read_b64_tr_b16 %6, %27\n\tds_read_b64_tr_b16 %7, %27 offset:%36\n\t"
        "ds_read_b64_tr_b16 %8, %28\n\tds_read_b64_tr_b16 %9, %28 offset:%36\n\tds_read_b64_tr_b16 %10, %29\n\tds_read_b64_tr_b16 %11, %29 offset:%36\n\t"
        "ds_read_b64_tr_b16 %12, %30\n\tds_read_b64_tr_b16 %13, %30 offset:%36\n\tds_read_b64_tr_b16 %14, %31\n\tds_read_b64_tr_b16 %15, %31 offset:%36\n\t"
        "ds_read_b64_tr_b16 %16, %32\n\tds_read_b64_tr_b16 %17, %32 offset:%36\n\tds_read_b64_tr_b16 %18, %33\n\tds_read_b64_tr_b16 %19, %33 offset:%36\n\t"
        "ds_read_b64_tr_b16 %20, %34\n\tds_read_b64_tr_b16 %21, %34 offset:%36\n\tds_read_b64_tr_b16 %22, %35\n\tds_read_b64_tr_b16 %23, %35 offset:%36\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]),
          "=&v"(x[9]), "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15]), "=&v"(x[16]),
          "=&v"(x[17]), "=&v"(x[18]), "=&v"(x[19]), "=&v"(x[20]), "=&v"(x[21]), "=&v"(x[22]), "=&v"(x[23])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7]), "v"(at[8]),
          "v"(at[9]), "v"(at[10]), "v"(at[11]), "n"(FOUR)
        : "memory");
  }
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) out[i] = Quad{x[2 * i][0], x[2 * i][1], x[2 * i + 1][0], x[2 * i + 1][1]};
}

// One operand's tile in LDS: how it is fetched and read.  Tiles go straight to LDS, 16 bytes a lane in the order of the
// lanes; where in memory a lane reads decides what lies where, and it is so that the lanes that read LDS together find
// different banks:
//   wide: lanes 16 apart read neighbouring accesses of a row, sixteen lanes their own rows; together go lanes 0 to 3, 12 to 15,
//     20 to 27 and such.  Access x of row r lies at x ^ key(r).  The sixteen rows follow each other, or, where a lane's results
//     are runs of neighbouring rows (RUNS), the matrix instruction's row i is row 8 (i / 4) + i % 4.
//   tall: sixteen neighbouring elements of a row are read from four rows by sixteen lanes, which hand them round (the read
//     turns them).  Such a block b of row k lies at b ^ (k % 4 + 4 (k / 8 % 2)).
// Tiles of half a row's 128 bytes ask the caches for every line twice, which a large tile's rate shows: it takes kDepth.
template <bool TALL, uint32_t ROWS, uint32_t THREADS, bool RUNS, uint32_t K>
struct Tile {
  static constexpr uint32_t kLoads = ROWS * K / 8 / THREADS;
  static_assert(kLoads * THREADS == ROWS * K / 8, "whole loads");
  static constexpr uint32_t kAcross = (TALL ? ROWS : K) / 8;   // accesses of a row
  uint32_t off[kLoads];

  static __device__ __forceinline__ uint32_t key(uint32_t r) {
    if (K == 64) return RUNS ? (r >> 1 & 1) | (r >> 3 & 3) << 1 : r >> 1 & 7;
    const uint32_t q = r >> (RUNS ? 3 : 2) & 3;
    return (q ^ q >> 1) % 2 * 2 + q / 2;   // 0, 2, 3, 1
  }
  // Byte offsets from the tile's first row on; tall: inside a row.  Rows that are not there are read as the last one.
  __device__ __forceinline__ void place(const Operand& o, uint32_t first) {
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) {
      const uint32_t slot = j * THREADS + threadIdx.x, r = slot / kAcross, x = slot % kAcross;
      if constexpr (TALL)
        off[j] = min((x ^ ((r & 3) | (r >> 3 & 1) << 2) << 1) * 8, o.along - first - 8) * 2;
      else
        off[j] = min(r, o.rows - first - 1) * (uint32_t)(o.stride * 2) + (x ^ key(r)) * 16;
    }
  }
  __device__ __forceinline__ void fetch(const Operand& o, uint32_t plane, uint32_t first, uint32_t k, uint8_t* to) const {
    const uint32_t row = TALL ? min(k, o.rows - 1) : first;   // a piece's K is padded, its last tile may begin behind its rows
    const uint8_t* p = reinterpret_cast<const uint8_t*>(o.p + plane * o.plane + row * o.stride + (TALL ? first : k));
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) {
      uint32_t at = off[j];
      if constexpr (TALL) at += min((j * THREADS + threadIdx.x) / kAcross, o.rows - 1 - row) * (uint32_t)(o.stride * 2);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + at),
                                       (__attribute__((address_space(3))) void*)(to + j * THREADS * 16), 16, 0, 0);
    }
  }
  // Where a lane reads what it takes to COUNT matrix instructions: its rows, of the sixteens from `rows` on, at 8 values of K, of
  // the tile's step-th kStep.
  template <uint32_t COUNT, uint32_t ALL>
  static __device__ __forceinline__ void turned_at(const uint8_t* tile, uint32_t rows, uint32_t step, uint32_t from, uint32_t (&at)[ALL]) {
    const uint32_t lane = lane_id(), row = lane & 15, k = (lane >> 4) * 8 + (row >> 2);   // and four rows on: the same bits of the order
    const uint32_t first = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)tile + (step * kStep + k) * (ROWS * 2) +
                           (rows / 16 ^ ((k & 3) | (k >> 3 & 1) << 2)) * 32 + (row & 3) * 8;
#pragma unroll
    for (uint32_t i = 0; i < COUNT; ++i) at[from + i] = first ^ i * 32;
  }
  template <uint32_t COUNT>
  static __device__ __forceinline__ void read(const uint8_t* tile, uint32_t rows, uint32_t step, Quad (&out)[COUNT]) {
    if constexpr (TALL) {
      uint32_t at[COUNT];
      turned_at<COUNT>(tile, rows, step, 0, at);
      turned<4 * ROWS * 2>(at, out);
    } else {
      const uint32_t lane = lane_id(), row = lane & 15, part = lane >> 4;
#pragma unroll
      for (uint32_t i = 0; i < COUNT; ++i) {
        const uint32_t r = rows + (RUNS ? (row >> 2) * 8 + (row & 3) + run_of(i) : i * 16 + row);
        out[i] = *reinterpret_cast<const Quad*>(tile + r * (K * 2) + ((step * 4 + part) ^ key(r)) * 16);
      }
    }
  }
};

// The tiles of one operand in the order in which they are multiplied: all of K for every plane in turn.
template <class T>
struct Walk {
  T tile;
  uint32_t pair, k;
  __device__ __forceinline__ void start(const Operand& o, uint32_t first, uint32_t at, uint32_t all_k) {
    tile.place(o, first);
    pair = at / all_k;
    k = at % all_k;
  }
  __device__ __forceinline__ void fetch(const Operand& o, uint32_t planes, uint32_t first, uint32_t step, uint32_t all_k, uint8_t* to) {
    tile.fetch(o, planes >> 4 * pair & 15, first, k, to);
    k += step;
    const bool over = k == all_k;
    k = over ? 0 : k;
    pair += over;
  }
};

// Where a wavefront's lane has its values: value r of acc[i][j] is row m + 16 i + r, or m + run_of(i) + r where the first
// operand is wide, and column n + 16 j.
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

// Waits until all but the last LOADS loads of this wavefront have arrived and its reads of LDS are done, and for all
// wavefronts to have come here.
template <uint32_t LOADS>
__device__ __forceinline__ void arrive() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <bool READS = false>
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  if (READS)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  else
    asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <class H, class S, bool TALL_A, bool TALL_B, class E>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Product g, E epilogue) {
  __shared__ __attribute__((aligned(128))) uint8_t lds[S::kStages * S::kStage];
  const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  Spot s;
  place(g, S::TM, S::TN, s);
  s.m0 = s.tile_m * S::TM;
  s.n0 = s.tile_n * S::TN;
  s.wm = wave / S::WN;
  s.wn = wave % S::WN;
  s.m = s.m0 + s.wm * S::MT * 16 + (lane >> 4) * (TALL_A ? 4 : 8);
  s.n = s.n0 + s.wn * S::NT * 16 + (lane & 15);
  const uint32_t all = g.pairs * (g.k / S::kK), per = (all + g.slices - 1) / g.slices;
  const uint32_t from = min(s.slice * per, all), count = min(from + per, all) - from;
  using TileA = Tile<TALL_A, S::TM, S::kThreads, !TALL_A, S::kK>;
  using TileB = Tile<TALL_B, S::TN, S::kThreads, false, S::kK>;
  Walk<TileA> wa;
  Walk<TileB> wb;
  wa.start(g.a, s.m0, from * S::kK, g.k);
  wb.start(g.b, s.n0, from * S::kK, g.k);
  auto fetch_a = [&](uint8_t* to) { wa.fetch(g.a, g.a_planes, s.m0, S::kK, g.k, to + wave * kWave * 16); };
  auto fetch_b = [&](uint8_t* to) { wb.fetch(g.b, g.b_planes, s.n0, S::kK, g.k, to + wave * kWave * 16); };
  Four acc[S::MT][S::NT];
#pragma unroll
  for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) acc[i][j] = Four{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr uint32_t kSets = S::kPairs ? 1 : 2;
  Quad a[kSets][S::MT], b[kSets][S::NT];
  auto read = [&](const uint8_t* la, const uint8_t* lb, uint32_t step, uint32_t o) {
    if constexpr (TALL_A && TALL_B) {
      static_assert(S::TM == S::TN, "rows equally far apart");
      uint32_t at[S::MT + S::NT];
      Quad both[S::MT + S::NT];
      TileA::template turned_at<S::MT>(la, s.wm * S::MT * 16, step, 0, at);
      TileB::template turned_at<S::NT>(lb, s.wn * S::NT * 16, step, S::MT, at);
      turned<8 * S::TM>(at, both);
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i) a[o][i] = both[i];
#pragma unroll
      for (uint32_t j = 0; j < S::NT; ++j) b[o][j] = both[S::MT + j];
    } else {
      TileB::read(lb, s.wn * S::NT * 16, step, b[o]);
      TileA::read(la, s.wm * S::MT * 16, step, a[o]);
    }
  };
  auto multiply = [&](uint32_t o) {
#pragma unroll
    for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
      for (uint32_t j = 0; j < S::NT; ++j) acc[i][j] = mfma<H>(a[o][i], b[o][j], acc[i][j]);
  };
  auto next = [&](uint32_t at) { return at + 1 == S::kStages ? 0 : at + 1; };
  uint32_t take = 0, fill = 0;                                        // places in the ring: read next, fetched into next
  if constexpr (S::kPairs) if (count) {
    // Two wavefronts share a SIMD, one half a turn behind the other: one reads a step's values from LDS while the other
    // multiplies; they meet after each.  The operands' tiles go round a ring, a, b, a, b: a place is fetched into when the tile
    // after the one it held is read, which those behind have read too by then; tiles have arrived, everybody's share of them, when
    // all meet after the reads before.
    const bool behind = wave & 4;
    auto to = [&]() {
      uint8_t* l = lds + fill * S::kStage;
      fill = next(fill);
      return l;
    };
    fetch_a(to());
    fetch_b(to());
    if (count > 1) fetch_a(to());
    arrive<0>();
    if (behind) meet<>();
    auto tile = [&](auto more_b, auto more_a) {   // loads of the next tile's b and of the a after it
      const uint8_t *la = lds + take * S::kStage, *lb = lds + next(take) * S::kStage;
      take = next(next(take));
      if (decltype(more_b)::value) fetch_b(to());
      read(la, lb, 0, 0);
      meet<true>();
      multiply(0);
      meet<>();
      if (decltype(more_a)::value) fetch_a(to());
      read(la, lb, 1, 0);
      arrive<decltype(more_a)::value ? TileA::kLoads : 0>();
      multiply(0);
      meet<>();
    };
    for (uint32_t t = 0; t + 2 < count; ++t) tile(std::true_type{}, std::true_type{});
    if (count > 1) tile(std::true_type{}, std::false_type{});
    tile(std::false_type{}, std::false_type{});
    if (!behind) meet<>();
  }
  if constexpr (!S::kPairs) if (count) {
    // A wavefront has its SIMD to itself: it reads the next tile into other registers before it multiplies.  A stage is
    // fetched into as soon as all have read the tile that it held.
    constexpr uint32_t kLoads = TileA::kLoads + TileB::kLoads;
    auto fetch = [&]() {
      uint8_t* l = lds + fill * S::kStage;
      fill = next(fill);
      fetch_a(l);
      fetch_b(l + S::TM * S::kK * 2);
    };
    auto read_next = [&](uint32_t o) {
      const uint8_t* l = lds + take * S::kStage;
      take = next(take);
      read(l, l + S::TM * S::kK * 2, 0, o);
    };
    for (uint32_t t = 0; t + 1 < S::kStages && t < count; ++t) fetch();
    arrive<0>();
    read_next(0);
    if (S::kStages - 1 < count) fetch();
    uint32_t t = 0;
    for (; t + S::kStages + 2 <= count; t += 2) {
#pragma unroll
      for (uint32_t o = 0; o < 2; ++o) {
        arrive<(S::kStages - 2) * kLoads>();
        fetch();
        read_next(o ^ 1);
        multiply(o);
      }
    }
    for (; t < count; t += 2) {
      arrive<0>();
      if (t + S::kStages < count) fetch();
      if (t + 1 < count) read_next(kSets - 1);
      multiply(0);
      if (t + 1 < count) {
        arrive<0>();
        if (t + 1 + S::kStages < count) fetch();
        if (t + 2 < count) read_next(0);
        multiply(kSets - 1);
      }
    }
  }
  __syncthreads();
  epilogue.template operator()<S>(acc, s, lds);
}

// ------------------------------------------------------------------------------ what becomes of it
// exp(x) for x <= 0 of a difference: the difference's rounding is small where the exponential is large.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 0x1.715476p+0f); }

// Rows are the vocabulary's, columns are tokens.  Every tile's largest logit and sum of exponentials per token.
struct StatsEnd {
  Rows who;
  uint32_t first, tile;     // the piece's first token of the vocabulary, and its first tile's number
  float scale;
  const Factors* factors;   // null: matrices are multiplied as they are
  float2* partial;          // [tile][token]
  float* answer;            // the logit of every token's label

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t* lds) const {
    if (s.m0 + S::TM <= who.vocab - first)
      tile_of<S, true>(acc, s, lds);
    else
      tile_of<S, false>(acc, s, lds);
  }
  template <class S, bool WHOLE>
  __device__ __forceinline__ void tile_of(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t* lds) const {
    float2* shared = reinterpret_cast<float2*>(lds);
    const uint32_t rest = who.vocab - first;   // rows that are there, counted from the piece's
    const float f = factors ? scale * (factors->down[0] * factors->down[1]) : scale;
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t token = s.n + j * 16;
      const int64_t label = token < who.n ? who.label(token) - first - s.m : -1;
      float top = -INFINITY, sum = 0.0f, z[S::MT][4];
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
          z[i][r] = acc[i][j][r] * f;
          if (WHOLE || s.m + run_of(i) + r < rest) top = fmaxf(top, z[i][r]);
        }
      if (label >= 0 && label < 16 * (int64_t)S::MT && label % 32 < 8) {
#pragma unroll
        for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
          for (uint32_t r = 0; r < 4; ++r)
            if (run_of(i) + r == (uint32_t)label) answer[token] = z[i][r];
      }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
#pragma unroll
      for (uint32_t i = 0; i < S::MT; ++i)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r)
          if (WHOLE || s.m + run_of(i) + r < rest) sum += exp_of(z[i][r] - top);
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
        sum += p.x > -INFINITY ? p.y * exp_of(p.x - top) : p.y;      // else nothing was there
      }
      partial[(uint64_t)(tile + s.tile_m) * who.n + s.n0 + t] = float2{top, sum};
    }
  }
};

// The tiles' statistics joined, and the losses: a workgroup has 2^tokens_log2 tokens, fewer where there are few, and more threads
// where there are many tiles to each (24 tokens, 3126 tiles: 8.9 us, 11.4 with 256).
constexpr uint32_t kJoinMost = 1024;
uint32_t join_block(uint32_t n, uint32_t tiles) { return n < 2048 && tiles > 1024 ? kJoinMost : 256; }
uint32_t join_tokens_log2(uint32_t n) { return n >= 16384 ? 4 : n >= 2048 ? 2 : 0; }
__global__ __launch_bounds__(kJoinMost) void loss_kernel(Rows who, uint32_t tiles, uint32_t tokens_log2, const float2* partial,
                                                          const float* answer, float* loss, float2* stats, uint32_t* status) {
  __shared__ float2 shared[kJoinMost];
  const uint32_t tokens = 1u << tokens_log2, rows = blockDim.x >> tokens_log2;
  const uint32_t x = threadIdx.x & (tokens - 1), y = threadIdx.x >> tokens_log2, token = (blockIdx.x << tokens_log2) + x;
  float2 all = {-INFINITY, 0.0f};
  auto add = [](float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x);
    if (top == -INFINITY) return float2{top, a.y + b.y};
    return float2{top, a.y * expf(a.x - top) + b.y * expf(b.x - top)};
  };
  if (token < who.n)
#pragma unroll 4
    for (uint32_t t = y; t < tiles; t += rows) all = add(all, partial[(uint64_t)t * who.n + token]);
  shared[threadIdx.x] = all;
  for (uint32_t half = rows / 2; half; half /= 2) {
    __syncthreads();
    if (y < half) shared[threadIdx.x] = all = add(all, shared[threadIdx.x + (half << tokens_log2)]);
  }
  if (y || token >= who.n) return;
  if (status && who.label(token) >= (int64_t)who.vocab) atomicOr(status, CVLC_DEV_INDEX);
  const bool live = who.live(token);
  if (loss) loss[token] = live ? who.weight(token) * (logf(all.y) + (all.x - answer[token])) : 0.0f;
  if (stats) stats[token] = live ? all : float2{0.0f, 0.0f};
}

// G in P planes, the vocabulary along the rows.  Rows and columns up to whole tiles of K are zeros.
template <class H, uint32_t P>
struct GradEnd {
  Rows who;
  uint32_t first;
  float scale;
  const float2* stats;
  const Factors* factors;
  uint32_t scaled;          // whether the operands were
  Half* g;
  float* rests;             // what is left of the label's entry, for dh
  uint64_t stride, plane, tokens;

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t*) const {
    const uint32_t rest = who.vocab - first;
    const float f = scaled ? scale * (factors->down[0] * factors->down[1]) : scale;
#pragma unroll
    for (uint32_t j = 0; j < S::NT; ++j) {
      const uint32_t token = s.n + j * 16;
      const bool live = token < who.n && who.live(token);
      const float2 st = live ? stats[token] : float2{0.0f, 1.0f};
      const float w = live ? who.weight(token) * scale * factors->grad : 0.0f, over = w / st.y;
      const int64_t label = live ? who.label(token) - first - s.m : -1;
      const bool here = label >= 0 && label < 16 * (int64_t)S::MT && label % 32 < 8;
      const uint32_t there = live && s.m < rest ? rest - s.m : 0u;      // of the lane's rows
      if (token >= tokens) continue;
#pragma unroll
      for (uint32_t i = 0; i < S::MT; i += 2) {
        Half out[8][P];
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) {
          float x = exp_of(acc[i + r / 4][j][r % 4] * f - st.x) * over;
          if (here && run_of(i) + r == (uint32_t)label) x -= w;
          x = run_of(i) + r < there ? x : 0.0f;
          split<H, P>(x, out[r]);
          if (here && run_of(i) + r == (uint32_t)label) rests[token] = x - (float)__builtin_bit_cast(H, out[r][0]);
        }
#pragma unroll
        for (uint32_t p = 0; p < P; ++p) {
          Quad q;
#pragma unroll
          for (uint32_t r = 0; r < 4; ++r) q[r] = out[2 * r][p] | (uint32_t)out[2 * r + 1][p] << 16;
          *reinterpret_cast<Quad*>(g + p * plane + token * stride + s.m + run_of(i)) = q;
        }
      }
    }
  }
};

// Rows are the result's columns, columns its rows (tokens for dh, the vocabulary's for dT): fp32 sums, a matrix for every slice
// of K.
struct SumsEnd {
  float* sums;
  uint64_t stride;          // of a row; whole fours
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
  const Factors* factors;
  uint32_t scaled;

  template <class S>
  __device__ __forceinline__ void operator()(const Four (&acc)[S::MT][S::NT], const Spot& s, uint8_t*) const {
    const float f = scaled ? back_of(*factors, 0) : factors->back;
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

// The slices added up.  dh, of rows that count: and what the rounding of the label's entry of G, its largest, has left.
struct JoinArgs {
  uint32_t rows, dim;
  const float* sums;
  uint64_t stride;
  uint32_t slices;
  const Factors* factors;
  uint32_t side;            // of Factors::down; 2: none
  uint32_t of_hidden, add;
  Rows who;
  const float* rests;
  Matrix table;
  uint64_t out_stride;
};
template <class T, class TO>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a, TO* out) {
  const uint32_t blocks = (a.dim + 1023) / 1024;
  const uint32_t c = blockIdx.x % blocks * 1024 + threadIdx.x * 4;
  if (c >= a.dim) return;
  const float f = a.side < 2 ? back_of(*a.factors, a.side) : a.factors->back;
  for (uint32_t i = blockIdx.x / blocks; i < a.rows; i += gridDim.x / blocks) {
    float x[4] = {};
    if (!a.of_hidden || a.who.live(i)) {
#pragma unroll 4
      for (uint32_t k = 0; k < a.slices; ++k) {
        const Four p = *reinterpret_cast<const Four*>(a.sums + ((uint64_t)k * a.rows + i) * a.stride + c);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) x[r] += p[r];
      }
      if (a.rests) {
        float t[4];
        load_row<4>(static_cast<const T*>(a.table.p) + (uint64_t)a.who.label(i) * a.table.stride, c, a.dim, 0.0f, t);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) x[r] = fmaf(a.rests[i], t[r], x[r]);
      }
    }
    float old[4] = {};
    if (a.add) load_row<4>(out + i * a.out_stride, c, a.dim, 0.0f, old);
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) x[r] = fmaf(x[r], f, old[r]);
    store_row<4>(out + i * a.out_stride, c, a.dim, x);
  }
}

// ------------------------------------------------------------------------------ few tokens
// z of up to 16 NT tokens and 64 rows of the table, which are read as they lie in memory, whatever their stride and alignment,
// once, straight into registers.  Bound by HBM: 24 x 2048 x 200 003 bf16 takes 166 us (4.95 TB/s), where tiles of 256 rows through
// LDS took 181 and wanted an aligned table.  For that a wavefront asks for 64 lines of 128 bytes, and the tokens' part, before it
// waits for the first, and eight share K out among them line by line (four 176 us, two 214, sixteen 198; loads past the caches'
// order 194).  Where the vocabulary is small it is what a CU has on its way: 4 x 4096 x 1472 takes 7.4 us, 57 as
// tiles with all of K.  fp32 rows are cut into three planes of bfloat16 on the way, which hold
// 8 + 8 + 8 bits, all there are, so that no row needs to be known before it is multiplied (24 x 2048 x 100 003 228 us, 3.6 TB/s; with
// K in an order that has four lanes read 64 bytes of a row at a time the same).
constexpr uint32_t kFewTokens = 64, kFewGap = 4, kFewWaves = 8, kNoRow = 0xFFFFFFFFu;
struct FewArgs {
  Matrix table;
  uint32_t dim;
  const Half* hidden;       // planes of tokens, rows and K padded with zeros
  uint64_t stride, plane;
};

template <class T>
constexpr uint32_t kFewPlanes = sizeof(T) == 4 ? 3 : 1;

// Eight values of a row as operands.
template <class T>
__device__ __forceinline__ void operands(const float (&x)[8], Quad (&q)[kFewPlanes<T>]) {
  if constexpr (sizeof(T) == 4) {
    float rest[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (uint32_t p = 0; p < 3; ++p) {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t low = __float_as_uint(rest[2 * i]), high = __float_as_uint(rest[2 * i + 1]);
        q[p][i] = low >> 16 | (high & 0xFFFF0000u);
        rest[2 * i] -= __uint_as_float(low & 0xFFFF0000u);
        rest[2 * i + 1] -= __uint_as_float(high & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      q[0][i] = (uint32_t)__builtin_bit_cast(Half, (T)x[2 * i]) | (uint32_t)__builtin_bit_cast(Half, (T)x[2 * i + 1]) << 16;
  }
}

template <class T, uint32_t NT, uint32_t MT, class E>
__global__ __launch_bounds__(kFewWaves* kWave) void few_kernel(FewArgs a, E epilogue) {
  using H = std::conditional_t<std::is_same_v<T, f16_t>, f16_t, bf16_t>;
  constexpr uint32_t P = kFewPlanes<T>, kRows = MT * 16, kWide = kRows + kFewGap, kWaves = kFewWaves;
  __shared__ __attribute__((aligned(16))) float z[kWaves][NT * 16][kWide];
  const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), first = blockIdx.x * kRows, part = (lane >> 4) * 8;
  const T* rows[MT];
#pragma unroll
  for (uint32_t i = 0; i < MT; ++i) rows[i] = static_cast<const T*>(a.table.p) + min(first + i * 16 + (lane & 15), a.table.rows - 1) * a.table.stride;
  const uint32_t token0 = blockIdx.y * kFewTokens;
  const Half* tokens = a.hidden + (token0 + (lane & 15)) * a.stride;
  Four acc[MT][NT];
#pragma unroll
  for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
    for (uint32_t j = 0; j < NT; ++j) acc[i][j] = Four{0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](uint32_t i, const Quad (&q)[P], const Quad (&b)[NT][P]) {
#pragma unroll
    for (uint32_t order = P == 1 ? 1 : P + 1; order-- > 0;)      // the last product of three planes, below 2^-30, is left out
#pragma unroll
      for (uint32_t p = order < P ? 0 : order - P + 1; p < P && p <= order; ++p)
#pragma unroll
        for (uint32_t j = 0; j < NT; ++j) acc[i][j] = mfma<H>(q[p], b[j][order - p], acc[i][j]);
  };
  auto take = [&](uint32_t k, Quad (&b)[NT][P]) {
#pragma unroll
    for (uint32_t j = 0; j < NT; ++j)
#pragma unroll
      for (uint32_t p = 0; p < P; ++p) b[j][p] = *reinterpret_cast<const Quad*>(tokens + p * a.plane + j * 16 * a.stride + k + part);
  };
  constexpr uint32_t kLine = 128 / sizeof(T), kSteps = kLine / kStep, kQuads = sizeof(T) / 2;
  const uint32_t lines = a.dim / kLine;
  for (uint32_t l = wave; l < lines; l += kWaves) {
    Quad raw[kSteps][MT][kQuads], b[kSteps][NT][P];
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) {
      const uint32_t k = l * kLine + s * kStep;
#pragma unroll
      for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
        for (uint32_t c = 0; c < kQuads; ++c) raw[s][i][c] = *reinterpret_cast<const UnalignedQuad*>(rows[i] + k + part + c * 16 / sizeof(T));
      take(k, b[s]);
    }
    // all of them on their way before the first is waited for: left to itself the compiler asks for each where it is used
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s)
#pragma unroll
      for (uint32_t i = 0; i < MT; ++i) {
        if constexpr (P == 1) {
          add(i, raw[s][i], b[s]);
        } else {
          float x[8];
          Quad q[P];
#pragma unroll
          for (uint32_t c = 0; c < 8; ++c) x[c] = __uint_as_float(raw[s][i][c / 4][c % 4]);
          operands<T>(x, q);
          add(i, q, b[s]);
        }
      }
  }
  if (wave == lines % kWaves)
    for (uint32_t k = lines * kLine; k < a.dim; k += kStep) {
      Quad b[NT][P];
      take(k, b);
#pragma unroll
      for (uint32_t i = 0; i < MT; ++i) {
        float x[8];
        Quad q[P];
        load_row<8>(rows[i], k + part, a.dim, 0.0f, x);
        operands<T>(x, q);
        add(i, q, b);
      }
    }
#pragma unroll
  for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
    for (uint32_t j = 0; j < NT; ++j) *reinterpret_cast<Four*>(&z[wave][j * 16 + (lane & 15)][i * 16 + (lane >> 4) * 4]) = acc[i][j];
  __syncthreads();
  // a wavefront has a token's rows at a time
  const bool mine = lane < kRows;
  for (uint32_t token = wave; token < max(NT * 16, min(epilogue.tokens, kFewTokens)); token += kWaves) {
    float sum = 0.0f;
    if (token < NT * 16 && mine)
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) sum += z[w][token][lane];
    epilogue(token0 + token, mine ? first + lane : kNoRow, sum);
  }
}

struct FewStats {
  Rows who;
  float scale;
  float2* partial;
  float* answer;
  uint32_t tokens;
  __device__ __forceinline__ void operator()(uint32_t token, uint32_t v, float product) const {
    if (token >= who.n) return;
    const bool there = v < who.vocab;
    const float x = product * scale, top = wave_max(there ? x : -INFINITY), sum = wave_sum(there ? exp_of(x - top) : 0.0f);
    if (lane_id() == 0) partial[(uint64_t)blockIdx.x * who.n + token] = float2{top, sum};
    if ((int64_t)v == who.label(token) && there) answer[token] = x;
  }
};

template <class H, uint32_t P>
struct FewGrad {
  Rows who;
  uint32_t first;
  float scale;
  const float2* stats;
  const Factors* factors;
  Half* g;
  float* rests;
  uint64_t stride, plane;
  uint32_t tokens;          // with the rows of zeros up to whole tiles of K
  __device__ __forceinline__ void operator()(uint32_t token, uint32_t row, float product) const {
    if (row == kNoRow) return;
    const bool live = token < who.n && who.live(token);
    float x = 0.0f;
    const int64_t v = (int64_t)first + row;
    if (live && v < (int64_t)who.vocab) {
      const float2 st = stats[token];
      const float w = who.weight(token) * scale * factors->grad;
      x = exp_of(product * scale - st.x) * (w / st.y);
      if (v == who.label(token)) x -= w;
    }
    Half out[P];
    split<H, P>(x, out);
    if (live && v == who.label(token)) rests[token] = x - (float)__builtin_bit_cast(H, out[0]);
#pragma unroll
    for (uint32_t p = 0; p < P; ++p) g[p * plane + token * stride + row] = out[p];
  }
};

template <class TO>
__global__ __launch_bounds__(256) void zero_rows_kernel(uint64_t rows, uint32_t dim, TO* out, uint64_t stride) {
  for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (uint32_t c = threadIdx.x; c < dim; c += 256) out[r * stride + c] = (TO)0.0f;
}

// ------------------------------------------------------------------------------ host
using Large = Shape<2, 4, 8, 4, 5>;   // 256 x 256, all of a CU's LDS: five operands' tiles
using Small = Shape<2, 2, 4, 4, 5>;   // 128 x 128, half of it

template <class T>
struct Kind {                      // how matrices of a type are multiplied
  using H = std::conditional_t<std::is_same_v<T, bf16_t>, bf16_t, f16_t>;
  static constexpr uint32_t P = sizeof(T) == 4 ? 2 : 1;
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

constexpr uint32_t kCus = 256;
uint64_t tiles(uint64_t m, uint64_t n, uint64_t tm, uint64_t tn) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); }
// What a product of m x n takes for each value of K, in hundredths of what 256 large tiles do (32 ns: 4096 x 16384 x 2048 262 us),
// one to a CU.  Of small tiles a CU has two, which together are half as large and take 88, or one, which takes 72.
uint64_t cost_large(uint64_t m, uint64_t n, uint64_t slices) { return (tiles(m, n, Large::TM, Large::TN) * slices + kCus - 1) / kCus * 100; }
uint64_t cost_small(uint64_t m, uint64_t n, uint64_t slices) {
  const uint64_t all = tiles(m, n, Small::TM, Small::TN) * slices, rest = all % (2 * kCus);
  return all / (2 * kCus) * 88 + (rest > kCus ? 88 : rest ? 72 : 0);
}
bool large_goes(const Product& g) { return cost_large(g.m, g.n, g.slices) <= cost_small(g.m, g.n, g.slices); }
uint64_t cost(uint64_t m, uint64_t n, uint64_t slices) { return std::min(cost_large(m, n, slices), cost_small(m, n, slices)); }

template <class H, bool TALL_A, bool TALL_B, class S, class E>
void run_as(const Product& g, const E& end, hipStream_t stream) {
  hipLaunchKernelGGL((product_kernel<H, S, TALL_A, TALL_B, E>), dim3((uint32_t)(tiles(g.m, g.n, S::TM, S::TN) * g.slices)), dim3(S::kThreads), 0,
                     stream, g, end);
}
template <class H, bool TALL_A, bool TALL_B, class E>
void run(const Product& g, const E& end, hipStream_t stream) {
  if (large_goes(g))
    run_as<H, TALL_A, TALL_B, Large>(g, end, stream);
  else
    run_as<H, TALL_A, TALL_B, Small>(g, end, stream);
}

// Rows of a workgroup of few tokens: fewer where 64 to each would not give every CU one (4 x 4096 x 1472 bf16 7.4 us, 15.2 with 64;
// 38 x 6205 x 1216 32, 49).
uint64_t few_rows(uint64_t vocab) { return vocab <= 64 * kCus ? 16 : 64; }
uint64_t few_blocks(uint64_t vocab) { return (vocab + 63) / 64 * (64 / few_rows(vocab)); }

struct Sizes {
  uint64_t depth, tokens, piece;      // dim and n in whole tiles of K; tokens of the vocabulary at a time
  uint32_t planes, g_planes, slices;
};
// Bytes of a piece's G and table, about.  More than the last-level cache holds, since fewer tokens of the vocabulary at a time end
// dh's sums, which every piece reads and writes, too often.
constexpr uint64_t kBudget = 320ull << 20;
constexpr uint64_t kSliceMin = 128;          // K that a product's slice has, at least ...
constexpr uint32_t kSlicesMost = 64;         // ... and slices, at most ...
constexpr uint64_t kSumsMost = 64ull << 20;  // ... and bytes of dT's slices; of which there is one where it has more small tiles than
constexpr uint64_t kTilesFew = kCus / 2;     // this: 2048 x 768 x 32 000 fp32 takes 1190 us so, 1310 with slices of a last piece's dT
constexpr uint64_t kLaunchCost = 30000;      // a launch's own time, about 10 us
constexpr uint32_t kManyTokens = 4096;       // from which on sums in fp32 are further off than two planes of bfloat16

// Into how many slices K of a product is cut, and what it costs then.  A slice's results are written and read again, 8 bytes
// a value at 5 TB/s, and added up in turn.
struct Slices {
  uint32_t count;
  uint64_t cost;
};
Slices slices_for(uint64_t m, uint64_t n, uint64_t k, uint64_t products, uint64_t most) {
  Slices best{1, cost(m, n, 1) * k * products};
  const uint64_t large = tiles(m, n, Large::TM, Large::TN), small = tiles(m, n, Small::TM, Small::TN);
  // as many as fill the CUs one to three times over with large tiles, or half, once and twice with small ones
  for (uint64_t s : {kCus / large, 2 * kCus / large, 3 * kCus / large, kCus / small, 2 * kCus / small, 4 * kCus / small}) {
    s = std::min({s, (uint64_t)kSlicesMost, most, k / kSliceMin});
    if (s < 2) continue;
    const uint64_t c = cost(m, n, s) * ((k + s - 1) / s) * products + s * (m * n / 200 + 300) + kLaunchCost / 2;
    if (c < best.cost) best = Slices{(uint32_t)s, c};
  }
  return best;
}
Slices table_slices(uint64_t rows, uint64_t dim, uint64_t depth, uint64_t tokens, uint64_t products) {
  const bool few = tiles(dim, rows, Small::TM, Small::TN) <= kTilesFew;
  return slices_for(dim, rows, tokens, products, few ? kSumsMost / (rows * depth * 4) : 1);
}
// G's planes; dtable: whether it is asked for.
uint32_t planes_of_g(uint32_t n, uint32_t type, uint32_t dtable_type, bool dtable) {
  if (type == CVLC_F32) return 2;
  if (!dtable) return 1;
  return type == CVLC_BF16 && dtable_type == CVLC_F32 && n < kManyTokens ? 3 : 2;
}
// g_planes: 0 for the loss.
Sizes sizes_for(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type, uint32_t g_planes) {
  Sizes z{};
  z.depth = pad_to(dim, kDepth);
  z.tokens = pad_to(n, kDepth);
  z.planes = type == CVLC_F32 ? 2 : 1;
  z.g_planes = g_planes;
  z.slices = 1;
  const uint64_t each = z.depth * z.planes * 2 + z.tokens * z.g_planes * 2;
  const uint64_t whole = pad_to(vocab, kPadTo) / kPadTo, most = std::min(whole, std::max<uint64_t>(1, kBudget / each / kPadTo));
  z.piece = most * kPadTo;
  if (!g_planes) return z;
  // A launch lasts as long as its fullest CU: of the pieces' sizes the one whose launches take least together.
  const uint64_t of_z = z.planes == 1 ? 1 : 3, of_g = z.planes == 1 ? z.g_planes : 3;
  auto of_piece = [&](uint64_t t, uint32_t* slices) {
    const uint64_t rows = t * kPadTo;
    const Slices h = slices_for(dim, n, rows, of_z, kSlicesMost);
    *slices = h.count;
    return h.cost + cost(rows, n, 1) * z.depth * of_z + table_slices(rows, dim, z.depth, z.tokens, of_g).cost + 3 * kLaunchCost;
  };
  uint64_t best = ~0ull;
  const uint64_t step = std::max<uint64_t>(1, most / 64);
  for (uint64_t t = most; t >= std::max<uint64_t>(1, most / 2); t -= std::min(step, t)) {
    uint32_t slices = 1, other;
    const uint64_t rest = whole % t, c = of_piece(t, &slices) * (whole / t) + (rest ? of_piece(rest, &other) : 0);
    if (c < best) {
      best = c;
      z.piece = t * kPadTo;
      z.slices = slices;
    }
  }
  return z;
}

struct Room {                          // parts of a workspace
  uint8_t* base;
  uint64_t used;
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
  Matrix hidden_matrix() const { return Matrix{hidden, hidden_stride, n}; }
  Matrix table_matrix(uint64_t first, uint32_t count) const {
    return Matrix{static_cast<const uint8_t*>(table) + first * table_stride * type_bytes(type), table_stride, count};
  }
};

// Whether a matrix can be multiplied as it is: rows that begin at 16 bytes and end with a tile of K, near enough to each other
// for 32-bit offsets inside a tile.
bool as_it_is(const void* p, uint64_t stride, uint32_t dim, uint32_t type) {
  return type != CVLC_F32 && dim % kDepth == 0 && stride % 8 == 0 && stride < (1u << 22) && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// Of more than 64, 64 at a time, while a CU has no more than one of them: 96 x 2816 x 1983 fp32 43 us against 113 of 16 small tiles
// (256 x 2816 x 4000, four to a CU, 152 against 115).
constexpr uint32_t kFewMany = 256;
bool few_of_many(uint32_t n, uint32_t vocab) {
  return n <= kFewMany && few_rows(vocab) == 16 && (n + kFewTokens - 1) / kFewTokens * few_blocks(vocab) <= kCus;
}
bool may_be_few(uint32_t n, uint32_t vocab) { return n <= kFewTokens || few_of_many(n, vocab); }

// Few tokens, that is whether logits come from the rows as they are.  Of more than 32, tiles that stay in LDS take less of a table
// that they can read as it is and that fills them: 60 x 2048 x 200 003 bf16 227 us against 292 (3 values to a row more 583 against
// 387, fp32 835 against 346 for half as many rows).
bool few_tokens(const Call& c) {
  if (c.n > kFewTokens) return few_of_many(c.n, c.vocab);
  return c.n <= kFewTokens / 2 || few_rows(c.vocab) == 16 || !as_it_is(c.table, c.table_stride, c.dim, c.type);
}

// The parts of a workspace; with base = null only its size.
struct Parts {
  Factors* factors;
  float* tops;
  Half *hidden, *table, *few;   // few: hidden rows beside a table that is read as it is
  Parts(Room& r, const Sizes& z, uint32_t n, uint32_t vocab) {
    factors = r.take<Factors>(1);
    tops = r.take<float>(z.planes > 1 ? 2 * kSurveyGrid : 0);
    hidden = r.take<Half>(z.planes * z.tokens * z.depth);
    table = r.take<Half>(z.planes * z.piece * z.depth);
    few = r.take<Half>(may_be_few(n, vocab) ? 3 * z.tokens * z.depth : 0);
  }
};
struct LossParts : Parts {
  float2* partial;
  float* answer;
  uint64_t bytes;
  LossParts(Room r, const Sizes& z, uint32_t n, uint32_t vocab) : Parts(r, z, n, vocab) {
    partial = r.take<float2>(std::max(may_be_few(n, vocab) ? few_blocks(vocab) : 0, vocab / Small::TM + vocab / z.piece + 2) * n);
    answer = r.take<float>(n);
    bytes = r.used;
  }
};
struct GradParts : Parts {
  Half* g;
  float *sums, *table_sums, *rests;
  uint64_t bytes;
  GradParts(Room r, const Sizes& z, uint32_t n, uint32_t vocab) : Parts(r, z, n, vocab) {
    g = r.take<Half>(z.g_planes * z.tokens * z.piece);
    sums = r.take<float>(z.slices * n * z.depth);
    table_sums = r.take<float>(std::min(kSumsMost / 4, kSlicesMost * z.piece * z.depth));
    rests = r.take<float>(n);
    bytes = r.used;
  }
};

// The factors that a call goes by.
void find_factors(const Call& c, const Sizes& z, const Parts& parts, uint32_t* status, hipStream_t stream) {
  const Matrix hidden = c.hidden_matrix(), table = c.table_matrix(0, c.vocab), none{};
  if (z.planes == 1) {
    hipLaunchKernelGGL(factors_kernel, dim3(1), dim3(1024), 0, stream, c.who, c.scale, nullptr, 0, none, none, c.dim, parts.factors, status);
  } else if ((uint64_t)(c.n + (uint64_t)c.vocab) * c.dim <= kSurveyAlone) {
    hipLaunchKernelGGL(factors_kernel, dim3(1), dim3(1024), 0, stream, c.who, c.scale, nullptr, 0, hidden, table, c.dim, parts.factors, status);
  } else {
    const uint32_t grid = (uint32_t)std::min<uint64_t>(((uint64_t)std::max(c.n, c.vocab) * c.dim + kSurveyEach - 1) / kSurveyEach, kSurveyGrid);
    hipLaunchKernelGGL(survey_kernel, dim3(grid, 2), dim3(kSurveyBlock), 0, stream, hidden, table, c.dim, c.who, parts.tops);
    hipLaunchKernelGGL(factors_kernel, dim3(1), dim3(1024), 0, stream, c.who, c.scale, parts.tops, grid, none, none, c.dim, parts.factors,
                       status);
  }
}

template <class T, class H = typename Kind<T>::H, uint32_t P = Kind<T>::P>
void pack(const Call& c, const PackArgs& first, const PackArgs& second, hipStream_t stream) {
  auto grid = [](const PackArgs& a) {
    return (uint32_t)std::min<uint64_t>(((uint64_t)a.rows_to * (a.stride / 8) + kPackBlock - 1) / kPackBlock, 1u << 16);
  };
  const uint32_t one = grid(first), two = grid(second);
  if (one + two)
    hipLaunchKernelGGL((pack_kernel<T, H, P>), dim3(one + two), dim3(kPackBlock), 0, stream, first, second, one, c.who);
}

// z of few tokens, from the table's rows [first, first + rows) as they are; the tokens' planes are made with the first.
template <class T, class E>
void run_few(const Call& c, const Sizes& z, const Parts& parts, uint64_t first, uint32_t rows, const E& end, hipStream_t stream) {
  constexpr uint32_t P = kFewPlanes<T>;
  using H = std::conditional_t<std::is_same_v<T, f16_t>, f16_t, bf16_t>;
  const uint32_t groups = (c.n + kFewTokens - 1) / kFewTokens;
  const uint64_t plane = groups * kFewTokens * z.depth;
  if (first == 0) pack<T, H, P>(c, PackArgs{c.hidden_matrix(), c.dim, groups * kFewTokens, parts.few, z.depth, plane, nullptr, 1}, PackArgs{}, stream);
  const FewArgs a{c.table_matrix(first, rows), c.dim, parts.few, z.depth, plane};
  auto go = [&](auto tokens) {
    constexpr uint32_t NT = decltype(tokens)::value;
    const uint32_t blocks = few_blocks(rows);
    if (few_rows(rows) == 16)
      hipLaunchKernelGGL((few_kernel<T, NT, 1, E>), dim3(blocks, groups), dim3(kFewWaves * kWave), 0, stream, a, end);
    else
      hipLaunchKernelGGL((few_kernel<T, NT, 4, E>), dim3(blocks, groups), dim3(kFewWaves * kWave), 0, stream, a, end);
  };
  if (c.n <= 16)
    go(std::integral_constant<uint32_t, 1>{});
  else if (c.n <= 32)
    go(std::integral_constant<uint32_t, 2>{});
  else
    go(std::integral_constant<uint32_t, 4>{});
}

template <class T>
void loss_of(const Call& c, const Sizes& z, const LossParts& parts, float* loss, float2* stats, uint32_t* status, hipStream_t stream) {
  using H = typename Kind<T>::H;
  constexpr uint32_t P = Kind<T>::P;
  uint32_t tile = 0;
  if (few_tokens(c)) {
    run_few<T>(c, z, parts, 0, c.vocab, FewStats{c.who, c.scale, parts.partial, parts.answer, 0}, stream);
    tile = few_blocks(c.vocab);
  } else {
    const bool hidden_goes = as_it_is(c.hidden, c.hidden_stride, c.dim, c.type), table_goes = as_it_is(c.table, c.table_stride, c.dim, c.type);
    if (P > 1) find_factors(c, z, parts, nullptr, stream);
    PackArgs hidden{c.hidden_matrix(), c.dim, c.n, parts.hidden, z.depth, z.tokens * z.depth, parts.factors->up, 0};
    if (hidden_goes) hidden.rows_to = 0;
    Product g{};
    g.b = hidden_goes ? Operand{static_cast<const Half*>(c.hidden), c.hidden_stride, 0, 0, c.n} : Operand{parts.hidden, z.depth, z.tokens * z.depth, 0, c.n};
    g.n = c.n;
    g.k = (uint32_t)z.depth;
    g.slices = 1;
    set_pairs(g, P, P);
    const uint64_t step = table_goes ? pad_to(c.vocab, kPadTo) : z.piece;
    for (uint64_t first = 0; first < c.vocab; first += step) {
      g.m = (uint32_t)std::min<uint64_t>(step, c.vocab - first);
      PackArgs table{c.table_matrix(first, g.m), c.dim, table_goes ? 0 : g.m, parts.table, z.depth, z.piece * z.depth, parts.factors->up + 1, 0};
      pack<T>(c, hidden, table, stream);
      hidden.rows_to = 0;
      g.a = table_goes ? Operand{static_cast<const Half*>(c.table) + first * c.table_stride, c.table_stride, 0, 0, g.m}
                       : Operand{parts.table, z.depth, z.piece * z.depth, 0, g.m};
      const StatsEnd end{c.who, (uint32_t)first, tile, c.scale, P > 1 ? parts.factors : nullptr, parts.partial, parts.answer};
      run<H, false, false>(g, end, stream);
      const uint32_t rows = large_goes(g) ? Large::TM : Small::TM;
      tile += (g.m + rows - 1) / rows;
    }
  }
  const uint32_t log2 = join_tokens_log2(c.n);
  hipLaunchKernelGGL(loss_kernel, dim3((c.n + (1u << log2) - 1) >> log2), dim3(join_block(c.n, tile)), 0, stream, c.who, tile, log2, parts.partial,
                     parts.answer, loss, stats, status);
}

template <class T, class TO>
void join(const JoinArgs& a, TO* out, hipStream_t stream) {
  const uint32_t blocks = (a.dim + 1023) / 1024;
  hipLaunchKernelGGL((join_kernel<T, TO>), dim3(std::min(a.rows, std::max(1u, 8192u / blocks)) * blocks), dim3(256), 0, stream, a, out);
}

template <class T, class TO, uint32_t PG>
void grad_of(const Call& c, const Sizes& z, const GradParts& parts, const float2* stats, T* dhidden, uint64_t dhidden_stride, TO* dtable,
             uint64_t dtable_stride, bool accumulate, uint32_t* status, hipStream_t stream) {
  using H = typename Kind<T>::H;
  constexpr uint32_t P = Kind<T>::P;
  const bool table_goes = as_it_is(c.table, c.table_stride, c.dim, c.type), few = few_tokens(c);
  find_factors(c, z, parts, status, stream);
  PackArgs hidden{c.hidden_matrix(), c.dim, (uint32_t)z.tokens, parts.hidden, z.depth, z.tokens * z.depth, parts.factors->up, 1};
  for (uint64_t first = 0; first < c.vocab; first += z.piece) {
    const uint32_t count = (uint32_t)std::min<uint64_t>(z.piece, c.vocab - first);
    PackArgs table{c.table_matrix(first, count), c.dim, table_goes || (few && !dhidden) ? 0 : count, parts.table, z.depth, z.piece * z.depth,
                   parts.factors->up + 1, 0};
    pack<T>(c, hidden, table, stream);
    hidden.rows_to = 0;
    Product g{};
    g.slices = 1;
    g.a = table_goes ? Operand{static_cast<const Half*>(c.table) + first * c.table_stride, c.table_stride, 0, c.dim, count}
                     : Operand{parts.table, z.depth, z.piece * z.depth, (uint32_t)z.depth, count};
    g.b = Operand{parts.hidden, z.depth, z.tokens * z.depth, (uint32_t)z.depth, (uint32_t)z.tokens};
    g.m = count;
    g.n = c.n;
    g.k = (uint32_t)z.depth;
    set_pairs(g, P, P);
    const Operand of_g{parts.g, z.piece, z.tokens * z.piece, (uint32_t)z.piece, (uint32_t)z.tokens};
    if (few)
      run_few<T>(c, z, parts, first, count, FewGrad<H, PG>{c.who, (uint32_t)first, c.scale, stats, parts.factors, parts.g, parts.rests, z.piece,
                                                           z.tokens * z.piece, (uint32_t)z.tokens}, stream);
    else
      run<H, false, false>(g, GradEnd<H, PG>{c.who, (uint32_t)first, c.scale, stats, parts.factors, P > 1, parts.g, parts.rests, z.piece,
                                             z.tokens * z.piece, z.tokens}, stream);
    if (dhidden) {
      Product y{};
      y.a = g.a;
      y.b = of_g;
      y.m = c.dim;
      y.n = c.n;
      y.k = (uint32_t)pad_to(count, kDepth);
      y.slices = z.slices;
      set_pairs(y, P, P);   // 16-bit results: G's first plane alone
      run<H, true, false>(y, SumsEnd{parts.sums, z.depth, c.n, first > 0}, stream);
    }
    if (dtable) {
      Product t{};
      t.a = g.b;
      t.b = of_g;
      t.m = c.dim;
      t.n = count;
      t.k = (uint32_t)z.tokens;
      set_pairs(t, P, PG);
      t.slices = table_slices(count, c.dim, z.depth, z.tokens, t.pairs).count;
      TO* out = dtable + first * dtable_stride;
      if (t.slices == 1) {
        run<H, true, true>(t, TableEnd<TO>{out, dtable_stride, c.dim, count, accumulate, parts.factors, P > 1}, stream);
      } else {
        run<H, true, true>(t, SumsEnd{parts.table_sums, z.depth, count, 0}, stream);
        join<T>(JoinArgs{count, c.dim, parts.table_sums, z.depth, t.slices, parts.factors, P > 1 ? 0u : 2u, 0, accumulate, c.who, nullptr, Matrix{},
                         dtable_stride}, out, stream);
      }
    }
  }
  if (dhidden)
    join<T>(JoinArgs{c.n, c.dim, parts.sums, z.depth, z.slices, parts.factors, P > 1 ? 1u : 2u, 1, 0, c.who, P == 1 ? parts.rests : nullptr,
                     c.table_matrix(0, c.vocab), dhidden_stride}, dhidden, stream);
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
  const uint64_t tiles = ((uint64_t)c.n / 128 + 1) * (pad_to(c.vocab, kPadTo) / 128), packs = ((uint64_t)std::max(c.n, c.vocab) / 64 + 1) * (c.dim / 64 + 1);
  if (tiles >= 1ull << 23 || packs >= 1ull << 24 || (c.n <= kFewTokens && c.vocab >= 1u << 28)) return CVLC_ERR_ARG;
  return CVLC_OK;
}

}  // namespace
}  // namespace cvlc

extern "C" {

size_t cvlc_linear_xent_workspace_bytes(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type) {
  using namespace cvlc;
  if (!n || !vocab || !dim) return 256;
  return (size_t)LossParts(Room{}, sizes_for(n, vocab, dim, type, 0), n, vocab).bytes;
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
  const Sizes z = sizes_for(n, vocab, dim, type, 0);
  const LossParts room(Room{static_cast<uint8_t*>(d_workspace), 0}, z, n, vocab);
  by_type(type, [&](auto t) {
    loss_of<decltype(t)>(c, z, room, d_loss, reinterpret_cast<float2*>(d_stats), d_status, static_cast<hipStream_t>(hip_stream));
  });
  return hip_check(hipGetLastError());
}

size_t cvlc_linear_xent_grad_workspace_bytes(uint32_t n, uint32_t vocab, uint32_t dim, uint32_t type, uint32_t dtable_type) {
  using namespace cvlc;
  if (!n || !vocab || !dim) return 256;
  uint64_t most = 0;
  for (bool dtable : {false, true}) most = std::max(most, GradParts(Room{}, sizes_for(n, vocab, dim, type, planes_of_g(n, type, dtable_type, dtable)), n, vocab).bytes);
  return (size_t)most;
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
  const Sizes z = sizes_for(n, vocab, dim, type, planes_of_g(n, type, out_type, d_dtable));
  const GradParts room(Room{static_cast<uint8_t*>(d_workspace), 0}, z, n, vocab);
  by_type(type, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto to, auto planes) {
      using TO = decltype(to);
      grad_of<T, TO, decltype(planes)::value>(c, z, room, reinterpret_cast<const float2*>(d_stats), static_cast<T*>(d_dhidden), dhidden_stride,
                                              static_cast<TO*>(d_dtable), dtable_stride, accumulate, d_status, stream);
    };
    using One = std::integral_constant<uint32_t, 1>;
    using Two = std::integral_constant<uint32_t, 2>;
    using Three = std::integral_constant<uint32_t, 3>;
    if constexpr (sizeof(T) == 4) {
      go(T{}, Two{});
    } else {
      if (!d_dtable)
        go(T{}, One{});
      else if (out_type == type)
        go(T{}, Two{});
      else if (z.g_planes == 2)
        go(0.0f, Two{});
      else if constexpr (std::is_same_v<T, bf16_t>)
        go(0.0f, Three{});
    }
  });
  return hip_check(hipGetLastError());
}

}  // extern "C"
