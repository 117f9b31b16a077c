// Orthogonalised updates: X <- a X + (b A + c A A) X, A = X X^T, from X = U / |U| (Frobenius), for all matrices of a layout in all replicas.
//
// An iteration is three launches over the tiles of a group of matrices: A (k_ortho_gram), B = b A + c A A (k_ortho_gram again, as A is its own
// transpose), and a X + B X (k_ortho_next; the last one, k_ortho_end, stores the matrix or takes the step).  A and B are symmetric: only the tiles of their
// lower half are computed, each stored twice, which leaves 3 p^2 q + p^3 of 4 p^2 q + 2 p^3 operations.  B X sums over X's rows: its tiles come into LDS as they
// lie and are turned on the way to the registers.
//
// Operands are half precision times a power of two (their spectral norms are bounded, so their elements are, see dadam_ortho.cpp).  Results of
// 32 bits have two halves an element (dadam_mfma.h): the error of five iterations is 2e-7 to 3e-6 of the result, by how fast the singular values
// fall.  For bfloat16 results one half is enough in the products, but not for X itself: what X loses to 11 bits in the directions of small singular
// values grows by a = 3.4 an iteration, 1e-3 of the result for equal singular values, 1.4e-2 for ones that fall by 1000 in 50.  a X is therefore taken
// from two halves as well (1.4e-3 and 5e-4), the second of which no product reads.  B's diagonal is most of it where q is much larger than p (A is near I / p), so it does not go
// through the product either, but into a X's factor, a row's own: the error of a random 150 x 1189 is 5.8e-4 instead of 1.6e-3, of 12 x 5948 7.1e-4 instead of 3.2e-3,
// of 1024 x 1024 7.4e-4 instead of 1.3e-3 (modelled; what bfloat16 itself costs is 1.7e-3).
#include "dadam_mfma.h"
#include "dadam_ortho.h"
#include "dadam_ortho_source.h"

namespace dadam {
namespace {

extern __shared__ char ortho_lds[];

// Of A and B, whose operands both lie by rows, and of a X + B X (transposed: q by p), whose X lies by columns.
template <int PLANES, int EDGE, int BUFFERS>
using GramTile = TileOf<Half, PLANES, EDGE, BUFFERS, false, false>;
template <int PLANES, int EDGE, int BUFFERS>
using NextTile = TileOf<Half, PLANES, EDGE, BUFFERS, true, false>;

__device__ __forceinline__ uint64_t x_at(const OrthoPlaces& w, uint32_t which) { return which ? w.x[1] : w.x[0]; }

// A workgroup's matrix, the tile of it and where its workspace begins.
struct Unit {
  OrthoTask t;
  uint32_t tile;
  uint64_t base;
};
enum Kind : int { kGram = 0, kWhole = 1, kCells = 2, kSmallGram = 3 };
template <Kind KIND>
__device__ __forceinline__ Unit find_unit(const OrthoSpan& s) {
  const uint32_t u = s.first_unit + die_run(blockIdx.x, gridDim.x, s.n_xcd);
  const uint32_t k = global<const uint32_t>(s.units)[u];
  Unit r;
  struct Words {
    uint32_t w[sizeof(OrthoTask) / 4];
  } words;
#pragma unroll
  for (uint32_t i = 0; i < sizeof(OrthoTask) / 4; ++i) words.w[i] = global<const uint32_t>(s.tasks + k)[i];
  r.t = __builtin_bit_cast(OrthoTask, words);
  r.tile = u - (KIND == kGram ? r.t.gram_units : KIND == kWhole ? r.t.whole_units : KIND == kCells ? r.t.cell_units : r.t.small_units);
  r.base = s.workspace + (uint64_t)blockIdx.y * s.stride + (r.t.at - s.before);
  return r;
}

// Where a cell of X begins in the matrix as it lies in memory, and the matrix's own rows and columns.
struct Cell {
  uint32_t r0, c0, rows, cols;
};
__device__ __forceinline__ Cell cell_of(const Unit& u) {
  const uint32_t across = u.t.Q / kOrthoCell, i = u.tile / across, j = u.tile % across;
  Cell c;
  c.r0 = (u.t.tall ? j : i) * kOrthoCell;
  c.c0 = (u.t.tall ? i : j) * kOrthoCell;
  c.rows = u.t.tall ? u.t.q : u.t.p;
  c.cols = u.t.tall ? u.t.p : u.t.q;
  return c;
}

// Squares of a cell, in 64 bits, to its place among the matrix's partial sums.  (Bound by memory, as k_ortho_begin is: 25 million elements of eight bfloat16 replicas, read
// twice, 40 and 72 us for 150 and 350 MB.)
template <typename GT, int PLANES, int N>
__global__ __launch_bounds__(256) void k_ortho_norm(OrthoBeginArgs<N> a) {
  const Unit u = find_unit<kCells>(a.s);
  const Cell c = cell_of(u);
  const uint32_t row = blockIdx.y, col = c.c0 + threadIdx.x % 16 * 8, n = left(c.cols, col);
  const uint64_t g = (uint64_t)a.grad[row], mh = (uint64_t)a.m_hat[row];
  double sum = 0.0;
  if (n)
    for (uint32_t r = c.r0 + threadIdx.x / 16; r < c.r0 + kOrthoCell && r < c.rows; r += 16) {
      const uint64_t e = u.t.first + (uint64_t)r * u.t.ld + col;
      float gv[8], m[8], v[8];
      load_source<GT>(a.c, a.source, g, mh, e, n, gv, m, v);
      sum = add_squares(v, sum);
    }
  __shared__ double parts[4];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) global<double>(u.base + ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts).sums)[u.tile] = parts[0] + parts[1] + parts[2] + parts[3];
}

// X from the matrix, and of a step lines 9 to 13 of Algorithm 3 for the first moment and the accumulator.
constexpr uint32_t kTurnPitch = kOrthoCell + 1;
template <typename GT, int PLANES, int N>
__global__ __launch_bounds__(256) void k_ortho_begin(OrthoBeginArgs<N> a) {
  const Unit u = find_unit<kCells>(a.s);
  const Cell c = cell_of(u);
  const uint32_t row = blockIdx.y, tiles = (u.t.P / kOrthoCell) * (u.t.Q / kOrthoCell);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  float DADAM_LDS* tile = (float DADAM_LDS*)ortho_lds;
  __shared__ double parts[4];
  double sum = 0.0;
  for (uint32_t k = threadIdx.x; k < tiles; k += 256) sum += global<const double>(u.base + w.sums)[k];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = sum;
  __syncthreads();
  const float factor = (float)((double)a.scale / (sqrt(parts[0] + parts[1] + parts[2] + parts[3]) + 1e-7));
  const uint64_t g = (uint64_t)a.grad[row], mh = (uint64_t)a.m_hat[row], acc = (uint64_t)a.acc[row];
  const uint32_t k8 = threadIdx.x % 16 * 8, n = left(c.cols, c.c0 + k8);
  for (uint32_t r = threadIdx.x / 16; r < kOrthoCell; r += 16) {
    float v[8] = {};
    if (c.r0 + r < c.rows && n) {
      const uint64_t e = u.t.first + (uint64_t)(c.r0 + r) * u.t.ld + c.c0 + k8;
      float gv[8], m[8];
      load_source<GT>(a.c, a.source, g, mh, e, n, gv, m, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= factor;
      if (a.source != kOrthoGiven) move_moment(a.c, a.phase, mh, acc, e, n, gv, m);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[r * kTurnPitch + k8 + k] = v[k];
  }
  __syncthreads();
  for (uint32_t r = threadIdx.x / 16; r < kOrthoCell; r += 16) {
    uint32_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = halves<Half>(u.t.tall ? tile[(k8 + k) * kTurnPitch + r] : tile[r * kTurnPitch + k8 + k]);
    const uint32_t p = (u.t.tall ? c.c0 : c.r0) + r, q = (u.t.tall ? c.r0 : c.c0) + k8;
    store8<PLANES>(u.base + w.x[0], p, u.t.Q, q, x);
    if constexpr (PLANES == 1) global<uint4v>(u.base + w.low + ((uint64_t)p * u.t.Q + q) * 2)[0] = highs(x);
  }
}

__device__ __forceinline__ void to_words(const float (&v)[8], uint32_t (&w)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[k]);
}

// The row of a tile among those of the lower half.
__device__ __forceinline__ uint32_t lower_row(uint32_t tile) {
  uint32_t i = (uint32_t)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);  // (the root may round across the border of a row of tiles)
  while (i * (i + 1) / 2 > tile) --i;
  while ((i + 1) * (i + 2) / 2 <= tile) ++i;
  return i;
}

// A tile (i, j), j <= i, of A = X X^T or of B = b A + c A A without its diagonal, and its mirror image.  (100 million elements of matrices 1024 wide: 690 TFLOP/s of the lower
// half by small tiles, bfloat16; 75 million in 32 bits 1070 of instructions by large ones.  What it loses to the products alone is the ends of its rounds of tiles.)
// A large tile on the diagonal mirrors its own lower quarter, as small tiles there do: with two planes the sums of an element and of its mirror image come in another order (low
// high and high low change places), and the tiles' size, which goes by the workspace, is to change no bit.
template <int PLANES, int EDGE, int BUFFERS, bool SQUARE>
__global__ __launch_bounds__(2 * EDGE) void k_ortho_gram(OrthoStepArgs a) {
  using T = GramTile<PLANES, EDGE, BUFFERS>;
  const Unit u = find_unit < EDGE == (int)kLargeEdge ? kGram : kSmallGram > (a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  const uint32_t i = lower_row(u.tile), j = u.tile - i * (i + 1) / 2, inner = SQUARE ? u.t.P : u.t.Q;
  const uint64_t pitch = (uint64_t)inner * 2 * PLANES;
  const uint64_t in = u.base + (SQUARE ? w.a : x_at(w, a.from));
  char DADAM_LDS* lds = (char DADAM_LDS*)ortho_lds;
  T t;
  t.product(operand(in + (uint64_t)i * T::kM * pitch, pitch), operand(in + (uint64_t)j * T::kN * pitch, pitch), (uint32_t)(pitch / kStageBytes), lds);
  const uint64_t out = u.base + (SQUARE ? w.b : w.a);
  constexpr bool kQuarters = EDGE == (int)kLargeEdge && PLANES == 2;
  auto above = [&](uint32_t m, uint32_t n) { return kQuarters && i == j && m / kSmallEdge < n / kSmallEdge; };  // of the quarter that is a mirror image
  t.hand_out(lds, i != j || kQuarters,
             [&](uint32_t m, uint32_t n) {
               if constexpr (SQUARE) return load8<PLANES>(u.base + w.a, j * T::kN + n, u.t.P, i * T::kM + m);
               else return Nothing{};
             },
             [&](uint32_t m, uint32_t n, float (&v)[8], const auto& held) {
               if (above(m, n)) return;
               uint32_t words[8];
               const uint32_t on_diagonal = j * T::kN + n - (i * T::kM + m);
#pragma unroll
               for (int k = 0; k < 8; ++k) {
                 if constexpr (SQUARE) {
                   v[k] = fmaf(value_of<Half, PLANES == 2>(held, k), a.gain, v[k] * a.fresh);
                   if (on_diagonal == (uint32_t)k) {
                     global<float>(u.base + w.diagonal)[j * T::kN + n] = v[k];
                     v[k] = 0.f;
                   }
                 } else {
                   v[k] *= a.fresh;
                 }
                 words[k] = operand_word<Half, PLANES>(v[k]);
                 v[k] = __uint_as_float(words[k]);
               }
               store8<PLANES>(out, j * T::kN + n, u.t.P, i * T::kM + m, words);
             },
             [&](uint32_t m, uint32_t n, const float (&v)[8]) {
               if (kQuarters && i == j && m / kSmallEdge <= n / kSmallEdge) return;
               uint32_t words[8];
               to_words(v, words);
               store8<PLANES>(out, i * T::kM + m, u.t.P, j * T::kN + n, words);
             });
}

// X X^T of a matrix whose tiles would leave most of the chip idle for the length of Q: a range of columns (blockIdx.z), 32 bits, with its mirror image.
template <int PLANES, int BUFFERS>
__global__ __launch_bounds__(2 * kSmallEdge) void k_ortho_part(OrthoStepArgs a) {
  using T = GramTile<PLANES, (int)kSmallEdge, BUFFERS>;
  const Unit u = find_unit<kSmallGram>(a.s);
  if (blockIdx.z >= u.t.parts) return;
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  const uint32_t i = lower_row(u.tile), j = u.tile - i * (i + 1) / 2;
  const uint64_t pitch = (uint64_t)u.t.Q * 2 * PLANES;
  const uint32_t stages = (uint32_t)(pitch / kStageBytes), from = (uint32_t)((uint64_t)stages * blockIdx.z / u.t.parts), to = (uint32_t)((uint64_t)stages * (blockIdx.z + 1) / u.t.parts);
  const uint64_t in = u.base + x_at(w, a.from) + (uint64_t)from * kStageBytes, out = u.base + w.parts + (uint64_t)blockIdx.z * u.t.P * u.t.P * 4;
  char DADAM_LDS* lds = (char DADAM_LDS*)ortho_lds;
  T t;
  t.product(operand(in + (uint64_t)i * T::kM * pitch, pitch), operand(in + (uint64_t)j * T::kN * pitch, pitch), to - from, lds);
  t.hand_out(lds, i != j, nothing_ahead,
             [&](uint32_t m, uint32_t n, float (&v)[8], const Nothing&) { F32::store8(out, (uint64_t)(j * T::kN + n) * u.t.P + i * T::kM + m, 8, v); },
             [&](uint32_t m, uint32_t n, const float (&v)[8]) { F32::store8(out, (uint64_t)(i * T::kM + m) * u.t.P + j * T::kN + n, 8, v); });
}

// A from its parts, in their order: 16 rows of a tile and of its mirror image (blockIdx.z), eight columns a thread.
template <int PLANES>
__global__ __launch_bounds__(256) void k_ortho_join(OrthoStepArgs a) {
  const Unit u = find_unit<kSmallGram>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  const uint32_t i = lower_row(u.tile), j = u.tile - i * (i + 1) / 2, m = blockIdx.z * 16 + threadIdx.x / 16, n = threadIdx.x % 16 * 8;
  for (int mirror = 0; mirror < (i == j ? 1 : 2); ++mirror) {
    const uint32_t r = (mirror ? j : i) * kSmallEdge + m, c = (mirror ? i : j) * kSmallEdge + n;
    const uint64_t e = (uint64_t)r * u.t.P + c, step = (uint64_t)u.t.P * u.t.P;
    float v[8] = {};
#pragma unroll 4
    for (uint32_t k = 0; k < u.t.parts; ++k) {
      float x[8];
      F32::load8(u.base + w.parts, k * step + e, 8, x);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += x[q];
    }
    uint32_t words[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) words[q] = operand_word<Half, PLANES>(v[q] * a.fresh);
    store8<PLANES>(u.base + w.a, r, u.t.P, c, words);
  }
}

// X of eight elements of a row, highs and lows, and what B's diagonal has there.
struct RowOfX {
  Eight x;
  float diagonal;
};
template <int PLANES>
__device__ __forceinline__ RowOfX load_x(uint64_t base, const OrthoPlaces& w, uint32_t which, const OrthoTask& t, uint32_t p, uint32_t q) {
  RowOfX r = {load8<PLANES>(base + x_at(w, which), p, t.Q, q), global<const float>(base + w.diagonal)[p]};
  if constexpr (PLANES == 1) r.x.low = global<const uint4v>(base + w.low + ((uint64_t)p * t.Q + q) * 2)[0];
  return r;
}

// The product of a tile of a X + B X, transposed: columns q of X against rows p of B (its own).
template <typename T, int PLANES>
__device__ __forceinline__ void next_product(T& t, const Unit& u, const OrthoPlaces& w, uint32_t from, uint32_t& q0, uint32_t& p0, char DADAM_LDS* lds) {
  const uint32_t across = u.t.P / T::kN;
  q0 = u.tile / across * T::kM;
  p0 = u.tile % across * T::kN;
  const uint64_t pitch = (uint64_t)u.t.P * 2 * PLANES;
  t.product(operand(u.base + x_at(w, from) + (uint64_t)q0 * 2 * PLANES, (uint64_t)u.t.Q * 2 * PLANES), operand(u.base + w.b + p0 * pitch, pitch),
            (uint32_t)(pitch / kStageBytes), lds);
}

// X of the next iteration.  (100 million elements of matrices 1024 wide, bfloat16: 306 us, 673 TFLOP/s and 2.6 TB/s; 75 million in 32 bits 473 us, 980 TFLOP/s of instructions
// and 1.9 TB/s.  Tiles of a round begin and end together, so that their products and the reading and writing of X take turns.)
template <int PLANES, int EDGE, int BUFFERS>
__global__ __launch_bounds__(2 * EDGE) void k_ortho_next(OrthoStepArgs a) {
  using T = NextTile<PLANES, EDGE, BUFFERS>;
  const Unit u = find_unit<kWhole>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  char DADAM_LDS* lds = (char DADAM_LDS*)ortho_lds;
  uint32_t q0, p0;
  T t;
  next_product<T, PLANES>(t, u, w, a.from, q0, p0, lds);
  t.hand_out(lds, false, [&](uint32_t m, uint32_t n) { return load_x<PLANES>(u.base, w, a.from, u.t, p0 + n, q0 + m); },
             [&](uint32_t m, uint32_t n, float (&v)[8], const RowOfX& row) {
               uint32_t words[8];
               const float gain = fmaf(row.diagonal, a.fresh, a.gain);
#pragma unroll
               for (int k = 0; k < 8; ++k) words[k] = halves<Half>(fmaf(value_of<Half, true>(row.x, k), gain, v[k] * a.fresh));
               store8<PLANES>(u.base + x_at(w, a.to), p0 + n, u.t.Q, q0 + m, words);
               if constexpr (PLANES == 1) global<uint4v>(u.base + w.low + ((uint64_t)(p0 + n) * u.t.Q + q0 + m) * 2)[0] = highs(words);
             },
             [](uint32_t, uint32_t, const float (&)[8]) {});
}

constexpr int kEarly = 3;  // sources whose elements are on their way together

// The last iteration, straight into the result: the matrix, or the parameters mixed and moved along it.
template <typename DT, int PLANES, int EDGE, int BUFFERS, int N>
__global__ __launch_bounds__(2 * EDGE) void k_ortho_end(OrthoEndArgs<N> a) {
  using T = NextTile<PLANES, EDGE, BUFFERS>;
  const Unit u = find_unit<kWhole>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES, u.t.parts);
  char DADAM_LDS* lds = (char DADAM_LDS*)ortho_lds;
  uint32_t q0, p0;
  T t;
  next_product<T, PLANES>(t, u, w, a.from, q0, p0, lds);
  const uint32_t replica = blockIdx.y, rows = u.t.tall ? u.t.q : u.t.p, cols = u.t.tall ? u.t.p : u.t.q;
  const uint64_t out = (uint64_t)a.out[replica];
  int32_t first = 0, last = 0;
  uint64_t own = 0, early[kEarly] = {};  // the first sources, and their weights
  float weights[kEarly] = {};
  if (a.mix) {
    first = global<const int32_t>(a.row_ptr)[a.first_row + replica];
    last = global<const int32_t>(a.row_ptr)[a.first_row + replica + 1];
    own = (uint64_t)a.x_src[a.first_row + replica];
#pragma unroll
    for (int32_t k = 0; k < kEarly; ++k) {
      if (first + k >= last) continue;
      early[k] = (uint64_t)a.x_src[global<const int32_t>(a.col)[first + k]];
      weights[k] = global<const float>(a.w)[first + k];
    }
  }
  // elements (r, c) ... of the matrix as it lies
  auto finish = [&](uint32_t r, uint32_t c, const float (&v)[8]) {
    const uint32_t n = r < rows ? left(cols, c) : 0;
    if (n == 0) return;
    const uint64_t e = u.t.first + (uint64_t)r * u.t.ld + c;
    if (!a.mix) {
      DT::store8(out, e, n, v);
      return;
    }
    float mixed[8], x[8];
    int32_t k = first;
    if (DT::is_whole(n)) {
      typename DT::Piece early_pieces[kEarly];
#pragma unroll
      for (int32_t q = 0; q < kEarly; ++q)
        if (first + q < last) early_pieces[q] = DT::piece(early[q], e);
#pragma unroll
      for (int32_t q = 0; q < kEarly; ++q)
        if (first + q < last) {
#pragma unroll
          for (int i = 0; i < 8; ++i) mixed[i] = q == 0 ? weights[q] * early_pieces[q][i] : fmaf(weights[q], early_pieces[q][i], mixed[i]);
        }
      k = first + kEarly;
    }
    for (; k < last; ++k) {
      const float weight = global<const float>(a.w)[k];
      DT::load8((uint64_t)a.x_src[global<const int32_t>(a.col)[k]], e, n, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) mixed[i] = k == first ? weight * x[i] : fmaf(weight, x[i], mixed[i]);
    }
    if (u.t.decay != 0.f) DT::load8(own, e, n, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float direction = u.t.scale * v[i];
      if (u.t.decay != 0.f) direction = fmaf(u.t.decay, x[i], direction);
      mixed[i] = fmaf(-a.lr, direction, mixed[i]);
    }
    DT::store8(out, e, n, mixed);
  };
  t.hand_out(lds, u.t.tall, [&](uint32_t m, uint32_t n) { return load_x<PLANES>(u.base, w, a.from, u.t, p0 + n, q0 + m); },
             [&](uint32_t m, uint32_t n, float (&v)[8], const RowOfX& row) {
               const float gain = fmaf(row.diagonal, a.fresh, a.gain);
#pragma unroll
               for (int k = 0; k < 8; ++k) v[k] = fmaf(value_of<Half, true>(row.x, k), gain, v[k] * a.fresh);
               if (!u.t.tall) finish(p0 + n, q0 + m, v);
             },
             [&](uint32_t m, uint32_t n, const float (&v)[8]) { finish(q0 + m, p0 + n, v); });
}

template <int N>
OrthoBeginArgs<N> shorter(const OrthoBeginArgs<kMaxRows>& a) {
  OrthoBeginArgs<N> s{};
  s.s = a.s, s.c = a.c, s.scale = a.scale, s.source = a.source, s.phase = a.phase;
  for (int k = 0; k < N; ++k) s.grad[k] = a.grad[k], s.m_hat[k] = a.m_hat[k], s.acc[k] = a.acc[k];
  return s;
}
template <int N>
OrthoEndArgs<N> shorter(const OrthoEndArgs<kMaxRows>& a) {
  OrthoEndArgs<N> s{};
  s.s = a.s, s.gain = a.gain, s.fresh = a.fresh, s.from = a.from, s.mix = a.mix, s.row_ptr = a.row_ptr, s.col = a.col, s.w = a.w, s.first_row = a.first_row, s.lr = a.lr;
  for (int k = 0; k < N; ++k) s.out[k] = a.out[k], s.x_src[k] = a.x_src[k];
  return s;
}

// Launches KERNEL, whose workgroups take `lds` bytes of LDS: more than 64 KB have to be asked for once on every device.
template <auto KERNEL, typename A>
int launch(const A& a, uint32_t threads, uint32_t units, uint32_t replicas, uint32_t lds, void* stream, uint32_t parts = 1) {
  if (lds > 65536)
    if (const int e = ask_for_lds<KERNEL>(lds)) return e;
  KERNEL<<<dim3(units, replicas, parts), threads, lds, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

template <typename GT, int PLANES>
int begin(bool norm, const OrthoBeginArgs<kMaxRows>& a, uint32_t units, uint32_t replicas, void* stream) {
  const uint32_t lds = kOrthoCell * kTurnPitch * 4;
  if (replicas <= (uint32_t)kOrthoFew) {
    const OrthoBeginArgs<kOrthoFew> s = shorter<kOrthoFew>(a);
    return norm ? launch<k_ortho_norm<GT, PLANES, kOrthoFew>>(s, 256, units, replicas, 0, stream) : launch<k_ortho_begin<GT, PLANES, kOrthoFew>>(s, 256, units, replicas, lds, stream);
  }
  return norm ? launch<k_ortho_norm<GT, PLANES, kMaxRows>>(a, 256, units, replicas, 0, stream) : launch<k_ortho_begin<GT, PLANES, kMaxRows>>(a, 256, units, replicas, lds, stream);
}
int begin_any(bool norm, int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  if (gdt == (int)DADAM_F32) return planes == 1 ? begin<F32, 1>(norm, a, units, replicas, stream) : begin<F32, 2>(norm, a, units, replicas, stream);
  return planes == 1 ? begin<B16, 1>(norm, a, units, replicas, stream) : begin<B16, 2>(norm, a, units, replicas, stream);
}

// fn(edge, buffers) as types, for a launch of small or large tiles.
template <typename Fn>
int with_tiles(uint32_t edge, uint32_t tiles, Fn fn) {
  using Large = std::integral_constant<int, 256>;
  using Small = std::integral_constant<int, 128>;
  if (edge == kLargeEdge) return fn(Large{}, std::integral_constant<int, 2>{});
  return tiles <= kOneEach ? fn(Small{}, std::integral_constant<int, 4>{}) : fn(Small{}, std::integral_constant<int, 2>{});
}

template <int PLANES>
int gram(bool square, uint32_t edge, const OrthoStepArgs& a, uint32_t units, uint32_t replicas, void* stream) {
  return with_tiles(edge, units * replicas, [&](auto e, auto b) {
    constexpr int kEdge = decltype(e)::value, kBuffers = decltype(b)::value;
    using T = GramTile<PLANES, kEdge, kBuffers>;
    return square ? launch<k_ortho_gram<PLANES, kEdge, kBuffers, true>>(a, T::kThreads, units, replicas, T::kLds, stream)
                  : launch<k_ortho_gram<PLANES, kEdge, kBuffers, false>>(a, T::kThreads, units, replicas, T::kLds, stream);
  });
}
template <int PLANES>
int parts(const OrthoStepArgs& a, uint32_t most, uint32_t units, uint32_t replicas, void* stream) {
  const int e = with_tiles(kSmallEdge, units * replicas * most, [&](auto, auto b) {
    constexpr int kBuffers = decltype(b)::value;
    using T = GramTile<PLANES, (int)kSmallEdge, kBuffers>;
    return launch<k_ortho_part<PLANES, kBuffers>>(a, T::kThreads, units, replicas, T::kLds, stream, most);
  });
  return e ? e : launch<k_ortho_join<PLANES>>(a, 256, units, replicas, 0, stream, kSmallEdge / 16);
}
template <int PLANES>
int next(uint32_t edge, const OrthoStepArgs& a, uint32_t units, uint32_t replicas, void* stream) {
  return with_tiles(edge, units * replicas, [&](auto e, auto b) {
    constexpr int kEdge = decltype(e)::value, kBuffers = decltype(b)::value;
    using T = NextTile<PLANES, kEdge, kBuffers>;
    return launch<k_ortho_next<PLANES, kEdge, kBuffers>>(a, T::kThreads, units, replicas, T::kLds, stream);
  });
}
template <typename DT, int PLANES>
int end(uint32_t edge, const OrthoEndArgs<kMaxRows>& a, uint32_t n_cols, uint32_t units, uint32_t replicas, void* stream) {
  return with_tiles(edge, units * replicas, [&](auto e, auto b) {
    constexpr int kEdge = decltype(e)::value, kBuffers = decltype(b)::value;
    using T = NextTile<PLANES, kEdge, kBuffers>;
    if (replicas <= (uint32_t)kOrthoFew && n_cols <= (uint32_t)kOrthoFew)
      return launch<k_ortho_end<DT, PLANES, kEdge, kBuffers, kOrthoFew>>(shorter<kOrthoFew>(a), T::kThreads, units, replicas, T::kLds, stream);
    return launch<k_ortho_end<DT, PLANES, kEdge, kBuffers, kMaxRows>>(a, T::kThreads, units, replicas, T::kLds, stream);
  });
}

}  // namespace

int launch_ortho_norm(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return begin_any(true, gdt, a, planes, units, replicas, stream);
}
int launch_ortho_begin(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return begin_any(false, gdt, a, planes, units, replicas, stream);
}
int launch_ortho_gram(bool square, uint32_t edge, const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return planes == 1 ? gram<1>(square, edge, a, units, replicas, stream) : gram<2>(square, edge, a, units, replicas, stream);
}
int launch_ortho_parts(const OrthoStepArgs& a, uint32_t planes, uint32_t most, uint32_t units, uint32_t replicas, void* stream) {
  return planes == 1 ? parts<1>(a, most, units, replicas, stream) : parts<2>(a, most, units, replicas, stream);
}
int launch_ortho_next(uint32_t edge, const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return planes == 1 ? next<1>(edge, a, units, replicas, stream) : next<2>(edge, a, units, replicas, stream);
}
int launch_ortho_end(int dtype, uint32_t edge, const OrthoEndArgs<kMaxRows>& a, uint32_t n_cols, uint32_t units, uint32_t replicas, void* stream) {
  return dtype == (int)DADAM_F32 ? end<F32, 2>(edge, a, n_cols, units, replicas, stream) : end<B16, 1>(edge, a, n_cols, units, replicas, stream);
}

}  // namespace dadam
