// Orthogonalised updates: X <- a X + (b A + c A A) X, A = X X^T, from X = U / |U| (Frobenius), for all matrices of a layout in all replicas.
//
// An iteration is three launches over the tiles of a group of matrices: A (k_ortho_gram), B = b A + c A A (k_ortho_gram again, as A is its own
// transpose), and a X + B X (k_ortho_next; the last one, k_ortho_end, stores the matrix or takes the step).  All three have the summed index innermost
// on both sides if X is there in both orientations, so every iteration writes X and its transpose.  A and B are symmetric: only the tiles of their
// lower half are computed, each stored twice, which leaves 3 p^2 q + p^3 of 4 p^2 q + 2 p^3 operations.
//
// Operands are half precision times a power of two (their spectral norms are bounded, so their elements are, see dadam_ortho.cpp).  Results of
// 32 bits have two halves an element (dadam_mfma.h): the error of five iterations is 2e-7 to 3e-6 of the result, by how fast the singular values
// fall.  For bfloat16 results one half is enough in the products, but not for X itself: what X loses to 11 bits in the directions of small singular
// values grows by a = 3.4 an iteration, 1e-3 of the result for equal singular values, 1.4e-2 for ones that fall by 1000 in 50.  a X is therefore taken
// from two halves as well (1.4e-3 and 5e-4), the second of which no product reads.
#include "dadam_mfma.h"
#include "dadam_ortho.h"

namespace dadam {
namespace {

extern __shared__ char ortho_lds[];

template <int PLANES>
using OrthoTile = Tile<Half, PLANES, 2, 2, 2, 2>;

// The turned copy of X: Q rows of P, the operand, and with one plane what the half leaves as a second array behind it.
template <int PLANES>
__device__ __forceinline__ void store_turned4(uint64_t base, const OrthoTask& t, uint32_t q, uint32_t p, const float4v& v) {
  store4<Half, PLANES>(base, q, t.P, p, v);
  if constexpr (PLANES == 1) {
    uint32_t h, l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) halves<Half>(v[e], h, l[e]);
    global<uint2v>(base + ((uint64_t)t.Q * t.P + (uint64_t)q * t.P + p) * 2)[0] = four(l);
  }
}
template <int PLANES>
__device__ __forceinline__ float4v load_turned4(uint64_t base, const OrthoTask& t, uint32_t q, uint32_t p) {
  float4v v = load4<Half, PLANES>(base, q, t.P, p);
  if constexpr (PLANES == 1) v += load4<Half, 1>(base + (uint64_t)t.Q * t.P * 2, q, t.P, p);
  return v;
}
template <int PLANES>
__device__ __forceinline__ float load_turned1(uint64_t base, const OrthoTask& t, uint32_t q, uint32_t p) {
  const uint64_t e = (uint64_t)q * t.P + p;
  if constexpr (PLANES == 1) return Half::value(global<const uint16_t>(base)[e]) + Half::value(global<const uint16_t>(base)[(uint64_t)t.Q * t.P + e]);
  const uint64_t at = (uint64_t)q * t.P * 2 + high_at(p);
  return Half::value(global<const uint16_t>(base)[at]) + Half::value(global<const uint16_t>(base)[at + 32]);
}

// A workgroup's matrix, the tile of it and where its workspace begins.
struct Unit {
  OrthoTask t;
  uint32_t tile;
  uint64_t base;
};
template <bool GRAM>
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
  r.tile = u - (GRAM ? r.t.gram_units : r.t.whole_units);
  r.base = s.workspace + (uint64_t)blockIdx.y * s.stride + (r.t.at - s.before);
  return r;
}

// Where a tile of X begins in the matrix as it lies in memory, and the matrix's own rows and columns.
struct Cell {
  uint32_t r0, c0, rows, cols;
};
__device__ __forceinline__ Cell cell_of(const Unit& u) {
  const uint32_t across = u.t.Q / kOrthoPad, i = u.tile / across, j = u.tile % across;
  Cell c;
  c.r0 = (u.t.tall ? j : i) * kOrthoPad;
  c.c0 = (u.t.tall ? i : j) * kOrthoPad;
  c.rows = u.t.tall ? u.t.q : u.t.p;
  c.cols = u.t.tall ? u.t.p : u.t.q;
  return c;
}

// What is orthogonalised, of one element: the gradient, the moment of line 6 of Algorithm 3, or that looked ahead.
__device__ __forceinline__ float source_value(const Scalars& c, uint32_t source, float g, float mh) {
  if (source == kOrthoGiven) return g;
  const float m = fmaf(c.beta1, mh, c.omb1 * g);
  return source == kOrthoMoment ? m : fmaf(c.beta1, m, c.omb1 * g);
}

// Squares of a tile, in 64 bits, to the tile's place among the matrix's partial sums.
template <typename GT, int PLANES, int N>
__global__ __launch_bounds__(256) void k_ortho_norm(OrthoBeginArgs<N> a) {
  const Unit u = find_unit<false>(a.s);
  const Cell c = cell_of(u);
  const uint32_t row = blockIdx.y;
  const uint64_t g = (uint64_t)a.grad[row], mh = (uint64_t)a.m_hat[row];
  const uint32_t lane_col = c.c0 + threadIdx.x % kOrthoPad;
  double sum = 0.0;
  if (lane_col < c.cols)
    for (uint32_t r = c.r0 + threadIdx.x / kOrthoPad; r < c.r0 + kOrthoPad && r < c.rows; r += 256 / kOrthoPad) {
      const uint64_t e = u.t.first + (uint64_t)r * u.t.ld + lane_col;
      const float v = source_value(a.c, a.source, GT::load(g, e), a.source == kOrthoGiven ? 0.f : F32::load(mh, e));
      sum += (double)v * (double)v;
    }
  __shared__ double parts[4];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) global<double>(u.base + ortho_places(u.t.P, u.t.Q, PLANES).sums)[u.tile] = parts[0] + parts[1] + parts[2] + parts[3];
}

// X and its transpose from the matrix, and of a step lines 9 to 13 of Algorithm 3 for the first moment and the accumulator.
constexpr uint32_t kTurnPitch = kOrthoPad + 1;
template <typename GT, int PLANES, int N>
__global__ __launch_bounds__(256) void k_ortho_begin(OrthoBeginArgs<N> a) {
  const Unit u = find_unit<false>(a.s);
  const Cell c = cell_of(u);
  const uint32_t row = blockIdx.y, tiles = (u.t.P / kOrthoPad) * (u.t.Q / kOrthoPad);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES);
  float DADAM_LDS* tile = (float DADAM_LDS*)ortho_lds;
  __shared__ double parts[4];
  double sum = 0.0;
  for (uint32_t k = threadIdx.x; k < tiles; k += 256) sum += global<const double>(u.base + w.sums)[k];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = sum;
  __syncthreads();
  const float factor = (float)((double)a.scale / (sqrt(parts[0] + parts[1] + parts[2] + parts[3]) + 1e-7));
  const uint64_t g = (uint64_t)a.grad[row], mh = (uint64_t)a.m_hat[row], acc = (uint64_t)a.acc[row];
  const uint32_t lane_col = threadIdx.x % kOrthoPad, col = c.c0 + lane_col;
  for (uint32_t r = threadIdx.x / kOrthoPad; r < kOrthoPad; r += 256 / kOrthoPad) {
    float v = 0.f;
    if (c.r0 + r < c.rows && col < c.cols) {
      const uint64_t e = u.t.first + (uint64_t)(c.r0 + r) * u.t.ld + col;
      const float gv = GT::load(g, e);
      float m = a.source == kOrthoGiven ? 0.f : F32::load(mh, e);
      v = source_value(a.c, a.source, gv, m) * factor;
      if (a.source != kOrthoGiven && a.phase != kUpdateOnly) {
        float b = gv * a.c.inv_s;
        if (a.phase == kPlain || a.phase == kFold) b = fmaf(gv, a.c.inv_s, F32::load(acc, e));
        if (a.phase == kFold || a.phase == kAlg1) F32::store(mh, e, fmaf(a.c.beta1, m, a.c.omb1 * b));
        if (a.phase != kAlg1) F32::store(acc, e, a.phase == kFold ? 0.f : b);
      }
    }
    tile[r * kTurnPitch + lane_col] = v;
  }
  __syncthreads();
  // as it lies: rows of four columns; turned: columns of four rows
  const uint32_t k4 = threadIdx.x % 32 * 4;
  for (uint32_t r = threadIdx.x / 32; r < kOrthoPad; r += 8) {
    float4v v, t;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = tile[r * kTurnPitch + k4 + e], t[e] = tile[(k4 + e) * kTurnPitch + r];
    if (u.t.tall) {
      store_turned4<PLANES>(u.base + w.turned[0], u.t, c.r0 + r, c.c0 + k4, v);
      store4<Half, PLANES>(u.base + w.x, c.c0 + r, u.t.Q, c.r0 + k4, t);
    } else {
      store4<Half, PLANES>(u.base + w.x, c.r0 + r, u.t.Q, c.c0 + k4, v);
      store_turned4<PLANES>(u.base + w.turned[0], u.t, c.c0 + r, c.r0 + k4, t);
    }
  }
}

// A tile (i, j), j <= i, of A = X X^T or of B = b A + c A A, and its mirror image.
template <int PLANES, bool SQUARE>
__global__ __launch_bounds__(256) void k_ortho_gram(OrthoStepArgs a) {
  using T = OrthoTile<PLANES>;
  const Unit u = find_unit<true>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES);
  uint32_t i = (uint32_t)((sqrtf(8.f * (float)u.tile + 1.f) - 1.f) * 0.5f);  // (the root may round across the border of a row of tiles)
  while (i * (i + 1) / 2 > u.tile) --i;
  while ((i + 1) * (i + 2) / 2 <= u.tile) ++i;
  const uint32_t j = u.tile - i * (i + 1) / 2, inner = SQUARE ? u.t.P : u.t.Q;
  const uint64_t pitch = (uint64_t)inner * 2 * PLANES;
  const char DADAM_GLOBAL* in = global<const char>(u.base + (SQUARE ? w.a : w.x));
  T t;
  t.product(in + (uint64_t)i * T::kM * pitch, pitch, in + (uint64_t)j * T::kN * pitch, pitch, (uint32_t)(pitch / kStageBytes), (char DADAM_LDS*)ortho_lds);
  const uint64_t out = u.base + (SQUARE ? w.b : w.a);
  t.each([&](uint32_t m, uint32_t n, float4v v) {
    m += i * T::kM;
    n += j * T::kN;
    v *= a.fresh;
    if constexpr (SQUARE) v += load4<Half, PLANES>(u.base + w.a, n, u.t.P, m) * a.gain;
    store4<Half, PLANES>(out, n, u.t.P, m, v);
    if (i != j)
#pragma unroll
      for (int e = 0; e < 4; ++e) store1<Half, PLANES>(out, m + e, u.t.P, n, v[e]);
  });
}

// A tile of a X + B X: rows p of B against columns q of X.
template <int PLANES>
__global__ __launch_bounds__(256) void k_ortho_next(OrthoStepArgs a) {
  using T = OrthoTile<PLANES>;
  const Unit u = find_unit<false>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES);
  const uint32_t across = u.t.Q / T::kN, i = u.tile / across, j = u.tile % across;
  const uint64_t pitch = (uint64_t)u.t.P * 2 * PLANES, from = u.base + w.turned[a.from], to = u.base + w.turned[a.to];
  T t;
  t.product(global<const char>(u.base + w.b) + (uint64_t)i * T::kM * pitch, pitch, global<const char>(from) + (uint64_t)j * T::kN * pitch, pitch,
            (uint32_t)(pitch / kStageBytes), (char DADAM_LDS*)ortho_lds);
  t.each([&](uint32_t m, uint32_t n, float4v v) {
    m += i * T::kM;
    n += j * T::kN;
    v = load_turned4<PLANES>(from, u.t, n, m) * a.gain + v * a.fresh;
    store_turned4<PLANES>(to, u.t, n, m, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) store1<Half, PLANES>(u.base + w.x, m + e, u.t.Q, n, v[e]);
  });
}

// The last iteration's tile, straight into the result: rows of the matrix as it lies in memory are the tile's rows, so of a tall one rows q of X
// against columns p of B (its own transpose).
template <typename DT, int PLANES, int N>
__global__ __launch_bounds__(256) void k_ortho_end(OrthoEndArgs<N> a) {
  using T = OrthoTile<PLANES>;
  const Unit u = find_unit<false>(a.s);
  const OrthoPlaces w = ortho_places(u.t.P, u.t.Q, PLANES);
  const Cell c = cell_of(u);
  const uint64_t pitch = (uint64_t)u.t.P * 2 * PLANES, from = u.base + w.turned[a.from], b = u.base + w.b;
  const char DADAM_GLOBAL* rows = global<const char>(u.t.tall ? from : b);
  const char DADAM_GLOBAL* cols = global<const char>(u.t.tall ? b : from);
  T t;
  t.product(rows + c.r0 * pitch, pitch, cols + c.c0 * pitch, pitch, (uint32_t)(pitch / kStageBytes), (char DADAM_LDS*)ortho_lds);
  const uint32_t replica = blockIdx.y;
  const uint64_t out = (uint64_t)a.out[replica];
  int32_t first = 0, last = 0;
  uint64_t own = 0;
  if (a.mix) {
    first = global<const int32_t>(a.row_ptr)[a.first_row + replica];
    last = global<const int32_t>(a.row_ptr)[a.first_row + replica + 1];
    own = (uint64_t)a.x_src[a.first_row + replica];
  }
  t.each([&](uint32_t m, uint32_t n, float4v v) {
    m += c.r0;
    n += c.c0;
    if (u.t.tall) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = load_turned1<PLANES>(from, u.t, m + e, n) * a.gain + v[e] * a.fresh;
    } else {
      v = load_turned4<PLANES>(from, u.t, n, m) * a.gain + v * a.fresh;
    }
    if (n >= c.cols) return;
    const uint64_t at = u.t.first + (uint64_t)m * u.t.ld + n;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (m + e >= c.rows) continue;
      const uint64_t x = at + (uint64_t)e * u.t.ld;
      float r = v[e];
      if (a.mix) {
        float mixed = 0.f;
        for (int32_t k = first; k < last; ++k) {
          const float weight = global<const float>(a.w)[k], value = DT::load((uint64_t)a.x_src[global<const int32_t>(a.col)[k]], x);
          mixed = k == first ? weight * value : fmaf(weight, value, mixed);
        }
        float direction = u.t.scale * r;
        if (u.t.decay != 0.f) direction = fmaf(u.t.decay, DT::load(own, x), direction);
        r = fmaf(-a.lr, direction, mixed);
      }
      DT::store(out, x, r);
    }
  });
}

template <typename K>
int reserve(K kernel, int bytes) {
  return bytes <= 65536 ? (int)hipSuccess : (int)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
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

template <typename K, typename A>
int launch(K kernel, const A& a, uint32_t units, uint32_t replicas, uint32_t lds, void* stream) {
  if (const int e = reserve(kernel, (int)lds)) return e;
  kernel<<<dim3(units, replicas), 256, lds, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

template <typename GT, int PLANES>
int begin(bool norm, const OrthoBeginArgs<kMaxRows>& a, uint32_t units, uint32_t replicas, void* stream) {
  const uint32_t lds = kOrthoPad * kTurnPitch * 4;
  if (replicas <= (uint32_t)kOrthoFew) {
    const OrthoBeginArgs<kOrthoFew> s = shorter<kOrthoFew>(a);
    return norm ? launch(k_ortho_norm<GT, PLANES, kOrthoFew>, s, units, replicas, 0, stream) : launch(k_ortho_begin<GT, PLANES, kOrthoFew>, s, units, replicas, lds, stream);
  }
  return norm ? launch(k_ortho_norm<GT, PLANES, kMaxRows>, a, units, replicas, 0, stream) : launch(k_ortho_begin<GT, PLANES, kMaxRows>, a, units, replicas, lds, stream);
}
int begin_any(bool norm, int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  if (gdt == (int)DADAM_F32) return planes == 1 ? begin<F32, 1>(norm, a, units, replicas, stream) : begin<F32, 2>(norm, a, units, replicas, stream);
  return planes == 1 ? begin<B16, 1>(norm, a, units, replicas, stream) : begin<B16, 2>(norm, a, units, replicas, stream);
}

template <typename DT, int PLANES>
int end(const OrthoEndArgs<kMaxRows>& a, uint32_t n_cols, uint32_t units, uint32_t replicas, void* stream) {
  const uint32_t lds = OrthoTile<PLANES>::kLds;
  if (replicas <= (uint32_t)kOrthoFew && n_cols <= (uint32_t)kOrthoFew) return launch(k_ortho_end<DT, PLANES, kOrthoFew>, shorter<kOrthoFew>(a), units, replicas, lds, stream);
  return launch(k_ortho_end<DT, PLANES, kMaxRows>, a, units, replicas, lds, stream);
}

}  // namespace

int launch_ortho_norm(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return begin_any(true, gdt, a, planes, units, replicas, stream);
}
int launch_ortho_begin(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return begin_any(false, gdt, a, planes, units, replicas, stream);
}
int launch_ortho_gram(bool square, const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  if (planes == 1) return launch(square ? k_ortho_gram<1, true> : k_ortho_gram<1, false>, a, units, replicas, OrthoTile<1>::kLds, stream);
  return launch(square ? k_ortho_gram<2, true> : k_ortho_gram<2, false>, a, units, replicas, OrthoTile<2>::kLds, stream);
}
int launch_ortho_next(const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  return planes == 1 ? launch(k_ortho_next<1>, a, units, replicas, OrthoTile<1>::kLds, stream) : launch(k_ortho_next<2>, a, units, replicas, OrthoTile<2>::kLds, stream);
}
int launch_ortho_end(int dtype, const OrthoEndArgs<kMaxRows>& a, uint32_t n_cols, uint32_t planes, uint32_t units, uint32_t replicas, void* stream) {
  // one plane where the result is bfloat16 (see the top)
  if (dtype == (int)DADAM_F32) return end<F32, 2>(a, n_cols, units, replicas, stream);
  (void)planes;
  return end<B16, 1>(a, n_cols, units, replicas, stream);
}

}  // namespace dadam
