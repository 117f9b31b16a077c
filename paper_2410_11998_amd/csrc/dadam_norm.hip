// Global gradient norms and clipping by them.
//
//   n_i = sqrt(sum_e g_i[e]^2),   out_i = g_i  or  g_i (max_norm / n_i)
//
// One pass over g for the norm, bound by reading it (8 rows of 355 million bfloat16 elements 831 to 886 us, 6.4 to 6.8 TB/s; 1e8 float32 elements 65 to 66 us,
// 6.1), one more to scale it (355 million float32 elements with both passes 654 to 665 us, 6.4 to 6.5 TB/s of the three streams).  A float32 square is exact
// in 64 bits (24 + 24 of 53), so sums in double lose next to nothing whatever their order, and nothing overflows or vanishes on the way; vector
// instructions fill 29 % of the issue slots in bfloat16.  Tried and dropped: clipping in reverse order, for what the norm's pass left in the 256 MB cache
// (704 against 681 us), and adding the partial sums up in every workgroup that clips (no counter; 683 to 820).
#include <hip/hip_runtime.h>

#include <cstring>

#include "dadam_granule.h"

namespace dadam {
namespace {

constexpr uint32_t kClipThreads = 256, kClipWaves = kClipThreads / kWave;
constexpr uint32_t kNormThreads = kWave * kNormWaves;

template <uint32_t WAVES>
__device__ __forceinline__ double group_sum(double sum, double (&partial)[WAVES], uint32_t lane, uint32_t wave) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if (lane == 0) partial[wave] = sum;
  __syncthreads();
  sum = partial[0];
#pragma unroll
  for (uint32_t w = 1; w < WAVES; ++w) sum += partial[w];
  return sum;
}

// The sum of a row's partial sums, the same in every workgroup that forms it.
__device__ __forceinline__ double row_sum(const double* partials, uint32_t count, double (&partial)[kNormWaves], uint32_t lane, uint32_t wave) {
  double sum = 0.0;
  for (uint32_t k = threadIdx.x; k < count; k += kNormThreads)
    sum += __hip_atomic_load(partials + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return group_sum(sum, partial, lane, wave);
}

__device__ __forceinline__ double with_square(double sum, float v) { return __builtin_fma((double)v, (double)v, sum); }

// A granule goes as 16-byte vectors, one (bfloat16) or two (float32) a lane.  Bits of `stored` say which elements of a vector count.
template <typename GT>
constexpr int kVectors = GT::bytes / 2;
template <typename GT>
constexpr int kVectorElems = 16 / GT::bytes;
template <typename GT, bool WHOLE>
__device__ __forceinline__ void add_squares(const u4& raw, uint32_t stored, double (&sums)[2]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  auto counted = [stored](uint32_t bits, int j) { return __uint_as_float(WHOLE || (stored >> j & 1) ? bits : 0u); };
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (GT::bytes == 4) {
      sums[j & 1] = with_square(sums[j & 1], counted(w[j], j));
    } else {
      sums[0] = with_square(sums[0], counted(w[j] << 16, 2 * j));
      sums[1] = with_square(sums[1], counted(w[j] & 0xFFFF0000u, 2 * j + 1));
    }
  }
}

// kAtOnce granules, `stride` apart; all loads are in flight before the first use.  Not WHOLE: some have padding, end behind the vector or lie
// there.
template <typename GT, int AT_ONCE, bool WHOLE, bool NT>
__device__ __forceinline__ void add_granules(const Span& s, const void* g, uint64_t i0, uint32_t stride, const uint32_t (&cut)[AT_ONCE], uint32_t lane,
                                             double (&sums)[2]) {
  constexpr int V = kVectors<GT>, E = kVectorElems<GT>;
  u4 raw[AT_ONCE][V];
  uint32_t stored[AT_ONCE][V];
#pragma unroll
  for (uint32_t k = 0; k < AT_ONCE; ++k)
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) {
      const uint64_t i = i0 + (uint64_t)k * stride, e = i * kGranule + v * (kGranule / V) + E * lane;
      stored[k][v] = WHOLE || e >= s.d ? 0u : stored_bits(s.cuts, cut[k], (uint32_t)(e % kGranule), E);
      raw[k][v] = u4{0, 0, 0, 0};
      if (WHOLE || e + E <= s.d) {
        raw[k][v] = vload<NT>(reinterpret_cast<const u4*>(static_cast<const char*>(g) + e * GT::bytes));
      } else if (e < s.d) {  // the vector's last elements
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (e + j < s.d) {
            if constexpr (GT::bytes == 4) w[j] = at<uint32_t>(g, e)[j];
            else w[j / 2] |= (uint32_t)at<uint16_t>(g, e)[j] << (16 * (j % 2));
          }
        raw[k][v] = u4{w[0], w[1], w[2], w[3]};
      }
    }
#pragma unroll
  for (uint32_t k = 0; k < AT_ONCE; ++k)
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) add_squares<GT, WHOLE>(raw[k][v], stored[k][v], sums);
}

// per_row workgroups share a row, each wavefront takes every (per_row * kNormWaves)-th granule, kAtOnce of them at a time.  The workgroup
// of a row that is done last adds up the row's partial sums in their fixed order: no second launch, and no sum that depends on
// who came first.
template <typename GT, bool NT, int N>
__global__ __launch_bounds__(kNormThreads) void k_grad_norm(const NormArgs<N> a) {
  __shared__ double partial[kNormWaves];
  __shared__ uint32_t last;
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group();
  const uint32_t row = blockIdx.x % a.s.n_rows, part = blockIdx.x / a.s.n_rows;
  const void* g = buffer<const void, 0>(a.row[row]);
  const uint32_t stride = a.per_row * kNormWaves, n = a.s.n_granules;
  constexpr int kAtOnce = 8 / kVectors<GT>;
  double sums[2] = {0.0, 0.0};
  for (uint64_t i0 = part * kNormWaves + wave; i0 < n; i0 += (uint64_t)kAtOnce * stride) {
    uint32_t cut[kAtOnce], any = i0 + (uint64_t)(kAtOnce - 1) * stride >= n;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint64_t i = i0 + (uint64_t)k * stride;
      cut[k] = i < n ? cut_of(a.s.cuts, (uint32_t)i) : 0u;
      any |= cut[k];
    }
    if (any == 0) add_granules<GT, kAtOnce, true, NT>(a.s, g, i0, stride, cut, lane, sums);
    else add_granules<GT, kAtOnce, false, NT>(a.s, g, i0, stride, cut, lane, sums);
  }
  const double sum = group_sum(sums[0] + sums[1], partial, lane, wave);
  if (a.per_row == 1) {  // nobody to wait for (the report and its answer take 3 us)
    if (threadIdx.x == 0) a.norms[row] = (float)__builtin_sqrt(sum);
  } else {
    double* row_partials = a.partials + (uint64_t)row * a.per_row;
    if (threadIdx.x == 0) {
      __hip_atomic_store(row_partials + part, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // The sum has to be there before the count.  On gfx950, and only by what its instructions do, not by the language's memory model (nothing there orders relaxed
      // operations on two places): stores and additions of the agent's scope go past the die's L2 to where all dies see them, vmcnt counts a
      // store until it is there, and the loads of row_sum, behind a barrier, go past the L2 too.  (A release of the agent's scope, which is
      // the portable form, writes the die's whole L2 back: norms and clipping of 4 x 1048576 elements 58 us, 13 us without.)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      last = __hip_atomic_fetch_add(a.arrived + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == a.per_row;
    }
    __syncthreads();  // (also: everybody has read the partial sums, which the next sum overwrites)
    if (last) {
      const double all = row_sum(row_partials, a.per_row, partial, lane, wave);
      if (threadIdx.x == 0) {
        a.norms[row] = (float)__builtin_sqrt(all);
        __hip_atomic_store(a.arrived + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
}

template <typename GT, bool WHOLE, bool NT>
__device__ __forceinline__ void clip_unit(const Cuts& cuts, const Units<2, 1>& u, const void* g, void* out, float factor) {
  float v[2][4];
  uint32_t bits[2];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    bits[k] = WHOLE ? 0xFu : u.bits(cuts, k);
    load_group<GT, WHOLE, NT>(based<GT>(g, u.base), u.at(k), bits[k], u.left, v[k]);
  }
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[k][j] *= factor;
    store_group<GT, NT>(based<GT>(out, u.base), u.at(k), bits[k], v[k]);
  }
}

template <typename GT, bool NT, int N>
__global__ __launch_bounds__(kClipThreads) void k_clip(const NormArgs<N> a) {
  const uint32_t lane = threadIdx.x % kWave;
  uint32_t piece, row;
  const bool active = die_block_piece(blockIdx.x, a.s.n_rows, a.s.n_xcd, (a.s.count + kClipWaves - 1) / kClipWaves, kDieBlockTiles, piece, row, a.s.run);
  const uint32_t i = a.s.first + piece * kClipWaves + wave_of_group();
  const void* g = buffer<const void, 0>(a.row[row]);
  void* out = buffer<void, 1>(a.row[row]);
  const float norm = a.norms[row];
  const bool scales = !(norm <= a.max_norm);  // NaN scales too: everything becomes NaN
  if (active && i < a.s.n_granules && (scales || g != out)) {
    const float factor = scales ? a.max_norm / norm : 1.0f;
    const Units<2, 1> u = units_from<2, NT>(i, a.s, lane);
    if (u.whole) clip_unit<GT, true, NT>(a.s.cuts, u, g, out, factor);
    else clip_unit<GT, false, NT>(a.s.cuts, u, g, out, factor);
  }
}

// Rows of at most kSmallGranules granules: one workgroup takes a row, holds it in registers (64 floats a lane at most) and does both.  One launch and one
// pass.  us, two launches / this: 16 rows of 13624 10.7 / 6.7, of 60000 10.6 / 9.2, one of 60000 bfloat16 11.0 / 10.6; 115 of 189 17.9 / 12.3.
constexpr uint32_t kSmallWaves = 16;
template <typename GT, int EACH, int N>
__global__ __launch_bounds__(kWave * kSmallWaves) void k_clip_small(const NormArgs<N> a) {
  __shared__ double partial[kSmallWaves];
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group();
  const RowPointers p = a.row[blockIdx.x];
  float v[EACH][2][4];
  uint32_t bits[EACH][2];
  double sums[2] = {0.0, 0.0};
#pragma unroll
  for (uint32_t q = 0; q < EACH; ++q) {
    const uint32_t i = wave + q * kSmallWaves;
    if (i < a.s.n_granules) {
      const Units<2, 1> u = units_from<2, false>(i, a.s, lane);
#pragma unroll
      for (uint32_t k = 0; k < 2; ++k) {
        bits[q][k] = u.bits(a.s.cuts, k);
        load_group<GT, false, false>(based<GT>(buffer<const void, 0>(p), u.base), u.at(k), bits[q][k], u.left, v[q][k]);
      }
    }
  }
#pragma unroll
  for (uint32_t q = 0; q < EACH; ++q)
    if (wave + q * kSmallWaves < a.s.n_granules) {
#pragma unroll
      for (uint32_t k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[j & 1] = with_square(sums[j & 1], v[q][k][j]);
    }
  const double sum = group_sum(sums[0] + sums[1], partial, lane, wave);
  const float norm = (float)__builtin_sqrt(sum);
  if (threadIdx.x == 0) a.norms[blockIdx.x] = norm;
  const bool scales = !(norm <= a.max_norm);
  if (scales || buffer<const void, 0>(p) != buffer<void, 1>(p)) {
    const float factor = scales ? a.max_norm / norm : 1.0f;
#pragma unroll
    for (uint32_t q = 0; q < EACH; ++q) {
      const uint32_t i = wave + q * kSmallWaves;
      if (i < a.s.n_granules) {
        const Units<2, 1> u = units_from<2, false>(i, a.s, lane);
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[q][k][j] *= factor;
          store_group<GT, false>(based<GT>(buffer<void, 1>(p), u.base), u.at(k), bits[q][k], v[q][k]);
        }
      }
    }
  }
}

template <int N>
NormArgs<N> shortened(const NormArgs<kMaxRows>& a) {
  NormArgs<N> f = few_rows<NormArgs<N>>(a);
  f.s = a.s; f.partials = a.partials; f.arrived = a.arrived; f.norms = a.norms; f.per_row = a.per_row; f.max_norm = a.max_norm;
  return f;
}

template <typename Fn>
int with_block(const NormArgs<kMaxRows>& a, Fn fn) {
  if (a.s.n_rows <= (uint32_t)kFewOperands) {
    NormArgs<kFewOperands> f = shortened<kFewOperands>(a);
    return fn(f);
  }
  NormArgs<kMaxRows> all = a;
  return fn(all);
}

template <int N>
KernelFn norm_kernel(int gdt, bool nt) {
  if (gdt == DADAM_BF16) return nt ? (KernelFn)k_grad_norm<TBF16, true, N> : (KernelFn)k_grad_norm<TBF16, false, N>;
  return nt ? (KernelFn)k_grad_norm<TF32, true, N> : (KernelFn)k_grad_norm<TF32, false, N>;
}
template <int N>
KernelFn clip_kernel(int gdt, bool nt) {
  if (gdt == DADAM_BF16) return nt ? (KernelFn)k_clip<TBF16, true, N> : (KernelFn)k_clip<TBF16, false, N>;
  return nt ? (KernelFn)k_clip<TF32, true, N> : (KernelFn)k_clip<TF32, false, N>;
}

template <int N>
int enqueue_norm(int gdt, NormArgs<N>& a, void* stream) {
  return enqueue_grid(norm_kernel<N>(gdt, a.s.streams), a.s.n_rows * a.per_row, kNormThreads, &a, 0, stream);
}
template <int N>
int enqueue_clip(int gdt, NormArgs<N>& a, void* stream) {
  return in_pieces(a, kClipWaves * a.s.n_xcd, a.s.n_rows * a.s.n_xcd, kClipThreads, [&](uint32_t grid) { return enqueue_grid(clip_kernel<N>(gdt, a.s.streams), grid, kClipThreads, &a, 0, stream); });
}

template <int N>
int enqueue_small(int gdt, NormArgs<N>& a, void* stream) {
  const bool few = a.s.n_granules <= kSmallGranules / 2;
  const KernelFn fn = gdt == DADAM_BF16 ? (few ? (KernelFn)k_clip_small<TBF16, kSmallGranules / kSmallWaves / 2, N> : (KernelFn)k_clip_small<TBF16, kSmallGranules / kSmallWaves, N>)
                                        : (few ? (KernelFn)k_clip_small<TF32, kSmallGranules / kSmallWaves / 2, N> : (KernelFn)k_clip_small<TF32, kSmallGranules / kSmallWaves, N>);
  return enqueue_grid(fn, a.s.n_rows, kWave * kSmallWaves, &a, 0, stream);
}

}  // namespace

int launch_clip_small(int gdt, const NormArgs<kMaxRows>& a, void* stream) {
  return with_block(a, [&](auto& block) { return enqueue_small(gdt, block, stream); });
}
int launch_norm(int gdt, const NormArgs<kMaxRows>& a, void* stream) {
  return with_block(a, [&](auto& block) { return enqueue_norm(gdt, block, stream); });
}
int launch_clip(int gdt, const NormArgs<kMaxRows>& a, void* stream) {
  return with_block(a, [&](auto& block) { return enqueue_clip(gdt, block, stream); });
}

}  // namespace dadam
