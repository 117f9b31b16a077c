// Orthogonalised updates of matrices that fit a compute unit: a workgroup holds one in LDS from the gradient to the parameters, in one launch where the tiles of
// dadam_ortho.hip take three an iteration, whose beginnings and ends are all that such matrices' time goes into.
//
// X (its short side's rows), A = X X^T and B without its diagonal (see dadam_ortho.hip) lie in LDS as words of two halves, 22 bits, whatever the result's
// type.  Rows are filled up to multiples of 32 and have four more words, so that eight rows' pieces of 16 bytes meet no bank twice.  A and B = b A + c A A by
// blocks of the lower half, a wavefront each; X X^T of one or three blocks by ranges of columns, joined in their order.  Columns of a X + B X depend on the same
// columns of X only: a wavefront has all rows of 32, and writes them where they were.
// Bound by latency: 64 x 48 and 48 x 192 take 42 us, of which an iteration is 7 (four barriers, and a chain of products that depend on each other; three sums, none of
// which waits for another, are slower: 44), 128 x 128 takes 70.
#include "dadam_mfma.h"
#include "dadam_ortho.h"
#include "dadam_ortho_source.h"

namespace dadam {
namespace {

constexpr uint32_t kWaves = kLoneThreads / 64;
extern __shared__ char lone_lds[];
typedef uint32_t DADAM_LDS* Words;

__device__ __forceinline__ int row_of(int r, int lane) { return (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3); }
__device__ __forceinline__ float value(uint32_t w) { return Half::value(w & 0xffffu) + Half::value(w >> 16); }

struct Fragment {
  half8 high, low;
};
__device__ __forceinline__ Fragment fragment(const uint32_t (&w)[8]) { return {__builtin_bit_cast(half8, lows(w)), __builtin_bit_cast(half8, highs(w))}; }
// Eight words of a row, and eight rows' words of a column.
__device__ __forceinline__ Fragment along(Words at) {
  const uint4v a = *(uint4v DADAM_LDS*)at, b = *(uint4v DADAM_LDS*)(at + 4);
  const uint32_t w[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return fragment(w);
}
__device__ __forceinline__ Fragment down(Words at, uint32_t pitch) {
  uint32_t w[8];
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) w[e] = at[e * pitch];
  return fragment(w);
}
__device__ __forceinline__ float16v multiply(const Fragment& a, const Fragment& b, float16v c) {
  c = Half::mfma(a.low, b.high, c);
  c = Half::mfma(a.high, b.low, c);
  return Half::mfma(a.high, b.high, c);
}
__device__ __forceinline__ float16v zeros() {
  float16v v;
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = 0.f;
  return v;
}

// Block (i, j) of rows i 32 .. times rows j 32 .. of an array, over steps of 16 columns.
__device__ __forceinline__ float16v block_product(Words x, uint32_t pitch, uint32_t i, uint32_t j, uint32_t from, uint32_t to, int lane) {
  float16v acc = zeros();
  const Words a = x + (i * 32 + (lane & 31)) * pitch + (lane >> 5) * 8, b = x + (j * 32 + (lane & 31)) * pitch + (lane >> 5) * 8;
  Fragment f = along(a + from * 16), g = along(b + from * 16);
  for (uint32_t s = from; s < to; ++s) {  // the next step's fragments on their way meanwhile
    const uint32_t next = s + 1 < to ? s + 1 : from;
    const Fragment nf = along(a + next * 16), ng = along(b + next * 16);
    acc = multiply(f, g, acc);
    f = nf, g = ng;
  }
  return acc;
}
// The n-th block of the lower half.
__device__ __forceinline__ void block_of(uint32_t n, uint32_t& i, uint32_t& j) {
  i = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
  j = n - i * (i + 1) / 2;
}

// A block's words and their mirror image.
__device__ __forceinline__ void put_block(Words a, uint32_t ap, uint32_t i, uint32_t j, const uint32_t (&w)[16], int lane) {
  const Words at = a + (i * 32 + row_of(0, lane)) * ap + j * 32 + (lane & 31), mirror = a + (j * 32 + (lane & 31)) * ap + i * 32 + row_of(0, lane);
#pragma unroll
  for (int r = 0; r < 16; ++r) at[row_of(r, 0) * ap] = w[r];
  if (i == j) return;
#pragma unroll
  for (int g = 0; g < 4; ++g) *(uint4v DADAM_LDS*)(mirror + g * 8) = uint4v{w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]};
}

// An iteration of a matrix of NB blocks of rows; the last leaves float32 values.
template <int NB>
__device__ __forceinline__ void iterate(Words x, Words a, Words diagonal, Words parts, uint32_t P, uint32_t Q, const LoneStep& s, bool last) {
  constexpr uint32_t kBlocks = NB * (NB + 1) / 2, kParts = NB == 1 ? 8 : NB == 2 ? 2 : 1, kEach = (kBlocks + kWaves - 1) / kWaves;
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), xp = Q + 4, ap = P + 4, column = lane & 31;
#pragma unroll
  for (uint32_t n = 0; n < kEach; ++n) {
    const uint32_t item = wave + n * kWaves;
    if (item >= kBlocks * kParts) continue;
    uint32_t i, j;
    block_of(item % kBlocks, i, j);
    const float16v acc = block_product(x, xp, i, j, Q / 16 * (item / kBlocks) / kParts, Q / 16 * (item / kBlocks + 1) / kParts, lane);
    if constexpr (kParts > 1) {
#pragma unroll
      for (int r = 0; r < 16; ++r) parts[item * 1024 + r * 64 + lane] = __float_as_uint(acc[r]);
    } else {
      uint32_t w[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] = halves<Half>(acc[r] * s.a_fresh);
      put_block(a, ap, i, j, w, lane);
    }
  }
  __syncthreads();
  if constexpr (kParts > 1) {
    for (uint32_t t = threadIdx.x; t < kBlocks * 1024; t += kLoneThreads) {
      const uint32_t block = t / 1024, e = t % 1024;
      float v = 0.f;
#pragma unroll
      for (uint32_t k = 0; k < kParts; ++k) v += __uint_as_float(parts[(k * kBlocks + block) * 1024 + e]);
      uint32_t i, j;
      block_of(block, i, j);
      const uint32_t m = i * 32 + row_of(e / 64, lane), c = j * 32 + column, w = halves<Half>(v * s.a_fresh);
      a[m * ap + c] = w;
      if (i != j) a[c * ap + m] = w;
    }
    __syncthreads();
  }
  uint32_t words[kEach][16];
#pragma unroll
  for (uint32_t n = 0; n < kEach; ++n) {
    const uint32_t item = wave + n * kWaves;
    if (item >= kBlocks) continue;
    uint32_t i, j;
    block_of(item, i, j);
    const float16v acc = block_product(a, ap, i, j, 0, P / 16, lane);
    const Words at = a + (i * 32 + row_of(0, lane)) * ap + j * 32 + column;
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = fmaf(value(at[row_of(r, 0) * ap]), s.b_gain, acc[r] * s.b_fresh);
#pragma unroll
    for (int r = 0; r < 16; ++r) words[n][r] = halves<Half>(v[r]);
    if (i != j) continue;
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool on = row_of(r, lane) == (int)column;
      mine = on ? v[r] : mine;
      words[n][r] = on ? 0 : words[n][r];
    }
    if ((column >> 2 & 1) == (uint32_t)(lane >> 5)) diagonal[i * 32 + column] = __float_as_uint(mine);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t n = 0; n < kEach; ++n) {
    const uint32_t item = wave + n * kWaves;
    if (item >= kBlocks) continue;
    uint32_t i, j;
    block_of(item, i, j);
    put_block(a, ap, i, j, words[n], lane);
  }
  __syncthreads();
  for (uint32_t q = wave; q < Q / 32; q += kWaves) {
    float16v acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[i] = zeros();
    const Words at = x + (lane >> 5) * 8 * xp + q * 32 + column, b = a + column * ap + (lane >> 5) * 8;
#pragma unroll 2
    for (uint32_t k = 0; k < NB * 2; ++k) {
      const Fragment f = down(at + k * 16 * xp, xp);
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = multiply(along(b + i * 32 * ap + k * 16), f, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const Words w = x + (i * 32 + row_of(0, lane)) * xp + q * 32 + column, d = diagonal + i * 32 + row_of(0, lane);
      float v[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = fmaf(value(w[row_of(r, 0) * xp]), fmaf(__uint_as_float(d[row_of(r, 0)]), s.x_fresh, s.x_gain), acc[i][r] * s.x_fresh);
      if (last) {
#pragma unroll
        for (int r = 0; r < 16; ++r) w[row_of(r, 0) * xp] = __float_as_uint(v[r]);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) w[row_of(r, 0) * xp] = halves<Half>(v[r]);
      }
    }
  }
  __syncthreads();
}

template <typename GT, typename DT, int N, int C>
__global__ __launch_bounds__(kLoneThreads) void k_ortho_lone(OrthoLoneArgs<N, C> a) {
  const uint64_t task = (uint64_t)(a.tasks + blockIdx.x);
  struct TaskWords {
    uint32_t w[sizeof(OrthoTask) / 4];
  } task_words;
#pragma unroll
  for (uint32_t i = 0; i < sizeof(OrthoTask) / 4; ++i) task_words.w[i] = global<const uint32_t>(task)[i];
  const OrthoTask t = __builtin_bit_cast(OrthoTask, task_words);
  const uint32_t replica = blockIdx.y, rows = t.tall ? t.q : t.p, cols = t.tall ? t.p : t.q, pieces = (cols + 7) / 8, xp = t.Q + 4;
  const Words x = (Words)lone_lds, A = x + t.P * xp, diagonal = A + t.P * (t.P + 4), parts = diagonal + t.P;
  const uint64_t g = (uint64_t)a.grad[replica], mh = (uint64_t)a.m_hat[replica], b = (uint64_t)a.acc[replica];
  for (uint32_t k = threadIdx.x; k < t.P * xp; k += kLoneThreads) x[k] = 0;
  __syncthreads();
  double sum = 0.0;
  for (uint32_t k = threadIdx.x; k < rows * pieces; k += kLoneThreads) {
    const uint32_t r = k / pieces, c = k % pieces * 8, n = left(cols, c);
    const uint64_t e = t.first + (uint64_t)r * t.ld + c;
    float gv[8], m[8], v[8];
    load_source<GT>(a.c, a.source, g, mh, e, n, gv, m, v);
    if (a.source != kOrthoGiven) move_moment(a.c, a.phase, mh, b, e, n, gv, m);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      if (i >= n) continue;
      sum = fma((double)v[i], (double)v[i], sum);
      x[t.tall ? (c + i) * xp + r : r * xp + c + i] = __float_as_uint(v[i]);
    }
  }
  __shared__ double sums[kWaves];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (uint32_t k = 0; k < kWaves; ++k) sum += sums[k];
  const float factor = (float)((double)a.scale / (sqrt(sum) + 1e-7));
  for (uint32_t k = threadIdx.x; k < t.P * xp; k += kLoneThreads) x[k] = halves<Half>(__uint_as_float(x[k]) * factor);
  __syncthreads();
  for (uint32_t k = 0; k < a.n_steps; ++k) {
    const bool last = k + 1 == a.n_steps;
    switch (t.P / 32) {
      case 1: iterate<1>(x, A, diagonal, parts, t.P, t.Q, a.step[k], last); break;
      case 2: iterate<2>(x, A, diagonal, parts, t.P, t.Q, a.step[k], last); break;
      case 3: iterate<3>(x, A, diagonal, parts, t.P, t.Q, a.step[k], last); break;
      default: iterate<4>(x, A, diagonal, parts, t.P, t.Q, a.step[k], last); break;
    }
  }
  const uint64_t out = (uint64_t)a.out[replica];
  const int32_t first = a.mix ? global<const int32_t>(a.row_ptr)[a.first_row + replica] : 0, end = a.mix ? global<const int32_t>(a.row_ptr)[a.first_row + replica + 1] : 0;
  for (uint32_t k = threadIdx.x; k < rows * pieces; k += kLoneThreads) {
    const uint32_t r = k / pieces, c = k % pieces * 8, n = left(cols, c);
    const uint64_t e = t.first + (uint64_t)r * t.ld + c;
    float v[8], source[8], mixed[8] = {};
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = i < n ? __uint_as_float(x[t.tall ? (c + i) * xp + r : r * xp + c + i]) : 0.f;
    if (!a.mix) {
      DT::store8(out, e, n, v);
      continue;
    }
    for (int32_t q = first; q < end; ++q) {
      const float weight = global<const float>(a.w)[q];
      DT::load8((uint64_t)a.x_src[global<const int32_t>(a.col)[q]], e, n, source);
#pragma unroll
      for (int i = 0; i < 8; ++i) mixed[i] = q == first ? weight * source[i] : fmaf(weight, source[i], mixed[i]);
    }
    if (t.decay != 0.f) DT::load8((uint64_t)a.x_src[a.first_row + replica], e, n, source);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float direction = t.scale * v[i];
      if (t.decay != 0.f) direction = fmaf(t.decay, source[i], direction);
      mixed[i] = fmaf(-a.lr, direction, mixed[i]);
    }
    DT::store8(out, e, n, mixed);
  }
}

template <auto KERNEL, typename A>
int launch(const A& a, uint32_t matrices, uint32_t replicas, uint32_t lds, void* stream) {
  if (lds > 65536)
    if (const int e = ask_for_lds<KERNEL>(kMostLoneLds)) return e;
  KERNEL<<<dim3(matrices, replicas), kLoneThreads, lds, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

template <int N, int C>
OrthoLoneArgs<N, C> shorter(const OrthoLoneArgs<kLoneRows, kMaxRows>& a) {
  OrthoLoneArgs<N, C> s{};
  s.tasks = a.tasks, s.n_steps = a.n_steps, s.source = a.source, s.phase = a.phase, s.mix = a.mix, s.first_row = a.first_row, s.scale = a.scale, s.lr = a.lr, s.c = a.c;
  s.row_ptr = a.row_ptr, s.col = a.col, s.w = a.w;
  for (uint32_t k = 0; k < DADAM_ORTHO_MAX_STEPS; ++k) s.step[k] = a.step[k];
  for (int k = 0; k < N; ++k) s.grad[k] = a.grad[k], s.m_hat[k] = a.m_hat[k], s.acc[k] = a.acc[k], s.out[k] = a.out[k];
  for (int k = 0; k < C; ++k) s.x_src[k] = a.x_src[k];
  return s;
}

template <typename GT, typename DT>
int lone(const OrthoLoneArgs<kLoneRows, kMaxRows>& a, uint32_t n_cols, uint32_t matrices, uint32_t replicas, uint32_t lds, void* stream) {
  if (replicas <= (uint32_t)kOrthoFew && n_cols <= (uint32_t)kOrthoFew)
    return launch<k_ortho_lone<GT, DT, kOrthoFew, kOrthoFew>>(shorter<kOrthoFew, kOrthoFew>(a), matrices, replicas, lds, stream);
  return launch<k_ortho_lone<GT, DT, kLoneRows, kMaxRows>>(a, matrices, replicas, lds, stream);
}

}  // namespace

int launch_ortho_lone(int gdt, int dtype, const OrthoLoneArgs<kLoneRows, kMaxRows>& a, uint32_t n_cols, uint32_t matrices, uint32_t replicas, uint32_t lds, void* stream) {
  if (gdt == (int)DADAM_F32)
    return dtype == (int)DADAM_F32 ? lone<F32, F32>(a, n_cols, matrices, replicas, lds, stream) : lone<F32, B16>(a, n_cols, matrices, replicas, lds, stream);
  return dtype == (int)DADAM_F32 ? lone<B16, F32>(a, n_cols, matrices, replicas, lds, stream) : lone<B16, B16>(a, n_cols, matrices, replicas, lds, stream);
}

}  // namespace dadam
