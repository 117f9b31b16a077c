// The loss of a language model's head: z = W h + bias, nll = log sum exp z - z[target], and with s the gradient's scale
//     dz = s (softmax z - e[target]),   dh = sum over words dz W,   dW = sum over tokens dz h,   dbias = sum over tokens dz.
//
// The logits never leave the chip.  A first product gives every token the largest logit and the sum of exponentials of every kHeadSlice words
// (k_head_logits), from which k_head_losses makes the logarithm of the sum; a second one recomputes the logits a piece of the vocabulary at a time
// and stores softmax - e[target] of it, both ways round, as the operand of the two gradient products.  dW of a piece is complete; dh adds up
// over pieces.  Four products of tokens x vocabulary x width, of which a program that keeps the logits (4 bytes for each, read and written
// several times) needs three.
//
// bfloat16 parameters and gradients: the operands are what is given, softmax - e[target] is rounded to bfloat16, 8 bits relative whatever its size;
// sums are float32.  Otherwise: two halves an element (dadam_mfma.h), times a power of two by the largest magnitude of the head and of the
// hidden vectors, so that an element is held to 22 bits or to 2^-39 of the largest.  Tokens without a target: their hidden vectors are taken as zeros,
// whatever they hold.
#include "dadam_head.h"
#include "dadam_mfma.h"

namespace dadam {
namespace {

extern __shared__ char head_lds[];

template <typename XT, typename GT>
struct Types;  // operands
template <>
struct Types<B16, B16> {
  using op = Brain;
  static constexpr int planes = 1;
};
template <>
struct Types<F32, F32> {
  using op = Half;
  static constexpr int planes = 2;
};
template <>
struct Types<B16, F32> : Types<F32, F32> {};
template <>
struct Types<F32, B16> : Types<F32, F32> {};

template <typename TY>
using HeadTile = Tile<typename TY::op, TY::planes, 2, 2, 2, 2>;

constexpr int kHeldAt = 13;  // operands of two planes are brought to at most 2^13, an eighth of what a half can hold

// The power of two that brings what is at most `most` (the bits of a finite float) to at most 2^kHeldAt.
__device__ __forceinline__ int held_power(uint32_t most) {
  const int e = (int)(most >> 23) - 126;  // below 2^e; -126 where it is subnormal or 0
  const int p = kHeldAt - e;
  return p > 120 ? 120 : p;
}

template <typename TY>
__device__ __forceinline__ int power_of(uint64_t base, const HeadArgs& a, HeadWord word) {
  if constexpr (TY::planes == 1) return 0;
  return held_power(global<const uint32_t>(base + a.w.words)[word]);
}

__device__ __forceinline__ uint64_t base_of(const HeadArgs& a) { return a.workspace + (uint64_t)blockIdx.z * a.stride; }

__device__ __forceinline__ bool has_target(const HeadArgs& a, uint64_t target, uint32_t t, int32_t& word) {
  word = -1;
  if (t >= a.s.tokens) return false;
  word = global<const int32_t>(target)[t];
  return word >= 0 && (uint32_t)word < a.s.vocab;
}

// The factor of the gradients and of the loss.
__device__ __forceinline__ float factor_of(uint64_t base, const HeadArgs& a) {
  const float count = global<const float>(base + a.w.words)[kHeadCount];
  return a.mean ? a.scale / fmaxf(count, 1.f) : a.scale;
}

// Tokens with a target, and the words of the largest magnitudes cleared.
__global__ __launch_bounds__(256) void k_head_count(HeadArgs a) {
  const uint64_t base = base_of(a), target = a.row[blockIdx.z].target;
  __shared__ uint32_t parts[4];
  uint32_t n = 0;
  int32_t word;
  for (uint32_t t = threadIdx.x; t < a.s.tokens; t += 256) n += has_target(a, target, t, word) ? 1 : 0;
#pragma unroll
  for (int step = 32; step; step >>= 1) n += __shfl_xor(n, step);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    global<float>(base + a.w.words)[kHeadCount] = (float)(parts[0] + parts[1] + parts[2] + parts[3]);
    global<uint32_t>(base + a.w.words)[kHeadMostHidden] = 0;
    global<uint32_t>(base + a.w.words)[kHeadMostHead] = 0;
  }
}

// Largest finite magnitudes: of the hidden vectors of tokens with a target (blockIdx.y 0) and of the head (1).  The largest is the same in any order.
constexpr uint32_t kMostEach = 16;  // elements a thread looks at
template <typename XT>
__global__ __launch_bounds__(256) void k_head_most(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const bool head = blockIdx.y;
  const uint64_t n = (uint64_t)(head ? a.s.vocab : a.s.tokens) * a.s.width, data = head ? row.head : row.hidden;
  uint32_t most = 0;
  uint64_t e = (uint64_t)blockIdx.x * (256 * kMostEach) + threadIdx.x;
#pragma unroll
  for (uint32_t k = 0; k < kMostEach; ++k, e += 256) {
    if (e >= n) continue;
    const uint32_t v = __float_as_uint(XT::load(data, e)) & 0x7fffffffu;
    int32_t word;
    const bool taken = head || has_target(a, row.target, (uint32_t)(e / a.s.width), word);
    if (taken && v < 0x7f800000u && v > most) most = v;
  }
#pragma unroll
  for (int step = 32; step; step >>= 1) {
    const uint32_t other = __shfl_xor(most, step);
    most = other > most ? other : most;
  }
  if (threadIdx.x % 64 == 0 && most)
    __hip_atomic_fetch_max(global<uint32_t>(base_of(a) + a.w.words) + (head ? kHeadMostHead : kHeadMostHidden), most, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A 64 x 64 tile of a matrix of `rows` rows and a.s.width columns as operands: as it lies (`plain`, of a.s.K columns), and if `turned` is there, the other
// way round (of `across` columns).  Beyond the matrix stand zeros.
constexpr uint32_t kCut = 64, kCutPitch = kCut + 1;
template <typename XT, typename TY>
__device__ __forceinline__ void operands(uint64_t data, uint32_t rows, uint32_t width, float factor, uint64_t plain, uint32_t K, uint64_t turned, uint32_t D,
                                         uint32_t across, uint64_t target, const HeadArgs& a) {
  using OP = typename TY::op;
  const uint32_t r0 = blockIdx.x * kCut, c0 = blockIdx.y * kCut, col = c0 + threadIdx.x % kCut;
  float DADAM_LDS* tile = (float DADAM_LDS*)head_lds;
  for (uint32_t r = threadIdx.x / kCut; r < kCut; r += 256 / kCut) {
    float v = 0.f;
    int32_t word;
    if (r0 + r < rows && col < width && (!target || has_target(a, target, r0 + r, word))) v = XT::load(data, (uint64_t)(r0 + r) * width + col) * factor;
    tile[r * kCutPitch + threadIdx.x % kCut] = v;
  }
  __syncthreads();
  const uint32_t k4 = threadIdx.x % 16 * 4;
  for (uint32_t r = threadIdx.x / 16; r < kCut; r += 16) {
    float4v v, t;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = tile[r * kCutPitch + k4 + e], t[e] = tile[(k4 + e) * kCutPitch + r];
    if (c0 < K) store4<OP, TY::planes>(plain, r0 + r, K, c0 + k4, v);
    if (turned && c0 < D) store4<OP, TY::planes>(turned, c0 + r, across, r0 + k4, t);
  }
}

template <typename XT, typename TY>
__global__ __launch_bounds__(256) void k_head_hidden(HeadArgs a, uint32_t gradient) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const float factor = ldexpf(1.f, power_of<TY>(base, a, kHeadMostHidden));
  operands<XT, TY>(row.hidden, a.s.tokens, a.s.width, factor, base + a.w.hidden_n, a.s.K, gradient ? base + a.w.hidden_t : 0, a.s.D, a.s.T, row.target, a);
}
template <typename XT, typename TY>
__global__ __launch_bounds__(256) void k_head_words(HeadArgs a, uint32_t turned) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const float factor = ldexpf(1.f, power_of<TY>(base, a, kHeadMostHead));
  const uint64_t bytes = sizeof(typename XT::type);
  operands<XT, TY>(row.head + (uint64_t)a.first_word * a.s.width * bytes, a.words, a.s.width, factor, base + a.w.head_n, a.s.K, turned ? base + a.w.head_t : 0, a.s.D,
                   a.s.piece, 0, a);
}

// The logits of a tile of words (m) and tokens (n).  Without gradients: the largest and the sum of exponentials of each wavefront's words, and the
// target's logit.  With: softmax - e[target], both ways round.
template <typename XT, typename TY, bool GRADIENT>
__global__ __launch_bounds__(256) void k_head_logits(HeadArgs a) {
  using T = HeadTile<TY>;
  using OP = typename TY::op;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.T / T::kN, u = die_run(blockIdx.x, gridDim.x, a.n_xcd), i = u / across, j = u % across;
  const uint64_t pitch = (uint64_t)a.s.K * 2 * TY::planes;
  T t;
  t.product(global<const char>(base + a.w.head_n) + (uint64_t)i * T::kM * pitch, pitch, global<const char>(base + a.w.hidden_n) + (uint64_t)j * T::kN * pitch, pitch,
            (uint32_t)(pitch / kStageBytes), (char DADAM_LDS*)head_lds);
  const float held = ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHidden) - power_of<TY>(base, a, kHeadMostHead));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % 2, wn = wave / 2;
#pragma unroll
  for (int jn = 0; jn < 2; ++jn) {
    const uint32_t n = j * T::kN + wn * 64 + jn * 32 + (lane & 31);
    int32_t target;
    const bool taken = has_target(a, row.target, n, target);
    const float lse = GRADIENT && taken ? global<const float>(base + a.w.lse)[n] : 0.f;
    float most = -INFINITY;
#pragma unroll
    for (int im = 0; im < 2; ++im)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t m = i * T::kM + wm * 64 + im * 32 + g * 8 + (lane >> 5) * 4;  // in the piece
        float4v z;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[e] = t.acc[im][jn][4 * g + e] * held;
          const uint32_t word = a.first_word + m + e;
          if (row.bias && m + e < a.words) z[e] += XT::load(row.bias, word);
          if constexpr (GRADIENT) {
            float p = 0.f;
            if (taken && m + e < a.words) p = word == (uint32_t)target ? expm1f(z[e] - lse) : __expf(z[e] - lse);
            z[e] = TY::planes == 1 ? p : p * (float)(1 << kHeldAt);
          } else {
            if (taken && word == (uint32_t)target) global<float>(base + a.w.hit)[n] = z[e];
            if (m + e >= a.words) z[e] = -INFINITY;
            most = fmaxf(most, z[e]);
            t.acc[im][jn][4 * g + e] = z[e];
          }
        }
        if constexpr (GRADIENT) {
          store4<OP, TY::planes>(base + a.w.p_n, n, a.s.piece, m, z);
#pragma unroll
          for (int e = 0; e < 4; ++e) store1<OP, TY::planes>(base + a.w.p_t, m + e, a.s.T, n, z[e]);
        }
      }
    if constexpr (!GRADIENT) {
      most = fmaxf(most, __shfl_xor(most, 32));
      float sum = 0.f;
      const float from = most == -INFINITY ? 0.f : most;  // nothing but words that cannot come: a sum of 0
#pragma unroll
      for (int im = 0; im < 2; ++im)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += __expf(t.acc[im][jn][r] - from);
      sum += __shfl_xor(sum, 32);
      if (lane < 32) {
        const uint32_t slice = (a.first_word + i * T::kM) / kHeadSlice + wm;
        global<float>(base + a.w.stats)[((uint64_t)slice * a.s.T + n) * 2] = most;
        global<float>(base + a.w.stats)[((uint64_t)slice * a.s.T + n) * 2 + 1] = sum;
      }
    }
  }
}

// Every token's logarithm of the sum of exponentials and its loss: 32 tokens a workgroup, eight threads a token.
__device__ __forceinline__ void join(float& most, float& sum, float other, float more) {
  const float top = fmaxf(most, other);
  if (top == -INFINITY) {  // words that cannot come, or NaN
    sum += more;
    return;
  }
  sum = sum * __expf(most - top) + more * __expf(other - top);
  most = top;
}
__global__ __launch_bounds__(256) void k_head_losses(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t n = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32;
  float most = -INFINITY, sum = 0.f;
  for (uint32_t s = part; s < a.s.slices; s += 8) {
    const uint64_t at = ((uint64_t)s * a.s.T + n) * 2;
    join(most, sum, global<const float>(base + a.w.stats)[at], global<const float>(base + a.w.stats)[at + 1]);
  }
  __shared__ float mosts[8][32], sums[8][32];
  mosts[part][threadIdx.x % 32] = most;
  sums[part][threadIdx.x % 32] = sum;
  __syncthreads();
  if (part == 0) {
    for (uint32_t k = 1; k < 8; ++k) join(most, sum, mosts[k][threadIdx.x], sums[k][threadIdx.x]);
    int32_t target;
    const bool taken = has_target(a, row.target, n, target);
    const float lse = most + logf(sum);
    global<float>(base + a.w.lse)[n] = lse;
    // (of a token that is as good as certain of its word the difference is the sum's rounding: never below 0)
    const float nll = taken ? lse - global<const float>(base + a.w.hit)[n] : 0.f;
    if (n < a.s.tokens && row.nll) global<float>(row.nll)[n] = nll;
    global<float>(base + a.w.hit)[n] = nll;
  }
}

// The loss of a replica, summed in 64 bits in the order of the tokens' numbers by 256.
__global__ __launch_bounds__(256) void k_head_sum(HeadArgs a) {
  const uint64_t base = base_of(a);
  __shared__ double parts[4];
  double sum = 0.0;
  for (uint32_t t = threadIdx.x; t < a.s.tokens; t += 256) sum += (double)global<const float>(base + a.w.hit)[t];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double count = (double)global<const float>(base + a.w.words)[kHeadCount], all = parts[0] + parts[1] + parts[2] + parts[3];
    global<float>(a.losses)[blockIdx.z] = (float)((double)a.scale * all / (a.mean && count > 1.0 ? count : 1.0));
  }
}

// dW of a tile of columns (m) and words (n).
template <typename XT, typename GT, typename TY>
__global__ __launch_bounds__(256) void k_head_dhead(HeadArgs a) {
  using T = HeadTile<TY>;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.D / T::kM, u = die_run(blockIdx.x, gridDim.x, a.n_xcd), i = u % across, j = u / across;
  const uint64_t pitch = (uint64_t)a.s.T * 2 * TY::planes;
  T t;
  t.product(global<const char>(base + a.w.hidden_t) + (uint64_t)i * T::kM * pitch, pitch, global<const char>(base + a.w.p_t) + (uint64_t)j * T::kN * pitch, pitch,
            (uint32_t)(pitch / kStageBytes), (char DADAM_LDS*)head_lds);
  const float factor = factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHidden) - kHeldAt));
  t.each([&](uint32_t m, uint32_t n, float4v v) {
    m += i * T::kM;
    n += j * T::kN;
    if (n >= a.words) return;
    const uint64_t e = (uint64_t)(a.first_word + n) * a.s.width + m;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (m + k >= a.s.width) continue;
      const float g = v[k] * factor;
      GT::store(row.dhead, e + k, a.add ? GT::load(row.dhead, e + k) + g : g);
    }
  });
}

// dbias: a wavefront a word.
template <typename GT, typename TY>
__global__ __launch_bounds__(256) void k_head_dbias(HeadArgs a) {
  using OP = typename TY::op;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t n = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
  if (n < a.words) {
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t t = lane * 4; t < a.s.T; t += 256) sum += load4<OP, TY::planes>(base + a.w.p_t, n, a.s.T, t);
    float all = sum[0] + sum[1] + (sum[2] + sum[3]);
#pragma unroll
    for (int step = 32; step; step >>= 1) all += __shfl_xor(all, step);
    if (lane == 0) {
      const float g = all * factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -kHeldAt));
      const uint64_t e = a.first_word + n;
      GT::store(row.dbias, e, a.add ? GT::load(row.dbias, e) + g : g);
    }
  }
}

// dh of a tile of columns (m) and tokens (n), over a part of the piece's words.
template <typename TY>
__global__ __launch_bounds__(256) void k_head_dhidden(HeadArgs a) {
  using T = HeadTile<TY>;
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.D / T::kM, u = die_run(blockIdx.x, gridDim.x, a.n_xcd), i = u % across, j = u / across, split = blockIdx.y;
  const uint64_t pitch = (uint64_t)a.s.piece * 2 * TY::planes;
  const uint32_t stages = (uint32_t)(((uint64_t)(a.words + kHeadTile - 1) / kHeadTile * kHeadTile * 2 * TY::planes) / kStageBytes);
  const uint32_t from = (uint32_t)((uint64_t)stages * split / a.s.splits), to = (uint32_t)((uint64_t)stages * (split + 1) / a.s.splits);
  T t;
  t.clear();
  if (from < to)
    t.product(global<const char>(base + a.w.head_t) + (uint64_t)i * T::kM * pitch + (uint64_t)from * kStageBytes, pitch,
              global<const char>(base + a.w.p_n) + (uint64_t)j * T::kN * pitch + (uint64_t)from * kStageBytes, pitch, to - from, (char DADAM_LDS*)head_lds);
  float4v DADAM_GLOBAL* sums = global<float4v>(base + a.w.sums + (uint64_t)split * a.s.T * a.s.D * 4);
  t.each([&](uint32_t m, uint32_t n, float4v v) {
    float4v DADAM_GLOBAL* at = sums + ((uint64_t)(j * T::kN + n) * a.s.D + i * T::kM + m) / 4;
    *at = a.later ? *at + v : v;
  });
}

template <typename XT, typename TY>
__global__ __launch_bounds__(256) void k_head_end(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a), each = (uint64_t)a.s.T * a.s.D;
  const float factor = factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHead) - kHeldAt));
  const uint32_t n = blockIdx.x;
  int32_t target;
  const bool taken = has_target(a, row.target, n, target);
  for (uint32_t c = threadIdx.x; c < a.s.width; c += 256) {
    float v = 0.f;
    if (taken)
      for (uint32_t s = 0; s < a.s.splits; ++s) v += global<const float>(base + a.w.sums)[s * each + (uint64_t)n * a.s.D + c];
    XT::store(row.dhidden, (uint64_t)n * a.s.width + c, v * factor);
  }
}

template <typename K, typename... A>
int launch(K kernel, dim3 grid, uint32_t lds, void* stream, const A&... a) {
  kernel<<<grid, 256, lds, (hipStream_t)stream>>>(a...);
  return (int)hipGetLastError();
}

// fn(types of parameters, gradients and operands) for a pair of element types.
template <typename Fn>
int with_types(int xdt, int gdt, Fn fn) {
  if (xdt == (int)DADAM_BF16) return gdt == (int)DADAM_BF16 ? fn(B16{}, B16{}, Types<B16, B16>{}) : fn(B16{}, F32{}, Types<B16, F32>{});
  return gdt == (int)DADAM_BF16 ? fn(F32{}, B16{}, Types<F32, B16>{}) : fn(F32{}, F32{}, Types<F32, F32>{});
}

constexpr uint32_t kCutLds = kCut * kCutPitch * 4;
uint32_t upto(uint64_t n, uint32_t each) { return (uint32_t)((n + each - 1) / each); }

}  // namespace

int launch_head_begin(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  int e = launch(k_head_count, dim3(1, 1, rows), 0, stream, a);
  if (e || (xdt == (int)DADAM_BF16 && gdt == (int)DADAM_BF16)) return e;
  const uint64_t n = (uint64_t)(a.s.vocab > a.s.tokens ? a.s.vocab : a.s.tokens) * a.s.width;
  const dim3 grid(upto(n, 256 * kMostEach), 2, rows);
  return xdt == (int)DADAM_BF16 ? launch(k_head_most<B16>, grid, 0, stream, a) : launch(k_head_most<F32>, grid, 0, stream, a);
}
int launch_head_hidden(int xdt, int gdt, bool gradient, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) {
    const uint32_t columns = gradient ? a.s.D : a.s.K;
    return launch(k_head_hidden<decltype(x), decltype(ty)>, dim3(a.s.T / kCut, upto(columns, kCut), rows), kCutLds, stream, a, (uint32_t)gradient);
  });
}
int launch_head_words(int xdt, int gdt, bool turned, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) {
    const uint32_t columns = turned ? a.s.D : a.s.K, words = upto(a.words, kHeadTile) * kHeadTile;
    return launch(k_head_words<decltype(x), decltype(ty)>, dim3(words / kCut, upto(columns, kCut), rows), kCutLds, stream, a, (uint32_t)turned);
  });
}
int launch_head_logits(int xdt, int gdt, bool gradient, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) {
    using X = decltype(x);
    using TY = decltype(ty);
    const dim3 grid(upto(a.words, kHeadTile) * (a.s.T / kHeadTile), 1, rows);
    return gradient ? launch(k_head_logits<X, TY, true>, grid, HeadTile<TY>::kLds, stream, a) : launch(k_head_logits<X, TY, false>, grid, HeadTile<TY>::kLds, stream, a);
  });
}
int launch_head_losses(const HeadArgs& a, uint32_t rows, void* stream) {
  if (const int e = launch(k_head_losses, dim3(a.s.T / 32, 1, rows), 0, stream, a)) return e;
  return launch(k_head_sum, dim3(1, 1, rows), 0, stream, a);
}
int launch_head_dhead(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto g, auto ty) {
    return launch(k_head_dhead<decltype(x), decltype(g), decltype(ty)>, dim3(upto(a.words, kHeadTile) * (a.s.D / kHeadTile), 1, rows), HeadTile<decltype(ty)>::kLds, stream, a);
  });
}
int launch_head_dbias(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto, auto g, auto ty) { return launch(k_head_dbias<decltype(g), decltype(ty)>, dim3(upto(a.words, 4), 1, rows), 0, stream, a); });
}
int launch_head_dhidden(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto, auto, auto ty) {
    return launch(k_head_dhidden<decltype(ty)>, dim3((a.s.T / kHeadTile) * (a.s.D / kHeadTile), a.s.splits, rows), HeadTile<decltype(ty)>::kLds, stream, a);
  });
}
int launch_head_end(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) { return launch(k_head_end<decltype(x), decltype(ty)>, dim3(a.s.tokens, 1, rows), 0, stream, a); });
}

}  // namespace dadam
