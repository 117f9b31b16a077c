// The loss of a language model's head: z = W h + bias, nll = log sum exp z - z[target], and with s the gradient's scale
//     dz = s (softmax z - e[target]),   dh = sum over words dz W,   dW = sum over tokens dz h,   dbias = sum over tokens dz.
//
// Two ways.  Where the workspace has room for 2 (or two planes: 4) bytes for every logit, the product of the logits stores the exponentials of each slice of
// words against the slice's largest logit, and k_head_scale makes softmax - e[target] of them in place once the sums are known: three products of tokens x
// vocabulary x width.  Elsewhere nothing of the logits leaves the chip but a piece of the vocabulary at a time.  A first product gives every token the largest
// logit and the sum of exponentials of some words (k_head_logits), from which k_head_losses makes the logarithm of the sum; a second one recomputes the logits
// a piece of the vocabulary at a time and stores softmax - e[target] of it, the operand of the two gradient products.  dW of a piece is complete; dh adds up over
// pieces.  Four products.  (Up to 64 tokens: dadam_head_few.hip.)
// All operands lie as they are made: the gradients sum over tokens and over words, so their tiles are turned on the way from LDS to the registers.
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

__device__ __forceinline__ uint32_t left(uint32_t n, uint32_t at) { return at < n ? n - at : 0; }

// Operands of two planes are brought to at most 2^15, half of what a half can hold: its smallest step is then 2^-38 of the largest or less, rounded 2^-39.
constexpr int kHeldAt = 15;

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

// Largest finite magnitudes: of the head (blockIdx.y 0) and of the hidden vectors of tokens with a target (1), of every workgroup's share.
__device__ __forceinline__ void larger(uint32_t& most, float v) {
  const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
  if (b < 0x7f800000u && b > most) most = b;
}
template <typename XT>
__global__ __launch_bounds__(256) void k_head_most(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  uint32_t most = 0;
  float v[8];
  if (blockIdx.y == 0) {
    const uint64_t n = (uint64_t)a.s.vocab * a.s.width;
    const uint64_t step = (uint64_t)gridDim.x * 2048;
    uint64_t e = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (row.head % 16 == 0)
      for (; e + 3 * step + 8 <= n; e += 4 * step) {  // four loads on their way at a time
        uint4v b[4][sizeof(typename XT::type) / 2];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
          for (uint32_t h = 0; h < sizeof(typename XT::type) / 2; ++h) b[k][h] = global<const uint4v>(row.head + (e + k * step) * sizeof(typename XT::type))[h];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
          for (uint32_t h = 0; h < sizeof(typename XT::type) / 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (sizeof(typename XT::type) == 4) {
                larger(most, __uint_as_float(b[k][h][i]));
              } else {
                larger(most, __uint_as_float(b[k][h][i] << 16));
                larger(most, __uint_as_float(b[k][h][i] & 0xffff0000u));
              }
            }
      }
    for (; e < n; e += step) {
      XT::load8(row.head, e, n - e < 8 ? (uint32_t)(n - e) : 8, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) larger(most, v[k]);
    }
  } else {
    int32_t word;
    for (uint32_t t = blockIdx.x; t < a.s.tokens; t += gridDim.x) {
      if (!has_target(a, row.target, t, word)) continue;
      for (uint32_t c = threadIdx.x * 8; c < a.s.width; c += 2048) {
        XT::load8(row.hidden, (uint64_t)t * a.s.width + c, left(a.s.width, c), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) larger(most, v[k]);
      }
    }
  }
#pragma unroll
  for (int step = 32; step; step >>= 1) {
    const uint32_t other = __shfl_xor(most, step);
    most = other > most ? other : most;
  }
  __shared__ uint32_t parts[4];
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 4; ++k) most = parts[k] > most ? parts[k] : most;
    global<uint32_t>(base_of(a) + a.w.words)[kHeadShares + blockIdx.y * kMostGroups + blockIdx.x] = most;
  }
}

// The power of two of an operand, by all threads of a workgroup: from the workgroups' largest, of which the first one here leaves the largest for the others, or (a later
// piece of the head) as it was left.
template <typename TY>
__device__ __forceinline__ int found_power(uint64_t base, const HeadArgs& a, HeadWord word) {
  if constexpr (TY::planes == 1) return 0;
  if (a.groups == 0) return power_of<TY>(base, a, word);
  const uint32_t DADAM_GLOBAL* shares = global<const uint32_t>(base + a.w.words) + kHeadShares + (word == kHeadMostHead ? 0 : kMostGroups);
  uint32_t most = 0;
  for (uint32_t k = threadIdx.x; k < a.groups; k += 256) most = shares[k] > most ? shares[k] : most;
#pragma unroll
  for (int step = 32; step; step >>= 1) {
    const uint32_t other = __shfl_xor(most, step);
    most = other > most ? other : most;
  }
  __shared__ uint32_t parts[4];
  if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = most;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) most = parts[k] > most ? parts[k] : most;
  if (blockIdx.x == 0 && threadIdx.x == 0) global<uint32_t>(base + a.w.words)[word] = most;
  return held_power(most);
}

// `rows` rows of `width` elements as an operand of a.s.D columns, `filled` rows in all; the rest zeros.  A thread takes eight elements, four times.
constexpr uint32_t kOperandPieces = 4;
template <typename XT, typename TY>
__device__ __forceinline__ void make_operand(uint64_t data, uint32_t rows, uint32_t filled, HeadWord most, uint64_t base, uint64_t to, uint64_t target, const HeadArgs& a) {
  using OP = typename TY::op;
  const uint32_t each = a.s.D / 8;
  float v[kOperandPieces][8];
#pragma unroll
  for (uint32_t i = 0; i < kOperandPieces; ++i) {
    const uint64_t e = ((uint64_t)blockIdx.x * kOperandPieces + i) * 256 + threadIdx.x;
    const uint32_t r = (uint32_t)(e / each), c = (uint32_t)(e % each) * 8, n = r < rows && r < filled ? left(a.s.width, c) : 0;
    int32_t word;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
    if (n && (!target || has_target(a, target, r, word))) XT::load8(data, (uint64_t)r * a.s.width + c, n, v[i]);
  }
  const float factor = ldexpf(1.f, found_power<TY>(base, a, most));  // (while the elements are on their way)
#pragma unroll
  for (uint32_t i = 0; i < kOperandPieces; ++i) {
    const uint64_t e = ((uint64_t)blockIdx.x * kOperandPieces + i) * 256 + threadIdx.x;
    const uint32_t r = (uint32_t)(e / each), c = (uint32_t)(e % each) * 8;
    if (r >= filled) return;
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = operand_word<OP, TY::planes>(v[i][k] * factor);
    store8<TY::planes>(to, r, a.s.D, c, w);
  }
}

// The operands that are not read as they lie: a piece of the head (blockIdx.y 0), the hidden vectors (1, or 0 where the head lies as it should).
template <typename XT, typename TY>
__global__ __launch_bounds__(256) void k_head_operands(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a), from = row.head + (uint64_t)a.first_word * a.s.width * sizeof(typename XT::type);
  if (blockIdx.y == 0 && !a.straight)
    make_operand<XT, TY>(from, a.words, (a.words + a.s.edge - 1) / a.s.edge * a.s.edge, kHeadMostHead, base, base + a.w.head, 0, a);
  else
    make_operand<XT, TY>(row.hidden, a.s.tokens, a.s.T, kHeadMostHidden, base, base + a.w.hidden, row.target, a);
}

// The piece's words as an operand, rows from `row` on: as they lie in the parameters, or their copy.
template <typename TY>
__device__ __forceinline__ Operand head_operand(uint64_t base, const HeadRow& row, const HeadArgs& a, uint32_t first, uint64_t offset) {
  const uint64_t pitch = (uint64_t)a.s.D * 2 * TY::planes;
  if (a.straight) return operand(row.head + (uint64_t)(a.first_word + first) * pitch + offset, pitch, a.words - first);
  return operand(base + a.w.head + first * pitch + offset, pitch);
}

// What a slice's exponentials, at most 1, are kept times.  For bfloat16 they are kept in half precision, which has three bits more than what is made of them: times
// 2^15 those down to 2^-29 have 11 bits, the others 2^-40 of the slice's largest.
template <typename TY>
__device__ __forceinline__ constexpr float kept_times() {
  return TY::planes == 1 ? 32768.f : (float)(1 << kHeldAt);
}

// The logits of a tile of words (m) and tokens (n).  Without gradients: the largest and the sum of exponentials of each wavefront's words, and the
// target's logit.  With: softmax - e[target].  (2048 tokens, 50257 words, width 1024, bfloat16, without gradients 219 us, 963 TFLOP/s; two replicas of 4096 tokens with the
// exponentials kept 1058 us, 796: behind its product a tile computes and stores 65536 exponentials while nobody multiplies.)
template <typename XT, typename TY, int EDGE, int BUFFERS, int MODE>
__global__ __launch_bounds__(2 * EDGE) void k_head_logits(HeadArgs a) {
  using T = TileOf<typename TY::op, TY::planes, EDGE, BUFFERS, false, false, TY::planes == 2 && BUFFERS == 4>;
  using OP = typename TY::op;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.T / T::kN;
  uint32_t i, j;
  banded(die_run(blockIdx.x, gridDim.x, a.n_xcd), across, gridDim.x / across, j, i);
  char DADAM_LDS* lds = (char DADAM_LDS*)head_lds;
  const uint64_t pitch = (uint64_t)a.s.D * 2 * TY::planes;
  T t;
  // (words beyond the piece come to nothing below, whatever stands for them)
  t.product(head_operand<TY>(base, row, a, i * T::kM, 0), operand(base + a.w.hidden + (uint64_t)j * T::kN * pitch, pitch), a.s.K * TY::planes / 64, lds);
  const float held = ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHidden) - power_of<TY>(base, a, kHeadMostHead));
  if constexpr (MODE == kHeadGradient) {
    struct Token {
      int32_t target;  // -1: none
      float2v top;
    };
    t.hand_out(lds, false,
               [&](uint32_t, uint32_t n) {
                 Token x;
                 if (!has_target(a, row.target, j * T::kN + n, x.target)) x.target = -1;
                 x.top = global<const float2v>(base + a.w.top)[j * T::kN + n];
                 return x;
               },
               [&](uint32_t m, uint32_t n, float (&v)[8], const Token& x) {
                 m += i * T::kM;
                 n += j * T::kN;
                 const bool taken = x.target >= 0;
                 const uint32_t words = left(a.words, m);
                 float bias[8] = {};
                 if (row.bias && words) XT::load8(row.bias, a.first_word + m, words, bias);
                 const uint32_t hit = (uint32_t)x.target - a.first_word - m;
                 uint32_t w[8];
#pragma unroll
                 for (uint32_t k = 0; k < 8; ++k) {
                   const float z = fmaf(v[k], held, bias[k]) - x.top[0];
                   float p = taken && k < words ? exponential<TY::planes == 2>(z) * x.top[1] : 0.f;
                   if (taken && k == hit) p = expm1f(-global<const float>(base + a.w.hit)[n]);
                   w[k] = operand_word<OP, TY::planes>(TY::planes == 1 ? p : p * (float)(1 << kHeldAt));
                 }
                 store8<TY::planes>(base + a.w.p, n, a.s.piece, m, w);
               },
               [](uint32_t, uint32_t, const float (&)[8]) {});
  } else {
    constexpr int MT = EDGE == 256 ? 4 : 2, WM = 2, WN = EDGE == 256 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
    // the words' bias; of words beyond the piece an infinity, so that they cannot come
    float DADAM_LDS* bias = (float DADAM_LDS*)lds;
    __syncthreads();
    if (threadIdx.x < EDGE) {
      const uint32_t m = i * T::kM + threadIdx.x;
      bias[threadIdx.x] = m >= a.words ? -INFINITY : row.bias ? XT::load(row.bias, a.first_word + m) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int jn = 0; jn < 2; ++jn) {
      const uint32_t n = j * T::kN + (jn * WN + wn) * 32 + (lane & 31);
      int32_t target;
      const uint32_t hit = has_target(a, row.target, n, target) ? (uint32_t)target - a.first_word - i * T::kM : 0xffffffffu;  // in the tile
      float most = -INFINITY;
      asm volatile("" ::: "memory");  // (the biases are read again rather than kept in registers)
#pragma unroll
      for (int im = 0; im < MT; ++im)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const uint32_t m = (wm * MT + im) * 32 + g * 8 + (lane >> 5) * 4;
          const float4v b = *(const float4v DADAM_LDS*)(bias + m);
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const float z = fmaf(t.acc[im][jn][4 * g + e], held, b[e]);
            if (m + e == hit) global<float>(base + a.w.hit)[n] = z;
            most = fmaxf(most, z);
            t.acc[im][jn][4 * g + e] = z;
          }
        }
      most = fmaxf(most, __shfl_xor(most, 32));
      float sum = 0.f;
      const float from = most == -INFINITY ? 0.f : most;  // nothing but words that cannot come: a sum of 0
#pragma unroll
      for (int im = 0; im < MT; ++im)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = exponential<TY::planes == 2>(t.acc[im][jn][r] - from);
          sum += e;
          t.acc[im][jn][r] = e;
        }
      sum += __shfl_xor(sum, 32);
      if (lane < 32) {
        const uint32_t slice = (a.first_word + i * T::kM) / (EDGE / 2) + wm;
        global<float2v>(base + a.w.stats)[(uint64_t)slice * a.s.T + n] = float2v{most, sum};
      }
    }
    if constexpr (MODE == kHeadKeep)
      t.hand_out(lds, false, nothing_ahead,
                 [&](uint32_t m, uint32_t n, float (&v)[8], Nothing) {
                   uint32_t w[8];
#pragma unroll
                   for (int k = 0; k < 8; ++k) w[k] = operand_word<Half, TY::planes>(v[k] * kept_times<TY>());
                   store8<TY::planes>(base + a.w.p, j * T::kN + n, a.s.piece, i * T::kM + m, w);
                 },
                 [](uint32_t, uint32_t, const float (&)[8]) {});
  }
}

// softmax - e[target] in place of the slices' exponentials: a thread takes eight words of a token.  (Bound by memory: 282 us for 1.6 GB.)
template <typename TY>
__global__ __launch_bounds__(256) void k_head_scale(HeadArgs a) {
  using OP = typename TY::op;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t each = (a.s.piece + 2047) / 2048, n = blockIdx.x / each, m = (blockIdx.x % each * 256 + threadIdx.x) * 8;  // (there may be more tokens than a grid's y)
  if (m >= a.s.piece) return;
  int32_t target;
  uint32_t w[8] = {};
  if (has_target(a, row.target, n, target)) {
    const float2v top = global<const float2v>(base + a.w.top)[n];
    const float most = global<const float2v>(base + a.w.stats)[(uint64_t)(m / (a.s.edge / 2)) * a.s.T + n][0];
    const float factor = exponential<TY::planes == 2>(most - top[0]) * top[1] * (TY::planes == 1 ? 1.f / kept_times<TY>() : 1.f);
    const Eight e = load8<TY::planes>(base + a.w.p, n, a.s.piece, m);
    const uint32_t hit = (uint32_t)target - m;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      float p = value_of<Half, TY::planes == 2>(e, k) * factor;
      if (k == hit) p = expm1f(-global<const float>(base + a.w.hit)[n]) * (TY::planes == 1 ? 1.f : (float)(1 << kHeldAt));
      w[k] = operand_word<OP, TY::planes>(p);
    }
  }
  store8<TY::planes>(base + a.w.p, n, a.s.piece, m, w);
}

// Every token's logarithm of the sum of exponentials and its loss: 16 tokens a workgroup, 16 threads a token.
__global__ __launch_bounds__(256) void k_head_losses(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t at = threadIdx.x % 16, part = threadIdx.x / 16, n = blockIdx.x * 16 + at;
  const float2v DADAM_GLOBAL* stats = global<const float2v>(base + a.w.stats) + n;
  __shared__ float parts[16][17];
  float most = -INFINITY, sum = 0.f;
#pragma unroll 4
  for (uint32_t s = part; s < a.s.slices; s += 16) most = fmaxf(most, stats[(uint64_t)s * a.s.T][0]);
  parts[part][at] = most;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 16; ++k) most = fmaxf(most, parts[k][at]);
  __syncthreads();
  // (a slice of words that cannot come has a sum of 0, one of NaN its NaN)
#pragma unroll 4
  for (uint32_t s = part; s < a.s.slices; s += 16) {
    const float2v v = stats[(uint64_t)s * a.s.T];
    sum += v[0] == -INFINITY ? v[1] : v[1] * exponential<true>(v[0] - most);
  }
  parts[part][at] = sum;
  __syncthreads();
  if (part == 0) {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += parts[k][at];
    int32_t target;
    const bool taken = has_target(a, row.target, n, target);
    global<float2v>(base + a.w.top)[n] = float2v{most, 1.f / sum};
    const float nll = taken ? logf(sum) + (most - global<const float>(base + a.w.hit)[n]) : 0.f;
    if (n < a.s.tokens && row.nll) global<float>(row.nll)[n] = nll;
    global<float>(base + a.w.hit)[n] = nll;
  }
}

// The loss of a replica, summed in 64 bits in the order of the tokens' numbers by 1024, and how many tokens have a target.
__global__ __launch_bounds__(1024) void k_head_sum(HeadArgs a) {
  const uint64_t base = base_of(a), target = a.row[blockIdx.z].target;
  __shared__ double parts[2][16];
  double sum = 0.0, count = 0.0;
  for (uint32_t t = threadIdx.x; t < a.s.tokens; t += 1024) {
    int32_t word;
    if (!has_target(a, target, t, word)) continue;
    sum += (double)global<const float>(base + a.w.hit)[t];
    count += 1.0;
  }
  sum = wave_sum(sum);
  count = wave_sum(count);
  if (threadIdx.x % 64 == 0) parts[0][threadIdx.x / 64] = sum, parts[1][threadIdx.x / 64] = count;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = count = 0.0;
    for (int k = 0; k < 16; ++k) sum += parts[0][k], count += parts[1][k];
    global<float>(base + a.w.words)[kHeadCount] = (float)count;
    global<float>(a.losses)[blockIdx.z] = (float)((double)a.scale * sum / (a.mean && count > 1.0 ? count : 1.0));
  }
}

// dW of a tile of columns (m) and words (n): both operands lie by tokens.  (Two replicas of 4096 tokens, 50257 words, width 1024, bfloat16: 783 and 53 us, 1007 TFLOP/s.)
template <typename GT, typename TY, int EDGE, int BUFFERS>
__global__ __launch_bounds__(2 * EDGE) void k_head_dhead(HeadArgs a) {
  using T = TileOf<typename TY::op, TY::planes, EDGE, BUFFERS, true, true>;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.D / T::kM;
  uint32_t i, j;
  banded(die_run(blockIdx.x, gridDim.x, a.n_xcd), across, gridDim.x / across, i, j);
  const uint64_t b = 2 * TY::planes;
  char DADAM_LDS* lds = (char DADAM_LDS*)head_lds;
  T t;
  t.product(operand(base + a.w.hidden + i * T::kM * b, a.s.D * b), operand(base + a.w.p + (a.skip + j * T::kN) * b, a.s.piece * b), a.s.T * TY::planes / 64, lds);
  const float factor = factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHidden) - kHeldAt));
  t.hand_out(lds, false, nothing_ahead,
             [&](uint32_t m, uint32_t n, float (&v)[8], Nothing) {
               m += i * T::kM;
               n += a.skip + j * T::kN;
               const uint32_t columns = n < a.words ? left(a.s.width, m) : 0;
               if (columns == 0) return;
               const uint64_t e = (uint64_t)(a.first_word + n) * a.s.width + m;
               float held[8] = {};
               if (a.add) GT::load8(row.dhead, e, columns, held);
#pragma unroll
               for (int k = 0; k < 8; ++k) held[k] = fmaf(v[k], factor, held[k]);
               GT::store8(row.dhead, e, columns, held);
             },
             [](uint32_t, uint32_t, const float (&)[8]) {});
}

// The same where there are so few tiles that the chip would wait for the tokens' sums: a part of the tokens (blockIdx.y), 32 bits, by rows of words.
template <typename TY>
__global__ __launch_bounds__(256) void k_head_dhead_part(HeadArgs a) {
  using T = TileOf<typename TY::op, TY::planes, 128, 4, true, true>;
  const uint64_t base = base_of(a), b = 2 * TY::planes;
  const uint32_t across = a.s.D / T::kM, i = blockIdx.x % across, j = blockIdx.x / across, stages = a.s.T * TY::planes / 64;
  const uint32_t from = (uint32_t)((uint64_t)stages * blockIdx.y / a.s.parts), to = (uint32_t)((uint64_t)stages * (blockIdx.y + 1) / a.s.parts);
  const uint64_t token = (uint64_t)from * (64 / TY::planes), out = base + a.w.parts + (uint64_t)blockIdx.y * a.s.piece * a.s.D * 4;
  char DADAM_LDS* lds = (char DADAM_LDS*)head_lds;
  T t;
  t.product(operand(base + a.w.hidden + (token * a.s.D + i * T::kM) * b, a.s.D * b), operand(base + a.w.p + (token * a.s.piece + j * T::kN) * b, a.s.piece * b), to - from, lds);
  t.hand_out(lds, false, nothing_ahead,
             [&](uint32_t m, uint32_t n, float (&v)[8], Nothing) { F32::store8(out, (uint64_t)(j * T::kN + n) * a.s.D + i * T::kM + m, 8, v); },
             [](uint32_t, uint32_t, const float (&)[8]) {});
}

// dW from its parts, in their order: eight columns of a word a thread.
template <typename GT, typename TY>
__global__ __launch_bounds__(256) void k_head_join(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t k = blockIdx.x * 256 + threadIdx.x, pieces = a.s.D / 8, n = k / pieces, m = k % pieces * 8, columns = n < a.words ? left(a.s.width, m) : 0;
  if (columns == 0) return;
  const uint64_t e = (uint64_t)(a.first_word + n) * a.s.width + m;
  float v[8] = {}, held[8] = {};
#pragma unroll 4
  for (uint32_t q = 0; q < a.s.parts; ++q) {
    float x[8];
    F32::load8(base + a.w.parts, ((uint64_t)q * a.s.piece + n) * a.s.D + m, 8, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += x[i];
  }
  const float factor = factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHidden) - kHeldAt));
  if (a.add) GT::load8(row.dhead, e, columns, held);
#pragma unroll
  for (int i = 0; i < 8; ++i) held[i] = fmaf(v[i], factor, held[i]);
  GT::store8(row.dhead, e, columns, held);
}

// dbias: 64 words a workgroup, 8 of them a thread; 32 threads share the tokens.
template <typename GT, typename TY>
__global__ __launch_bounds__(256) void k_head_dbias(HeadArgs a) {
  using OP = typename TY::op;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t k8 = threadIdx.x % 8 * 8, m = blockIdx.x * 64 + k8, part = threadIdx.x / 8;
  __shared__ float parts[32][65];
  float sum[8] = {};
#pragma unroll 4
  for (uint32_t t = part; t < a.s.T; t += 32) {
    const Eight p = load8<TY::planes>(base + a.w.p, t, a.s.piece, m);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] += value_of<OP, TY::planes == 2>(p, k);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) parts[part][k8 + k] = sum[k];
  __syncthreads();
  const uint32_t n = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x < 64 && n < a.words) {
    float all = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) all += parts[k][threadIdx.x];
    const float g = all * factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -kHeldAt));
    const uint64_t e = a.first_word + n;
    GT::store(row.dbias, e, a.add ? GT::load(row.dbias, e) + g : g);
  }
}

// dh of a tile of columns (m) and tokens (n), over a part of the piece's words: the head lies by words.  (Two replicas as above: 788 us, 1069
// TFLOP/s.)
template <typename TY, int EDGE, int BUFFERS>
__global__ __launch_bounds__(2 * EDGE) void k_head_dhidden(HeadArgs a) {
  using T = TileOf<typename TY::op, TY::planes, EDGE, BUFFERS, true, false>;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a);
  const uint32_t across = a.s.D / T::kM, down = a.s.T / T::kN, u = die_run(blockIdx.x, gridDim.x, a.n_xcd), split = u / (across * down);
  uint32_t i, j;
  banded(u % (across * down), across, down, i, j);
  const uint64_t b = 2 * TY::planes, pitch = a.s.piece * b;
  constexpr uint32_t kEach = 64 / TY::planes;  // words of a stage
  const uint32_t stages = (a.words + kEach - 1) / kEach;
  const uint32_t from = (uint32_t)((uint64_t)stages * split / a.s.splits), to = (uint32_t)((uint64_t)stages * (split + 1) / a.s.splits);
  char DADAM_LDS* lds = (char DADAM_LDS*)head_lds;
  T t;
  t.clear();
  if (from < to)  // (of words beyond the piece softmax is 0, and the last word stands for them)
    t.product(head_operand<TY>(base, row, a, from * kEach, i * T::kM * b), operand(base + a.w.p + (uint64_t)j * T::kN * pitch + (uint64_t)from * kStageBytes, pitch), to - from, lds);
  const uint64_t sums = base + a.w.sums + (uint64_t)split * a.s.T * a.s.D * 4;
  struct Held {
    float4v a, b;
  };
  auto at = [&](uint32_t m, uint32_t n) { return global<float4v>(sums + ((uint64_t)(j * T::kN + n) * a.s.D + i * T::kM + m) * 4); };
  t.hand_out(lds, false, [&](uint32_t m, uint32_t n) { return a.later && j * T::kN + n < a.s.tokens ? Held{at(m, n)[0], at(m, n)[1]} : Held{}; },
             [&](uint32_t m, uint32_t n, float (&v)[8], const Held& held) {
               if (j * T::kN + n >= a.s.tokens) return;
               at(m, n)[0] = float4v{v[0], v[1], v[2], v[3]} + held.a;
               at(m, n)[1] = float4v{v[4], v[5], v[6], v[7]} + held.b;
             },
             [](uint32_t, uint32_t, const float (&)[8]) {});
}

// dh of 256 columns of a token, four a thread, from the parts of its sum.
template <typename XT, typename TY>
__global__ __launch_bounds__(64) void k_head_end(HeadArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = base_of(a), each = (uint64_t)a.s.T * a.s.D * 4;
  const float factor = factor_of(base, a) * (TY::planes == 1 ? 1.f : ldexpf(1.f, -power_of<TY>(base, a, kHeadMostHead) - kHeldAt));
  const uint32_t n = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x * 4;
  if (c >= a.s.width) return;
  int32_t target;
  float4v v = {0.f, 0.f, 0.f, 0.f};
  if (has_target(a, row.target, n, target)) {
    const uint64_t at = base + a.w.sums + ((uint64_t)n * a.s.D + c) * 4;
#pragma unroll 8
    for (uint32_t s = 0; s < a.s.splits; ++s) v += global<const float4v>(at + s * each)[0];
  }
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k)
    if (c + k < a.s.width) XT::store(row.dhidden, (uint64_t)n * a.s.width + c + k, v[k] * factor);
}

template <auto KERNEL, typename... A>
int launch(dim3 grid, uint32_t threads, uint32_t lds, void* stream, const A&... a) {
  if (lds > 65536)
    if (const int e = ask_for_lds<KERNEL>(lds)) return e;
  KERNEL<<<grid, threads, lds, (hipStream_t)stream>>>(a...);
  return (int)hipGetLastError();
}

// fn(types of parameters, gradients and operands) for a pair of element types.
template <typename Fn>
int with_types(int xdt, int gdt, Fn fn) {
  if (xdt == (int)DADAM_BF16) return gdt == (int)DADAM_BF16 ? fn(B16{}, B16{}, Types<B16, B16>{}) : fn(B16{}, F32{}, Types<B16, F32>{});
  return gdt == (int)DADAM_BF16 ? fn(F32{}, B16{}, Types<F32, B16>{}) : fn(F32{}, F32{}, Types<F32, F32>{});
}

uint32_t upto(uint64_t n, uint32_t each) { return (uint32_t)((n + each - 1) / each); }

// fn(types of parameters, gradients and operands, edge and buffers of the tiles as types), for a launch of so many tiles.
template <typename Fn>
int with_tiles(int xdt, int gdt, uint32_t edge, uint32_t tiles, Fn fn) {
  using Large = std::integral_constant<int, 256>;
  using Small = std::integral_constant<int, 128>;
  return with_types(xdt, gdt, [&](auto x, auto g, auto ty) {
    if (edge == 256) return fn(x, g, ty, Large{}, std::integral_constant<int, 2>{});
    return tiles <= kOneEach ? fn(x, g, ty, Small{}, std::integral_constant<int, 4>{}) : fn(x, g, ty, Small{}, std::integral_constant<int, 2>{});
  });
}

}  // namespace

uint32_t head_most_groups(const HeadArgs& a) {
  const uint32_t head = upto((uint64_t)a.s.vocab * a.s.width, 2048), most = head > a.s.tokens ? head : a.s.tokens;
  return most < kMostGroups ? most : kMostGroups;
}
int launch_head_most(int xdt, const HeadArgs& a, uint32_t rows, void* stream) {
  const dim3 grid(a.groups, 2, rows);
  return xdt == (int)DADAM_BF16 ? launch<k_head_most<B16>>(grid, 256, 0, stream, a) : launch<k_head_most<F32>>(grid, 256, 0, stream, a);
}
int launch_head_operands(int xdt, int gdt, const HeadArgs& a, bool hidden, uint32_t rows, void* stream) {
  const uint32_t words = a.straight ? 0 : upto((uint64_t)upto(a.words, a.s.edge) * a.s.edge * a.s.D, kOperandPieces * 2048),
                 vectors = hidden ? upto((uint64_t)a.s.T * a.s.D, kOperandPieces * 2048) : 0;
  const dim3 grid(words > vectors ? words : vectors, (words ? 1 : 0) + (vectors ? 1 : 0), rows);
  if (grid.x == 0) return 0;
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) { return launch<k_head_operands<decltype(x), decltype(ty)>>(grid, 256, 0, stream, a); });
}
int launch_head_logits(int xdt, int gdt, HeadMode mode, const HeadArgs& a, uint32_t rows, void* stream) {
  const dim3 grid(upto(a.words, a.s.edge) * (a.s.T / a.s.edge), 1, rows);
  return with_tiles(xdt, gdt, a.s.edge, grid.x * rows, [&](auto x, auto, auto ty, auto edge, auto buffers) {
    using X = decltype(x);
    using TY = decltype(ty);
    constexpr int kEdge = decltype(edge)::value, kBuffers = decltype(buffers)::value;
    using T = TileOf<typename TY::op, TY::planes, kEdge, kBuffers, false, false, TY::planes == 2 && kBuffers == 4>;
    if (mode == kHeadStatistics) return launch<k_head_logits<X, TY, kEdge, kBuffers, kHeadStatistics>>(grid, T::kThreads, T::kLds, stream, a);
    if (mode == kHeadKeep) return launch<k_head_logits<X, TY, kEdge, kBuffers, kHeadKeep>>(grid, T::kThreads, T::kLds, stream, a);
    return launch<k_head_logits<X, TY, kEdge, kBuffers, kHeadGradient>>(grid, T::kThreads, T::kLds, stream, a);
  });
}
int launch_head_scale(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto, auto, auto ty) { return launch<k_head_scale<decltype(ty)>>(dim3(a.s.T * upto(a.s.piece, 2048), 1, rows), 256, 0, stream, a); });
}
int launch_head_losses(const HeadArgs& a, uint32_t rows, void* stream) {
  if (const int e = launch<k_head_losses>(dim3(a.s.T / 16, 1, rows), 256, 0, stream, a)) return e;
  return launch<k_head_sum>(dim3(1, 1, rows), 1024, 0, stream, a);
}
int launch_head_dhead(int xdt, int gdt, uint32_t edge, const HeadArgs& a, uint32_t rows, void* stream) {
  const dim3 grid(upto(a.words - a.skip, edge) * (a.s.D / edge), 1, rows);
  return with_tiles(xdt, gdt, edge, grid.x * rows, [&](auto, auto g, auto ty, auto edge_, auto buffers) {
    using TY = decltype(ty);
    using T = TileOf<typename TY::op, TY::planes, decltype(edge_)::value, decltype(buffers)::value, true, true>;
    return launch<k_head_dhead<decltype(g), TY, decltype(edge_)::value, decltype(buffers)::value>>(grid, T::kThreads, T::kLds, stream, a);
  });
}
int launch_head_dhead_parts(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  const dim3 grid(upto(a.words, 128) * (a.s.D / 128), a.s.parts, rows);
  const int e = with_types(xdt, gdt, [&](auto, auto, auto ty) {  // (parts make no more tiles than compute units: four stages)
    using TY = decltype(ty);
    using T = TileOf<typename TY::op, TY::planes, 128, 4, true, true>;
    return launch<k_head_dhead_part<TY>>(grid, T::kThreads, T::kLds, stream, a);
  });
  const dim3 pieces(upto((uint64_t)a.words * (a.s.D / 8), 256), 1, rows);
  return e ? e : with_types(xdt, gdt, [&](auto, auto g, auto ty) { return launch<k_head_join<decltype(g), decltype(ty)>>(pieces, 256, 0, stream, a); });
}
int launch_head_dbias(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto, auto g, auto ty) { return launch<k_head_dbias<decltype(g), decltype(ty)>>(dim3(upto(a.words, 64), 1, rows), 256, 0, stream, a); });
}
int launch_head_dhidden(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  const dim3 grid((a.s.T / a.s.edge) * (a.s.D / a.s.edge) * a.s.splits, 1, rows);
  return with_tiles(xdt, gdt, a.s.edge, grid.x * rows, [&](auto, auto, auto ty, auto edge, auto buffers) {
    using TY = decltype(ty);
    using T = TileOf<typename TY::op, TY::planes, decltype(edge)::value, decltype(buffers)::value, true, false>;
    return launch<k_head_dhidden<TY, decltype(edge)::value, decltype(buffers)::value>>(grid, T::kThreads, T::kLds, stream, a);
  });
}
int launch_head_end(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream) {
  return with_types(xdt, gdt, [&](auto x, auto, auto ty) { return launch<k_head_end<decltype(x), decltype(ty)>>(dim3(a.s.tokens, upto(a.s.width, 256), rows), 64, 0, stream, a); });
}

}  // namespace dadam
