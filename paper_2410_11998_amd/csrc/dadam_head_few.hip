// The loss of a language model's head for few tokens (up to kFewTokens): what there is to read and write of the head counts, so it is read as it lies, once for the
// logits and once for the hidden vectors' gradients, and its gradient is written; nothing of its size is copied.
//
// Operands come to the registers straight from memory; LDS holds the sums of wavefronts that share a row's width, and the tokens' values for softmax.
// Logits: 32 words by 32 tokens, every lane its own row's pieces of 16 bytes.  dW: 32 words by 128 columns, summed over
// the tokens; dh: the tokens by 128 columns, summed over a range of words, whose rows the lanes read four columns each.  In both, column 4 n + j belongs to block j of 32,
// so that a lane's four blocks' elements of a row are side by side in memory.  The logits (4 bytes for a token and a word, at most 64 of 2 or 4 bytes times the width) are kept.
// bfloat16 parameters and gradients: 16 summed elements an instruction, softmax - e[target] rounded to bfloat16.  Otherwise float32 instructions, whose sixteenth part
// of the rate is enough here: 6.6e9 operations beside 400 MB (32 tokens, 50257 words, width 1024).
// 16 tokens, 50257 words, width 1024, bfloat16: 118 us, 44 of them for both gradients (206 MB, 4.7 TB/s) and 34 for the logits (103 MB, 3 TB/s: every instruction's
// lanes read 32 rows); 32-bit heads reach 3.2 to 3.5 TB/s, as their products take half of that time.
#include "dadam_head.h"
#include "dadam_mfma.h"

namespace dadam {
namespace {

template <typename XT, typename GT>
struct FewOp {  // float32
  static constexpr bool brain = false;
};
template <>
struct FewOp<B16, B16> {
  static constexpr bool brain = true;
};

__device__ __forceinline__ float16v mfma32(float a, float b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float16v nothing() {
  float16v v;
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = 0.f;
  return v;
}
// Row (of 32) of element r of a block's sums that a lane holds.
__device__ __forceinline__ uint32_t row_of(int r, int lane) { return (uint32_t)((r >> 2) * 8 + (lane >> 5) * 4 + (r & 3)); }

__device__ __forceinline__ uint64_t few_base(const FewArgs& a) { return a.workspace + (uint64_t)blockIdx.z * a.stride; }
__device__ __forceinline__ uint32_t rest(uint32_t n, uint32_t at) { return at < n ? n - at : 0; }
__device__ __forceinline__ bool few_target(const FewArgs& a, uint64_t target, uint32_t t, int32_t& word) {
  word = -1;
  if (t >= a.s.tokens) return false;
  word = global<const int32_t>(target)[t];
  return word >= 0 && (uint32_t)word < a.s.vocab;
}

// Eight bfloat16s of a row from column k on; beyond the row zeros.
__device__ __forceinline__ brain8 eight(uint64_t row, uint32_t width, uint32_t k) {
  uint4v v = {0, 0, 0, 0};
  if (k + 8 <= width) {
    v = global<const uint4u>(row + (uint64_t)k * 2)[0];
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e)
      if (k + e < width) v[e / 2] |= (uint32_t)global<const uint16_t>(row)[k + e] << 16 * (e & 1);
  }
  return __builtin_bit_cast(brain8, v);
}

// Logits of a block of words, their largest and their sum of exponentials, and the target's.  A wavefront takes a block or, where there are so few blocks that the chip
// would wait for them, SHARE of a workgroup take a part of its width each (2009 words, 11 tokens, 12 KB a row, four replicas: 154 us by one, 40 by four, 36 by eight;
// 145 words, one token, six replicas 45 and 28).
template <typename XT, bool BRAIN, int NB, uint32_t SHARE>
__global__ __launch_bounds__(SHARE == 8 ? 512 : 256) void k_few_logits(FewArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = few_base(a);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), block = SHARE > 1 ? blockIdx.x : blockIdx.x * 4 + wave;
  if (block >= a.s.blocks) return;
  const uint32_t mine = block * kFewWords + (lane & 31), word = mine < a.s.vocab ? mine : a.s.vocab - 1;
  const uint64_t size = sizeof(typename XT::type), w = row.head + (uint64_t)word * a.s.width * size;
  uint64_t h[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint32_t t = b * 32 + (lane & 31);
    h[b] = row.hidden + (uint64_t)(t < a.s.tokens ? t : a.s.tokens - 1) * a.s.width * size;
  }
  // float32 products go to four sums in turn (two of 64 tokens): one sum of 1327 elements, rounded at every
  // second one, leaves gradients off by 1.1e-6 of their norm, four 2.9e-7.
  constexpr int kSums = BRAIN ? 1 : 4 / NB;
  float16v sums[kSums][NB];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[k][b] = nothing();
  constexpr uint32_t kStep = BRAIN ? 16 : 8;
  const uint32_t steps = (a.s.width + kStep - 1) / kStep, from = SHARE > 1 ? steps * wave / SHARE * kStep : 0, to = SHARE > 1 ? steps * (wave + 1) / SHARE * kStep : steps * kStep;
  const uint32_t whole = to < a.s.width ? to : a.s.width / kStep * kStep;  // up to here whole pieces
  uint32_t k0 = from;
  constexpr uint32_t kAhead = NB == 1 ? 8 : 4;  // pieces of a row on their way at once
  for (; k0 + kAhead * kStep <= whole; k0 += kAhead * kStep) {
    const uint32_t k = k0 + half * (kStep / 2);
    if constexpr (BRAIN) {
      brain8 x[kAhead], y[kAhead][NB];
#pragma unroll
      for (uint32_t s = 0; s < kAhead; ++s) {
        x[s] = __builtin_bit_cast(brain8, (uint4v)global<const uint4u>(w + (uint64_t)(k + s * kStep) * 2)[0]);
#pragma unroll
        for (int b = 0; b < NB; ++b) y[s][b] = __builtin_bit_cast(brain8, (uint4v)global<const uint4u>(h[b] + (uint64_t)(k + s * kStep) * 2)[0]);
      }
#pragma unroll
      for (uint32_t s = 0; s < kAhead; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) sums[0][b] = Brain::mfma(x[s], y[s][b], sums[0][b]);
    } else {
      float x[kAhead][4], y[kAhead][NB][4];
#pragma unroll
      for (uint32_t s = 0; s < kAhead; ++s) {
        XT::load4(w, k + s * kStep, 4, x[s]);
#pragma unroll
        for (int b = 0; b < NB; ++b) XT::load4(h[b], k + s * kStep, 4, y[s][b]);
      }
#pragma unroll
      for (uint32_t s = 0; s < kAhead; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int b = 0; b < NB; ++b) sums[e % kSums][b] = mfma32(x[s][e], y[s][b][e], sums[e % kSums][b]);
    }
  }
  for (; k0 < to; k0 += kStep) {
    const uint32_t k = k0 + half * (kStep / 2);
    if constexpr (BRAIN) {
      const brain8 x = eight(w, a.s.width, k);
#pragma unroll
      for (int b = 0; b < NB; ++b) sums[0][b] = Brain::mfma(x, eight(h[b], a.s.width, k), sums[0][b]);
    } else {
      float x[4], y[NB][4];
      XT::load4(w, k, rest(a.s.width, k), x);
#pragma unroll
      for (int b = 0; b < NB; ++b) XT::load4(h[b], k, rest(a.s.width, k), y[b]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int b = 0; b < NB; ++b) sums[e % kSums][b] = mfma32(x[e], y[b][e], sums[e % kSums][b]);
    }
  }
  float16v acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    acc[b] = sums[0][b];
    if constexpr (kSums == 2) acc[b] += sums[1][b];
    if constexpr (kSums == 4) acc[b] = (acc[b] + sums[1][b]) + (sums[2][b] + sums[3][b]);
  }
  if constexpr (SHARE > 1) {
    __shared__ float parts[SHARE - 1][NB][16][64];
    if (wave > 0)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) parts[wave - 1][b][r][lane] = acc[b][r];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float pairs[SHARE / 2];
        pairs[0] = acc[b][r] + parts[0][b][r][lane];
#pragma unroll
        for (uint32_t k = 1; k < SHARE / 2; ++k) pairs[k] = parts[2 * k - 1][b][r][lane] + parts[2 * k][b][r][lane];
        acc[b][r] = pairs[0] + pairs[1];
        if constexpr (SHARE == 8) acc[b][r] += pairs[2] + pairs[3];
      }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint32_t t = b * 32 + (lane & 31);
    int32_t target;
    const bool taken = few_target(a, row.target, t, target);
    float most = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t v = block * kFewWords + row_of(r, lane);
      float z = -INFINITY;
      if (v < a.s.vocab) z = acc[b][r] + (row.bias ? XT::load(row.bias, v) : 0.f);
      if (taken && v == (uint32_t)target) global<float>(base + a.w.hit)[t] = z;
      most = fmaxf(most, z);
      acc[b][r] = z;
    }
    most = fmaxf(most, __shfl_xor(most, 32));
    const float from = most == -INFINITY ? 0.f : most;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += exponential<!BRAIN>(acc[b][r] - from);
    sum += __shfl_xor(sum, 32);
    const uint64_t at = base + a.w.z + ((uint64_t)block * a.s.T + t) * (kFewWords * 4);
#pragma unroll
    for (int g = 0; g < 4; ++g) global<float4v>(at)[g * 2 + half] = float4v{acc[b][4 * g], acc[b][4 * g + 1], acc[b][4 * g + 2], acc[b][4 * g + 3]};
    if (half == 0) global<float2v>(base + a.w.stats)[(uint64_t)block * a.s.T + t] = float2v{most, sum};
  }
}

// Every token's loss and the replica's: T tokens and 1024 / T threads for each.
template <int NB>
__global__ __launch_bounds__(1024) void k_few_losses(FewArgs a) {
  constexpr uint32_t T = NB * 32, kParts = 1024 / T;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = few_base(a);
  const uint32_t t = threadIdx.x % T, part = threadIdx.x / T;
  const float2v DADAM_GLOBAL* stats = global<const float2v>(base + a.w.stats) + t;
  __shared__ float parts[kParts][T + 1];
  // eight blocks at a time; their sums come to the largest so far (a sum of NaN has no largest: it is taken as it is)
  float most = -INFINITY, sum = 0.f;
  for (uint32_t b0 = part; b0 < a.s.blocks; b0 += 8 * kParts) {
    float2v v[8];
    float top = most;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = b0 + k * kParts < a.s.blocks ? stats[(uint64_t)(b0 + k * kParts) * T] : float2v{-INFINITY, 0.f};
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) top = fmaxf(top, v[k][0]);
    if (most != -INFINITY) sum *= exponential<true>(most - top);
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) sum += v[k][0] == -INFINITY ? v[k][1] : v[k][1] * exponential<true>(v[k][0] - top);
    most = top;
  }
  parts[part][t] = most;
  __syncthreads();
  float top = most;
#pragma unroll
  for (uint32_t k = 0; k < kParts; ++k) top = fmaxf(top, parts[k][t]);
  __syncthreads();
  if (most != -INFINITY) sum *= exponential<true>(most - top);
  most = top;
  parts[part][t] = sum;
  __syncthreads();
  __shared__ double all[T];
  __shared__ uint32_t count[T];
  if (part == 0) {
    sum = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kParts; ++k) sum += parts[k][t];
    int32_t target;
    const bool taken = few_target(a, row.target, t, target);
    global<float2v>(base + a.w.top)[t] = float2v{most, 1.f / sum};
    const float nll = taken ? logf(sum) + (most - global<const float>(base + a.w.hit)[t]) : 0.f;
    if (t < a.s.tokens && row.nll) global<float>(row.nll)[t] = nll;
    global<float>(base + a.w.hit)[t] = nll;
    all[t] = (double)nll;
    count[t] = taken ? 1 : 0;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double loss = 0.0;
    uint32_t n = 0;
    for (uint32_t k = 0; k < T; ++k) loss += all[k], n += count[k];
    const double divisor = a.mean && n > 1 ? (double)n : 1.0;
    global<float>(a.losses)[blockIdx.z] = (float)((double)a.scale * loss / divisor);
    global<float>(base + a.w.words)[kHeadCount] = (float)n;
  }
}

__device__ __forceinline__ float few_factor(uint64_t base, const FewArgs& a) {
  return a.mean ? a.scale / fmaxf(global<const float>(base + a.w.words)[kHeadCount], 1.f) : a.scale;
}

// softmax - e[target] (blockIdx.y 0: a wavefront a block of words, a lane a word and half of the tokens) with the bias's gradient, and the hidden vectors of tokens with a
// target as an operand (1).
template <typename XT, typename GT, bool BRAIN, int NB>
__global__ __launch_bounds__(256) void k_few_softmax(FewArgs a) {
  constexpr uint32_t T = NB * 32;
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = few_base(a);
  int32_t target;
  if (blockIdx.y == 1) {
    const uint32_t e = blockIdx.x * 256 + threadIdx.x, t = BRAIN ? e % T : e / a.s.D, d = BRAIN ? e / T : e % a.s.D;
    if (e >= T * a.s.D) return;
    const float v = d < a.s.width && few_target(a, row.target, t, target) ? XT::load(row.hidden, (uint64_t)t * a.s.width + d) : 0.f;
    if constexpr (BRAIN) B16::store(base + a.w.hidden, e, v);
    else F32::store(base + a.w.hidden, e, v);
    return;
  }
  __shared__ float2v tops[T];
  __shared__ float hits[T];
  __shared__ int32_t targets[T];
  if (threadIdx.x < T) {
    tops[threadIdx.x] = global<const float2v>(base + a.w.top)[threadIdx.x];
    hits[threadIdx.x] = global<const float>(base + a.w.hit)[threadIdx.x];
    targets[threadIdx.x] = few_target(a, row.target, threadIdx.x, target) ? target : -1;
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const uint32_t block = blockIdx.x * 4 + threadIdx.x / 64, word = block * kFewWords + (lane & 31);
  if (block >= a.s.blocks) return;
  float sum = 0.f;
#pragma unroll
  for (uint32_t t0 = 0; t0 < T; t0 += 16) {  // eight tokens a lane: 16 bytes of the turned operand
    float p[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) p[k] = global<const float>(base + a.w.z)[((uint64_t)block * T + t0 + half * 8 + k) * kFewWords + (lane & 31)];
    uint4v turned = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      const uint32_t t = t0 + half * 8 + k;
      p[k] = targets[t] >= 0 && word < a.s.vocab ? exponential<!BRAIN>(p[k] - tops[t][0]) * tops[t][1] : 0.f;
      if (targets[t] >= 0 && word == (uint32_t)targets[t]) p[k] = expm1f(-hits[t]);
      const uint64_t e = ((uint64_t)block * T + t) * kFewWords + (lane & 31);
      if constexpr (BRAIN) {
        const uint32_t bits = Brain::bits(p[k]);
        p[k] = Brain::value(bits);
        turned[k / 2] |= bits << 16 * (k & 1);
        global<uint16_t>(base + a.w.p)[e] = (uint16_t)bits;
      } else {
        F32::store(base + a.w.z, e, p[k]);
      }
      sum += p[k];
    }
    if constexpr (BRAIN) global<uint4v>(base + a.w.p_turned)[(((uint64_t)block * kFewWords + (lane & 31)) * T + t0) / 8 + half] = turned;
  }
  sum += __shfl_xor(sum, 32);
  if (row.dbias && half == 0 && word < a.s.vocab) {
    const float g = sum * few_factor(base, a);
    GT::store(row.dbias, word, a.add ? GT::load(row.dbias, word) + g : g);
  }
}

// dW of a block of words and 128 columns.
template <typename GT, bool BRAIN, int NB>
__device__ __forceinline__ void few_dhead(const FewArgs& a, const HeadRow& row, uint64_t base, uint32_t block, uint32_t d0, int lane) {
  constexpr uint32_t T = NB * 32;
  const int half = lane >> 5;
  const uint32_t n = (uint32_t)(lane & 31), d = d0 + 4 * n;
  float16v acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = nothing();
  if constexpr (BRAIN) {
#pragma unroll
    for (uint32_t t = 0; t < T; t += 16) {
      const brain8 p = global<const brain8>(base + a.w.p_turned)[(((uint64_t)block * kFewWords + n) * T + t) / 8 + half];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) acc[j] = Brain::mfma(p, global<const brain8>(base + a.w.hidden)[((uint64_t)(d + j) * T + t) / 8 + half], acc[j]);
    }
  } else {
#pragma unroll 4
    for (uint32_t t0 = 0; t0 < T; t0 += 2) {
      const uint32_t t = t0 + half;
      const float p = global<const float>(base + a.w.z)[((uint64_t)block * T + t) * kFewWords + n];
      const float4v h = global<const float4v>(base + a.w.hidden)[((uint64_t)t * a.s.D + d) / 4];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = mfma32(p, h[j], acc[j]);
    }
  }
  const float factor = few_factor(base, a);
  const uint32_t columns = rest(a.s.width, d);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const uint32_t word = block * kFewWords + row_of(r, lane);
    if (word >= a.s.vocab || columns == 0) continue;
    const uint64_t e = (uint64_t)word * a.s.width + d;
    float g[4] = {};
    if (a.add) GT::load4(row.dhead, e, columns, g);
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = fmaf(acc[j][r], factor, g[j]);
    GT::store4(row.dhead, e, columns, g);
  }
}

// A range's part of dh, 128 columns.
template <typename XT, bool BRAIN, int NB, bool WIDE>
__device__ __forceinline__ void few_dhidden(const FewArgs& a, const HeadRow& row, uint64_t base, uint32_t range, uint32_t d0, int lane) {
  constexpr uint32_t T = NB * 32;
  const int half = lane >> 5;
  const uint32_t n = (uint32_t)(lane & 31), d = d0 + 4 * n, columns = rest(a.s.width, d);
  const uint32_t from = WIDE && columns == 0 ? 0 : d;  // WIDE: a thread has four columns or, reading the first ones, none
  const uint32_t end = (range + 1) * a.s.each < a.s.blocks ? (range + 1) * a.s.each : a.s.blocks;
  float16v acc[NB][4];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[b][j] = nothing();
  for (uint32_t block = range * a.s.each; block < end; ++block) {
    if constexpr (BRAIN) {
#pragma unroll
      for (uint32_t s = 0; s < kFewWords; s += 16) {
        // eight words' four columns, turned into four columns' eight words
        uint2v w[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
          const uint32_t mine = block * kFewWords + s + half * 8 + e, word = mine < a.s.vocab ? mine : a.s.vocab - 1;
          const uint64_t at = row.head + ((uint64_t)word * a.s.width + from) * 2;
          if (WIDE) {
            w[e] = global<const uint2u>(at)[0];
          } else {
            w[e] = uint2v{0, 0};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
              if (j < columns) w[e][j / 2] |= (uint32_t)global<const uint16_t>(at)[j] << 16 * (j & 1);
          }
        }
        brain8 p[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b] = global<const brain8>(base + a.w.p)[(((uint64_t)block * T + b * 32 + n) * kFewWords + s) / 8 + half];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint4v x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_perm(w[2 * e + 1][j / 2], w[2 * e][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int b = 0; b < NB; ++b) acc[b][j] = Brain::mfma(p[b], __builtin_bit_cast(brain8, x), acc[b][j]);
        }
      }
    } else {
#pragma unroll
      for (uint32_t s = 0; s < kFewWords; s += 8) {
        float4v p[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b] = global<const float4v>(base + a.w.z)[(((uint64_t)block * T + b * 32 + n) * kFewWords + s) / 4 + half];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const uint32_t mine = block * kFewWords + s + half * 4 + e, word = mine < a.s.vocab ? mine : a.s.vocab - 1;
          float w[4];
          XT::load4(row.head, (uint64_t)word * a.s.width + from, WIDE ? 4 : columns, w);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int b = 0; b < NB; ++b) acc[b][j] = mfma32(p[b][e], w[j], acc[b][j]);
        }
      }
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t t = b * 32 + row_of(r, lane);
      if (t < a.s.tokens)
        global<float4v>(base + a.w.sums)[(((uint64_t)range * a.s.tokens + t) * a.s.D + d) / 4] = float4v{acc[b][0][r], acc[b][1][r], acc[b][2][r], acc[b][3][r]};
    }
}

// Wavefronts 0 .. : dh of a range and 128 columns each; behind them dW of a block and 128 columns.
template <typename XT, typename GT, bool BRAIN, int NB>
__global__ __launch_bounds__(256) void k_few_gradients(FewArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = few_base(a);
  const int lane = threadIdx.x & 63;
  const uint32_t chunks = a.s.D / kFewColumns, first = row.dhidden ? a.s.ranges * chunks : 0;
  uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  if (item < first) {
    if (item % chunks * kFewColumns + kFewColumns <= a.s.width || a.s.width % 4 == 0) few_dhidden<XT, BRAIN, NB, true>(a, row, base, item / chunks, item % chunks * kFewColumns, lane);
    else few_dhidden<XT, BRAIN, NB, false>(a, row, base, item / chunks, item % chunks * kFewColumns, lane);
  } else if (row.dhead && item - first < a.s.blocks * chunks) {
    item -= first;
    few_dhead<GT, BRAIN, NB>(a, row, base, item / chunks, item % chunks * kFewColumns, lane);
  }
}

// dh of a token's 64 columns from its ranges' parts: four columns a thread, sixteen threads share the parts.
template <typename XT>
__global__ __launch_bounds__(256) void k_few_end(FewArgs a) {
  const HeadRow& row = a.row[blockIdx.z];
  const uint64_t base = few_base(a);
  const uint32_t t = blockIdx.x, k = threadIdx.x % 16, c = blockIdx.y * 64 + k * 4, part = threadIdx.x / 16;
  __shared__ float4v parts[16][16];
  float4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (uint32_t s = part; s < a.s.ranges; s += 16) v += global<const float4v>(base + a.w.sums)[(((uint64_t)s * a.s.tokens + t) * a.s.D + c) / 4];
  parts[part][k] = v;
  __syncthreads();
  if (part == 0) {
    for (int s = 1; s < 16; ++s) v += parts[s][k];
    int32_t target;
    const float factor = few_target(a, row.target, t, target) ? few_factor(base, a) : 0.f;
    const float g[4] = {factor == 0.f ? 0.f : v[0] * factor, factor == 0.f ? 0.f : v[1] * factor, factor == 0.f ? 0.f : v[2] * factor, factor == 0.f ? 0.f : v[3] * factor};
    XT::store4(row.dhidden, (uint64_t)t * a.s.width + c, rest(a.s.width, c), g);
  }
}

template <typename K, typename A>
int launch(K kernel, dim3 grid, uint32_t threads, void* stream, const A& a) {
  kernel<<<grid, threads, 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}
constexpr uint32_t kFewBlocks = 2048;  // eight wavefronts a compute unit
uint32_t upto(uint64_t n, uint32_t each) { return (uint32_t)((n + each - 1) / each); }

// fn(types of parameters and gradients, whether operands are bfloat16, blocks of tokens).
template <typename Fn>
int with_few(int xdt, int gdt, const FewArgs& a, Fn fn) {
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  auto with = [&](auto x, auto g) {
    constexpr bool brain = FewOp<decltype(x), decltype(g)>::brain;
    return a.s.T <= 32 ? fn(x, g, std::integral_constant<bool, brain>{}, One{}) : fn(x, g, std::integral_constant<bool, brain>{}, Two{});
  };
  if (xdt == (int)DADAM_BF16) return gdt == (int)DADAM_BF16 ? with(B16{}, B16{}) : with(B16{}, F32{});
  return gdt == (int)DADAM_BF16 ? with(F32{}, B16{}) : with(F32{}, F32{});
}

}  // namespace

int launch_few_logits(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream) {
  return with_few(xdt, gdt, a, [&](auto x, auto, auto brain, auto nb) {
    using X = decltype(x);
    constexpr bool kBrain = decltype(brain)::value;
    constexpr int kNB = decltype(nb)::value;
    const uint32_t blocks = a.s.blocks * rows;
    if constexpr (kNB == 1)  // (the parts of 64 tokens do not fit the registers)
      if (blocks < kFewBlocks / 4) return launch(k_few_logits<X, kBrain, kNB, 8>, dim3(a.s.blocks, 1, rows), 512, stream, a);
    if (blocks < kFewBlocks) return launch(k_few_logits<X, kBrain, kNB, 4>, dim3(a.s.blocks, 1, rows), 256, stream, a);
    return launch(k_few_logits<X, kBrain, kNB, 1>, dim3(upto(a.s.blocks, 4), 1, rows), 256, stream, a);
  });
}
int launch_few_losses(const FewArgs& a, uint32_t rows, void* stream) {
  return a.s.T <= 32 ? launch(k_few_losses<1>, dim3(1, 1, rows), 1024, stream, a) : launch(k_few_losses<2>, dim3(1, 1, rows), 1024, stream, a);
}
int launch_few_softmax(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream) {
  return with_few(xdt, gdt, a, [&](auto x, auto g, auto brain, auto nb) {
    const uint32_t words = upto(a.s.blocks, 4), hidden = upto((uint64_t)a.s.T * a.s.D, 256);
    return launch(k_few_softmax<decltype(x), decltype(g), decltype(brain)::value, decltype(nb)::value>, dim3(words > hidden ? words : hidden, 2, rows), 256, stream, a);
  });
}
int launch_few_gradients(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream) {
  return with_few(xdt, gdt, a, [&](auto x, auto g, auto brain, auto nb) {
    const uint64_t items = ((uint64_t)(a.row[0].dhidden ? a.s.ranges : 0) + (a.row[0].dhead ? a.s.blocks : 0)) * (a.s.D / kFewColumns);
    return launch(k_few_gradients<decltype(x), decltype(g), decltype(brain)::value, decltype(nb)::value>, dim3(upto(items, 4), 1, rows), 256, stream, a);
  });
}
int launch_few_end(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream) {
  const dim3 grid(a.s.tokens, upto(a.s.width, 64), rows);
  (void)gdt;
  return xdt == (int)DADAM_BF16 ? launch(k_few_end<B16>, grid, 256, stream, a) : launch(k_few_end<F32>, grid, 256, stream, a);
}

}  // namespace dadam
