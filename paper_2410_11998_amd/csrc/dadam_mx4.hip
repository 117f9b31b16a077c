// Microscaled 4-bit messages: quantisation of what a worker sends, the mixing matrix times such messages, the gossip update
// from that product, and the whole round in one pass where all replicas are here.
//
// A block of 32 elements is eight lanes' groups of four: its largest magnitude takes three exchanges inside those lanes.  The type's own
// conversions (round to nearest even, saturating at 6) do the rest; the power of two goes into the weight of the sum.
#include <hip/hip_runtime.h>

#include <cstring>

#include "dadam_granule.h"

namespace dadam {
namespace {

constexpr uint32_t kMixWaves = 4;

// The largest of the eight lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
  auto other = [](uint32_t v, uint32_t o) { return v > o ? v : o; };
  m = other(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  m = other(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));   // lane ^ 2
  m = other(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));  // 7 - lane of eight: the other four
  return m;
}

// The power of two that byte b of a message stands for: 2^(b - 127), NaN for 255.
__device__ __forceinline__ float power_of(uint32_t b) {
  return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7FC00000u : b << 23);
}

// The four values of 16 bits of codes, without their power of two.
__device__ __forceinline__ void decode(uint32_t codes, float (&q)[4]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0);
  const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
  q[0] = a.x; q[1] = a.y; q[2] = b.x; q[3] = b.y;
}

// A lane's group u of a block (padding: zeros) as 16 bits of codes, the block's scale byte, and the values these stand for.
__device__ __forceinline__ void encode(const float (&u)[4], uint32_t& codes, uint32_t& scale, float (&value)[4]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t magnitude = __float_as_uint(u[j]) & 0x7FFFFFFFu;  // as a whole number: NaN and infinity are the largest
    m = m > magnitude ? m : magnitude;
  }
  const uint32_t exponent = block_max(m) >> 23;  // floor(log2) + 127; 0: below 2^-126
  const bool finite = exponent != 255;
  scale = !finite ? 255u : exponent > 3 ? exponent - 2 : 1u;
  const float power = power_of(scale);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, u[0], u[1], power, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[2], u[3], power, 1) & 0xFFFFu;
  if (!finite) codes = 0;
  decode(codes, value);
#pragma unroll
  for (int j = 0; j < 4; ++j) value[j] *= power;
}

template <typename XT, int N>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_encode(const EncodeArgs<N> a) {
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group();
  const uint32_t row = a.s.row0 + blockIdx.x % a.s.n_rows, i = a.s.first + blockIdx.x / a.s.n_rows * kMixWaves + wave;
  if (i < a.s.n_granules) {
    const RowPointers p = a.row[row];
    const void* x = buffer<const void, 0>(p);
    const void* before = buffer<const void, 1>(p);
    void* behind = buffer<void, 2>(p);
    uint8_t* message = buffer<uint8_t, 3>(p);
    const uint32_t cut = cut_of(a.s.cuts, i);
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
      const uint64_t e = (uint64_t)i * kGranule + half * 256 + 4 * lane;
      const uint32_t bits = group_bits(a.s.cuts, cut, half, lane);
      float u[4], copy[4] = {0.f, 0.f, 0.f, 0.f}, value[4];
      load_group<XT, false>(x, e, bits, u);
      if (before) {
        load_group<TF32, false>(before, e, bits, copy);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] -= copy[j];
      }
      uint32_t codes, scale;
      encode(u, codes, scale, value);
      if (e / 2 < a.scale_offset) {  // blocks end behind the vector where d is no multiple of 32, granules behind the blocks
        *reinterpret_cast<uint16_t*>(message + e / 2) = (uint16_t)codes;
        if (lane % 8 == 0) message[a.scale_offset + e / kMxBlock] = (uint8_t)scale;
      }
      if (behind) {
        if (before) {
#pragma unroll
          for (int j = 0; j < 4; ++j) value[j] = copy[j] + value[j];
        }
        store_group<TF32, false>(behind, e, bits, value);
      }
    }
  }
}

template <typename XT, int MODE, int N, int C>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_mix(const MixArgs<N, C> a) {
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group();
  const uint32_t row = blockIdx.x % a.s.n_rows, i = a.s.first + blockIdx.x / a.s.n_rows * kMixWaves + wave;
  if (i < a.s.n_granules) {
    const RowPointers p = a.row[row];
    void* sum = buffer<void, 0>(p);
    const void* copy = buffer<const void, 1>(p);
    const void* x = buffer<const void, 2>(p);
    void* behind = buffer<void, 3>(p);
    const uint32_t cut = cut_of(a.s.cuts, i);
    const uint64_t e0 = (uint64_t)i * kGranule + 4 * lane;
    const uint32_t bits[2] = {group_bits(a.s.cuts, cut, 0, lane), group_bits(a.s.cuts, cut, 1, lane)};
    float mixed[2][4] = {};
    const int32_t first = a.lists.row_ptr[a.s.row0 + row], end = a.lists.row_ptr[a.s.row0 + row + 1];
    for (int32_t k = first; k < end; ++k) {
      const uint8_t* message = buffer(a.message[a.lists.col[k]]);
      const float w = a.lists.w[k];
#pragma unroll
      for (uint32_t half = 0; half < 2; ++half) {
        const uint64_t e = e0 + half * 256;
        if (bits[half] != 0) {
          float q[4];
          decode(*reinterpret_cast<const uint16_t*>(message + e / 2), q);
          const float weight = w * power_of(message[a.scale_offset + e / kMxBlock]);
#pragma unroll
          for (int j = 0; j < 4; ++j) mixed[half][j] = __builtin_fmaf(weight, q[j], mixed[half][j]);
        }
      }
    }
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
      const uint64_t e = e0 + half * 256;
      if constexpr (MODE != kMixStore) {
        float s[4];
        load_group<TF32, false>(sum, e, bits[half], s);
#pragma unroll
        for (int j = 0; j < 4; ++j) mixed[half][j] = s[j] + mixed[half][j];
      }
      if constexpr (MODE == kMixGossip) {
        float c[4], v[4];
        load_group<TF32, false>(copy, e, bits[half], c);
        load_group<XT, false>(x, e, bits[half], v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_fmaf(a.gamma, mixed[half][j] - c[j], v[j]);
        store_group<XT, false>(behind, e, bits[half], v);
      }
      store_group<TF32, false>(sum, e, bits[half], mixed[half]);
    }
  }
}

// One workgroup takes 256 elements of all rows: its wavefronts deal the rows among themselves, park their messages in LDS,
// and after one barrier take the neighbours' from there.  What a row holds in registers until then is its x, its copy and its sum.
constexpr uint32_t kRoundElems = kWave * 4, kRoundMessage = kRoundElems / 2 + kRoundElems / kMxBlock;
constexpr uint32_t kRoundWaves = 16;
template <typename XT, int ROWS, int N>
__global__ __launch_bounds__(kWave * kRoundWaves) void k_mx4_round(const RoundArgs<N> a) {
  extern __shared__ uint8_t lds[];  // of every row: 128 bytes of codes, 8 of scales
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group(), waves = blockDim.x / kWave;
  const uint32_t tile = a.s.first * 2 + blockIdx.x;  // first, count and n_granules count granules, which are two tiles
  const uint64_t e = (uint64_t)tile * kRoundElems + 4 * lane;
  const uint32_t bits = group_bits(a.s.cuts, cut_of(a.s.cuts, tile / 2), tile % 2, lane);
  float x[ROWS][4], copy[ROWS][4];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const uint32_t row = wave + k * waves;
    if (row < a.s.n_rows) {
      load_group<XT, false>(buffer<const void, 0>(a.row[row]), e, bits, x[k]);
      load_group<TF32, false>(buffer<const void, 2>(a.row[row]), e, bits, copy[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const uint32_t row = wave + k * waves;
    if (row < a.s.n_rows) {
      float u[4], value[4];
      uint32_t codes, scale;
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = x[k][j] - copy[k][j];
      encode(u, codes, scale, value);
#pragma unroll
      for (int j = 0; j < 4; ++j) copy[k][j] = copy[k][j] + value[j];
      store_group<TF32, false>(buffer<void, 2>(a.row[row]), e, bits, copy[k]);
      *reinterpret_cast<uint16_t*>(lds + row * kRoundMessage + 2 * lane) = (uint16_t)codes;
      if (lane % 8 == 0) lds[row * kRoundMessage + kRoundElems / 2 + lane / 8] = (uint8_t)scale;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const uint32_t row = wave + k * waves;
    if (row < a.s.n_rows) {
      float sum[4], mixed[4] = {};
      load_group<TF32, false>(buffer<const void, 3>(a.row[row]), e, bits, sum);
      const int32_t first = a.lists.row_ptr[row], end = a.lists.row_ptr[row + 1];
      for (int32_t n = first; n < end; ++n) {
        const uint8_t* message = lds + a.lists.col[n] * kRoundMessage;
        float q[4];
        decode(*reinterpret_cast<const uint16_t*>(message + 2 * lane), q);
        const float weight = a.lists.w[n] * power_of(message[kRoundElems / 2 + lane / 8]);
#pragma unroll
        for (int j = 0; j < 4; ++j) mixed[j] = __builtin_fmaf(weight, q[j], mixed[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[j] = sum[j] + mixed[j];
        x[k][j] = __builtin_fmaf(a.gamma, sum[j] - copy[k][j], x[k][j]);
      }
      store_group<TF32, false>(buffer<void, 3>(a.row[row]), e, bits, sum);
      store_group<XT, false>(buffer<void, 1>(a.row[row]), e, bits, x[k]);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------
template <int N>
int enqueue_encode(int xdt, EncodeArgs<N> a, void* stream) {
  const KernelFn fn = xdt == DADAM_BF16 ? (KernelFn)k_mx4_encode<TBF16, N> : (KernelFn)k_mx4_encode<TF32, N>;
  return in_pieces(a, kMixWaves, a.s.n_rows, kWave * kMixWaves, [&](uint32_t grid) { return enqueue_grid(fn, grid, kWave * kMixWaves, &a, 0, stream); });
}

template <int N, int C>
KernelFn mix_kernel(int xdt, MixMode mode) {
  if (mode == kMixStore) return (KernelFn)k_mx4_mix<TF32, kMixStore, N, C>;
  if (mode == kMixAdd) return (KernelFn)k_mx4_mix<TF32, kMixAdd, N, C>;
  return xdt == DADAM_BF16 ? (KernelFn)k_mx4_mix<TBF16, kMixGossip, N, C> : (KernelFn)k_mx4_mix<TF32, kMixGossip, N, C>;
}
template <int N, int C>
int enqueue_mix(int xdt, MixMode mode, MixArgs<N, C> a, void* stream) {
  const KernelFn fn = mix_kernel<N, C>(xdt, mode);
  return in_pieces(a, kMixWaves, a.s.n_rows, kWave * kMixWaves, [&](uint32_t grid) { return enqueue_grid(fn, grid, kWave * kMixWaves, &a, 0, stream); });
}

template <int N>
KernelFn round_kernel(int xdt, uint32_t rows_per_wave) {
  const bool b = xdt == DADAM_BF16;
#define DADAM_ROUND(ROWS) (b ? (KernelFn)k_mx4_round<TBF16, ROWS, N> : (KernelFn)k_mx4_round<TF32, ROWS, N>)
  if (rows_per_wave <= 1) return DADAM_ROUND(1);
  if constexpr (N > kFewOperands) {
    if (rows_per_wave <= 2) return DADAM_ROUND(2);
    if (rows_per_wave <= 4) return DADAM_ROUND(4);
    return DADAM_ROUND(10);
  }
#undef DADAM_ROUND
  return nullptr;
}
template <int N>
int enqueue_round(int xdt, RoundArgs<N> a, void* stream) {
  const uint32_t waves = a.s.n_rows < kRoundWaves ? a.s.n_rows : kRoundWaves;
  const KernelFn fn = round_kernel<N>(xdt, (a.s.n_rows + waves - 1) / waves);
  if (fn == nullptr) return (int)hipErrorInvalidDeviceFunction;
  const uint32_t last = (uint32_t)((a.s.d + kRoundElems - 1) / kRoundElems);  // the last granule may hold one tile only
  return in_pieces(a, 1, 2, kWave * waves, [&](uint32_t grid) {
    const uint32_t from = a.s.first * 2;
    return enqueue_grid(fn, from + grid > last ? last - from : grid, kWave * waves, &a, a.s.n_rows * kRoundMessage, stream);
  });
}

}  // namespace

int launch_encode(int xdt, const EncodeArgs<kMaxRows>& a, void* stream) {
  if (a.s.n_rows > (uint32_t)kFewOperands) return enqueue_encode(xdt, a, stream);
  auto f = few_rows<EncodeArgs<kFewOperands>>(a);
  f.s = a.s; f.scale_offset = a.scale_offset;
  return enqueue_encode(xdt, f, stream);
}

int launch_mix4(int xdt, MixMode mode, uint32_t n_cols, const MixArgs<kMessageRows, kMaxRows>& a, void* stream) {
  if (a.s.n_rows > (uint32_t)kFewOperands || n_cols > (uint32_t)kFewOperands) return enqueue_mix(xdt, mode, a, stream);
  auto f = few_rows<MixArgs<kFewOperands, kFewOperands>>(a);
  memcpy((void*)f.message, (const void*)a.message, sizeof(f.message));
  f.s = a.s; f.lists = a.lists; f.scale_offset = a.scale_offset; f.gamma = a.gamma;
  return enqueue_mix(xdt, mode, f, stream);
}

int launch_round(int xdt, const RoundArgs<kMaxRows>& a, void* stream) {
  if (a.s.n_rows > (uint32_t)kFewOperands) return enqueue_round(xdt, a, stream);
  auto f = few_rows<RoundArgs<kFewOperands>>(a);
  f.s = a.s; f.lists = a.lists; f.gamma = a.gamma;
  return enqueue_round(xdt, f, stream);
}

}  // namespace dadam
