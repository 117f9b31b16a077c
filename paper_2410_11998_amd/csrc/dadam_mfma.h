// Matrix products on the matrix cores, shared by the kernels of orthogonalised updates and of a head's loss (included by their .hip files only).
//
// Every product here is C[m][n] = sum_k A[m][k] B[n][k]: both operands have the summed index innermost, rows a multiple of the tile and the summed
// index a multiple of kStageBytes, the padding zero.  An operand element is 16 bits (bfloat16, or half precision times a power of two that keeps it
// in range) or, where 32 bits are called for, two halves that together hold 22 bits of it: element = high + low.  Then a row holds 32 highs, their
// 32 lows, the next 32 highs and so on, and a product takes three instructions instead of one (high high, high low, low high; low low is below the
// last place that is kept).  Sums are float32 throughout.
#ifndef DADAM_MFMA_H_
#define DADAM_MFMA_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dadam {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

#define DADAM_GLOBAL __attribute__((address_space(1)))
#define DADAM_LDS __attribute__((address_space(3)))

// Addresses that come out of tables are global memory.
template <typename T>
__device__ __forceinline__ T DADAM_GLOBAL* global(uint64_t address) {
  return (T DADAM_GLOBAL*)address;
}
template <typename T>
__device__ __forceinline__ T DADAM_GLOBAL* global(const void* p) {
  return (T DADAM_GLOBAL*)(uint64_t)p;
}

struct Half {
  using vec = half8;
  static __device__ __forceinline__ float16v mfma(vec a, vec b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  static __device__ __forceinline__ float value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
};
struct Brain {
  using vec = brain8;
  static __device__ __forceinline__ float16v mfma(vec a, vec b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  static __device__ __forceinline__ float value(uint32_t b) { return __uint_as_float(b << 16); }
};

// Elements of parameters, gradients and state.
struct F32 {
  using type = float;
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return global<const float>(p)[e]; }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<float>(p)[e] = v; }
};
struct B16 {
  using type = uint16_t;
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return Brain::value(global<const uint16_t>(p)[e]); }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<uint16_t>(p)[e] = (uint16_t)Brain::bits(v); }
};

constexpr int kStageBytes = 128;  // of a row's elements that a stage takes: 64 elements of one plane, 32 of two

// Where element k of a row of a two-plane operand has its high (the low is 32 behind it).
__device__ __forceinline__ uint32_t high_at(uint32_t k) { return (k & ~31u) * 2 + (k & 31u); }

__device__ __forceinline__ uint32_t pair(uint32_t low, uint32_t high) { return low | high << 16; }
__device__ __forceinline__ uint2v four(const uint32_t (&b)[4]) { return uint2v{pair(b[0], b[1]), pair(b[2], b[3])}; }

// A value as the halves of an operand.
template <typename OP>
__device__ __forceinline__ void halves(float v, uint32_t& high, uint32_t& low) {
  high = OP::bits(v);
  low = OP::bits(v - OP::value(high));
}

// Elements k .. k+3 (k % 4 == 0) of row r of an operand of `cols` columns.
template <typename OP, int PLANES>
__device__ __forceinline__ void store4(uint64_t base, uint64_t r, uint32_t cols, uint32_t k, const float4v& v) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) halves<OP>(v[e], h[e], l[e]);
  if constexpr (PLANES == 1) {
    global<uint2v>(base + (r * cols + k) * 2)[0] = four(h);
  } else {
    global<uint2v>(base + (r * cols * 2 + high_at(k)) * 2)[0] = four(h);
    global<uint2v>(base + (r * cols * 2 + high_at(k) + 32) * 2)[0] = four(l);
  }
}
template <typename OP, int PLANES>
__device__ __forceinline__ void store1(uint64_t base, uint64_t r, uint32_t cols, uint32_t k, float v) {
  uint32_t h, l;
  halves<OP>(v, h, l);
  if constexpr (PLANES == 1) {
    global<uint16_t>(base)[r * cols + k] = (uint16_t)h;
  } else {
    global<uint16_t>(base)[r * cols * 2 + high_at(k)] = (uint16_t)h;
    global<uint16_t>(base)[r * cols * 2 + high_at(k) + 32] = (uint16_t)l;
  }
}
template <typename OP, int PLANES>
__device__ __forceinline__ float4v load4(uint64_t base, uint64_t r, uint32_t cols, uint32_t k) {
  auto unpack = [](uint2v b) { return float4v{OP::value(b[0] & 0xffff), OP::value(b[0] >> 16), OP::value(b[1] & 0xffff), OP::value(b[1] >> 16)}; };
  if constexpr (PLANES == 1) return unpack(global<const uint2v>(base + (r * cols + k) * 2)[0]);
  return unpack(global<const uint2v>(base + (r * cols * 2 + high_at(k)) * 2)[0]) + unpack(global<const uint2v>(base + (r * cols * 2 + high_at(k) + 32) * 2)[0]);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int step = 32; step; step >>= 1) v += __shfl_xor(v, step);
  return v;
}

// Shape of a workgroup's tile: WM x WN wavefronts, each MT x NT blocks of 32 x 32.
template <typename OP, int PLANES, int MT, int NT, int WM, int WN>
struct Tile {
  static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
  static constexpr int kM = WM * MT * 32, kN = WN * NT * 32;
  static constexpr int kStage = (kM + kN) * kStageBytes;  // LDS of a stage
  static constexpr int kLds = 2 * kStage;
  using vec = typename OP::vec;

  float16v acc[MT][NT];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  }

  // One stage of ROWS rows into LDS, straight from memory: a wavefront's instruction brings 8 rows of 128 bytes, lane l the 16 bytes that
  // belong at l * 16 of them.  The 16-byte pieces of row r lie in the order piece ^ (r & 7), so that the lanes of a fragment, which read one piece
  // of 32 rows, touch all banks.
  template <int ROWS>
  static __device__ __forceinline__ void fetch(const char DADAM_GLOBAL* rows, uint64_t pitch, char DADAM_LDS* lds, int wave, int lane) {
    const uint32_t own = (uint32_t)(lane >> 3) * (uint32_t)pitch + (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
#pragma unroll
    for (int j = 0; j < ROWS / 8 / kWaves; ++j) {
      const int eight = j * kWaves + wave;
      __builtin_amdgcn_global_load_lds((const uint32_t DADAM_GLOBAL*)(rows + (uint64_t)eight * 8 * pitch + own), (uint32_t DADAM_LDS*)(lds + eight * 1024), 16, 0, 0);
    }
  }

  __device__ __forceinline__ void multiply(const char DADAM_LDS* stage, int wm, int wn, int lane) {
    const uint32_t order = (uint32_t)((lane >> 5) ^ (lane & 7));
    const char DADAM_LDS* a0 = stage + (wm * MT * 32 + (lane & 31)) * kStageBytes;
    const char DADAM_LDS* b0 = stage + (kM + wn * NT * 32 + (lane & 31)) * kStageBytes;
    auto piece = [&](const char DADAM_LDS* rows, int i, int s) {
      return *(const vec DADAM_LDS*)(rows + i * 32 * kStageBytes + ((order ^ (uint32_t)(s << 1)) << 4));
    };
    if constexpr (PLANES == 1) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        vec a[MT], b[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) a[i] = piece(a0, i, s);
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = piece(b0, j, s);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = OP::mfma(a[i], b[j], acc[i][j]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        vec ah[MT], bh[NT], al[MT], bl[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) ah[i] = piece(a0, i, s), al[i] = piece(a0, i, s + 2);
#pragma unroll
        for (int j = 0; j < NT; ++j) bh[j] = piece(b0, j, s), bl[j] = piece(b0, j, s + 2);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            acc[i][j] = OP::mfma(al[i], bh[j], acc[i][j]);
            acc[i][j] = OP::mfma(ah[i], bl[j], acc[i][j]);
            acc[i][j] = OP::mfma(ah[i], bh[j], acc[i][j]);
          }
      }
    }
  }

  // The sums over `stages` stages, from zero on.  a and b: the tile's first rows, at their first stage; pitches in bytes.
  __device__ __forceinline__ void product(const char DADAM_GLOBAL* a, uint64_t a_pitch, const char DADAM_GLOBAL* b, uint64_t b_pitch, uint32_t stages, char DADAM_LDS* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    clear();
    fetch<kM>(a, a_pitch, lds, wave, lane);
    fetch<kN>(b, b_pitch, lds + kM * kStageBytes, wave, lane);
    for (uint32_t s = 0; s < stages; ++s) {
      __syncthreads();
      if (s + 1 < stages) {
        char DADAM_LDS* next = lds + ((s + 1) & 1) * kStage;
        fetch<kM>(a + (uint64_t)(s + 1) * kStageBytes, a_pitch, next, wave, lane);
        fetch<kN>(b + (uint64_t)(s + 1) * kStageBytes, b_pitch, next + kM * kStageBytes, wave, lane);
      }
      multiply(lds + (s & 1) * kStage, wm, wn, lane);
    }
  }

  // Calls fn(m, n, four sums) for what the lane holds: C[m .. m+3][n] of the tile.
  template <typename Fn>
  __device__ __forceinline__ void each(Fn fn) const {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4v v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
          fn((uint32_t)(wm * MT * 32 + i * 32 + g * 8 + (lane >> 5) * 4), (uint32_t)(wn * NT * 32 + j * 32 + (lane & 31)), v);
        }
  }
};

// Workgroup b of n as its die takes it: consecutive workgroup ids go to the dies in turn, each die takes a contiguous run of tiles, whose operands
// its L2 then holds.
__device__ __forceinline__ uint32_t die_run(uint32_t b, uint32_t n, uint32_t dies) {
  const uint32_t each = n / dies, more = n % dies, die = b % dies, at = b / dies;
  return die * each + (die < more ? die : more) + at;
}

}  // namespace
}  // namespace dadam

#endif  // DADAM_MFMA_H_
