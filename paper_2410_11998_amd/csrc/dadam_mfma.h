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

#include <atomic>

namespace dadam {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

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

// Elements of parameters, gradients and state: one, or up to eight side by side (a whole piece where the buffer's 16 bytes allow it; beyond n: zeros, not
// stored).
struct F32 {
  using type = float;
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return global<const float>(p)[e]; }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<float>(p)[e] = v; }
  static __device__ __forceinline__ void load8(uint64_t p, uint64_t e, uint32_t n, float (&v)[8]) {
    if (n >= 8 && (p + e * 4) % 16 == 0) {
      const float4v a = global<const float4v>(p + e * 4)[0], b = global<const float4v>(p + e * 4)[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store8(uint64_t p, uint64_t e, uint32_t n, const float (&v)[8]) {
    if (n >= 8 && (p + e * 4) % 16 == 0) {
      global<float4v>(p + e * 4)[0] = float4v{v[0], v[1], v[2], v[3]};
      global<float4v>(p + e * 4)[1] = float4v{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
};
struct B16 {
  using type = uint16_t;
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return Brain::value(global<const uint16_t>(p)[e]); }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<uint16_t>(p)[e] = (uint16_t)Brain::bits(v); }
  static __device__ __forceinline__ void load8(uint64_t p, uint64_t e, uint32_t n, float (&v)[8]) {
    if (n >= 8 && (p + e * 2) % 16 == 0) {
      const uint4v a = global<const uint4v>(p + e * 2)[0];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[2 * k] = Brain::value(a[k] & 0xffffu), v[2 * k + 1] = Brain::value(a[k] >> 16);
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store8(uint64_t p, uint64_t e, uint32_t n, const float (&v)[8]) {
    if (n >= 8 && (p + e * 2) % 16 == 0) {
      uint4v r;
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = Brain::bits(v[2 * k]) | Brain::bits(v[2 * k + 1]) << 16;
      global<uint4v>(p + e * 2)[0] = r;
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
};

constexpr int kStageBytes = 128;  // of a row's elements that a stage takes: 64 elements of one plane, 32 of two

// Where element k of a row of a two-plane operand has its high (the low is 32 behind it).
__device__ __forceinline__ uint32_t high_at(uint32_t k) { return (k & ~31u) * 2 + (k & 31u); }

// A value as the halves of an operand, the high in the low half of the word.
template <typename OP>
__device__ __forceinline__ uint32_t halves(float v) {
  const uint32_t high = OP::bits(v);
  return high | OP::bits(v - OP::value(high)) << 16;
}

// The same where an operand of PLANES planes is all that is made of it.
template <typename OP, int PLANES>
__device__ __forceinline__ uint32_t operand_word(float v) {
  if constexpr (PLANES == 1) return OP::bits(v);
  return halves<OP>(v);
}

// Eight values in their order, from the low or the high halves of eight words.
__device__ __forceinline__ uint4v lows(const uint32_t (&w)[8]) {
  uint4v r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100u);
  return r;
}
__device__ __forceinline__ uint4v highs(const uint32_t (&w)[8]) {
  uint4v r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
  return r;
}

// Elements k .. k+7 (k % 8 == 0) of row r of an operand of `cols` columns, from words that halves() gives.
template <int PLANES>
__device__ __forceinline__ void store8(uint64_t base, uint64_t r, uint32_t cols, uint32_t k, const uint32_t (&w)[8]) {
  if constexpr (PLANES == 1) {
    global<uint4v>(base + (r * cols + k) * 2)[0] = lows(w);
  } else {
    const uint64_t at = base + (r * cols * 2 + high_at(k)) * 2;
    global<uint4v>(at)[0] = lows(w);
    global<uint4v>(at + 64)[0] = highs(w);
  }
}
template <typename OP>
__device__ __forceinline__ void add8(float (&v)[8], uint64_t at) {
  const uint4v b = global<const uint4v>(at)[0];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[2 * e] += OP::value(b[e] & 0xffffu), v[2 * e + 1] += OP::value(b[e] >> 16);
}
// Their sum onto v.
template <typename OP, int PLANES>
__device__ __forceinline__ void load8(float (&v)[8], uint64_t base, uint64_t r, uint32_t cols, uint32_t k) {
  if constexpr (PLANES == 1) {
    add8<OP>(v, base + (r * cols + k) * 2);
  } else {
    const uint64_t at = base + (r * cols * 2 + high_at(k)) * 2;
    add8<OP>(v, at);
    add8<OP>(v, at + 64);
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int step = 32; step; step >>= 1) v += __shfl_xor(v, step);
  return v;
}

// Shape of a workgroup's tile: WM x WN wavefronts, each MT x NT blocks of 32 x 32; block (i, j) of wavefront (wm, wn) has rows (wm MT + i) 32 ... and columns
// (j WN + wn) 32 ...  The large tile (256 x 256, eight wavefronts) is bound by LDS as much as by the matrix cores: a stage reads 192 KB and is written 64 KB, 2048
// cycles, for 2048 cycles of products.  The small one (128 x 128, four) takes 768 cycles of LDS for 512 of products, and is for what has too few large tiles.
// TFLOP/s, large / small / library, 8192 x 8192 x 8192 1119 / 914 / 1319, x 1024 1061 / 805 / 1078, 1024 x 49152 x 4096 1087 / 915 / 1295.
template <typename OP, int PLANES, int MT, int NT, int WM, int WN>
struct Tile {
  static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
  static constexpr int kM = WM * MT * 32, kN = WN * NT * 32;
  static constexpr int kStage = (kM + kN) * kStageBytes;  // LDS of a stage
  static constexpr int kRows = WN * 32;                   // columns of C that are finished at a time
  static constexpr int kLds = 2 * kStage > kRows * kM * 4 ? 2 * kStage : kRows * kM * 4;
  static constexpr int kSteps = PLANES == 1 ? 4 : 2;      // of 16 summed elements, in a stage
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
  // of 32 rows, touch all banks.  LIMITED: beyond `limit` rows (at least 1) the last one is brought again.
  template <int ROWS, bool LIMITED>
  static __device__ __forceinline__ void fetch(const char DADAM_GLOBAL* rows, uint64_t pitch, uint32_t limit, char DADAM_LDS* lds, int wave, int lane) {
    const uint32_t piece = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u, own = (uint32_t)(lane >> 3) * (uint32_t)pitch + piece;
#pragma unroll
    for (int j = 0; j < ROWS / 8 / kWaves; ++j) {
      const int eight = j * kWaves + wave;
      const char DADAM_GLOBAL* from = rows + (uint64_t)eight * 8 * pitch + own;
      if constexpr (LIMITED) {
        const uint32_t row = (uint32_t)(eight * 8 + (lane >> 3));
        from = rows + (uint64_t)(row < limit ? row : limit - 1) * (uint32_t)pitch + piece;
      }
      __builtin_amdgcn_global_load_lds((const uint32_t DADAM_GLOBAL*)from, (uint32_t DADAM_LDS*)(lds + eight * 1024), 16, 0, 0);
    }
  }

  // Fragments of a step: lane l has elements 8 (l / 32) ... of row l % 32 of every block.
  struct Fragments {
    vec a[PLANES][MT], b[PLANES][NT];
  };
  static __device__ __forceinline__ void read(Fragments& f, const char DADAM_LDS* stage, int step, int wm, int wn, int lane) {
    const uint32_t order = (uint32_t)((lane >> 5) ^ (lane & 7)), row = (uint32_t)(lane & 31) * kStageBytes;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      const char DADAM_LDS* at = stage + row + ((order ^ (uint32_t)((step + 2 * p) << 1)) << 4);
#pragma unroll
      for (int i = 0; i < MT; ++i) f.a[p][i] = *(const vec DADAM_LDS*)(at + (wm * MT + i) * 32 * kStageBytes);
#pragma unroll
      for (int j = 0; j < NT; ++j) f.b[p][j] = *(const vec DADAM_LDS*)(at + (kM + (j * WN + wn) * 32) * kStageBytes);
    }
  }
  __device__ __forceinline__ void multiply(const Fragments& f) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if constexpr (PLANES == 2) {
          acc[i][j] = OP::mfma(f.a[1][i], f.b[0][j], acc[i][j]);
          acc[i][j] = OP::mfma(f.a[0][i], f.b[1][j], acc[i][j]);
        }
        acc[i][j] = OP::mfma(f.a[0][i], f.b[0][j], acc[i][j]);
      }
  }

  // The sums over `stages` stages, from zero on.  a and b: the tile's first rows, at their first stage; pitches in bytes.  While a stage is multiplied
  // the next one is on its way, and with one plane (two have no registers for it) while a step is multiplied the next one's fragments are: 128 x 128 x 1024
  // tiles 805 TFLOP/s instead of 695.
  template <bool LIMITED = false>
  __device__ __forceinline__ void product(const char DADAM_GLOBAL* a, uint64_t a_pitch, const char DADAM_GLOBAL* b, uint64_t b_pitch, uint32_t stages, char DADAM_LDS* lds,
                                          uint32_t a_limit = 0, uint32_t b_limit = 0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    auto bring = [&](uint32_t s) {
      char DADAM_LDS* to = lds + (s & 1) * kStage;
      fetch<kM, LIMITED>(a + (uint64_t)s * kStageBytes, a_pitch, a_limit, to, wave, lane);
      fetch<kN, LIMITED>(b + (uint64_t)s * kStageBytes, b_pitch, b_limit, to + kM * kStageBytes, wave, lane);
    };
    clear();
    bring(0);
    if constexpr (PLANES == 1) {
      Fragments f[2];
      __syncthreads();
      read(f[0], lds, 0, wm, wn, lane);
      for (uint32_t s = 0; s < stages; ++s) {
        if (s + 1 < stages) bring(s + 1);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          if (k + 1 < kSteps) {
            read(f[(k + 1) & 1], lds + (s & 1) * kStage, k + 1, wm, wn, lane);
          } else {
            __syncthreads();  // everybody has read this stage, and the next one is there
            if (s + 1 < stages) read(f[(k + 1) & 1], lds + ((s + 1) & 1) * kStage, 0, wm, wn, lane);
          }
          __builtin_amdgcn_sched_barrier(0);
          multiply(f[k & 1]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
      for (uint32_t s = 0; s < stages; ++s) {
        __syncthreads();
        if (s + 1 < stages) bring(s + 1);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          Fragments f;
          read(f, lds + (s & 1) * kStage, k, wm, wn, lane);
          multiply(f);
        }
      }
    }
  }

  // Hands the sums out by whole pieces of rows and of columns, through LDS (a lane holds four rows of one column of every block; stored from there, an
  // instruction writes 16 bytes each to 32 lines).  kRows columns at a time: column(m, n, v) gets C[m .. m+7][n] in v and may replace them by 32-bit values of its
  // own; with `turned`, row(m, n, v) then gets those of C[m][n .. n+7].  The 16-byte pieces of a column lie in the order piece ^ n ^ n / 8, so that neither
  // the lanes that write, 32 columns of one piece, nor those that read, 128 columns of one row, meet in a bank.
  template <typename Column, typename Row>
  __device__ __forceinline__ void hand_out(char DADAM_LDS* lds, bool turned, Column column, Row row) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    auto place = [&](uint32_t n, uint32_t piece) { return lds + n * (kM * 4) + ((piece ^ ((n ^ (n >> 3)) & 31u)) << 4); };
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4v v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
          *(float4v DADAM_LDS*)place((uint32_t)(wn * 32 + (lane & 31)), (uint32_t)((wm * MT + i) * 8 + g * 2 + (lane >> 5))) = v;
        }
      __syncthreads();
#pragma unroll 2
      for (uint32_t k = threadIdx.x; k < (uint32_t)(kRows * kM / 8); k += kThreads) {
        const uint32_t n = k / (kM / 8), m = k % (kM / 8) * 8;
        float v[8];
        float4v DADAM_LDS* low = (float4v DADAM_LDS*)place(n, m / 4);
        float4v DADAM_LDS* high = (float4v DADAM_LDS*)place(n, m / 4 + 1);
        const float4v a = *low, b = *high;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        column(m, (uint32_t)(j * kRows) + n, v);
        if (turned) {
          *low = float4v{v[0], v[1], v[2], v[3]};
          *high = float4v{v[4], v[5], v[6], v[7]};
        }
      }
      if (!turned) continue;
      __syncthreads();
#pragma unroll 2
      for (uint32_t k = threadIdx.x; k < (uint32_t)(kRows * kM / 8); k += kThreads) {
        const uint32_t n = k % (kRows / 8) * 8, m = k / (kRows / 8);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *(const float DADAM_LDS*)(place(n + e, m / 4) + (m & 3) * 4);
        row(m, (uint32_t)(j * kRows) + n, v);
      }
    }
  }
};

template <typename OP, int PLANES>
using LargeTile = Tile<OP, PLANES, 4, 2, 2, 4>;
template <typename OP, int PLANES>
using SmallTile = Tile<OP, PLANES, 2, 2, 2, 2>;

// Workgroup b of n as its die takes it: consecutive workgroup ids go to the dies in turn, each die takes a contiguous run of tiles, whose operands
// its L2 then holds.
__device__ __forceinline__ uint32_t die_run(uint32_t b, uint32_t n, uint32_t dies) {
  const uint32_t each = n / dies, more = n % dies, die = b % dies, at = b / dies;
  return die * each + (die < more ? die : more) + at;
}

// The LDS of KERNEL's workgroups beyond what a launch may take unasked: said once on every device.
template <auto KERNEL>
int ask_for_lds(uint32_t bytes) {
  static std::atomic<uint64_t> asked{0};
  int device = 0;
  if (const hipError_t e = hipGetDevice(&device)) return (int)e;
  const uint64_t bit = 1ull << (device & 63);
  if (device < 64 && (asked.load(std::memory_order_relaxed) & bit)) return (int)hipSuccess;
  const hipError_t e = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess) asked.fetch_or(bit, std::memory_order_relaxed);
  return (int)e;
}

}  // namespace
}  // namespace dadam

#endif  // DADAM_MFMA_H_
