// Matrix products on the matrix cores, shared by the kernels of orthogonalised updates and of a head's loss (included by their .hip files only).
//
// Every product here is C[m][n] = sum_k A[m][k] B[n][k].  An operand lies by rows (m or n, the summed index innermost) or by columns (rows of the summed
// index); either way its rows, columns and the summed index are filled up to the tiles with zeros, or with what comes to nothing.  An element is 16 bits
// (bfloat16, or half precision times a power of two that keeps it in range) or, where 32 bits are called for, two halves that together hold 22 bits of it:
// element = high + low.  Then 32 highs are followed by their 32 lows, the next 32 highs and so on, and a product takes three instructions instead of one
// (high high, high low, low high; low low is below the last place that is kept).  Sums are float32 throughout.
#ifndef DADAM_MFMA_H_
#define DADAM_MFMA_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

namespace dadam {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// The same where elements lie as a caller's buffer has them, at a multiple of an element's size only (memory takes such pieces at any address; element by element, a vector of
// odd width takes three times as long).
typedef float4v float4u __attribute__((aligned(4)));
typedef uint2v uint2u __attribute__((aligned(2)));
typedef uint4v uint4u __attribute__((aligned(2)));

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

// Elements of parameters, gradients and state: one, or up to four or eight side by side (beyond n: zeros, not stored).
struct F32 {
  using type = float;
  static __device__ __forceinline__ void load4(uint64_t p, uint64_t e, uint32_t n, float (&v)[4]) {
    if (n >= 4) {
      const float4v a = global<const float4u>(p + e * 4)[0];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = a[k];
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store4(uint64_t p, uint64_t e, uint32_t n, const float (&v)[4]) {
    if (n >= 4) {
      global<float4u>(p + e * 4)[0] = float4v{v[0], v[1], v[2], v[3]};
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
  struct Piece {  // eight elements as they lie, of a whole piece
    float4v a, b;
    __device__ __forceinline__ float operator[](int k) const { return k < 4 ? a[k] : b[k - 4]; }
  };
  static __device__ __forceinline__ bool is_whole(uint32_t n) { return n >= 8; }
  static __device__ __forceinline__ Piece piece(uint64_t p, uint64_t e) { return {global<const float4u>(p + e * 4)[0], global<const float4u>(p + e * 4)[1]}; }
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return global<const float>(p)[e]; }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<float>(p)[e] = v; }
  static __device__ __forceinline__ void load8(uint64_t p, uint64_t e, uint32_t n, float (&v)[8]) {
    if (n >= 8) {
      const float4v a = global<const float4u>(p + e * 4)[0], b = global<const float4u>(p + e * 4)[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store8(uint64_t p, uint64_t e, uint32_t n, const float (&v)[8]) {
    if (n >= 8) {
      global<float4u>(p + e * 4)[0] = float4v{v[0], v[1], v[2], v[3]};
      global<float4u>(p + e * 4)[1] = float4v{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
};
struct B16 {
  using type = uint16_t;
  static __device__ __forceinline__ void load4(uint64_t p, uint64_t e, uint32_t n, float (&v)[4]) {
    if (n >= 4) {
      const uint2v a = global<const uint2u>(p + e * 2)[0];
      v[0] = Brain::value(a[0] & 0xffffu), v[1] = Brain::value(a[0] >> 16), v[2] = Brain::value(a[1] & 0xffffu), v[3] = Brain::value(a[1] >> 16);
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store4(uint64_t p, uint64_t e, uint32_t n, const float (&v)[4]) {
    if (n >= 4) {
      global<uint2u>(p + e * 2)[0] = uint2v{Brain::bits(v[0]) | Brain::bits(v[1]) << 16, Brain::bits(v[2]) | Brain::bits(v[3]) << 16};
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
  struct Piece {
    uint4v a;
    __device__ __forceinline__ float operator[](int k) const { return Brain::value(a[k / 2] >> 16 * (k & 1) & 0xffffu); }
  };
  static __device__ __forceinline__ bool is_whole(uint32_t n) { return n >= 8; }
  static __device__ __forceinline__ Piece piece(uint64_t p, uint64_t e) { return {global<const uint4u>(p + e * 2)[0]}; }
  static __device__ __forceinline__ float load(uint64_t p, uint64_t e) { return Brain::value(global<const uint16_t>(p)[e]); }
  static __device__ __forceinline__ void store(uint64_t p, uint64_t e, float v) { global<uint16_t>(p)[e] = (uint16_t)Brain::bits(v); }
  static __device__ __forceinline__ void load8(uint64_t p, uint64_t e, uint32_t n, float (&v)[8]) {
    if (n >= 8) {
      const uint4v a = global<const uint4u>(p + e * 2)[0];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[2 * k] = Brain::value(a[k] & 0xffffu), v[2 * k + 1] = Brain::value(a[k] >> 16);
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < n ? load(p, e + k) : 0.f;
  }
  static __device__ __forceinline__ void store8(uint64_t p, uint64_t e, uint32_t n, const float (&v)[8]) {
    if (n >= 8) {
      uint4v r;
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = Brain::bits(v[2 * k]) | Brain::bits(v[2 * k + 1]) << 16;
      global<uint4u>(p + e * 2)[0] = r;
      return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
      if (k < n) store(p, e + k, v[k]);
  }
};

// e^x for x <= 0 (or NaN), with CLOSE to about two places of float32: the instruction's 2^y of y = x log2(e) in two parts, y = high + low, 2^low = 1 + low ln 2.  Without, the
// rounding of y makes it |x| 2^-24 of the value.
template <bool CLOSE>
__device__ __forceinline__ float exponential(float x) {
  if constexpr (!CLOSE) return __expf(x);
  x = x < -200.f ? -200.f : x;  // (0 as well, and no infinity less an infinity)
  const float high = x * 1.44269502f, low = fmaf(x, 1.44269502f, -high) + x * 1.92596299e-8f, e = __builtin_amdgcn_exp2f(high);
  return fmaf(e, low * 0.693147181f, e);
}

// Where a tile's side of an operand begins (at the first stage), its rows' distance in bytes (a stage's rows within 2^32 of each other), and how many of
// them there are: beyond, the last one is taken again.
struct Operand {
  uint64_t at;
  uint32_t pitch, rows;
};
constexpr uint32_t kNoLimit = 0xffffffffu;
__device__ __forceinline__ Operand operand(uint64_t at, uint64_t pitch, uint32_t rows = kNoLimit) { return {at, (uint32_t)pitch, rows}; }
// The same for the whole wavefront, in scalar registers.
__device__ __forceinline__ Operand uniform(const Operand& o) {
  const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)o.at), high = __builtin_amdgcn_readfirstlane((uint32_t)(o.at >> 32));
  return {(uint64_t)high << 32 | low, (uint32_t)__builtin_amdgcn_readfirstlane(o.pitch), (uint32_t)__builtin_amdgcn_readfirstlane(o.rows)};
}

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
// Elements k .. k+7 of row r of an operand, as loaded: their highs and lows.
struct Eight {
  uint4v high, low;
};
template <int PLANES>
__device__ __forceinline__ Eight load8(uint64_t base, uint64_t r, uint32_t cols, uint32_t k) {
  if constexpr (PLANES == 1) return {global<const uint4v>(base + (r * cols + k) * 2)[0], uint4v{0, 0, 0, 0}};
  const uint64_t at = base + (r * cols * 2 + high_at(k)) * 2;
  return {global<const uint4v>(at)[0], global<const uint4v>(at + 64)[0]};
}
template <typename OP, bool LOW>
__device__ __forceinline__ float value_of(const Eight& x, int e) {
  const float high = OP::value(x.high[e / 2] >> 16 * (e & 1) & 0xffffu);
  return LOW ? high + OP::value(x.low[e / 2] >> 16 * (e & 1) & 0xffffu) : high;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int step = 32; step; step >>= 1) v += __shfl_xor(v, step);
  return v;
}

// 16 bytes a lane from `offset` of a buffer to LDS, 1 KB side by side from `to` on.  Nothing waits for it but everybody_has_loaded().  (In assembly, as the compiler
// takes the builtin's load for one that any LDS read may depend on: of the global loads it then waits for all fragments where it needs the older ones only,
// and before a read that turns for all loads.  No register is written but m0, which nothing else here uses.)
__device__ __forceinline__ void load_to_lds(uint4v buffer, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer) : "memory");
}

// What this wavefront has asked for is in LDS, but for its LEFT last loads, and so is what the others have; and nobody reads what was there before.  (Not
// __syncthreads(), which waits for all loads that the compiler knows of.)  Nothing else is under way either: scalar loads that are, and are not needed before the
// products' end, make the compiler wait for all fragments where it needs the older ones only.
template <int LEFT>
__device__ __forceinline__ void everybody_has_loaded() {
  static_assert(LEFT < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (LEFT & 15) | (LEFT >> 4) << 14);  // vmcnt(LEFT) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Fragments of blocks that lie by columns: elements of two times four rows, AT and NEXT bytes behind at[...].
template <int AT, int NEXT, typename V, int N>
__device__ __forceinline__ void read_turned(V (&out)[N], const uint32_t (&at)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v DADAM_LDS*)(uintptr_t)(at[i] + AT));
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v DADAM_LDS*)(uintptr_t)(at[i] + NEXT));
    out[i] = __builtin_bit_cast(V, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

// Shape of a workgroup's tile: WM x WN wavefronts, each MT x NT blocks of 32 x 32; block (i, j) of wavefront (wm, wn) has rows (wm MT + i) 32 ... and columns
// (j WN + wn) 32 ...  The large tile (256 x 256, eight wavefronts) is bound by LDS as much as by the matrix cores: a stage reads 192 KB and is written 64 KB, 2048
// cycles, for 2048 cycles of products.  The small one (128 x 128, four) takes 768 cycles of LDS for 512 of products, and is for what has too few large tiles.
// TFLOP/s of products alone, large / small / library's whole product: 8192 x 8192 x 8192 1293 / 1081 / 1347, x 1024 1162 / 1020 / 1092, 4096 x 50176 x 1024 1190 / 1040 / 1096;
// with two planes, of instructions, 1383, 1324 and 1287.  (Zeros reach 1600 to 1900: what random numbers cost beyond that is the power that the chip may take.)
// A_DOWN, B_DOWN: that operand lies by columns.  BUFFERS: stages in LDS, of which all but one are on their way.
// APART: products with a low half have sums of their own, so that a sum of large values is rounded a third as often (32-bit logits of a width of 2304 and more:
// gradients off by 7e-7 instead of 1.3e-6 of their norm).  It has to be the only tile of its compute unit: two of them would not fit the registers, nor a large one.
template <typename OP, int PLANES, int MT, int NT, int WM, int WN, bool A_DOWN, bool B_DOWN, int BUFFERS, bool APART = false>
struct Tile {
  static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
  static constexpr int kM = WM * MT * 32, kN = WN * NT * 32;
  static constexpr int kStage = (kM + kN) * kStageBytes;  // LDS of a stage
  static constexpr int kRows = WN * 32;                   // columns of C that are finished at a time
  static constexpr int kLds = BUFFERS * kStage;
  static_assert(kLds >= kRows * kM * 4, "columns that are finished find room");
  static constexpr int kSteps = PLANES == 1 ? 4 : 2;      // of 16 summed elements, in a stage
  using vec = typename OP::vec;

  float16v acc[MT][NT];
  float16v lows_apart[APART ? MT : 1][APART ? NT : 1];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          acc[i][j][r] = 0.f;
          if constexpr (APART) lows_apart[i][j][r] = 0.f;
        }
  }

  // By columns, the 32-byte pieces of row k of a stage lie in the order piece ^ mixed(k): a fragment's instruction reads two pieces side by side of
  // rows k .. k+3 and k+8 .. k+11, which are then all different.
  template <int SIDE>
  static __device__ __forceinline__ uint32_t mixed(uint32_t k) {
    constexpr uint32_t kPieces = SIDE * 2 * PLANES / 32;
    return ((k & 3) << 1 | (k >> 3 & 1) << 3) & (kPieces - 1);
  }

  // A stage of SIDE rows (DOWN: columns) of an operand into LDS, straight from memory; a wavefront's instruction brings 1 KB, lane l the 16 bytes that belong at
  // l * 16 of it.  By rows that is 8 rows of 128 bytes, whose 16-byte pieces lie in the order piece ^ (row / 2 & 7): the lanes of a fragment read one piece of 32
  // rows, sixteen of them at a time, which are then in sixteen different places of 256 bytes.  (With row & 7 in eight: half of the LDS cycles were conflicts.)  `rows`: of the operand from the stage on.
  static constexpr uint32_t kSummed = 16 * kSteps;  // of a stage
  template <int SIDE, bool DOWN>
  static __device__ __forceinline__ void fetch(uint64_t at, uint32_t pitch, uint32_t rows, char DADAM_LDS* lds, int wave, int lane) {
    const uint4v buffer = {(uint32_t)at, (uint32_t)(at >> 32), 0xffffffffu, 0x00020000u};
#pragma unroll
    for (int j = 0; j < SIDE / 8 / kWaves; ++j) {
      const int part = j * kWaves + wave;
      uint32_t from;
      if constexpr (DOWN) {
        constexpr int kRowBytes = SIDE * 2 * PLANES, kPieces = kRowBytes / 16;
        const uint32_t k = (uint32_t)(part * 64 + lane) / kPieces, piece = (uint32_t)(lane % kPieces) ^ (mixed<SIDE>(k) << 1);
        from = (k < rows ? k : rows - 1) * pitch + piece * 16;
      } else {
        const uint32_t row = (uint32_t)(part * 8 + (lane >> 3)), piece = (uint32_t)(lane & 7) ^ (row >> 1 & 7);
        from = (row < rows ? row : rows - 1) * pitch + piece * 16;
      }
      load_to_lds(buffer, from, (uint32_t)(uintptr_t)(lds + part * 1024));
    }
  }

  // Fragments of a step: lane l has elements 8 (l / 32) ... of row l % 32 of every block.
  struct Fragments {
    vec a[PLANES][MT], b[PLANES][NT];
  };
  // By rows: block `block` of 32.
  static __device__ __forceinline__ vec fragment(const char DADAM_LDS* side, int block, int plane, int step, int lane) {
    const uint32_t piece = (uint32_t)((lane >> 5) ^ (lane >> 1 & 7)) ^ (uint32_t)((step + 2 * plane) << 1);
    return *(const vec DADAM_LDS*)(side + (block * 32 + (lane & 31)) * kStageBytes + piece * 16);
  }
  // By columns: where the lane's part of block `block` of SIDE begins.  Sixteen lanes get four rows of sixteen columns, every lane the four of its column.
  template <int SIDE>
  static __device__ __forceinline__ uint32_t column_part(const char DADAM_LDS* side, int block, int plane, int lane) {
    const uint32_t k = (uint32_t)(lane >> 5) * 8 + ((uint32_t)(lane & 15) >> 2);
    const uint32_t piece = (uint32_t)(block * 2 * PLANES + plane * 2 + (lane >> 4 & 1)) ^ mixed<SIDE>(k);
    return (uint32_t)(uintptr_t)(side + k * (SIDE * 2 * PLANES) + piece * 32 + (lane & 3) * 8);
  }
  template <int STEP>
  static __device__ __forceinline__ void read(Fragments& f, const char DADAM_LDS* stage, int wm, int wn, int lane) {
    const char DADAM_LDS* b_side = stage + kM * kStageBytes;
    static_assert(kM == kN, "rows of either side have the same length");
    constexpr int kAt = STEP * 16 * kM * 2 * PLANES, kNext = kAt + 4 * kM * 2 * PLANES;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      if constexpr (!A_DOWN)
#pragma unroll
        for (int i = 0; i < MT; ++i) f.a[p][i] = fragment(stage, wm * MT + i, p, STEP, lane);
      if constexpr (!B_DOWN)
#pragma unroll
        for (int j = 0; j < NT; ++j) f.b[p][j] = fragment(b_side, j * WN + wn, p, STEP, lane);
    }
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      if constexpr (A_DOWN && B_DOWN) {
        uint32_t at[MT + NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) at[i] = column_part<kM>(stage, wm * MT + i, p, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) at[MT + j] = column_part<kN>(b_side, j * WN + wn, p, lane);
        vec out[MT + NT];
        read_turned<kAt, kNext>(out, at);
#pragma unroll
        for (int i = 0; i < MT; ++i) f.a[p][i] = out[i];
#pragma unroll
        for (int j = 0; j < NT; ++j) f.b[p][j] = out[MT + j];
      } else if constexpr (A_DOWN) {
        uint32_t at[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) at[i] = column_part<kM>(stage, wm * MT + i, p, lane);
        read_turned<kAt, kNext>(f.a[p], at);
      }
    }
    static_assert(A_DOWN || !B_DOWN, "an operand that lies by columns is the first one");
  }
  __device__ __forceinline__ void multiply(const Fragments& f) {
    // (one product of all blocks after the other: three in a row onto the same sums would wait for each other)
#pragma unroll
    for (int p = PLANES == 1 ? 2 : 0; p < 3; ++p)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float16v& sum = APART && p < 2 ? lows_apart[APART ? i : 0][APART ? j : 0] : acc[i][j];
          sum = OP::mfma(f.a[p == 0 ? PLANES - 1 : 0][i], f.b[p == 1 ? PLANES - 1 : 0][j], sum);
        }
  }

  // The sums over `stages` stages (of 64 summed elements, or 32 of two planes), from zero on.  While a stage is multiplied the next one is on its way, and while a
  // step is multiplied the next one's fragments are.
  __device__ __forceinline__ void product(const Operand& a, const Operand& b, uint32_t stages, char DADAM_LDS* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const Operand ua = uniform(a), ub = uniform(b);
    auto stage_at = [&](uint32_t s) { return lds + s % BUFFERS * kStage; };
    auto bring = [&](uint32_t s) {
      char DADAM_LDS* to = stage_at(s);
      fetch<kM, A_DOWN>(ua.at + (A_DOWN ? (uint64_t)s * kSummed * ua.pitch : (uint64_t)s * kStageBytes), ua.pitch, A_DOWN ? ua.rows - s * kSummed : ua.rows, to, wave, lane);
      fetch<kN, B_DOWN>(ub.at + (B_DOWN ? (uint64_t)s * kSummed * ub.pitch : (uint64_t)s * kStageBytes), ub.pitch, B_DOWN ? ub.rows - s * kSummed : ub.rows,
                        to + kM * kStageBytes, wave, lane);
    };
    // Stage s is there: only the loads of the stages behind it, as many as have been asked for, may be left.
    constexpr int kLoads = (kM + kN) / 8 / kWaves;
    auto loaded = [&](uint32_t s) {
      const uint32_t behind = stages - 1 - s < (uint32_t)(BUFFERS - 2) ? stages - 1 - s : (uint32_t)(BUFFERS - 2);
      if (BUFFERS > 3 && behind == 2) return everybody_has_loaded<2 * kLoads>();
      if (BUFFERS > 2 && behind == 1) return everybody_has_loaded<kLoads>();
      return everybody_has_loaded<0>();
    };
    static_assert(BUFFERS == 2 || BUFFERS == 4, "loaded() counts for these");
    clear();
#pragma unroll
    for (uint32_t s = 0; s + 1 < (uint32_t)BUFFERS; ++s)
      if (s < stages) bring(s);
    Fragments f[2];
    loaded(0);
    read<0>(f[0], lds, wm, wn, lane);
    for (uint32_t s = 0; s < stages; ++s) {
      const char DADAM_LDS* stage = stage_at(s);
      if (s + BUFFERS - 1 < stages) bring(s + BUFFERS - 1);
      auto step = [&](int k) {
        __builtin_amdgcn_sched_barrier(0);
        multiply(f[k & 1]);
        __builtin_amdgcn_sched_barrier(0);
      };
      read<1>(f[1], stage, wm, wn, lane);
      step(0);
      if constexpr (kSteps == 4) {
        read<2>(f[0], stage, wm, wn, lane);
        step(1);
        read<3>(f[1], stage, wm, wn, lane);
        step(2);
      }
      if (s + 1 < stages) {
        loaded(s + 1);  // and everybody has read this stage
        read<0>(f[0], stage_at(s + 1), wm, wn, lane);
      }
      step(1);
    }
    if constexpr (APART) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] += lows_apart[i][j];
    }
  }

  // Hands the sums out by whole pieces of rows and of columns, through LDS (a lane holds four rows of one column of every block; stored from there, an
  // instruction writes 16 bytes each to 32 lines).  kRows columns at a time: column(m, n, v, held) gets C[m .. m+7][n] in v, and what ahead(m, n) has loaded;
  // with `turned` it leaves 32-bit values in v, of which row(m, n, v) then gets those of C[m][n .. n+7].  Loads go out four pieces at a time, before anything is
  // stored: one by one, each waits for memory behind the last one's store (half of the time of a tile of 1024 summed elements).
  // The 16-byte pieces of a column lie in the order piece ^ n ^ n / 8, so that neither the lanes that write, 32 columns of one piece, nor those that read,
  // 128 columns of one row, meet in a bank.
  template <typename Ahead, typename Column, typename Row>
  __device__ __forceinline__ void hand_out(char DADAM_LDS* lds, bool turned, Ahead ahead, Column column, Row row) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    constexpr int kEach = kRows * kM / 8 / kThreads, kAhead = 4;  // pieces of a thread
    static_assert(kEach % kAhead == 0, "whole batches");
    auto place = [&](uint32_t n, uint32_t piece) { return lds + n * (kM * 4) + ((piece ^ ((n ^ (n >> 3)) & 31u)) << 4); };
    auto m_of = [&](int k) { return (threadIdx.x + (uint32_t)k * kThreads) % (kM / 8) * 8; };
    auto n_of = [&](int k) { return (threadIdx.x + (uint32_t)k * kThreads) / (kM / 8); };
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      decltype(ahead(0u, 0u)) held[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) held[k] = ahead(m_of(k), (uint32_t)(j * kRows) + n_of(k));
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4v v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
          *(float4v DADAM_LDS*)place((uint32_t)(wn * 32 + (lane & 31)), (uint32_t)((wm * MT + i) * 8 + g * 2 + (lane >> 5))) = v;
        }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const uint32_t n = n_of(k), m = m_of(k);
        float v[8];
        float4v DADAM_LDS* low = (float4v DADAM_LDS*)place(n, m / 4);
        float4v DADAM_LDS* high = (float4v DADAM_LDS*)place(n, m / 4 + 1);
        const float4v a = *low, b = *high;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        if (k && k % kAhead == 0) {
#pragma unroll
          for (int x = 0; x < kAhead; ++x) held[x] = ahead(m_of(k + x), (uint32_t)(j * kRows) + n_of(k + x));
        }
        column(m, (uint32_t)(j * kRows) + n, v, held[k % kAhead]);
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

// ahead of hand_out where there is nothing to load.
struct Nothing {};
__device__ __forceinline__ Nothing nothing_ahead(uint32_t, uint32_t) { return {}; }

// Small tiles of a launch that gives every compute unit one at most keep four stages: a stage then has three times as long to come, and it is the length of a tile that
// counts.  (Two tiles of two stages each fit a compute unit otherwise.)
template <typename OP, int PLANES, int EDGE, int BUFFERS, bool A_DOWN, bool B_DOWN, bool APART = false>
using TileOf =
    typename std::conditional<EDGE == 256, Tile<OP, PLANES, 4, 2, 2, 4, A_DOWN, B_DOWN, BUFFERS>, Tile<OP, PLANES, 2, 2, 2, 2, A_DOWN, B_DOWN, BUFFERS, APART>>::type;
constexpr uint32_t kOneEach = 256;  // compute units

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

// Tile u of `across` x `down`, in bands of kBand across: the workgroups that a die runs at a time, neighbours in this order, then share few rows and columns of
// the operands.  8192 x 8192 x 1024 by large tiles: 1196 TFLOP/s in bands of 8, 999 row by row.
constexpr uint32_t kBand = 8;
__device__ __forceinline__ void banded(uint32_t u, uint32_t across, uint32_t down, uint32_t& i, uint32_t& j) {
  const uint32_t band = u / (kBand * down), in = u % (kBand * down), wide = across - band * kBand < kBand ? across - band * kBand : kBand;
  i = band * kBand + in % wide;
  j = in / wide;
}

}  // namespace
}  // namespace dadam

#endif  // DADAM_MFMA_H_
