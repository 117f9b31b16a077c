// Microscaled 4-bit messages: quantisation of what a worker sends, the mixing matrix times such messages, the gossip update
// from that product, and the whole round in one pass where all replicas are here.
//
//   encode   u = x - h;  e = max(floor(log2 max|u|) - 2, -126);  q = u 2^-e on the grid 0, 1/2, 1, 3/2, 2, 3, 4, 6;  h += q 2^e
//   product  out_i (+)= sum_k w_ik value(msg_k)
//   gossip   s_i += that sum;  x_i += gamma (s_i - h_i)
//
// A block of 32 elements is eight lanes' groups of four: its largest magnitude takes three exchanges inside those lanes.  The type's own
// conversions (round to nearest even, saturating at 6; the power of two is their operand) do the rest.  All of it is bound by HBM where launches are large:
// 17 bytes a block of a message beside 8 to 24 an element of float32 vectors, against 12 vector instructions an element to quantise and 2.2 an element
// and listed source to sum up.
#include <hip/hip_runtime.h>

#include <cstring>
#include <type_traits>

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

// The four values of 16 bits of codes in a block of scale byte b.  The conversion takes the exponent of its scale operand as such a byte:
// 2^(b - 127), 0 included, and NaN for 255.
__device__ __forceinline__ void decode(uint32_t codes, uint32_t b, float (&value)[4]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(b << 23);
  const f2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const f2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  value[0] = x.x; value[1] = x.y; value[2] = y.x; value[3] = y.y;
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
  const float power = __uint_as_float(scale << 23);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, u[0], u[1], power, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[2], u[3], power, 1) & 0xFFFFu;
  if (!finite) codes = 0;
  decode(codes, scale, value);
}

template <typename XT, bool WHOLE, bool NT>
__device__ __forceinline__ void encode_unit(const Cuts& cuts, const Units<2, 1>& t, const RowPointers& p, uint64_t scale_offset) {
  const void* x = based<XT>(buffer<const void, 0>(p), t.base);
  const bool differs = buffer<const void, 1>(p) != nullptr, moves = buffer<void, 2>(p) != nullptr;
  const void* before = based<TF32>(buffer<const void, 1>(p), t.base);
  void* behind = based<TF32>(buffer<void, 2>(p), t.base);
  uint8_t* codes_to = buffer<uint8_t, 3>(p) + t.base / 2;
  uint8_t* scales_to = buffer<uint8_t, 3>(p) + scale_offset + t.base / kMxBlock;
  const uint32_t end = (uint32_t)(2 * scale_offset - t.base < 0x7FFFFFFFu ? 2 * scale_offset - t.base : 0x7FFFFFFFu);  // of the last block
  float u[2][4], copy[2][4] = {};
  uint32_t bits[2];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    bits[k] = WHOLE ? 0xFu : t.bits(cuts, k);
    load_group<XT, WHOLE, NT>(x, t.at(k), bits[k], t.left, u[k]);
  }
  if (differs) {
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) load_group<TF32, WHOLE, NT>(before, t.at(k), bits[k], t.left, copy[k]);
  }
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    const uint32_t e = t.at(k);
    if (differs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) u[k][j] -= copy[k][j];
    }
    uint32_t codes, scale;
    float value[4];
    encode(u[k], codes, scale, value);
    if (WHOLE || e < end) {  // blocks end behind the vector where d is no multiple of 32, granules behind the blocks
      *reinterpret_cast<uint16_t*>(codes_to + e / 2) = (uint16_t)codes;
      if (threadIdx.x % 8 == 0) scales_to[e / kMxBlock] = (uint8_t)scale;
    }
    if (moves) {
      if (differs) {
#pragma unroll
        for (int j = 0; j < 4; ++j) value[j] = copy[k][j] + value[j];
      }
      store_group<TF32, NT>(behind, e, bits[k], value);
    }
  }
}

// A wavefront takes a unit of one row, all of its loads in flight before the first use.  355 million bfloat16 elements without a copy before 373 us
// (6.2 TB/s, 366 to 377 over machines; vector instructions fill 46 % of the issue slots), 8 float32 rows of 3e7 329 us (6.2).
template <typename XT, int S, int N>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_encode(const EncodeArgs<N> a) {
  constexpr bool NT = S == kStreamsHinted;
  const uint32_t lane = threadIdx.x % kWave;
  uint32_t piece, row;
  const bool active = die_block_piece(blockIdx.x, a.s.n_rows, a.s.n_xcd, (a.s.count + kMixWaves - 1) / kMixWaves, kDieBlockTiles, piece, row, a.s.run);
  const uint32_t i = a.s.first + piece * kMixWaves + wave_of_group();
  if (active && i < a.s.n_granules) {
    const Units<2, 1> t = units_from<2, S != kStreamsNot>(i, a.s, lane);
    if (t.whole) encode_unit<XT, true, NT>(a.s.cuts, t, a.row[row], a.scale_offset);
    else encode_unit<XT, false, NT>(a.s.cuts, t, a.row[row], a.scale_offset);
  }
}

__device__ __forceinline__ MixRow mix_row(const Lists& l, uint32_t position) {
  typedef const MixRow __attribute__((address_space(4))) * Constant;
  return *reinterpret_cast<const MixRow*>((const MixRow*)((Constant)l.rows + position));
}
__device__ __forceinline__ MixEntry mix_entry(const Lists& l, uint32_t at) {
  typedef const MixEntry __attribute__((address_space(4))) * Constant;
  return *reinterpret_cast<const MixEntry*>((const MixEntry*)((Constant)l.entries + at));
}

// Messages [first, end) of the lists times their weights, for a lane's G groups.
template <bool WHOLE, int U, int G, typename A>
__device__ __forceinline__ void mix_unit(const A& a, int32_t first, int32_t end, const Units<2, U>& t, const uint32_t (&bits)[G], float (&mixed)[G][4]) {
  uint32_t e[G];
#pragma unroll
  for (uint32_t k = 0; k < G; ++k) {
    // groups without an element may lie behind the message: their lanes look at what the units count from instead
    e[k] = WHOLE || bits[k] != 0 ? t.at(k) : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) mixed[k][j] = 0.0f;
  }
  for (int32_t n = first; n < end; n += kMixAtOnce) {
    uint32_t codes[kMixAtOnce][G], scale[kMixAtOnce][G];
    float w[kMixAtOnce];
#pragma unroll
    for (int q = 0; q < kMixAtOnce; ++q) {
      const MixEntry entry = mix_entry(a.lists, (uint32_t)(n + q));
      w[q] = entry.w;
      if (n + q >= end) continue;
      const uint8_t* message = buffer(a.message[entry.col]) + t.base / 2;
      const uint8_t* scales = buffer(a.message[entry.col]) + a.scale_offset + t.base / kMxBlock;
#pragma unroll
      for (uint32_t k = 0; k < G; ++k) {
        codes[q][k] = *reinterpret_cast<const uint16_t*>(message + e[k] / 2);
        scale[q][k] = scales[e[k] / kMxBlock];
      }
    }
#pragma unroll
    for (int q = 0; q < kMixAtOnce; ++q) {
      if (n + q >= end) continue;
#pragma unroll
      for (uint32_t k = 0; k < G; ++k) {
        float value[4];
        decode(codes[q][k], scale[q][k], value);
#pragma unroll
        for (int j = 0; j < 4; ++j) mixed[k][j] = __builtin_fmaf(w[q], value[j], mixed[k][j]);
      }
    }
  }
}

// What one row does with its neighbours' sum.
template <typename XT, int MODE, int U, bool WHOLE, bool NT, typename A>
struct RowUpdate {
  static constexpr int G = 2 * U;
  float s[G][4], c[G][4], x[G][4];
  __device__ __forceinline__ void load(const A& a, uint32_t p, const Units<2, U>& t, const uint32_t (&bits)[G]) {
#pragma unroll
    for (uint32_t k = 0; k < G; ++k) {
      const uint32_t e = t.at(k);
      if constexpr (MODE != kMixStore) load_group<TF32, WHOLE, NT>(based<TF32>(buffer<const void, 0>(a.row[p]), t.base), e, bits[k], t.left, s[k]);
      if constexpr (MODE == kMixGossip) {
        load_group<TF32, WHOLE, NT>(based<TF32>(buffer<const void, 1>(a.row[p]), t.base), e, bits[k], t.left, c[k]);
        load_group<XT, WHOLE, NT>(based<XT>(buffer<const void, 2>(a.row[p]), t.base), e, bits[k], t.left, x[k]);
      }
    }
  }
  __device__ __forceinline__ void store(const A& a, uint32_t p, const Units<2, U>& t, const uint32_t (&bits)[G], const float (&mixed)[G][4]) {
#pragma unroll
    for (uint32_t k = 0; k < G; ++k) {
      const uint32_t e = t.at(k);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[k][j] = MODE == kMixStore ? mixed[k][j] : s[k][j] + mixed[k][j];
        if constexpr (MODE == kMixGossip) x[k][j] = __builtin_fmaf(a.gamma, s[k][j] - c[k][j], x[k][j]);
      }
      store_group<TF32, NT>(based<TF32>(buffer<void, 0>(a.row[p]), t.base), e, bits[k], s[k]);
      if constexpr (MODE == kMixGossip) store_group<XT, NT>(based<XT>(buffer<void, 3>(a.row[p]), t.base), e, bits[k], x[k]);
    }
  }
};

// The whole sum of a list, part by part.
template <bool WHOLE, int U, int G, typename A>
__device__ __forceinline__ void mix_list(const A& a, const MixRow& r, const Units<2, U>& t, const uint32_t (&bits)[G], float (&mixed)[G][4]) {
  mix_unit<WHOLE>(a, r.first_entry, r.first_entry + (r.part < r.n_entries ? r.part : r.n_entries), t, bits, mixed);
  for (int32_t n = r.part; n < r.n_entries; n += r.part) {
    float part[G][4];
    mix_unit<WHOLE>(a, r.first_entry + n, r.first_entry + (n + r.part < r.n_entries ? n + r.part : r.n_entries), t, bits, part);
#pragma unroll
    for (uint32_t k = 0; k < G; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) mixed[k][j] += part[k][j];
  }
}

template <typename XT, int MODE, bool WHOLE, bool NT, int U, typename A>
__device__ __forceinline__ void mix_position(const A& a, const Units<2, U>& t, uint32_t p) {
  constexpr int G = 2 * U;
  uint32_t bits[G];
#pragma unroll
  for (uint32_t k = 0; k < G; ++k) bits[k] = WHOLE ? 0xFu : t.bits(a.s.cuts, k);
  float mixed[G][4];
  RowUpdate<XT, MODE, U, WHOLE, NT, A> row;
  row.load(a, p, t, bits);
  mix_list<WHOLE>(a, mix_row(a.lists, p), t, bits, mixed);
  row.store(a, p, t, bits, mixed);
}

// A wavefront takes kMixUnits units of one row.  One row of 355 million in bfloat16 with three messages 977 us (6.4 TB/s), 16 rows of 2e7 with five
// 1050 us (6.3 TB/s of what has to move), 124 million decoded and summed from three 126 to 132 us (5.3 to 5.6).  All rows of a unit run on one die, whose L2 then holds the unit's messages; where handles stream
// a die walks runs of units row after row.  Two units where nothing but messages is read: their loads are then twice as many (us, one unit /
// two, ring of 8 of 3e7 elements 268 / 216, exp. graph of 16 of 2e7 420 / 333, four 430; adding 315 / 390, 458 / 512: their registers leave too few wavefronts).
template <int MODE>
constexpr uint32_t kMixUnits = MODE == kMixStore ? 2 : 1;
template <typename XT, int MODE, int S, int N, int C>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_mix(const MixArgs<N, C> a) {
  constexpr bool NT = S == kStreamsHinted;
  constexpr uint32_t U = kMixUnits<MODE>;
  uint32_t piece, p;
  const bool active = die_block_piece(blockIdx.x, a.s.n_rows, a.s.n_xcd, (a.s.count + kMixWaves * U - 1) / (kMixWaves * U), kDieBlockTiles, piece, p, a.s.run);
  const uint32_t i = a.s.first + (piece * kMixWaves + wave_of_group()) * U;
  if (active && i < a.s.n_granules) {
    const Units<2, U> t = units_from<2, S != kStreamsNot, U>(i, a.s, threadIdx.x % kWave);
    if (t.whole) mix_position<XT, MODE, true, NT>(a, t, p);
    else mix_position<XT, MODE, false, NT>(a, t, p);
  }
}

// Rows that share their sum, products of many granules: a wavefront takes a unit of all rows and forms the sums once.  (Two or four units, so that
// more of a row is written at a time, change nothing for 32 rows and lose 10 to 30 % for 100.)
template <typename XT, int MODE, bool WHOLE, bool NT, typename A>
__device__ __forceinline__ void mix_rows(const A& a, const Units<2, 1>& t) {
  uint32_t bits[2];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) bits[k] = WHOLE ? 0xFu : t.bits(a.s.cuts, k);
  float mixed[2][4];
  int32_t group = -1;
  for (uint32_t p = 0; p < a.s.n_rows; ++p) {
    RowUpdate<XT, MODE, 1, WHOLE, NT, A> row;
    row.load(a, p, t, bits);
    const MixRow r = mix_row(a.lists, p);
    if (r.group != group) mix_list<WHOLE>(a, r, t, bits, mixed);
    group = r.group;
    row.store(a, p, t, bits, mixed);
  }
}

template <int MODE, int S, int N, int C>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_products(const MixArgs<N, C> a) {
  constexpr bool NT = S == kStreamsHinted;
  const uint32_t pieces = (a.s.count + kMixWaves - 1) / kMixWaves;
  const uint32_t i = a.s.first + die_block_order(blockIdx.x, pieces, a.s.n_xcd, kDieBlockTiles) * kMixWaves + wave_of_group();
  if (i < a.s.n_granules) {
    const Units<2, 1> t = units_from<2, S != kStreamsNot>(i, a.s, threadIdx.x % kWave);
    if (t.whole) mix_rows<TF32, MODE, true, NT>(a, t);
    else mix_rows<TF32, MODE, false, NT>(a, t);
  }
}

// The other rows of products that share their sum, from the row that has it.
template <bool WHOLE, bool NT, typename A>
__device__ __forceinline__ void copy_unit(const A& a, const Units<2, 1>& t, const RowPointers& p) {
  uint32_t bits[2];
  float v[2][4];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    bits[k] = WHOLE ? 0xFu : t.bits(a.s.cuts, k);
    load_group<TF32, WHOLE, false>(based<TF32>(buffer<const void, 1>(p), t.base), t.at(k), bits[k], t.left, v[k]);
  }
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) store_group<TF32, NT>(based<TF32>(buffer<void, 0>(p), t.base), t.at(k), bits[k], v[k]);
}
template <int S, int N, int C>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_copy(const MixArgs<N, C> a) {
  constexpr bool NT = S == kStreamsHinted;
  uint32_t piece, p;
  const bool active = die_block_piece(blockIdx.x, a.s.n_rows, a.s.n_xcd, (a.s.count + kMixWaves - 1) / kMixWaves, kDieBlockTiles, piece, p, a.s.run);
  const uint32_t i = a.s.first + piece * kMixWaves + wave_of_group();
  if (active && i < a.s.n_granules) {
    const Units<2, 1> t = units_from<2, S != kStreamsNot>(i, a.s, threadIdx.x % kWave);
    if (t.whole) copy_unit<true, NT>(a, t, a.row[p]);
    else copy_unit<false, NT>(a, t, a.row[p]);
  }
}

// Rows that share their sum: a workgroup takes a unit of `rows_each` positions.  For every run of rows with the same list its wavefronts
// form a part of the sum each, add the parts up through LDS, all in the same order, and deal the rows among themselves.
template <typename XT, int MODE, bool WHOLE, bool NT, typename A>
__device__ __forceinline__ void mix_shared(const A& a, const Units<2, 1>& t, uint32_t from, uint32_t to, f4 (&parts)[kMixParts][2][kWave]) {
  static_assert(kMixParts == kMixWaves, "a part a wavefront");
  const uint32_t lane = threadIdx.x % kWave, wave = wave_of_group();
  constexpr int G = 2;
  uint32_t bits[G];
#pragma unroll
  for (uint32_t k = 0; k < G; ++k) bits[k] = WHOLE ? 0xFu : t.bits(a.s.cuts, k);
  while (from < to) {
    const MixRow r = mix_row(a.lists, from);
    uint32_t end = from + 1;
    while (end < to && mix_row(a.lists, end).group == r.group) ++end;
    float mixed[G][4];
    const int32_t n = (int32_t)wave * r.part, last = n + r.part < r.n_entries ? n + r.part : r.n_entries;
    mix_unit<WHOLE>(a, r.first_entry + n, r.first_entry + last, t, bits, mixed);
#pragma unroll
    for (uint32_t k = 0; k < G; ++k) parts[wave][k][lane] = f4{mixed[k][0], mixed[k][1], mixed[k][2], mixed[k][3]};
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < G; ++k) {
      f4 sum = parts[0][k][lane];
      for (int32_t q = 1; q < kMixParts; ++q)
        if (q * r.part < r.n_entries) sum += parts[q][k][lane];
      mixed[k][0] = sum.x; mixed[k][1] = sum.y; mixed[k][2] = sum.z; mixed[k][3] = sum.w;
    }
    for (uint32_t p = from + wave; p < end; p += kMixWaves) {
      RowUpdate<XT, MODE, 1, WHOLE, NT, A> row;
      row.load(a, p, t, bits);
      row.store(a, p, t, bits, mixed);
    }
    __syncthreads();
    from = end;
  }
}

template <typename XT, int MODE, int S, int N, int C>
__global__ __launch_bounds__(kWave * kMixWaves) void k_mx4_shared(const MixArgs<N, C> a) {
  constexpr bool NT = S == kStreamsHinted;
  __shared__ f4 parts[kMixParts][2][kWave];
  static_assert(sizeof(parts) == kSharedBytes, "what the host allows for");
  uint32_t i, part;
  const bool active = die_block_piece(blockIdx.x, (a.s.n_rows + a.rows_each - 1) / a.rows_each, a.s.n_xcd, a.s.count, kDieBlockTiles, i, part, a.s.run);
  if (active) {
    const uint32_t from = part * a.rows_each, to = from + a.rows_each < a.s.n_rows ? from + a.rows_each : a.s.n_rows;
    const Units<2, 1> t = units_from<2, S != kStreamsNot>(a.s.first + i, a.s, threadIdx.x % kWave);
    if (t.whole) mix_shared<XT, MODE, true, NT>(a, t, from, to, parts);
    else mix_shared<XT, MODE, false, NT>(a, t, from, to, parts);
  }
}

// Both sides of a round are elementwise in the vector and couple rows only through messages: with all rows of a unit in one workgroup the messages
// need not leave the chip, and x and the copy are read once (24 bytes an element in float32 instead of 33 in two calls).  16 rows of 124 million on the
// exponential graph 7.7 to 8.1 ms (5.9 to 6.2 TB/s), 8 bfloat16 rows of 3e7 786 to 803 us (6.2 to 6.4).
// One workgroup takes a unit of all rows: its wavefronts deal the rows among themselves, park their messages in LDS,
// and after one barrier take the neighbours' from there.  What a row holds in registers until then is its x and its copy.
static_assert(kRoundMessage<1> == kUnitElems<1> / 2 + kUnitElems<1> / kMxBlock && kRoundMessage<2> == 2 * kRoundMessage<1>, "codes and scales");

// Entries [first, end) of the lists, from the messages in LDS.
template <int V, typename A>
__device__ __forceinline__ void mix_parked(const A& a, int32_t first, int32_t end, const uint8_t* lds, uint32_t lane, float (&part)[V][4]) {
#pragma unroll
  for (uint32_t k = 0; k < V; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) part[k][j] = 0.0f;
  for (int32_t n = first; n < end; n += kMixAtOnce) {
#pragma unroll
    for (int m = 0; m < kMixAtOnce; ++m) {
      if (n + m >= end) continue;
      const MixEntry entry = mix_entry(a.lists, (uint32_t)(n + m));
      const uint8_t* message = lds + entry.col * kRoundMessage<V>;
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
        float value[4];
        decode(*reinterpret_cast<const uint16_t*>(message + k * 128 + 2 * lane), message[128 * V + k * 8 + lane / 8], value);
#pragma unroll
        for (int j = 0; j < 4; ++j) part[k][j] = __builtin_fmaf(entry.w, value[j], part[k][j]);
      }
    }
  }
}

template <typename XT, int ROWS, int V, bool WHOLE, bool NT, typename A>
__device__ __forceinline__ void round_unit(const A& a, const Units<V, 1>& t, uint32_t each, uint8_t* lds) {
  const uint32_t lane = threadIdx.x % kWave, from = wave_of_group() * each;
  uint32_t bits[V];
#pragma unroll
  for (uint32_t k = 0; k < V; ++k) bits[k] = WHOLE ? 0xFu : t.bits(a.s.cuts, k);
  float x[ROWS][V][4], copy[ROWS][V][4];
#pragma unroll
  for (uint32_t q = 0; q < ROWS; ++q) {
    const uint32_t p = from + q;
    if (q < each && p < a.s.n_rows) {
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
        load_group<XT, WHOLE, NT>(based<XT>(buffer<const void, 0>(a.row[p]), t.base), t.at(k), bits[k], t.left, x[q][k]);
        load_group<TF32, WHOLE, NT>(based<TF32>(buffer<const void, 2>(a.row[p]), t.base), t.at(k), bits[k], t.left, copy[q][k]);
      }
    }
  }
#pragma unroll
  for (uint32_t q = 0; q < ROWS; ++q) {
    const uint32_t p = from + q;
    if (q < each && p < a.s.n_rows) {
      uint8_t* message = lds + mix_row(a.lists, p).row * kRoundMessage<V>;
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
        float u[4], value[4];
        uint32_t codes, scale;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = x[q][k][j] - copy[q][k][j];
        encode(u, codes, scale, value);
#pragma unroll
        for (int j = 0; j < 4; ++j) copy[q][k][j] = copy[q][k][j] + value[j];
        store_group<TF32, NT>(based<TF32>(buffer<void, 2>(a.row[p]), t.base), t.at(k), bits[k], copy[q][k]);
        *reinterpret_cast<uint16_t*>(message + k * 128 + 2 * lane) = (uint16_t)codes;
        if (lane % 8 == 0) message[128 * V + k * 8 + lane / 8] = (uint8_t)scale;
      }
    }
  }
  __syncthreads();
  // Lists that many rows share: a part of a sum to a wavefront, through LDS.  (Every wavefront its own sum: complete graph on 61 rows of 2e6 in
  // bfloat16 715 us.)
  f4* parts = reinterpret_cast<f4*>(lds + a.s.n_rows * kRoundMessage<V> + (a.s.n_rows * kRoundMessage<V> & 8));
  if (a.n_groups != 0) {
    for (uint32_t task = wave_of_group(); task < a.n_groups * kMixParts; task += blockDim.x / kWave) {
      const Lists firsts = {a.firsts, a.lists.entries};
      const MixRow r = mix_row(firsts, task / kMixParts);
      const int32_t n = (int32_t)(task % kMixParts) * r.part;
      float part[V][4];
      mix_parked<V>(a, r.first_entry + n, r.first_entry + (n + r.part < r.n_entries ? n + r.part : r.n_entries), lds, lane, part);
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) parts[(task * V + k) * kWave + lane] = f4{part[k][0], part[k][1], part[k][2], part[k][3]};
    }
    __syncthreads();
  }
  float mixed[V][4];
  int32_t group = -1;
#pragma unroll
  for (uint32_t q = 0; q < ROWS; ++q) {
    const uint32_t p = from + q;
    if (q < each && p < a.s.n_rows) {
      float s[V][4];
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) load_group<TF32, WHOLE, NT>(based<TF32>(buffer<const void, 3>(a.row[p]), t.base), t.at(k), bits[k], t.left, s[k]);
      const MixRow r = mix_row(a.lists, p);
      if (r.group != group) {
        group = r.group;
        for (int32_t n = 0; n < r.n_entries; n += r.part) {
          float part[V][4];
          if (a.n_groups != 0) {
#pragma unroll
            for (uint32_t k = 0; k < V; ++k) {
              const f4 v = parts[((r.group * kMixParts + n / r.part) * V + k) * kWave + lane];
              part[k][0] = v.x; part[k][1] = v.y; part[k][2] = v.z; part[k][3] = v.w;
            }
          } else {
            mix_parked<V>(a, r.first_entry + n, r.first_entry + (n + r.part < r.n_entries ? n + r.part : r.n_entries), lds, lane, part);
          }
#pragma unroll
          for (uint32_t k = 0; k < V; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) mixed[k][j] = n == 0 ? part[k][j] : mixed[k][j] + part[k][j];
        }
      }
#pragma unroll
      for (uint32_t k = 0; k < V; ++k) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[k][j] = s[k][j] + mixed[k][j];
          x[q][k][j] = __builtin_fmaf(a.gamma, s[k][j] - copy[q][k][j], x[q][k][j]);
        }
        store_group<TF32, NT>(based<TF32>(buffer<void, 3>(a.row[p]), t.base), t.at(k), bits[k], s[k]);
        store_group<XT, NT>(based<XT>(buffer<void, 1>(a.row[p]), t.base), t.at(k), bits[k], x[q][k]);
      }
    }
  }
}

template <typename XT, int ROWS, int V, int S, int N>
__global__ __launch_bounds__(kWave * kRoundWaves) void k_mx4_round(const RoundArgs<N> a) {
  constexpr bool NT = S == kStreamsHinted;
  extern __shared__ __align__(16) uint8_t lds[];  // of every row: the codes of a unit, then its scales; then parts of shared sums
  const uint32_t waves = blockDim.x / kWave, each = (a.s.n_rows + waves - 1) / waves;
  const uint32_t i = a.s.first * (kGranule / kUnitElems<V>) + die_block_order(blockIdx.x, gridDim.x, a.s.n_xcd, kDieBlockTiles);
  const Units<V, 1> t = units_from<V, S != kStreamsNot>(i, a.s, threadIdx.x % kWave);
  if (t.whole) round_unit<XT, ROWS, V, true, NT>(a, t, each, lds);
  else round_unit<XT, ROWS, V, false, NT>(a, t, each, lds);
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------
// pick(std::integral_constant<int, S>) for the Streams of a launch
template <typename Pick>
KernelFn for_streams(uint32_t streams, Pick pick) {
  if (streams == kStreamsHinted) return pick(std::integral_constant<int, kStreamsHinted>());
  if (streams == kStreamsApart) return pick(std::integral_constant<int, kStreamsApart>());
  return pick(std::integral_constant<int, kStreamsNot>());
}

template <int N>
int enqueue_encode(int xdt, EncodeArgs<N> a, void* stream) {
  const KernelFn fn = for_streams(a.s.streams, [&](auto s) {
    return xdt == DADAM_BF16 ? (KernelFn)k_mx4_encode<TBF16, decltype(s)::value, N> : (KernelFn)k_mx4_encode<TF32, decltype(s)::value, N>;
  });
  return in_pieces(a, kMixWaves * a.s.n_xcd, a.s.n_rows * a.s.n_xcd, kWave * kMixWaves,
                   [&](uint32_t grid) { return enqueue_grid(fn, grid, kWave * kMixWaves, &a, 0, stream); });
}

// Only what the host's rules ask for (fill_span's calls, share_rows, copies_rows) has a kernel; anything else is refused by the launch.
template <int N, int C, int S>
KernelFn mix_kernel(int xdt, MixMode mode, uint32_t work) {
  const bool by_group = work == kMixByGroup;
  if (mode == kMixGossip) {
    if (xdt == DADAM_BF16) return by_group ? (KernelFn)k_mx4_shared<TBF16, kMixGossip, S, N, C> : (KernelFn)k_mx4_mix<TBF16, kMixGossip, S, N, C>;
    return by_group ? (KernelFn)k_mx4_shared<TF32, kMixGossip, S, N, C> : (KernelFn)k_mx4_mix<TF32, kMixGossip, S, N, C>;
  }
  // Few rows that stream are long: their products go by wavefronts.
  if constexpr (S == kStreamsNot || N > kFewOperands)
    if (mode == kMixAdd && by_group) return (KernelFn)k_mx4_shared<TF32, kMixAdd, S, N, C>;
  if (mode == kMixAdd && work == kMixAllRows) return (KernelFn)k_mx4_products<kMixAdd, S, N, C>;
  if constexpr (S != kStreamsApart) {  // (rows that do not share their sum, and products that store, keep the hint)
    if (mode == kMixAdd && work == kMixByRow) return (KernelFn)k_mx4_mix<TF32, kMixAdd, S, N, C>;
    if constexpr (S == kStreamsNot || N > kFewOperands)
      if (mode == kMixStore && by_group) return (KernelFn)k_mx4_shared<TF32, kMixStore, S, N, C>;
    if (mode == kMixStore && work == kMixAllRows) return (KernelFn)k_mx4_products<kMixStore, S, N, C>;
    if (mode == kMixStore && work == kMixByRow) return (KernelFn)k_mx4_mix<TF32, kMixStore, S, N, C>;
    if constexpr (S == kStreamsHinted)
      if (work == kMixCopy) return (KernelFn)k_mx4_copy<S, N, C>;
  }
  return nullptr;
}
template <int N, int C>
int enqueue_mix(int xdt, MixMode mode, MixArgs<N, C> a, void* stream) {
  const KernelFn fn = for_streams(a.s.streams, [&](auto s) { return mix_kernel<N, C, decltype(s)::value>(xdt, mode, a.work); });
  if (fn == nullptr) return (int)hipErrorInvalidDeviceFunction;
  const uint32_t X = a.s.n_xcd;  // kernels that walk rows have as many workgroups on every die
  uint32_t units = kMixWaves, groups = 1;
  if (a.work == kMixByRow) {
    units = kMixWaves * (mode == kMixStore ? kMixUnits<kMixStore> : kMixUnits<kMixAdd>) * X;
    groups = a.s.n_rows * X;
  } else if (a.work == kMixCopy) {
    units = kMixWaves * X;
    groups = a.s.n_rows * X;
  } else if (a.work == kMixByGroup) {
    units = X;
    groups = (a.s.n_rows + a.rows_each - 1) / a.rows_each * X;
  }
  return in_pieces(a, units, groups, kWave * kMixWaves, [&](uint32_t grid) { return enqueue_grid(fn, grid, kWave * kMixWaves, &a, 0, stream); });
}

// Rows a wavefront holds, and its groups a lane: what 128 registers have room for.  Up to kFewOperands rows: one where handles do not stream, up to three
// where they do; more rows: two at least, where handles stream three.
template <int N, int S>
KernelFn round_kernel(int xdt, uint32_t each) {
  const bool b = xdt == DADAM_BF16;
#define DADAM_ROUND(ROWS, V) (b ? (KernelFn)k_mx4_round<TBF16, ROWS, V, S, N> : (KernelFn)k_mx4_round<TF32, ROWS, V, S, N>)
  if constexpr (N <= kFewOperands) {
    if (each <= 1) return DADAM_ROUND(1, 2);
    if constexpr (S != kStreamsNot) return each <= 2 ? DADAM_ROUND(2, 2) : DADAM_ROUND(3, 2);
    return nullptr;
  } else {
    if constexpr (S == kStreamsNot)
      if (each <= 2) return DADAM_ROUND(2, 2);
    if (each <= 3) return DADAM_ROUND(3, 2);
    if (each <= 4) return DADAM_ROUND(4, 2);
    if (each <= 6) return DADAM_ROUND(6, 1);
    if (each <= 8) return DADAM_ROUND(8, 1);
    return DADAM_ROUND(10, 1);
  }
#undef DADAM_ROUND
}
template <int N>
int enqueue_round(int xdt, RoundArgs<N> a, void* stream) {
  const RoundShape r = round_shape(a.s.n_rows, a.s.streams != kStreamsNot);
  const KernelFn fn = for_streams(a.s.streams, [&](auto s) { return round_kernel<N, decltype(s)::value>(xdt, r.each); });
  if (fn == nullptr) return (int)hipErrorInvalidDeviceFunction;
  return in_pieces(a, 1, r.units, kWave * r.waves,
                   [&](uint32_t grid) { return enqueue_grid(fn, grid, kWave * r.waves, &a, round_bytes(r, a.n_groups), stream); });
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
  f.s = a.s; f.lists = a.lists; f.scale_offset = a.scale_offset; f.rows_each = a.rows_each; f.work = a.work; f.gamma = a.gamma;
  return enqueue_mix(xdt, mode, f, stream);
}

int launch_round(int xdt, const RoundArgs<kMaxRows>& a, void* stream) {
  if (a.s.n_rows > (uint32_t)kFewOperands) return enqueue_round(xdt, a, stream);
  auto f = few_rows<RoundArgs<kFewOperands>>(a);
  f.s = a.s; f.lists = a.lists; f.firsts = a.firsts; f.n_groups = a.n_groups; f.gamma = a.gamma;
  return enqueue_round(xdt, f, stream);
}

}  // namespace dadam
