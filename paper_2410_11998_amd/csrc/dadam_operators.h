// Internal interface between the host side of the operators around the step (dadam_operators.cpp: gradient norms and
// clipping, microscaled 4-bit messages) and their kernels (dadam_norm.hip, dadam_mx4.hip).
#ifndef DADAM_OPERATORS_H_
#define DADAM_OPERATORS_H_

#include <stdint.h>

#include "dadam_internal.h"

namespace dadam {

constexpr uint32_t kMxBlock = DADAM_MX4_BLOCK;  // elements that share one power of two
constexpr uint32_t kGranule = 512;              // elements a wavefront takes at a time: two groups of four a lane
constexpr uint32_t kGranuleBlocks = kGranule / kMxBlock;

// Up to four buffers of one row.  With 160 rows four plain addresses each would not fit the 4 KB of kernel arguments: these
// are 16-byte aligned and below 2^52 (the host checks both), so 32 low and 16 high bits of address / 16 name them.
struct RowPointers {
  uint32_t low[4], high[2];
};
struct ColPointer {
  uint32_t low, high;
};

// Which elements of a granule belong to a tensor.  index[granule]: 0 all of them, else 1 + where its kGranuleBlocks words of 32
// bits stand in masks.  index == nullptr: every granule is whole.
struct Cuts {
  const uint32_t* index;
  const uint32_t* masks;
};

// Neighbour lists of a slot (device), see MixRow: positions [first, first + the launch's rows) of its rows.
struct Lists {
  const MixRow* rows;
  const MixEntry* entries;
};

// How launches of handles that stream go: lanes lie apart (see units_from), and accesses carry the non-temporal hint.  Buffers that do not all begin
// at a multiple of 128 bytes (rows of one tensor often do not): apart only, as stores with the hint then write parts of lines.  us, three processes each in
// turn, with the hint / without: round of 16 rows of 2e7 1757, 1758, 1558 / 1584, 1417, 1394, of 61 of 2.3e6 in bfloat16 724, 689, 606 / 593, 499, 533, quantising 8 of
// 3e7 437, 429, 430 / 378, 358, 369, gossip of 8 bfloat16 rows of 3e7 795, 796, 758 / 727, 700, 688, adding product of 32 rows that share their sum 1446, 1451, 1371 / 1366, 1297,
// 1354.  Clipping (468 / 468) and products that store (749 / 757) keep it, as do other adding products (478 / 500).  On whole lines: quantising 329 / 353, gossip of 16 rows
// of 2e7 1058 / 1165.
enum Streams : uint32_t { kStreamsNot = 0, kStreamsHinted = 1, kStreamsApart = 2 };

// What all these launches have in common: units [first, first + count) of n_rows rows.
struct Span {
  Cuts cuts;
  uint64_t d;
  uint32_t n_granules;  // of the whole vector; as many units
  uint32_t first, count;
  uint32_t n_rows;
  uint32_t n_xcd;
  uint32_t run;         // pieces of a row that a die takes one after the other (see die_block_piece)
  uint32_t streams;     // Streams
};

constexpr int kFewOperands = 16;  // rows and sources of the short argument block (see kFewRows)
constexpr uint32_t kNormWaves = 16;       // of a workgroup of k_grad_norm
constexpr uint32_t kSmallGranules = 128;  // see k_clip_small
constexpr int kMessageRows = 96;  // rows of one launch that also carries the addresses of kMaxRows messages

template <int N>
struct NormArgs {
  RowPointers row[N];  // 0 gradient, 1 scaled gradient
  Span s;
  double* partials;    // [row][per_row]
  uint32_t* arrived;   // [row], zero between launches
  float* norms;        // [row]
  uint32_t per_row;    // workgroups that share a row
  float max_norm;
};

template <int N>
struct EncodeArgs {
  RowPointers row[N];  // 0 x, 1 copy before (may be null), 2 copy behind (may be null), 3 message
  Span s;
  uint64_t scale_offset;
};

template <int N, int C>
struct MixArgs {
  RowPointers row[N];  // by position: 0 sum or output, 1 copy, 2 x, 3 x behind
  ColPointer message[C];
  Span s;
  Lists lists;
  uint64_t scale_offset;
  uint32_t work;       // MixWork
  uint32_t rows_each;  // kMixByGroup: positions a workgroup takes
  float gamma;
};

template <int N>
struct RoundArgs {
  RowPointers row[N];  // by position: 0 x, 1 x behind, 2 copy, 3 sum
  Span s;
  Lists lists;
  const MixRow* firsts;  // the first row of every list
  uint32_t n_groups;     // lists whose sums the wavefronts of a workgroup form together, 0: every wavefront its own
  float gamma;
};

// Who does what of a launch: a wavefront a row, a workgroup several rows that share their sum, a wavefront all rows; or rows are copies of
// others (row 0 the copy, 1 what it is of).
enum MixWork : uint32_t { kMixByRow = 0, kMixByGroup = 1, kMixAllRows = 2, kMixCopy = 3 };
static_assert(sizeof(NormArgs<kMaxRows>) <= 4096 && sizeof(EncodeArgs<kMaxRows>) <= 4096 && sizeof(RoundArgs<kMaxRows>) <= 4096 &&
                  sizeof(MixArgs<kMessageRows, kMaxRows>) <= 4096, "the argument block of a launch holds 4 KB");

enum MixMode : int { kMixStore = 0, kMixAdd = 1, kMixGossip = 2 };

constexpr uint32_t kSharedBytes = kMixParts * 2 * kWave * 16;  // LDS of a workgroup that forms a sum together (k_mx4_shared)

// How a round is dealt to a workgroup: rows a wavefront holds, its wavefronts, units of a granule, and the LDS that the messages of a unit take.
// Streaming handles: three rows a wavefront, or as many as there are.  Up to four rows a wavefront has two groups of four a lane, beyond that one.
constexpr uint32_t kRoundWaves = 16;
template <int V>
constexpr uint32_t kRoundMessage = 128 * V + 8 * V;  // bytes of a row's message of a unit of 256 V elements, by lane
struct RoundShape {
  uint32_t each, waves, units, messages;
};
inline RoundShape round_shape(uint32_t n_rows, bool streams) {
  const uint32_t least = (n_rows + kRoundWaves - 1) / kRoundWaves, most = n_rows < 3 ? n_rows : 3;
  const uint32_t each = streams && least < most ? most : least, units = each <= 4 ? 1 : 2;
  return {each, (n_rows + each - 1) / each, units, n_rows * (units == 1 ? kRoundMessage<2> : kRoundMessage<1>)};
}
// The LDS of a workgroup: the messages, and the parts of the sums that it forms together.
inline uint32_t round_bytes(const RoundShape& r, uint32_t n_groups) {
  return n_groups == 0 ? r.messages : r.messages + (r.messages & 8) + n_groups * kMixParts * (2 / r.units) * kWave * 16;
}

// Launchers: enqueue on `stream`, return the hipError_t of the launch as int.  The large block is given; launches of few rows
// and sources send the short one.
int launch_norm(int gdt, const NormArgs<kMaxRows>& a, void* stream);
int launch_clip(int gdt, const NormArgs<kMaxRows>& a, void* stream);
int launch_clip_small(int gdt, const NormArgs<kMaxRows>& a, void* stream);  // norms and clipping of up to kSmallGranules granules
int launch_encode(int xdt, const EncodeArgs<kMaxRows>& a, void* stream);
int launch_mix4(int xdt, MixMode mode, uint32_t n_cols, const MixArgs<kMessageRows, kMaxRows>& a, void* stream);
int launch_round(int xdt, const RoundArgs<kMaxRows>& a, void* stream);

}  // namespace dadam

#endif  // DADAM_OPERATORS_H_
