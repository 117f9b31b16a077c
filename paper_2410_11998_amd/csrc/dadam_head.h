// Internal interface between the host side of a head's loss (dadam_head.cpp) and its kernels (dadam_head.hip).
#ifndef DADAM_HEAD_H_
#define DADAM_HEAD_H_

#include <stdint.h>

#include "dadam_internal.h"

namespace dadam {

constexpr int kHeadRows = 32;         // replicas of a launch

struct HeadRow {  // device addresses, 0 where there is none
  uint64_t head, bias, hidden, target, nll, dhidden, dhead, dbias;
};

// HeadPlaces::words: how many tokens have a target, largest magnitudes, and from kHeadShares on those of kMostGroups workgroups, of the head and of the hidden vectors.
enum HeadWord : uint32_t { kHeadCount = 0, kHeadMostHidden = 1, kHeadMostHead = 2, kHeadShares = 16 };
constexpr uint32_t kMostGroups = 512;

// Workspace of a replica.  Operands have `planes` halves or bfloat16s an element: hidden vectors and a piece of the head by rows of D, softmax - e[target] of a
// piece by rows of its words, a token each.
struct HeadPlaces {
  uint64_t words, top, hit, stats, hidden, head, p, sums, parts, bytes;
};
struct HeadShape {
  uint32_t tokens, vocab, width;
  uint32_t edge;           // of the products' tiles: 128 or 256
  uint32_t T, D, K;        // tokens and width filled up to the edge, width filled up to a stage
  uint32_t piece, slices;  // words of a piece (a multiple of the edge), slices of edge / 2 of all words
  uint32_t splits;         // parts that the sum over words of a hidden vector's gradient goes in
  uint32_t parts;          // that the sum over tokens of the head's gradient goes in
  uint32_t keeps;          // softmax of all words is kept from the statistics on: one piece
};
inline constexpr HeadPlaces head_places(const HeadShape& s, uint64_t planes, bool gradient) {
  HeadPlaces w{};
  uint64_t at = 0, b = 2 * planes;
  auto take = [&at](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  w.words = take((kHeadShares + 2 * kMostGroups) * 4);
  w.top = take((uint64_t)s.T * 8);  // a token's largest logit and 1 / its sum of exponentials
  w.hit = take((uint64_t)s.T * 4);
  w.stats = take((uint64_t)s.slices * s.T * 8);
  w.hidden = take((uint64_t)s.T * s.D * b);
  w.head = take((uint64_t)s.piece * s.D * b);
  if (gradient) {
    w.p = take((uint64_t)s.T * s.piece * b);
    w.sums = take((uint64_t)s.splits * s.T * s.D * 4);
    if (s.parts > 1) w.parts = take((uint64_t)s.parts * s.piece * s.D * 4);
  }
  w.bytes = at;
  return w;
}

struct HeadArgs {
  HeadShape s;
  HeadPlaces w;
  uint64_t workspace, stride;
  float* losses;        // [row]
  float scale;
  uint32_t mean, add;
  uint32_t first_word, words;  // of the piece
  uint32_t skip;        // words of the piece that another launch of launch_head_dhead takes: those before
  uint32_t groups;      // whose largest magnitudes the operands go by, 0: they are known
  uint32_t later;       // a piece before this one has begun the sums
  uint32_t n_xcd;
  uint32_t straight;    // the head is an operand as it lies
  HeadRow row[kHeadRows];
};
static_assert(sizeof(HeadArgs) <= 4096, "the argument block of a launch holds 4 KB");

// The way of few tokens (dadam_head_few.hip): the head is read as it lies, 32 words at a time.
constexpr uint32_t kFewTokens = 64, kFewWords = 32, kFewColumns = 128;
struct FewPlaces {
  uint64_t words, top, hit, stats, z, p, p_turned, hidden, sums, bytes;
};
struct FewShape {
  uint32_t tokens, vocab, width;
  uint32_t T, D;             // tokens filled up to 32, width to kFewColumns
  uint32_t blocks;           // of kFewWords words
  uint32_t each, ranges;     // blocks of a range that a wavefront sums a hidden vector's gradient over, and ranges
};
inline constexpr FewPlaces few_places(const FewShape& s, uint64_t planes, bool gradient) {
  FewPlaces w{};
  uint64_t at = 0;
  auto take = [&at](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  w.words = take(64);
  w.top = take((uint64_t)s.T * 8);
  w.hit = take((uint64_t)s.T * 4);
  w.stats = take((uint64_t)s.blocks * s.T * 8);
  w.z = take((uint64_t)s.blocks * s.T * kFewWords * 4);  // of a block: T rows of kFewWords logits, with two planes softmax - e[target] in their place
  if (gradient) {
    if (planes == 1) {
      w.p = take((uint64_t)s.blocks * s.T * kFewWords * 2);         // as bfloat16
      w.p_turned = take((uint64_t)s.blocks * s.T * kFewWords * 2);  // and turned: kFewWords rows of T
    }
    w.hidden = take((uint64_t)s.T * s.D * 4);  // rows of D, with one plane D rows of T bfloat16s
    w.sums = take((uint64_t)s.ranges * s.tokens * s.D * 4);
  }
  w.bytes = at;
  return w;
}
struct FewArgs {
  FewShape s;
  FewPlaces w;
  uint64_t workspace, stride;
  float* losses;
  float scale;
  uint32_t mean, add;
  HeadRow row[kHeadRows];
};
static_assert(sizeof(FewArgs) <= 4096, "the argument block of a launch holds 4 KB");
int launch_few_logits(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream);
int launch_few_losses(const FewArgs& a, uint32_t rows, void* stream);
int launch_few_softmax(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream);    // and the bias's gradient
int launch_few_gradients(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream);
int launch_few_end(int xdt, int gdt, const FewArgs& a, uint32_t rows, void* stream);

// Launchers, of `rows` replicas.  xdt: type of parameters and hidden vectors, gdt of gradients; two planes unless both are bfloat16.
uint32_t head_most_groups(const HeadArgs& a);
int launch_head_most(int xdt, const HeadArgs& a, uint32_t rows, void* stream);  // with two planes only
int launch_head_operands(int xdt, int gdt, const HeadArgs& a, bool hidden, uint32_t rows, void* stream);  // of a piece, and of the hidden vectors
// Statistics; statistics, and the slices' exponentials kept; or the logits' gradient.
enum HeadMode : int { kHeadStatistics = 0, kHeadKeep = 1, kHeadGradient = 2 };
int launch_head_logits(int xdt, int gdt, HeadMode mode, const HeadArgs& a, uint32_t rows, void* stream);
int launch_head_losses(const HeadArgs& a, uint32_t rows, void* stream);
int launch_head_scale(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream);                   // the logits' gradient from what was kept
int launch_head_dhead(int xdt, int gdt, uint32_t edge, const HeadArgs& a, uint32_t rows, void* stream);
// The same by small tiles, in HeadShape::parts of the tokens, and their sum.
int launch_head_dhead_parts(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream);
int launch_head_dbias(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream);
int launch_head_dhidden(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream);                 // a piece's part of the sums
int launch_head_end(int xdt, int gdt, const HeadArgs& a, uint32_t rows, void* stream);                     // the hidden vectors' gradients from the sums

}  // namespace dadam

#endif  // DADAM_HEAD_H_
