// Internal interface between the host side of orthogonalised updates (dadam_ortho.cpp) and their kernels (dadam_ortho.hip).
#ifndef DADAM_ORTHO_H_
#define DADAM_ORTHO_H_

#include <stdint.h>

#include "dadam_internal.h"

namespace dadam {

constexpr uint32_t kOrthoCell = 128;               // side of the tiles that the iteration's beginning goes by
constexpr uint32_t kSmallEdge = 128, kLargeEdge = 256;  // sides of the products' tiles

// One matrix, the same for every replica.  X has p rows and q >= p columns: the matrix itself, or its transpose where it is tall.
struct OrthoTask {
  uint64_t first;        // its first element in the packed vector
  uint64_t at;           // bytes of workspace of the matrices before it, for one replica
  uint32_t ld;           // elements from row to row
  uint32_t p, q, P, Q;   // P, Q: filled up to a multiple of the products' tiles
  uint32_t tall;
  uint32_t gram_units, whole_units, cell_units, small_units;  // tiles of the matrices before it: of the lower half of P x P, of P x Q, cells of P x Q, and
                                                              // small tiles of the lower half
  float scale, decay;
  uint32_t edge;         // of the products' tiles
  uint32_t parts;        // X X^T of so many ranges of columns, or 0: in one
};

// Workspace of a matrix, one replica: X twice (an iteration reads one and writes the other), with one plane what the half leaves of it (see dadam_ortho.hip),
// A = X X^T, B = b A + c A A without its diagonal, which lies apart in 32 bits, partial sums of the norm, the ranges' parts of X X^T.
struct OrthoPlaces {
  uint64_t x[2], low, a, b, diagonal, sums, parts, bytes;
};
inline constexpr OrthoPlaces ortho_places(uint64_t P, uint64_t Q, uint64_t planes, uint64_t parts) {
  OrthoPlaces w{};
  uint64_t at = 0;
  w.x[0] = at, at += P * Q * 2 * planes;
  w.x[1] = at, at += P * Q * 2 * planes;
  w.low = at, at += planes == 1 ? P * Q * 2 : 0;
  w.a = at, at += P * P * 2 * planes;
  w.b = at, at += P * P * 2 * planes;
  w.diagonal = at, at += P * 4;  // (P is a multiple of 128)
  w.sums = at, at += ((P / kOrthoCell) * (Q / kOrthoCell) * 8 + 255) / 256 * 256;
  w.parts = at, at += parts * P * P * 4;
  w.bytes = at;
  return w;
}

// What all launches of a group of matrices have in common.
struct OrthoSpan {
  const OrthoTask* tasks;   // device, of all matrices
  const uint32_t* units;    // device: the matrix of every tile, of this launch's kind
  uint64_t workspace, stride;  // of the group's first matrix and replica, and from replica to replica
  uint64_t before;          // OrthoTask::at of the group's first matrix
  uint32_t first_unit;      // tiles before the group
  uint32_t n_xcd;
};

enum OrthoSource : int { kOrthoGiven = 0, kOrthoMoment = 1, kOrthoNesterov = 2 };

template <int N>
struct OrthoBeginArgs {
  OrthoSpan s;
  const void* grad[N];   // by replica of the group
  float* m_hat[N];
  float* acc[N];
  Scalars c;
  float scale;           // power of two that X is held times
  uint32_t source;       // OrthoSource
  uint32_t phase;        // Phase
};

struct OrthoStepArgs {
  OrthoSpan s;
  float gain, fresh;     // what is stored of the term held already, and of the new product
  uint32_t from, to;     // which X is read and written
};

template <int N>
struct OrthoEndArgs {
  OrthoSpan s;
  float gain, fresh;
  uint32_t from;
  uint32_t mix;          // 0: out = the matrix, 1: the step
  void* out[N];          // by replica of the group
  const void* x_src[N];
  const int32_t* row_ptr;  // of the slot (device)
  const int32_t* col;
  const float* w;
  uint32_t first_row;
  float lr;
};

// Matrices that a workgroup holds in LDS (dadam_ortho_lone.hip): their rows and columns are filled up to multiples of kLoneEdge, and no workspace is theirs.
constexpr uint32_t kLoneEdge = 32, kLoneThreads = 512, kMostLoneLds = 160 * 1024 - 256;
constexpr int kLoneRows = 64;
inline constexpr uint64_t lone_lds_bytes(uint64_t P, uint64_t Q) {
  return P > 4 * kLoneEdge ? ~0ull : (P * (Q + 4) + P * (P + 4) + P + (P <= 2 * kLoneEdge ? 8192 : 0)) * 4;
}
// What is stored of a product, and of the term held already.
struct LoneStep {
  float a_fresh, b_gain, b_fresh, x_gain, x_fresh;
};
template <int N, int C>
struct OrthoLoneArgs {
  const OrthoTask* tasks;  // device, the first of them
  uint32_t n_steps, source, phase, mix, first_row;
  float scale, lr;
  Scalars c;
  const int32_t* row_ptr;
  const int32_t* col;
  const float* w;
  LoneStep step[DADAM_ORTHO_MAX_STEPS];
  const void* grad[N];
  float* m_hat[N];
  float* acc[N];
  void* out[N];
  const void* x_src[C];
};
static_assert(sizeof(OrthoLoneArgs<kLoneRows, kMaxRows>) <= 4096, "the argument block of a launch holds 4 KB");

constexpr int kOrthoFew = 16;
static_assert(sizeof(OrthoBeginArgs<kMaxRows>) <= 4096 && sizeof(OrthoEndArgs<kMaxRows>) <= 4096, "the argument block of a launch holds 4 KB");

// Launchers.  units: tiles of the group, replicas: of the group.  planes: 1 or 2 (see dadam_mfma.h); of launch_ortho_end 1 for bfloat16, 2 for float32.
int launch_ortho_norm(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream);
int launch_ortho_begin(int gdt, const OrthoBeginArgs<kMaxRows>& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream);
int launch_ortho_gram(bool square, uint32_t edge, const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream);
// The same of ranges of columns, by small tiles, and their sum: most is the largest OrthoTask::parts.
int launch_ortho_parts(const OrthoStepArgs& a, uint32_t planes, uint32_t most, uint32_t units, uint32_t replicas, void* stream);
int launch_ortho_next(uint32_t edge, const OrthoStepArgs& a, uint32_t planes, uint32_t units, uint32_t replicas, void* stream);
int launch_ortho_end(int dtype, uint32_t edge, const OrthoEndArgs<kMaxRows>& a, uint32_t n_cols, uint32_t units, uint32_t replicas, void* stream);
int launch_ortho_lone(int gdt, int dtype, const OrthoLoneArgs<kLoneRows, kMaxRows>& a, uint32_t n_cols, uint32_t matrices, uint32_t replicas, uint32_t lds, void* stream);

}  // namespace dadam

#endif  // DADAM_ORTHO_H_
