// What the kernels of orthogonalised updates read and what they make of the state, eight elements at a time (dadam_ortho.hip, dadam_ortho_lone.hip).
#ifndef DADAM_ORTHO_SOURCE_H_
#define DADAM_ORTHO_SOURCE_H_

#include "dadam_mfma.h"
#include "dadam_ortho.h"

namespace dadam {

// Elements of a row of the matrix from column `col` on.
__device__ __forceinline__ uint32_t left(uint32_t cols, uint32_t col) { return col < cols ? cols - col : 0; }

// What is orthogonalised: the gradient, the moment of line 6 of Algorithm 3, or that looked ahead.
template <typename GT>
__device__ __forceinline__ void load_source(const Scalars& c, uint32_t source, uint64_t grad, uint64_t m_hat, uint64_t e, uint32_t n, float (&g)[8], float (&m)[8],
                                            float (&v)[8]) {
  GT::load8(grad, e, n, g);
  if (source != kOrthoGiven) F32::load8(m_hat, e, n, m);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = g[k];
    if (source == kOrthoGiven) continue;
    v[k] = fmaf(c.beta1, m[k], c.omb1 * g[k]);
    if (source == kOrthoNesterov) v[k] = fmaf(c.beta1, v[k], c.omb1 * g[k]);
  }
}

__device__ __forceinline__ double add_squares(const float (&v)[8], double sum) {
#pragma unroll
  for (int k = 0; k < 8; ++k) sum = fma((double)v[k], (double)v[k], sum);
  return sum;
}

// Lines 9 to 13 of Algorithm 3 of the first moment.
__device__ __forceinline__ void move_moment(const Scalars& c, uint32_t phase, uint64_t m_hat, uint64_t acc, uint64_t e, uint32_t n, const float (&g)[8], float (&m)[8]) {
  if (phase == kUpdateOnly) return;
  float b[8] = {};
  if (phase == kPlain || phase == kFold) F32::load8(acc, e, n, b);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    b[k] = phase == kPlain || phase == kFold ? fmaf(g[k], c.inv_s, b[k]) : g[k] * c.inv_s;
    m[k] = fmaf(c.beta1, m[k], c.omb1 * b[k]);
    if (phase == kFold) b[k] = 0.f;
  }
  if (phase == kFold || phase == kAlg1) F32::store8(m_hat, e, n, m);
  if (phase != kAlg1) F32::store8(acc, e, n, b);
}

}  // namespace dadam

#endif  // DADAM_ORTHO_SOURCE_H_
