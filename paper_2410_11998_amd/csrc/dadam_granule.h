// What the kernels of the operators around the step share: granules of 512 elements (a wavefront's share: lane l holds elements
// 4 l .. 4 l + 3 and 256 + 4 l .. 256 + 4 l + 3, so that every access covers one contiguous run), the padding that cuts them, and
// the addresses of a row's buffers.
#ifndef DADAM_GRANULE_H_
#define DADAM_GRANULE_H_

#include "dadam_device.h"
#include "dadam_operators.h"

namespace dadam {
namespace {

template <typename T>
__device__ __forceinline__ T* global_pointer(uint64_t address) {
  typedef T __attribute__((address_space(1))) * Global;
  return (T*)(Global)address;
}
// Buffer K of a row.
template <typename T, int K>
__device__ __forceinline__ T* buffer(const RowPointers& r) {
  const uint64_t high = (r.high[K / 2] >> (16 * (K % 2))) & 0xFFFFu;
  return global_pointer<T>(((high << 32) | r.low[K]) << 4);
}
__device__ __forceinline__ const uint8_t* buffer(const ColPointer& c) {
  return global_pointer<const uint8_t>((((uint64_t)c.high << 32) | c.low) << 4);
}

__device__ __forceinline__ uint32_t wave_of_group() { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)); }

// 1 + where the masks of a granule stand, 0 if no padding cuts it.
__device__ __forceinline__ uint32_t cut_of(const Cuts& c, uint32_t granule) {
  typedef const uint32_t __attribute__((address_space(4))) * Constant;
  return c.index ? ((Constant)c.index)[granule] : 0u;
}
// Which of the n elements from e on (multiples of n, 4 or 8; inside the vector) belong to a tensor; cut: of their granule.
__device__ __forceinline__ uint32_t stored_bits(const Cuts& c, uint32_t cut, uint32_t e, int n) {
  const uint32_t all = (1u << n) - 1;
  return cut == 0 ? all : (c.masks[cut - 1 + e % kGranule / kMxBlock] >> (e % kMxBlock)) & all;
}

// Where a wavefront's unit of 512 elements (V = 2) or 256 (V = 1) lies: lane l holds V groups of four from a place of its own on, 64 or 256
// elements apart; eight lanes side by side hold a block of 32 elements.  In order: one run.  SPREAD: as streaming kernels have it (see lane_start, V
// vectors a lane), the two halves of the wavefront work 8192 V elements apart, in blocks of twice that many elements that lie inside
// the vector.  A wavefront takes U units at a time, side by side; those behind the vector have no element.
// Places count from `base`, the same for all lanes: addresses are then a scalar and 32 bits a lane.
template <int V, int U>
struct Units {
  uint64_t base;     // a multiple of kGranule, below d
  uint32_t left;     // elements from there to the end of the vector (2^31 - 1: so many or more)
  uint32_t first[U];
  uint32_t step;
  uint32_t cut[U];   // of the granule that the lane's groups of a unit lie in
  bool whole;        // no padding in them
  __device__ __forceinline__ uint32_t at(uint32_t k) const { return first[k / V] + k % V * step; }  // group k of the lane's U V
  __device__ __forceinline__ Units<V, 1> one(uint32_t u) const { return {base, left, {first[u]}, step, {cut[u]}, whole}; }
  __device__ __forceinline__ uint32_t bits(const Cuts& c, uint32_t k) const { return at(k) < left ? stored_bits(c, cut[k / V], at(k), 4) : 0u; }
};
template <int V>
constexpr uint32_t kUnitElems = 256 * V;
template <int V, bool SPREAD, int U = 1>
__device__ __forceinline__ Units<V, U> units_from(uint32_t i, const Span& s, uint32_t lane) {
  constexpr uint32_t kFar = 8192 * V, kUnits = 2 * kFar / kUnitElems<V>;
  static_assert(kUnits % U == 0, "units side by side lie in one block");
  const uint64_t block = (uint64_t)(i & ~(kUnits - 1)) * kUnitElems<V>;
  const bool spread = SPREAD && block + 2 * kFar <= s.d;
  Units<V, U> units;
  units.base = spread ? block : (uint64_t)i * kUnitElems<V> / kGranule * kGranule;
  units.left = s.d - units.base < 0x7FFFFFFFu ? (uint32_t)(s.d - units.base) : 0x7FFFFFFFu;
  units.step = spread ? 64 : 256;
  units.whole = true;
  const uint32_t granule = (uint32_t)(units.base / kGranule);
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    if (spread) {
      const uint32_t at = (i % kUnits + u) * (kUnitElems<V> / 2);
      units.first[u] = at + (V == 2 ? 4 * (lane & 15) + 8 * (lane & 16) : 4 * (lane & 31)) + (lane >> 5) * kFar;
      const uint32_t near = cut_of(s.cuts, granule + at / kGranule), far = cut_of(s.cuts, granule + (at + kFar) / kGranule);
      units.whole &= (near | far) == 0;
      units.cut[u] = lane >> 5 ? far : near;
    } else {
      const uint32_t at = (uint32_t)((uint64_t)i * kUnitElems<V> - units.base) + u * kUnitElems<V>;
      units.first[u] = at + 4 * lane;
      units.cut[u] = at < units.left ? cut_of(s.cuts, granule + at / kGranule) : 0u;
      units.whole &= at < units.left && units.cut[u] == 0;
    }
  }
  return units;
}
// Where the elements of a buffer begin that units count from.
template <typename T>
__device__ __forceinline__ const void* based(const void* buffer, uint64_t base) { return static_cast<const char*>(buffer) + base * T::bytes; }
template <typename T>
__device__ __forceinline__ void* based(void* buffer, uint64_t base) { return static_cast<char*>(buffer) + base * T::bytes; }

// A lane's group of four elements at e (a multiple of 4), widened to float.  Elements that `bits` leaves out read as zero: whole groups
// are loaded wherever they end within the buffer (`left` elements), so that no load waits for the masks.
template <typename T, bool WHOLE, bool NT>
__device__ __forceinline__ void load_group(const void* base, uint32_t e, uint32_t bits, uint32_t left, float (&v)[4]) {
  if (WHOLE || e + 4 <= left) {
    if constexpr (T::bytes == 4) {
      const f4 x = vload<NT>(reinterpret_cast<const f4*>(at<float>(base, e)));
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
      const u2 x = vload<NT>(reinterpret_cast<const u2*>(at<uint16_t>(base, e)));
      v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xFFFF0000u);
      v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) v[j] = bits >> j & 1 ? load_elem<T>(at<typename T::elem>(base, e), j) : 0.0f;
  }
  if constexpr (!WHOLE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = bits >> j & 1 ? v[j] : 0.0f;
  }
}

template <typename T, bool NT>
__device__ __forceinline__ void store_group(void* base, uint32_t e, uint32_t bits, const float (&v)[4]) {
  if (bits == 0xFu) {
    if constexpr (T::bytes == 4) {
      const f4 x = {v[0], v[1], v[2], v[3]};
      vstore<NT>(reinterpret_cast<f4*>(at<float>(base, e)), x);
    } else {
      const u2 x = {f32_to_bf16_bits(v[0]) | (f32_to_bf16_bits(v[1]) << 16), f32_to_bf16_bits(v[2]) | (f32_to_bf16_bits(v[3]) << 16)};
      vstore<NT>(reinterpret_cast<u2*>(at<uint16_t>(base, e)), x);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (bits >> j & 1) store_elem<T>(at<typename T::elem>(base, e), j, v[j]);
  }
}

}  // namespace

// The part of a large argument block that a launch of at most kFewOperands rows (and sources) needs.
template <typename Few, typename All>
Few few_rows(const All& a) {
  Few f;
  memcpy((void*)f.row, (const void*)a.row, sizeof(f.row));
  return f;
}

// The status of the launch itself; the runtime's copy of a failure is taken away (the call that reports it is this one).
inline int enqueue_grid(KernelFn fn, uint32_t grid, uint32_t block, void* args, uint32_t lds, void* stream) {
  if (grid == 0) return (int)hipSuccess;
  void* list[] = {args};
  const hipError_t e = hipLaunchKernel(fn, dim3(grid), dim3(block), list, lds, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) (void)hipGetLastError();
  return (int)e;
}

inline constexpr uint32_t kMostThreads = 0xFFFFFFFFu;  // of one launch

// Runs `launch` over granules [first, first + count) in pieces whose grid stays below 2^32 threads, `per` granules and `threads` a
// workgroup, `groups` workgroups for each.
template <typename Args, typename Launch>
int in_pieces(Args& a, uint32_t per, uint32_t groups, uint32_t threads, Launch launch) {
  const uint32_t most = kMostThreads / threads / groups;
  uint64_t left = a.s.count;
  int e = (int)hipSuccess;
  while (left > 0 && e == (int)hipSuccess) {
    const uint64_t works = (left + per - 1) / per;
    const uint32_t now = works < most ? (uint32_t)works : most;
    a.s.count = (uint32_t)((uint64_t)now * per < left ? (uint64_t)now * per : left);  // kernels number the pieces of their launch
    e = launch(now * groups);
    a.s.first += a.s.count;
    left -= a.s.count;
  }
  return e;
}

}  // namespace dadam

#endif  // DADAM_GRANULE_H_
