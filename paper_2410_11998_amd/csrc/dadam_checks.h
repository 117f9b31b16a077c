// What the entry points that take their buffers in the call check before they launch (included by the host code only).
#ifndef DADAM_CHECKS_H_
#define DADAM_CHECKS_H_

#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>

#include "dadam_handle.h"

namespace dadam {

// No exception leaves an entry point.
template <typename Fn>
int guarded(dadam_handle* h, Fn fn) {
  try {
    return fn();
  } catch (const std::bad_alloc&) {
    return fail(h, DADAM_EINVAL, "out of host memory");
  }
}

constexpr uint64_t kMostElems = 1ull << 36;  // index and masks count in 32 bits

// One argument of a call: n buffers of `bytes` bytes (of none: they may be null, and lie anywhere).
struct Table {
  const void* const* p;
  uint32_t n;
  size_t bytes;
  const char* name;
  bool written;
  int in_place_of;  // the table whose entry of the same number this one's may be, -1 none
  uint32_t align = 16;
};

struct Range {
  uintptr_t lo, hi;
  int table;
  uint32_t index;
};

constexpr int kMostTables = 8;  // of a call
constexpr uintptr_t kHighest = (uintptr_t)1 << 52;

// Nothing that is written overlaps anything else, but the same entry of the table it may be in place of.
inline int check_overlaps(const dadam_handle* h, const Table* t, int n_tables) {
  Range all[kMostTables * DADAM_MAX_ROWS], open[kMostTables * DADAM_MAX_ROWS];  // open: earlier ranges that reach beyond where the walk is
  uint32_t n = 0, n_open = 0;
  for (int k = 0; k < n_tables; ++k)
    for (uint32_t i = 0; t[k].p && t[k].bytes && i < t[k].n; ++i) all[n++] = {(uintptr_t)t[k].p[i], (uintptr_t)t[k].p[i] + t[k].bytes, k, i};
  std::sort(all, all + n, [](const Range& a, const Range& b) { return a.lo < b.lo; });
  for (uint32_t q = 0; q < n; ++q) {
    const Range& r = all[q];
    n_open = (uint32_t)(std::remove_if(open, open + n_open, [&](const Range& o) { return o.hi <= r.lo; }) - open);
    for (uint32_t k = 0; k < n_open; ++k) {
      const Range& o = open[k];
      if (!t[r.table].written && !t[o.table].written) continue;
      const bool pair = t[r.table].in_place_of == o.table || t[o.table].in_place_of == r.table;
      if (pair && r.lo == o.lo && r.index == o.index) continue;
      return fail(h, DADAM_EALIAS, "%s[%u] overlaps %s[%u]", t[r.table].name, r.index, t[o.table].name, o.index);
    }
    open[n_open++] = r;
  }
  return DADAM_OK;
}

// Every buffer is there, aligned and within reach, and does not overlap what it must not.
inline int check_tables(const dadam_handle* h, const Table* t, int n_tables) {
  if (h->cfg.d > kMostElems) return fail(h, DADAM_EINVAL, "the operators around the step take up to 2^36 elements");
  bool apart = true;  // tables of increasing buffers, one table's behind the other's: nothing overlaps
  uintptr_t lows[kMostTables], highs[kMostTables];
  int n_used = 0;
  for (int k = 0; k < n_tables; ++k) {
    if (!t[k].p || t[k].n == 0 || t[k].bytes == 0) continue;
    uintptr_t end = 0;
    for (uint32_t i = 0; i < t[k].n; ++i) {
      const uintptr_t at = (uintptr_t)t[k].p[i];
      if (!at) return fail(h, DADAM_EINVAL, "%s[%u] is null", t[k].name, i);
      if (at & (t[k].align - 1)) return fail(h, DADAM_EALIGN, "%s[%u] is not %u-byte aligned", t[k].name, i, t[k].align);
      if (at >= kHighest || t[k].bytes > kHighest - at) return fail(h, DADAM_EINVAL, "%s[%u] reaches above address 2^52", t[k].name, i);
      apart &= at >= end;
      end = at + t[k].bytes;
    }
    lows[n_used] = (uintptr_t)t[k].p[0];
    highs[n_used++] = end;
  }
  for (int k = 0; k < n_used; ++k)
    for (int m = 0; m < k; ++m) apart &= highs[k] <= lows[m] || highs[m] <= lows[k];
  return apart ? DADAM_OK : check_overlaps(h, t, n_tables);
}

inline int check_slot(const dadam_handle* h, uint32_t slot) {
  if (slot >= DADAM_MAX_SLOTS) return fail(h, DADAM_EINVAL, "slot %u out of range", slot);
  if (!h->slots[slot].set) return fail(h, DADAM_ESTATE, "slot %u has no topology", slot);
  return DADAM_OK;
}

// Whether work on the stream is being recorded; a stream that cannot be asked counts as one.
inline bool captures(void* stream) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(reinterpret_cast<hipStream_t>(stream), &status) == hipSuccess) return status != hipStreamCaptureStatusNone;
  (void)hipGetLastError();
  return true;
}

}  // namespace dadam

#endif  // DADAM_CHECKS_H_
