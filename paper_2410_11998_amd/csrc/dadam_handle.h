// The handle, and what every entry point does with it (not part of the public C ABI; included by the host code only).
#ifndef DADAM_HANDLE_H_
#define DADAM_HANDLE_H_

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>
#include <utility>
#include <vector>

#include "dadam_internal.h"

namespace dadam {

inline thread_local std::string g_init_error;

struct Slot {
  bool set = false;
  std::vector<int32_t> row_ptr, col;
  std::vector<float> w;
  int32_t max_degree = 0;             // longest row
  uint32_t n_read = 0;                // sources that some row lists
  std::vector<int32_t> order;         // rows ordered so that neighbours share sources (empty: nothing is shared)
  bool reuse = false;                 // some source is read by two or more rows
  // Loops: rows that list the same sources with the same weights.  Filled only where the loop kernel may take the
  // slot (see find_loops).
  std::vector<Loop> loops;
  std::vector<int32_t> loop_of_row, loop_of_source;  // the loop a row is in / that reads a source (-1: none)
  std::vector<int32_t> sole_reader;   // per source: the only row reading it, -1 none, -2 several
  // one device allocation holding everything the kernels read (see StepArgs)
  char* d_lists = nullptr;
  const int32_t *d_row_ptr = nullptr, *d_col = nullptr;                                    // tile kernel
  const float* d_w = nullptr;
  const int32_t *d_row_len = nullptr, *d_list_col = nullptr, *d_row_order = nullptr;        // direct kernel
  const float* d_list_w = nullptr;
  const int32_t *d_loop_col = nullptr, *d_loop_rows = nullptr;                              // loop kernel
  const float* d_loop_w = nullptr;
  const Loop* d_loops = nullptr;
  // What the products with 4-bit messages read: made with the handle's OperatorState, and from then on with the slot.
  std::vector<MixRow> mix_rows;       // see MixRow
  std::vector<MixEntry> mix_entries;
  std::vector<MixRow> mix_firsts;     // the first row of every list
  const MixRow *d_mix_rows = nullptr, *d_mix_firsts = nullptr;
  const MixEntry* d_mix_entries = nullptr;
  char* d_mix = nullptr;              // the allocation of a slot that was set later than the state
};

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev != dev) {
      err = hipSetDevice(dev);
      switched = (err == hipSuccess);
    }
  }
  ~DeviceGuard() {
    if (switched) (void)hipSetDevice(prev);
  }
};

struct OperatorState;

}  // namespace dadam

using namespace dadam;

struct dadam_handle {
  dadam_config cfg{};
  std::vector<dadam_tensor_desc> tensors;
  std::vector<uint32_t> tensor_seg;  // segment of each non-empty tensor, UINT32_MAX for empty ones
  std::vector<Segment> segs;
  std::vector<uint32_t> seg_work[kNumGrids];  // per Grid: number of work items (tiles; per row in direct mode) in earlier segments
  // Layouts of many short tensors side by side: no search and no tile launched twice, but one dense grid over the whole vector and a byte
  // for every four elements that says which are stored and decay (build_map).
  bool mapped = false;
  float map_decay = 0.f;      // of the tensors that decay
  uint8_t* d_map = nullptr;
  Segment* d_segs = nullptr;     // the segments, and behind them
  uint32_t* d_seg_work = nullptr;  // their first work items, per Grid (what the kernels search)
  double* d_partials = nullptr;  // kConsensusPartials doubles of scratch for the consensus error
  // Cleared when the handle is made and by every pass after use; false after a pass that could not be enqueued whole,
  // and the next one clears them itself.  Passes that are recorded into a graph neither rely on it nor change it.
  bool partials_clear = true;
  // Handles with more than kInlineRows rows or sources: device copies of the bound pointer tables, two per
  // binding (as bound, and with x_src / x_dst exchanged), DADAM_BINDINGS_KEPT bindings in a ring.
  BoundTables* d_tables = nullptr;
  uint32_t binding = 0;  // ring position of the current binding
  bool swapped = false;  // dadam_swap_x flips between the binding's two copies
  double* d_static_partials = nullptr;  // the same in the library's device image (dadam_mix_consensus_static)
  uint32_t static_capacity = 0;         // doubles it holds
  TileShape shape{4, 1, false};
  TileShape mix_shape{4, 1, false};  // shape of the mixing-only launch (more bytes in flight per wavefront)
  uint32_t mix_tile_elems = 0, mix_lds_bytes = 0;
  uint64_t n_work_m = 0;
  bool nontemporal = false;  // every launch streams (steps of few rows may all the same, see few_rows_stream)
  bool decays = false;  // some tensor carries weight decay
  // Segments of fewer than 65536 elements on average: lanes are hardly ever spread and most tiles need their segment searched, so
  // streaming launches keep the shapes and orders of contiguous lanes.  (By the share of elements in whole blocks, which takes a long tensor
  // beside many short ones for long, steps of GPT-2 shapes with decay gain nothing and unfused steps lose up to 7 % at 16 rows.)  Fraction of 8 TB/s, contiguous / spread choices, segments of
  // 1100 elements: exp. graph of 16 0.74 / 0.70, of 64 0.68 / 0.66, pairs of 64 0.53 / 0.51.
  bool short_segments = false;
  int vec = 4;
  uint32_t tile_elems = 0, direct_elems = 0, lds_bytes = 0;
  bool tile_possible = false;
  uint64_t n_elems = 0;  // elements of the tensors
  uint64_t n_work_t = 0, n_work_d = 0, n_work_v = 0;
  Slot slots[DADAM_MAX_SLOTS];
  bool bound = false;
  const void* x_src[kMaxRows] = {};
  void* x_dst[kMaxRows] = {};
  float* m_hat[kMaxRows] = {};
  float* v_hat[kMaxRows] = {};
  float* acc[kMaxRows] = {};
  std::vector<int32_t> inplace_cols[kMaxRows];  // every source buffer that x_dst[i] coincides with
  uint32_t lds_limit = 65536;  // LDS one workgroup may use
  uint32_t n_xcds = 8;         // dies consecutive workgroup ids are dealt over
  // Gradient tables that passed check_grads against the current outputs: a caller that cycles a few
  // gradient sets (or issues a step bucket by bucket) is checked once per set, not once per call.
  struct CheckedGrads { uint64_t gen; std::vector<const void*> ptrs; };
  std::vector<CheckedGrads> checked;
  size_t checked_next = 0;
  // Names the set of output buffers: dadam_bind moves on to the next even number, dadam_swap_x flips
  // the lowest bit (two exchanges give back the same tables).
  uint64_t outputs_gen = 0;
  std::vector<std::pair<uintptr_t, uintptr_t>> outputs_sorted[2];  // [lo, hi) of x_dst, m_hat, v_hat, b, by lo
  uint64_t outputs_sorted_gen[2] = {~0ull, ~0ull};
  float lr = 0.f;
  double betav = 0.0;
  mutable std::string err;
  // What the operators around the step keep for this handle (dadam_operators.cpp makes it on their first call), what frees it, and what gives
  // a slot that is set later its lists.
  OperatorState* operators = nullptr;
  void (*free_operators)(OperatorState*) = nullptr;
  int (*add_mix_lists)(dadam_handle*, Slot*) = nullptr;
};

namespace dadam {

inline int fail(const dadam_handle* h, int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  if (h) h->err = buf; else g_init_error = buf;
  return code;
}

inline size_t dtype_bytes(uint32_t dt) { return dt == DADAM_BF16 ? 2 : 4; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The last check before a launch, after every argument has been validated (so that a host-only
// handle reports what is wrong with a call exactly as a device handle would).
inline int check_device(const dadam_handle* h) {
  if (h->cfg.device == DADAM_DEVICE_NONE)
    return fail(h, DADAM_ESTATE, "host-only handle (device = DADAM_DEVICE_NONE) cannot launch");
  return DADAM_OK;
}

}  // namespace dadam

#endif  // DADAM_HANDLE_H_
