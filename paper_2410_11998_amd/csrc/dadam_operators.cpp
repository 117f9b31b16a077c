// Host side of the operators around the step (include/dadam.h, "Around the step"): validation, what a handle keeps for them on
// the device, and launch set-up.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <map>
#include <memory>
#include <new>
#include <vector>

#include "dadam_checks.h"
#include "dadam_handle.h"
#include "dadam_operators.h"

namespace dadam {

struct OperatorState {
  char* memory = nullptr;      // one allocation: partial sums, counters, index and masks, lists of the slots
  double* partials = nullptr;  // per_row partial sums a row
  uint32_t* arrived = nullptr;
  uint32_t per_row = 1;
  Cuts cuts{};
};

namespace {

uint64_t granules_of(const dadam_handle* h) { return (h->cfg.d + kGranule - 1) / kGranule; }

// Index and masks of the layout's granules (see Cuts), the masks behind the granules_of(h) words of the index; empty if all granules are whole.
// A granule is whole if one segment covers it; the others get a word of bits for each of their blocks.  Segments that touch (they differ in decay)
// may cover a granule between them: its bits are then all set.
std::vector<uint32_t> build_cuts(const dadam_handle* h) {
  const uint64_t n = granules_of(h);
  std::vector<uint32_t> index, masks;
  auto cut = [&](uint64_t g) -> uint32_t* {
    if (index.empty()) index.assign(n, 0);
    if (index[g] == 0) {
      masks.resize(masks.size() + kGranuleBlocks, 0u);
      index[g] = (uint32_t)(masks.size() - kGranuleBlocks) + 1;
    }
    return masks.data() + index[g] - 1;
  };
  auto part = [&](uint64_t lo, uint64_t hi) {  // of one granule
    if (lo >= hi) return;
    uint32_t* m = cut(lo / kGranule);
    const uint32_t first = (uint32_t)(lo % kGranule), last = first + (uint32_t)(hi - lo) - 1;
    for (uint32_t w = first / kMxBlock; w <= last / kMxBlock; ++w) {
      const uint32_t from = w == first / kMxBlock ? first % kMxBlock : 0, to = w == last / kMxBlock ? last % kMxBlock : kMxBlock - 1;
      m[w] |= (~0u << from) & (~0u >> (kMxBlock - 1 - to));
    }
  };
  uint64_t done = 0;  // granules before this one are whole or have their entry
  for (const Segment& s : h->segs) {
    const uint64_t first = (s.lo + kGranule - 1) / kGranule, last = s.hi / kGranule;  // whole granules [first, last)
    for (; done < s.lo / kGranule; ++done) cut(done);  // nothing but padding, or begun by the segment before
    if (first <= last) {
      part(s.lo, first * kGranule);
      part(last * kGranule, s.hi);
    } else {
      part(s.lo, s.hi);
    }
    done = std::max(done, std::max(first, last));
  }
  for (; done < n; ++done) cut(done);
  if (masks.empty()) return {};
  index.insert(index.end(), masks.begin(), masks.end());
  return index;
}

// Rows and entries as the products with 4-bit messages take them (see MixRow), in order of the first row of each group.
void find_mix_rows(uint32_t R, Slot& s) {
  s.mix_rows.clear();
  s.mix_firsts.clear();
  s.mix_entries.clear();
  std::map<std::vector<std::pair<int32_t, float>>, std::vector<int32_t>> by_list;
  std::vector<std::vector<std::pair<int32_t, float>>> sorted(R);
  for (uint32_t i = 0; i < R; ++i) {
    for (int32_t k = s.row_ptr[i]; k < s.row_ptr[i + 1]; ++k) sorted[i].push_back({s.col[k], s.w[k]});
    std::sort(sorted[i].begin(), sorted[i].end());
    by_list[sorted[i]].push_back((int32_t)i);
  }
  for (uint32_t i = 0; i < R; ++i) {
    const std::vector<int32_t>& rows = by_list[sorted[i]];
    if (rows.front() != (int32_t)i) continue;
    const int32_t first = (int32_t)s.mix_entries.size();
    if (rows.size() > 1) {
      for (const auto& e : sorted[i]) s.mix_entries.push_back({e.first, e.second});
    } else {
      for (int32_t k = s.row_ptr[i]; k < s.row_ptr[i + 1]; ++k) s.mix_entries.push_back({s.col[k], s.w[k]});
    }
    const int32_t n = (int32_t)s.mix_entries.size() - first;
    while (s.mix_entries.size() % kMixAtOnce) s.mix_entries.push_back({s.mix_entries.back().col, 0.f});
    const int32_t all = (int32_t)s.mix_entries.size() - first, step = kMixAtOnce * (rows.size() > 1 ? kMixParts : 1);
    const int32_t part = rows.size() > 1 ? (all + step - 1) / step * kMixAtOnce : all;
    const int16_t group = (int16_t)s.mix_firsts.size();
    for (int32_t row : rows) s.mix_rows.push_back({(int16_t)row, group, first, n, part});
    s.mix_firsts.push_back({(int16_t)i, group, first, n, part});
  }
}

// A slot's rows and entries in an image of device memory.
struct ListPlaces {
  size_t rows, firsts, entries;
};
ListPlaces add_lists(const Slot& s, std::vector<char>* image) {
  auto add = [image](const auto& v) {
    const size_t at = (image->size() + 15) / 16 * 16;
    image->resize(at + v.size() * sizeof(v[0]));
    memcpy(image->data() + at, v.data(), v.size() * sizeof(v[0]));
    return at;
  };
  return {add(s.mix_rows), add(s.mix_firsts), add(s.mix_entries)};
}
void point_lists(Slot* s, const char* memory, const ListPlaces& at) {
  s->d_mix_rows = reinterpret_cast<const MixRow*>(memory + at.rows);
  s->d_mix_firsts = reinterpret_cast<const MixRow*>(memory + at.firsts);
  s->d_mix_entries = reinterpret_cast<const MixEntry*>(memory + at.entries);
}

// Lists of a slot that is set on a handle with state, with the handle's device current.
int add_mix_lists(dadam_handle* h, Slot* s) {
  return guarded(h, [&] {
    find_mix_rows(h->cfg.n_rows, *s);
    std::vector<char> image;
    const ListPlaces at = add_lists(*s, &image);
    hipError_t e = hipMalloc((void**)&s->d_mix, image.size());
    if (e == hipSuccess) e = hipMemcpy(s->d_mix, image.data(), image.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return fail(h, DADAM_EHIP, "uploading the neighbour list failed: %s", hipGetErrorString(e));
    }
    point_lists(s, s->d_mix, at);
    return DADAM_OK;
  });
}

void free_state(OperatorState* s) {
  if (!s) return;
  if (s->memory) (void)hipFree(s->memory);
  delete s;
}

int make_state(dadam_handle* h) {
  std::unique_ptr<OperatorState, void (*)(OperatorState*)> s(new OperatorState(), free_state);
  const std::vector<uint32_t> cuts = build_cuts(h);
  // Workgroups of the norm, sixteen wavefronts each, for all rows together: one a compute unit, four granules a wavefront and more, so that few
  // have to report.  us, 256 / 512 workgroups: 1e8 float32 elements 64.7 / 64.3, 9 rows of 3.9e6 bfloat16 18.3 / 20.4, 87 of 5.8e5 22.6 / 25.3; two / four / eight
  // granules: 4e6 elements 10.1 / 8.0 / 8.7, 3 rows of 707 small tensors 8.3 / 8.0 / 10.2.  (1024 workgroups of four wavefronts: the first 73, the second 23.)
  s->per_row = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((granules_of(h) + 4 * kNormWaves - 1) / (4 * kNormWaves), 256 / h->cfg.n_rows));
  const size_t sums = (size_t)s->per_row * h->cfg.n_rows * sizeof(double), head = sums + DADAM_MAX_ROWS * sizeof(uint32_t);
  std::vector<char> image(head + cuts.size() * sizeof(uint32_t), 0);
  if (!cuts.empty()) memcpy(image.data() + head, cuts.data(), cuts.size() * sizeof(uint32_t));
  ListPlaces places[DADAM_MAX_SLOTS];
  for (uint32_t k = 0; k < DADAM_MAX_SLOTS; ++k) {
    if (!h->slots[k].set) continue;
    find_mix_rows(h->cfg.n_rows, h->slots[k]);
    places[k] = add_lists(h->slots[k], &image);
  }
  hipError_t e = hipMalloc((void**)&s->memory, image.size());
  if (e == hipSuccess) e = hipMemcpy(s->memory, image.data(), image.size(), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return fail(h, DADAM_EHIP, "setting up the operators around the step failed: %s", hipGetErrorString(e));
  }
  s->partials = reinterpret_cast<double*>(s->memory);
  s->arrived = reinterpret_cast<uint32_t*>(s->memory + sums);
  if (!cuts.empty()) {
    s->cuts.index = reinterpret_cast<uint32_t*>(s->memory + head);
    s->cuts.masks = s->cuts.index + granules_of(h);
  }
  for (uint32_t k = 0; k < DADAM_MAX_SLOTS; ++k)
    if (h->slots[k].set) point_lists(&h->slots[k], s->memory, places[k]);
  h->operators = s.release();
  h->free_operators = free_state;
  h->add_mix_lists = add_mix_lists;
  return DADAM_OK;
}

int check_norms(const dadam_handle* h, const float* norms) {
  if (!norms) return fail(h, DADAM_EINVAL, "norms is null");
  if ((uintptr_t)norms & 3u) return fail(h, DADAM_EALIGN, "norms is not 4-byte aligned");
  return DADAM_OK;
}

int check_gamma(const dadam_handle* h, float gamma) {
  if (!(gamma > 0.f && gamma <= 1.f)) return fail(h, DADAM_EINVAL, "gamma must be in (0, 1]");
  return DADAM_OK;
}

// A pointer as the kernels take it (see RowPointers).
void put(RowPointers* r, int k, const void* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p >> 4;
  r->low[k] = (uint32_t)v;
  r->high[k / 2] |= (uint32_t)(v >> 32) << (16 * (k % 2));
}
void put(ColPointer* c, const void* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p >> 4;
  c->low = (uint32_t)v;
  c->high = (uint32_t)(v >> 32);
}

bool lines_are_whole(const Table* t, int n_tables) {
  uintptr_t bits = 0;
  for (int k = 0; k < n_tables; ++k)
    for (uint32_t i = 0; t[k].p && i < t[k].n; ++i) bits |= (uintptr_t)t[k].p[i];
  return bits % 128 == 0;
}

// whole: all buffers that are streamed begin on a line, or cut lines do not matter (see Streams).
void fill_span(const dadam_handle* h, bool whole, Span* s) {
  s->cuts = h->operators->cuts;
  s->d = h->cfg.d;
  s->n_granules = (uint32_t)granules_of(h);
  s->first = 0;
  s->count = s->n_granules;
  s->n_rows = h->cfg.n_rows;
  s->n_xcd = h->n_xcds;
  s->streams = !h->nontemporal ? kStreamsNot : whole ? kStreamsHinted : kStreamsApart;
  s->run = s->streams ? kDieRunPieces : 1;
}

uint64_t blocks_of(const dadam_handle* h) { return (h->cfg.d + kMxBlock - 1) / kMxBlock; }
size_t message_bytes(const dadam_handle* h) { return (size_t)((blocks_of(h) * 17 + 15) / 16 * 16); }

// Who takes what of a launch of n_rows positions (MixArgs::work, rows_each).  Lists that fewer than four rows share on average: a wavefront
// for every unit and row.  Otherwise products of 1536 granules and more: a wavefront takes a unit of all rows and forms the sum once; all
// others: a workgroup does, its wavefronts share the list and the rows, and rows are split until there are 4096 workgroups.
// us, by workgroup / by wavefront, complete graph, product of 100 rows of 4e6 elements 456 / 370, of 1e6 137 / 119, of 4e5 55 / 78, of 32 rows of 4e6 147 / 111,
// of 2e6 48 / 53, of 4e5 15.5 / 22, of 8 rows of 2e6 18 / 13.5; gossip of 100 rows of 2e6 777 / 845, of 32 rows of 2e6 237 / 259, of 8 rows of 1e6 33 / 35.5.
// Handles whose workgroups may not use the 8 KB that a shared sum takes go by wavefronts.
constexpr uint64_t kProductGranules = 1536, kSharedGroups = 4096;
bool shares_rows(const dadam_handle* h, const Slot& s) { return h->cfg.n_rows >= 4 * s.mix_firsts.size(); }
void share_rows(const dadam_handle* h, const Slot& s, MixMode mode, uint32_t n_rows, uint32_t* work, uint32_t* rows_each) {
  const uint64_t granules = granules_of(h);
  *work = kMixByRow;
  *rows_each = 1;
  if (!shares_rows(h, s)) return;
  const bool room = h->lds_limit >= kSharedBytes;
  if (mode != kMixGossip && (granules >= kProductGranules || !room)) {
    *work = kMixAllRows;
    return;
  }
  if (!room) return;
  const uint64_t parts = (kSharedGroups + granules - 1) / granules;
  *work = kMixByGroup;
  *rows_each = std::min((uint32_t)((n_rows + parts - 1) / parts + kMixParts - 1) / kMixParts * kMixParts, n_rows);
}

// Rounds whose wavefronts form shared sums together: up to kRoundGroups lists (their parts lie in LDS) of kRoundEntries entries and more on average.
// Where the parts do not fit beside the messages every wavefront forms its own, the same bits.
constexpr size_t kRoundGroups = 4, kRoundEntries = 12;
uint32_t round_groups(const dadam_handle* h, const Slot& s) {
  const size_t n = s.mix_firsts.size();
  const bool shares = shares_rows(h, s) && n <= kRoundGroups && s.mix_entries.size() >= kRoundEntries * n;
  return shares && round_bytes(round_shape(h->cfg.n_rows, h->nontemporal), (uint32_t)n) <= h->lds_limit ? (uint32_t)n : 0;
}

// Products of 1e8 elements in all rows whose rows share sums: one row of every list is formed, and the others are copied from it, a die taking
// a run of 256 pieces of one row after the other, with what it copies in its L2.  (A wavefront that writes all rows has as many places of
// memory in use at a time as there are wavefronts on the chip.)  us, a wavefront for all rows / copies, complete graph: 32 rows of 2.6e7 951 / 731, 12 of 3e7 349 /
// 309, 100 of 4e6 373 / 330, of 1e6 129 / 110; 8 rows of 8e6 45 / 59.  Runs of 32 / 128 / 1024 pieces: the first 802 / 759 / 1050.
bool copies_rows(const dadam_handle* h, const Slot& s, MixMode mode) {
  return mode == kMixStore && h->cfg.d * h->cfg.n_rows >= kManyElems && shares_rows(h, s) && granules_of(h) >= kProductGranules;
}

// Runs the launches of a call whose arguments have passed, with the handle's device current and its state made.  (Allocating it would end a
// capture of the caller's.)
template <typename Launch>
int on_device(dadam_handle* h, void* stream, Launch launch) {
  DeviceGuard guard(h->cfg.device);
  if (guard.err != hipSuccess) return fail(h, DADAM_EHIP, "hipSetDevice: %s", hipGetErrorString(guard.err));
  if (!h->operators) {
    if (captures(stream))
      return fail(h, DADAM_ESTATE, "the first call of an operator around the step on a handle allocates: make one before the stream is captured");
    const int rc = make_state(h);
    if (rc) return rc;
  }
  const int e = launch();
  if (e != (int)hipSuccess) return fail(h, DADAM_EHIP, "kernel launch failed: %s", hipGetErrorString((hipError_t)e));
  return DADAM_OK;
}

int norm_impl(dadam_handle* h, const void* const* grads, void* const* out, float max_norm, float* norms, void* stream) {
  const uint32_t R = h->cfg.n_rows;
  const size_t gb = (size_t)h->cfg.d * dtype_bytes(h->cfg.grad_dtype);
  const Table tables[2] = {{grads, R, gb, "grads", false, -1}, {out, out ? R : 0, gb, "out", true, 0}};
  int rc = check_norms(h, norms);
  if (!rc) rc = check_tables(h, tables, 2);
  if (!rc && out)  // the norms lie outside the table's checks: they need not be 16-byte aligned
    for (uint32_t i = 0; i < R && !rc; ++i)
      if ((uintptr_t)norms < (uintptr_t)out[i] + gb && (uintptr_t)out[i] < (uintptr_t)(norms + R)) rc = fail(h, DADAM_EALIAS, "norms overlaps out[%u]", i);
  for (uint32_t i = 0; i < R && !rc; ++i)
    if ((uintptr_t)norms < (uintptr_t)grads[i] + gb && (uintptr_t)grads[i] < (uintptr_t)(norms + R)) rc = fail(h, DADAM_EALIAS, "norms overlaps grads[%u]", i);
  if (!rc) rc = check_device(h);
  if (rc) return rc;
  return on_device(h, stream, [&] {
    NormArgs<kMaxRows> a;
    memset((void*)&a, 0, sizeof(a));
    for (uint32_t i = 0; i < R; ++i) {
      put(&a.row[i], 0, grads[i]);
      if (out) put(&a.row[i], 1, out[i]);
    }
    fill_span(h, true, &a.s);
    a.partials = h->operators->partials;
    a.arrived = h->operators->arrived;
    a.per_row = h->operators->per_row;
    a.norms = norms;
    a.max_norm = max_norm;
    if (out && a.s.n_granules <= kSmallGranules) return launch_clip_small((int)h->cfg.grad_dtype, a, stream);
    int e = launch_norm((int)h->cfg.grad_dtype, a, stream);
    if (e == (int)hipSuccess && out) e = launch_clip((int)h->cfg.grad_dtype, a, stream);
    return e;
  });
}

int mix_impl(dadam_handle* h, uint32_t slot, const void* const* msg, float* const* sum, MixMode mode, const float* const* copy,
             const void* const* x_src, void* const* x_dst, float gamma, void* stream) {
  const uint32_t R = h->cfg.n_rows, C = h->cfg.n_cols;
  const size_t sb = (size_t)h->cfg.d * 4, xb = (size_t)h->cfg.d * dtype_bytes(h->cfg.param_dtype);
  int rc = check_slot(h, slot);
  const Table tables[5] = {{msg, C, message_bytes(h), "msg", false, -1},
                           {(const void* const*)sum, R, sb, mode == kMixGossip ? "sum" : "out", true, -1},
                           {(const void* const*)copy, R, sb, "copy", false, -1},
                           {x_src, R, xb, "x_src", false, -1},
                           {x_dst, R, xb, "x_dst", true, 3}};
  if (!rc) rc = check_tables(h, tables, mode == kMixGossip ? 5 : 2);
  if (!rc) rc = check_device(h);
  if (rc) return rc;
  return on_device(h, stream, [&] {
    const Slot& lists = h->slots[slot];
    const bool copies = copies_rows(h, lists, mode);
    std::vector<std::pair<int32_t, int32_t>> pairs;  // (copy, of), before anything is launched: host memory may run out
    if (copies)
      for (const MixRow& r : lists.mix_rows)
        if (r.row != lists.mix_firsts[r.group].row) pairs.push_back({r.row, lists.mix_firsts[r.group].row});
    // Positions [0, count) of `rows` in as few launches as the argument block allows, of about the same number each.
    MixArgs<kMessageRows, kMaxRows> a;
    memset((void*)&a, 0, sizeof(a));
    fill_span(h, (mode != kMixGossip && !(mode == kMixAdd && shares_rows(h, lists))) || lines_are_whole(tables + 1, mode == kMixGossip ? 4 : 1), &a.s);
    for (uint32_t c = 0; c < C; ++c) put(&a.message[c], msg[c]);
    a.scale_offset = 16 * blocks_of(h);
    a.gamma = gamma;
    auto in_launches = [&](uint32_t count, auto fill) {
      const uint32_t launches = (count + kMessageRows - 1) / kMessageRows, each = launches ? (count + launches - 1) / launches : 0;
      int e = (int)hipSuccess;
      for (uint32_t p0 = 0; p0 < count && e == (int)hipSuccess; p0 += each) {
        memset((void*)a.row, 0, sizeof(a.row));
        a.s.n_rows = std::min(each, count - p0);
        for (uint32_t p = 0; p < a.s.n_rows; ++p) fill(&a.row[p], p0 + p);
        fill(nullptr, p0);
        e = launch_mix4((int)h->cfg.param_dtype, mode, C, a, stream);
      }
      return e;
    };
    const std::vector<MixRow>& rows = copies ? lists.mix_firsts : lists.mix_rows;
    int e = in_launches((uint32_t)rows.size(), [&](RowPointers* r, uint32_t p) {
      if (!r) {
        a.lists = {(copies ? lists.d_mix_firsts : lists.d_mix_rows) + p, lists.d_mix_entries};
        a.work = kMixByRow;
        if (!copies) share_rows(h, lists, mode, a.s.n_rows, &a.work, &a.rows_each);
        return;
      }
      const int32_t i = rows[p].row;
      put(r, 0, sum[i]);
      if (mode != kMixGossip) return;
      put(r, 1, copy[i]);
      put(r, 2, x_src[i]);
      put(r, 3, x_dst[i]);
    });
    if (e != (int)hipSuccess || !copies) return e;
    a.work = kMixCopy;
    return in_launches((uint32_t)pairs.size(), [&](RowPointers* r, uint32_t p) {
      if (!r) return;
      put(r, 0, sum[pairs[p].first]);
      put(r, 1, sum[pairs[p].second]);
    });
  });
}

}  // namespace
}  // namespace dadam

extern "C" {

int dadam_grad_norm(dadam_handle* h, const void* const* grads, float* norms, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!grads) return fail(h, DADAM_EINVAL, "grads is null");
  return guarded(h, [&] { return norm_impl(h, grads, nullptr, 0.f, norms, hip_stream); });
}

int dadam_clip_grads(dadam_handle* h, const void* const* grads, void* const* out, float max_norm, float* norms, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!grads || !out) return fail(h, DADAM_EINVAL, "grads or out is null");
  if (!(max_norm >= 0.f) || !std::isfinite(max_norm)) return fail(h, DADAM_EINVAL, "max_norm must be finite and >= 0");
  return guarded(h, [&] { return norm_impl(h, grads, out, max_norm, norms, hip_stream); });
}

int dadam_mx4_get_info(const dadam_handle* h, dadam_mx4_info* out) {
  if (!h) return DADAM_EINVAL;
  if (!out) return fail(h, DADAM_EINVAL, "out is null");
  out->n_blocks = blocks_of(h);
  out->scale_offset = 16 * out->n_blocks;
  out->bytes = message_bytes(h);
  return DADAM_OK;
}

int dadam_mx4_encode(dadam_handle* h, const void* const* x, const float* const* copy_in, float* const* copy_out, void* const* msg,
                     void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!x || !msg) return fail(h, DADAM_EINVAL, "x or msg is null");
  return guarded(h, [&] {
    const uint32_t R = h->cfg.n_rows;
    const size_t sb = (size_t)h->cfg.d * 4, xb = (size_t)h->cfg.d * dtype_bytes(h->cfg.param_dtype);
    const Table tables[4] = {{x, R, xb, "x", false, -1},
                             {(const void* const*)copy_in, R, sb, "copy_in", false, -1},
                             {(const void* const*)copy_out, R, sb, "copy_out", true, 1},
                             {msg, R, message_bytes(h), "msg", true, -1}};
    int rc = check_tables(h, tables, 4);
    if (!rc) rc = check_device(h);
    if (rc) return rc;
    return on_device(h, hip_stream, [&] {
      EncodeArgs<kMaxRows> a;
      memset((void*)&a, 0, sizeof(a));
      for (uint32_t i = 0; i < R; ++i) {
        put(&a.row[i], 0, x[i]);
        if (copy_in) put(&a.row[i], 1, copy_in[i]);
        if (copy_out) put(&a.row[i], 2, copy_out[i]);
        put(&a.row[i], 3, msg[i]);
      }
      fill_span(h, lines_are_whole(tables, 3), &a.s);
      a.scale_offset = 16 * blocks_of(h);
      return launch_encode((int)h->cfg.param_dtype, a, hip_stream);
    });
  });
}

int dadam_mx4_product(dadam_handle* h, uint32_t slot, const void* const* msg, float* const* out, uint32_t flags, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!msg || !out) return fail(h, DADAM_EINVAL, "msg or out is null");
  if (flags & ~DADAM_MX4_ADD) return fail(h, DADAM_EINVAL, "unknown flags %u", flags);
  return guarded(h, [&] {
    return mix_impl(h, slot, msg, out, flags & DADAM_MX4_ADD ? kMixAdd : kMixStore, nullptr, nullptr, nullptr, 0.f, hip_stream);
  });
}

int dadam_mx4_gossip(dadam_handle* h, uint32_t slot, const void* const* msg, float* const* sum, const float* const* copy,
                     const void* const* x_src, void* const* x_dst, float gamma, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!msg || !sum || !copy || !x_src || !x_dst) return fail(h, DADAM_EINVAL, "null table");
  if (int rc = check_gamma(h, gamma)) return rc;
  return guarded(h, [&] { return mix_impl(h, slot, msg, sum, kMixGossip, copy, x_src, x_dst, gamma, hip_stream); });
}

int dadam_mx4_round(dadam_handle* h, uint32_t slot, const void* const* x_src, void* const* x_dst, float* const* copy, float* const* sum,
                    float gamma, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!x_src || !x_dst || !copy || !sum) return fail(h, DADAM_EINVAL, "null table");
  if (h->cfg.n_rows != h->cfg.n_cols) return fail(h, DADAM_ESTATE, "a round needs every replica in the handle (n_rows == n_cols)");
  if (int rc = check_gamma(h, gamma)) return rc;
  const uint32_t lds = round_bytes(round_shape(h->cfg.n_rows, h->nontemporal), 0);
  if (lds > h->lds_limit)
    return fail(h, DADAM_EINVAL, "the messages of a round take %u bytes of LDS, the handle's limit is %u: use dadam_mx4_encode and dadam_mx4_gossip", lds, h->lds_limit);
  return guarded(h, [&] {
    const uint32_t R = h->cfg.n_rows;
    const size_t sb = (size_t)h->cfg.d * 4, xb = (size_t)h->cfg.d * dtype_bytes(h->cfg.param_dtype);
    int rc = check_slot(h, slot);
    const Table tables[4] = {{x_src, R, xb, "x_src", false, -1},
                             {x_dst, R, xb, "x_dst", true, 0},
                             {(const void* const*)copy, R, sb, "copy", true, -1},
                             {(const void* const*)sum, R, sb, "sum", true, -1}};
    if (!rc) rc = check_tables(h, tables, 4);
    if (!rc) rc = check_device(h);
    if (rc) return rc;
    return on_device(h, hip_stream, [&] {
      RoundArgs<kMaxRows> a;
      memset((void*)&a, 0, sizeof(a));
      const Slot& lists = h->slots[slot];
      for (uint32_t p = 0; p < R; ++p) {
        const int32_t i = lists.mix_rows[p].row;
        put(&a.row[p], 0, x_src[i]);
        put(&a.row[p], 1, x_dst[i]);
        put(&a.row[p], 2, copy[i]);
        put(&a.row[p], 3, sum[i]);
      }
      fill_span(h, lines_are_whole(tables, 4), &a.s);
      a.lists = {lists.d_mix_rows, lists.d_mix_entries};
      a.firsts = lists.d_mix_firsts;
      a.n_groups = round_groups(h, lists);
      a.gamma = gamma;
      return launch_round((int)h->cfg.param_dtype, a, hip_stream);
    });
  });
}

}  // extern "C"
