// The lists of 4-bit messages on a modelled HIP runtime (memory is the host's) with modelled launchers, under AddressSanitizer and
// UndefinedBehaviorSanitizer (tests/test_operators_calls.py builds it): random matrices whose rows share lists or do not, set before a handle's
// first call and behind it, over and over.  What a launch is given is checked against the matrix: every row is formed once, with its entries and
// weights, or copied from a row of the same list that was formed before; rows of one list follow each other; sums fall into parts as
// they should; entries are filled up inside the allocation.  Prints "launches N bad <number of mismatches>".
#include "dadam.h"
#include "dadam_operators.h"
#include <hip/hip_runtime_api.h>
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <utility>
#include <vector>

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t a, int) {
  *v = a == hipDeviceAttributeNumberOfXccs ? 8 : 160 * 1024;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t n) { *p = malloc(n); memset(*p, 0xA5, n); return hipSuccess; }
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { memcpy(d, s, n); return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "modelled"; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
}

typedef std::vector<std::pair<int32_t, float>> List;
static long bad = 0, launches = 0;
static std::vector<List> rows_of;       // the matrix of the call at hand, entries as listed
static std::vector<int> formed;         // by row: -1 not yet, else its group
static uint32_t lds_limit;
static List sorted(List l) { std::sort(l.begin(), l.end()); return l; }
static std::vector<List> in_order;      // the same by source
static std::vector<char> together;      // whether another row has the same list
static void use(const std::vector<List>& matrix) {
  rows_of = in_order = matrix;
  for (List& l : in_order) l = sorted(l);
  together.assign(matrix.size(), 0);
  for (size_t i = 0; i < matrix.size(); ++i)
    for (size_t k = 0; k < i; ++k)
      if (in_order[i] == in_order[k]) together[i] = together[k] = 1;
}
constexpr uint64_t kBase = 1ull << 33, kStep = 1ull << 30;
static uint32_t row_of(const dadam::RowPointers& r, int k) {
  return (uint32_t)((((((uint64_t)((r.high[k / 2] >> (16 * (k % 2))) & 0xFFFF) << 32) | r.low[k]) << 4) - kBase) / kStep % DADAM_MAX_ROWS);
}

namespace dadam {
static double sums[kConsensusPartials];
int launch_tile(int, int, Phase, TileShape, const StepArgs&, uint32_t, uint32_t, void*) { return 0; }
int launch_direct(int, int, Phase, bool, bool, bool, const StepArgs&, uint32_t, void*) { return 0; }
int launch_accumulate(int, Phase, bool, bool, const StepArgs&, uint32_t, void*, int) { return 0; }
int launch_consensus_zero(double*, void*) { return 0; }
int launch_consensus_sum(double*, double*, void*) { return 0; }
int static_partials(double** out, uint32_t* capacity) { *out = sums; *capacity = kConsensusPartials; return 0; }
int vec_elems(int xdt) { return xdt == DADAM_BF16 ? 8 : 4; }
bool tile_shape_supported(TileShape s) { return s.waves <= 16 && s.ut <= 2; }
int launch_norm(int, const NormArgs<kMaxRows>&, void*) { return 0; }
int launch_clip(int, const NormArgs<kMaxRows>&, void*) { return 0; }
int launch_clip_small(int, const NormArgs<kMaxRows>&, void*) { return 0; }
int launch_encode(int, const EncodeArgs<kMaxRows>&, void*) { return 0; }

// One row's list as the kernels read it.
static void check_list(const MixRow& r, const MixEntry* entries) {
  const List& want = rows_of[(uint32_t)r.row];
  const bool parts = together[(size_t)r.row];
  if (r.first_entry % kMixAtOnce || r.part % kMixAtOnce || r.part <= 0 || r.n_entries != (int32_t)want.size()) { ++bad; return; }
  const int32_t up = (r.n_entries + kMixAtOnce - 1) / kMixAtOnce * kMixAtOnce;
  if (parts ? kMixParts * r.part < r.n_entries : r.part < r.n_entries) ++bad;
  List got;
  for (int32_t k = 0; k < up; ++k) {  // all of them are loaded
    const MixEntry& e = entries[r.first_entry + k];
    if (k < r.n_entries) got.push_back({e.col, e.w});
    else if (e.w != 0.f || e.col < 0) ++bad;
  }
  if (got != (parts ? in_order[(size_t)r.row] : want)) ++bad;
}
int launch_mix4(int, MixMode mode, uint32_t, const MixArgs<kMessageRows, kMaxRows>& a, void*) {
  ++launches;
  if (a.s.n_rows == 0 || a.s.n_rows > (uint32_t)kMessageRows) ++bad;
  if (a.work == kMixByGroup && (a.rows_each == 0 || lds_limit < kSharedBytes)) ++bad;
  if (a.work == kMixCopy && mode != kMixStore) ++bad;
  int last = -1;
  std::vector<char> done(DADAM_MAX_ROWS, 0);
  for (uint32_t p = 0; p < a.s.n_rows; ++p) {
    const uint32_t row = row_of(a.row[p], 0);
    if (row >= rows_of.size() || formed[row] != -1) { ++bad; continue; }
    if (a.work == kMixCopy) {
      const uint32_t of = row_of(a.row[p], 1);
      if (of >= rows_of.size() || formed[of] < 0 || in_order[of] != in_order[row]) ++bad;
      formed[row] = -2;
      continue;
    }
    const MixRow& r = a.lists.rows[p];
    if ((uint32_t)r.row != row) { ++bad; continue; }
    if (r.group != last && done[(size_t)r.group]) ++bad;  // a run of its own
    done[(size_t)(last = r.group)] = 1;
    formed[row] = r.group;
    check_list(r, a.lists.entries);
  }
  return 0;
}
int launch_round(int, const RoundArgs<kMaxRows>& a, void*) {
  ++launches;
  const RoundShape shape = round_shape(a.s.n_rows, a.s.streams != kStreamsNot);
  if (a.s.n_rows != rows_of.size() || round_bytes(shape, a.n_groups) > lds_limit) ++bad;
  for (uint32_t p = 0; p < a.s.n_rows; ++p) {
    const MixRow& r = a.lists.rows[p];
    const uint32_t row = row_of(a.row[p], 0);
    if ((uint32_t)r.row != row || formed[row] != -1) { ++bad; continue; }
    formed[row] = r.group;
    check_list(r, a.lists.entries);
    if (a.n_groups == 0) continue;
    if ((uint32_t)r.group >= a.n_groups) { ++bad; continue; }
    const MixRow& f = a.firsts[r.group];
    if (f.group != r.group || f.first_entry != r.first_entry || f.n_entries != r.n_entries || f.part != r.part) ++bad;
  }
  return 0;
}
}  // namespace dadam

int main() {
  std::mt19937_64 rng(11);
  for (int iter = 0; iter < 260; ++iter) {
    const uint32_t R = 1 + rng() % (iter % 3 ? 40 : DADAM_MAX_ROWS), C = iter % 4 ? R : 1 + rng() % DADAM_MAX_ROWS;
    const uint64_t kinds[5] = {100, 5000, 900000, 30000000 / R + 5, 110000000 / R + 5}, d = kinds[rng() % 5];
    const dadam_tensor_desc t = {0, d, 0.f, 0};
    const uint32_t limits[4] = {0, 1024, 8192, 20000};
    dadam_config cfg{};
    cfg.abi_version = DADAM_ABI_VERSION; cfg.n_rows = R; cfg.n_cols = C; cfg.d = d; cfg.n_tensors = 1; cfg.tensors = &t;
    cfg.lr = 1e-3f; cfg.accum_s = 1; cfg.beta_vhat = -1.f; cfg.eps = 1e-8f; cfg.lds_limit_bytes = limits[rng() % 4];
    lds_limit = cfg.lds_limit_bytes ? cfg.lds_limit_bytes : 160 * 1024;
    dadam_handle* h = nullptr;
    if (dadam_init(&cfg, &h) != DADAM_OK) { printf("init: %s\n", dadam_last_error(nullptr)); return 1; }
    std::vector<void*> tables[6];
    for (uint64_t k = 0; k < 6; ++k)
      for (uint64_t i = 0; i < DADAM_MAX_ROWS; ++i) tables[k].push_back((void*)(kBase + (k * DADAM_MAX_ROWS + i) * kStep));
    auto in = [&](int k) { return (const void* const*)tables[k].data(); };
    auto out = [&](int k) { return (void* const*)tables[k].data(); };
    auto f = [&](int k) { return (float* const*)tables[k].data(); };
    std::vector<std::vector<List>> slots(4);
    for (int turn = 0; turn < 8; ++turn) {
      const uint32_t slot = rng() % 4;
      if (slots[slot].empty() || rng() % 2) {
        // a few lists that rows pick from, in orders of their own; one in four lists anew for a row by itself
        const uint32_t n = 1 + rng() % (rng() % 2 ? 4 : R);
        std::vector<List> pool(n);
        for (List& l : pool) {
          std::vector<int32_t> cols(C);
          for (uint32_t c = 0; c < C; ++c) cols[c] = (int32_t)c;
          std::shuffle(cols.begin(), cols.end(), rng);
          const uint32_t len = 1 + rng() % std::min<uint32_t>(C, rng() % 2 ? 5 : 160);
          for (uint32_t k = 0; k < len; ++k) l.push_back({cols[k], 1.f / (float)len});
        }
        std::vector<List> matrix(R);
        std::vector<int32_t> ptr(1, 0), col;
        std::vector<float> w;
        for (List& l : matrix) {
          l = pool[rng() % n];
          std::shuffle(l.begin(), l.end(), rng);
          for (const auto& e : l) { col.push_back(e.first); w.push_back(e.second); }
          ptr.push_back((int32_t)col.size());
        }
        if (dadam_set_topology(h, slot, ptr.data(), col.data(), w.data(), nullptr) != DADAM_OK) { printf("topology: %s\n", dadam_last_error(h)); return 1; }
        slots[slot] = matrix;
      }
      use(slots[slot]);
      for (int call = 0; call < (R == C ? 4 : 3); ++call) {
        formed.assign(R, -1);
        int rc;
        if (call < 2) rc = dadam_mx4_product(h, slot, in(5), f(0), call ? DADAM_MX4_ADD : 0, nullptr);
        else if (call == 2) rc = dadam_mx4_gossip(h, slot, in(5), f(0), f(1), in(2), out(3), 0.5f, nullptr);
        else rc = dadam_mx4_round(h, slot, in(0), out(1), f(2), f(3), 0.5f, nullptr);
        if (call == 3 && rc == DADAM_EINVAL && dadam::round_bytes(dadam::round_shape(R, d * R * 24.0 > 512.0 * 1024 * 1024), 0) > lds_limit) continue;
        if (rc) { ++bad; printf("refused: %s\n", dadam_last_error(h)); continue; }
        for (uint32_t i = 0; i < R; ++i) bad += formed[i] == -1;
      }
    }
    dadam_destroy(h);
  }
  printf("launches %ld bad %ld\n", launches, bad);
  return bad != 0;
}
