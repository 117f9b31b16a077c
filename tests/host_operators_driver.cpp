// The host code of the operators around the step on a modelled HIP runtime (memory is the host's) with modelled launchers, under
// AddressSanitizer and UndefinedBehaviorSanitizer (tests/test_operators_host.py builds it): random layouts, what the kernels are
// told about padding against the tensor list, and the addresses they are given.  Prints "bad <number of mismatches>".
#include "dadam.h"
#include "dadam_operators.h"
#include <hip/hip_runtime_api.h>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
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

static long bad = 0, launches = 0;
static std::vector<char> stored;  // of the layout at hand
static uint64_t at_base;          // buffer k of table t of row i lies at base + ((i * 8 + t) << 24)
static uint64_t address_of(uint32_t row, uint32_t table) { return at_base + ((uint64_t)(row * 8 + table) << 24); }

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

static void check_span(const Span& s) {
  ++launches;
  const uint64_t d = stored.size(), n = (d + kGranule - 1) / kGranule;
  if (s.d != d || s.n_granules != n || s.first != 0 || s.count != n) ++bad;
  for (uint64_t g = 0; g < n; ++g) {
    const uint32_t cut = s.cuts.index ? s.cuts.index[g] : 0;
    for (uint32_t b = 0; b < kGranuleBlocks; ++b) {
      uint32_t want = 0;
      for (uint32_t j = 0; j < kMxBlock; ++j) {
        const uint64_t e = g * kGranule + b * kMxBlock + j;
        if (e < d && stored[e]) want |= 1u << j;
      }
      if ((cut ? s.cuts.masks[cut - 1 + b] : ~0u) != want) ++bad;
    }
  }
}
static uint64_t address(const RowPointers& r, int k) {
  return (((uint64_t)((r.high[k / 2] >> (16 * (k % 2))) & 0xFFFF) << 32) | r.low[k]) << 4;
}
static void check_rows(const RowPointers* r, const Span& s, int n_tables, const MixRow* order = nullptr) {
  for (uint32_t i = 0; i < s.n_rows; ++i)
    for (int k = 0; k < n_tables; ++k)
      if (address(r[i], k) != address_of(order ? (uint32_t)order[i].row : i, k)) ++bad;
}
int launch_norm(int, const NormArgs<kMaxRows>& a, void*) {
  check_span(a.s);
  check_rows(a.row, a.s, 1);
  for (uint32_t k = 0; k < a.per_row * a.s.n_rows; ++k) bad += a.partials[k] != 0.0;
  for (uint32_t i = 0; i < a.s.n_rows; ++i) bad += a.arrived[i] != 0;
  return 0;
}
int launch_clip(int, const NormArgs<kMaxRows>& a, void*) { check_span(a.s); check_rows(a.row, a.s, 2); return 0; }
int launch_clip_small(int gdt, const NormArgs<kMaxRows>& a, void* stream) { return launch_norm(gdt, a, stream) | launch_clip(gdt, a, stream); }
int launch_encode(int, const EncodeArgs<kMaxRows>& a, void*) { check_span(a.s); check_rows(a.row, a.s, 4); return 0; }
int launch_mix4(int, MixMode mode, uint32_t n_cols, const MixArgs<kMessageRows, kMaxRows>& a, void*) {
  check_span(a.s);
  check_rows(a.row, a.s, mode == kMixGossip ? 4 : 1, a.lists.rows);
  for (uint32_t c = 0; c < n_cols; ++c)
    if ((((uint64_t)a.message[c].high << 32) | a.message[c].low) << 4 != address_of(c, 5)) ++bad;
  return 0;
}
int launch_round(int, const RoundArgs<kMaxRows>& a, void*) { check_span(a.s); check_rows(a.row, a.s, 4, a.lists.rows); return 0; }
}  // namespace dadam

int main() {
  std::mt19937_64 rng(7);
  for (int iter = 0; iter < 400; ++iter) {
    const uint32_t R = 1 + rng() % (iter % 3 ? 8 : DADAM_MAX_ROWS), n = 1 + rng() % 30;
    std::vector<dadam_tensor_desc> ts(n);
    uint64_t at = iter % 4 == 0 ? rng() % 3000 : 0;
    for (auto& t : ts) {
      at += iter % 5 == 0 ? 0 : rng() % 4 == 0 ? rng() % 3000 : rng() % 9;
      const uint64_t kinds[6] = {0, 1, 512, rng() % 40, rng() % 1500, rng() % 20000};
      t = {at, kinds[rng() % 6], rng() % 4 == 0 ? 0.01f : 0.f, 0};
      at += t.numel;
    }
    const uint64_t d = at + (iter % 2 ? rng() % 1200 : 0) + (at == 0 ? 1 : 0);
    stored.assign(d, 0);
    for (auto& t : ts) memset(stored.data() + t.offset_elems, 1, t.numel);
    dadam_config cfg{};
    cfg.abi_version = DADAM_ABI_VERSION; cfg.n_rows = cfg.n_cols = R; cfg.d = d; cfg.n_tensors = n; cfg.tensors = ts.data();
    cfg.lr = 1e-3f; cfg.accum_s = 1; cfg.beta_vhat = -1.f; cfg.eps = 1e-8f;
    dadam_handle* h = nullptr;
    if (dadam_init(&cfg, &h) != DADAM_OK) { printf("init: %s\n", dadam_last_error(nullptr)); return 1; }
    std::vector<int32_t> ptr(R + 1), col(R);
    std::vector<float> w(R, 1.f);
    for (uint32_t i = 0; i < R; ++i) { ptr[i + 1] = (int32_t)i + 1; col[i] = (int32_t)i; }
    dadam_set_topology(h, 3, ptr.data(), col.data(), w.data(), nullptr);
    at_base = iter % 2 ? 1ull << 40 : (1ull << 51) + (rng() % 1000 << 4);
    std::vector<void*> tables[6];
    for (uint32_t t = 0; t < 6; ++t)
      for (uint32_t i = 0; i < R; ++i) tables[t].push_back((void*)address_of(i, t));
    auto in = [&](int t) { return (const void* const*)tables[t].data(); };
    auto out = [&](int t) { return (void* const*)tables[t].data(); };
    auto f = [&](int t) { return (float* const*)tables[t].data(); };
    float* norms = (float*)(1ull << 30);
    int rc = dadam_grad_norm(h, in(0), norms, nullptr);
    rc |= dadam_clip_grads(h, in(0), out(1), 1.f, norms, nullptr);
    rc |= dadam_mx4_encode(h, in(0), f(1), f(2), out(3), nullptr);
    rc |= dadam_mx4_product(h, 3, in(5), f(0), DADAM_MX4_ADD, nullptr);
    rc |= dadam_mx4_gossip(h, 3, in(5), f(0), f(1), in(2), out(3), 0.5f, nullptr);
    rc |= dadam_mx4_round(h, 3, in(0), out(1), f(2), f(3), 0.5f, nullptr);
    if (rc) { ++bad; printf("refused: %s\n", dadam_last_error(h)); }
    dadam_destroy(h);
  }
  printf("launches %ld bad %ld\n", launches, bad);
  return bad != 0;
}
