// What the calls around the step ask of the HIP runtime, without a GPU: the built library on a modelled runtime (this program defines
// the calls, so the library's references resolve here) that says what it was asked for.  Reads commands, a line each, and prints one
// line for each: the command, the call's answer, and the allocations, copies and launches (kernel, grid x block, bytes of LDS) that it made; behind
// launches of products and gossip the rows whose sums they form, or "copy<of" where they copy rows.
// tests/test_operators_calls.py builds and runs it.
//
//   handle ROWS COLS D PARAM_TYPE GRAD_TYPE LDS_LIMIT     one tensor of D elements
//   tensors COUNT LEN                                     a row of COUNT tensors of LEN elements, up to two apart: dadam_init and a first norm; behind
//                                                         the answer the microseconds that the host spent in each, the shortest of five
//   topology SLOT lists N                                 N complete graphs side by side (rows = cols); N = rows: the identity
//   topology SLOT ring                                    every row, the one before and the one behind
//   call NAME SLOT                                        norm, clip, encode, product, add, gossip, round
//   capture 0|1                                           streams are being captured from now on
//   shift BYTES                                           by which every other buffer misses the beginning of a line from now on
//   kernels                                               the kernels of these calls that the library has
//   memory N                                              of the next call's allocations of host memory the N-th fails, 0 none; answers 0
//   left                                                  N less those made since, 0 or less: the N-th failed
#include "dadam.h"
#include "dadam_operators.h"
#include <hip/hip_runtime_api.h>
#include <algorithm>
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <map>
#include <new>
#include <sstream>
#include <string>
#include <vector>

static uint32_t R, C;
static uint64_t d;
static std::string events;
static bool capturing = false;
static std::map<const void*, std::string>& kernels() { static std::map<const void*, std::string> m; return m; }
struct Outside {  // the modelled runtime's own strings and tables do not count
  bool was;
  Outside();
  ~Outside();
};
static void note(const std::string& what);

// Host memory of the library's calls (inside a call only: the program's own goes through).
static bool in_call = false;
static long until = 0;
void* operator new(size_t n) {
  if (in_call && until-- == 1) throw std::bad_alloc();
  void* p = malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
// Buffer i of table t lies at base + (t * DADAM_MAX_ROWS + i) * step, every other one `shift` bytes further.
static uint64_t step = 1, shift = 0;
constexpr uint64_t kBase = 1ull << 32;
static uint64_t row_of(const dadam::RowPointers& r, int k) {
  const uint64_t at = (((uint64_t)((r.high[k / 2] >> (16 * (k % 2))) & 0xFFFF) << 32) | r.low[k]) << 4;
  return (at - kBase) / step;  // outputs are table 0
}
template <typename A>
static void note_rows(const std::string& name, const A& a) {
  std::string text = "rows";
  for (uint32_t p = 0; p < a.s.n_rows; ++p) {
    const uint64_t row = row_of(a.row[p], 0);
    text += " " + std::to_string(row);
    if (name.find("k_mx4_copy") != std::string::npos) text += "<" + std::to_string(row_of(a.row[p], 1));
    else if ((uint64_t)a.lists.rows[p].row != row) text += "!";  // the list of another row
  }
  note(text);
}
Outside::Outside() : was(in_call) { in_call = false; }
Outside::~Outside() { in_call = was; }
static void note(const std::string& what) { events += " | " + what; }
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* module; return &module; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { kernels()[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t a, int) {
  *v = a == hipDeviceAttributeNumberOfXccs ? 8 : 160 * 1024;
  return hipSuccess;
}
// A real runtime refuses both while a stream is being captured, and ends the capture.
hipError_t hipMalloc(void** p, size_t n) {
  Outside o;
  note("malloc " + std::to_string(n));
  if (capturing) return hipErrorStreamCaptureUnsupported;
  *p = malloc(n);
  return hipSuccess;
}
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) {
  Outside o;
  note("memcpy " + std::to_string(n));
  if (capturing) return hipErrorStreamCaptureImplicit;
  memcpy(d, s, n);
  return hipSuccess;
}
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, const void*) { static double array[1024]; *p = array; return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipLaunchKernel(const void* fn, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t) {
  Outside o;
  note("launch " + kernels()[fn] + " " + std::to_string(grid.x) + "x" + std::to_string(block.x) + " " + std::to_string(lds));
  const std::string& name = kernels()[fn];
  using namespace dadam;
  if (name.find("MixArgs") == std::string::npos) return hipSuccess;
  if (name.find("Li16ELi16EEE") != std::string::npos) note_rows(name, *(const MixArgs<kFewOperands, kFewOperands>*)args[0]);
  else note_rows(name, *(const MixArgs<kMessageRows, kMaxRows>*)args[0]);
  return hipSuccess;
}
}

static int topology(dadam_handle* h, std::istringstream& in) {
  uint32_t slot, n = 0;
  std::string kind;
  in >> slot >> kind >> n;
  std::vector<int32_t> ptr(1, 0), col;
  std::vector<float> w;
  for (uint32_t i = 0; i < R; ++i) {
    if (kind == "lists") {
      const uint32_t each = R / n, first = i / each * each;
      for (uint32_t k = 0; k < each; ++k) col.push_back((int32_t)(first + k));
    } else {
      for (uint32_t k : {i, (i + R - 1) % R, (i + 1) % R}) col.push_back((int32_t)k);
    }
    w.resize(col.size(), 1.f / (float)(col.size() - (size_t)ptr.back()));
    ptr.push_back((int32_t)col.size());
  }
  return dadam_set_topology(h, slot, ptr.data(), col.data(), w.data(), nullptr);
}

static int call(dadam_handle* h, std::istringstream& in) {
  std::string name;
  uint32_t slot = 0;
  in >> name >> slot;
  // addresses only: nothing is read or written
  step = (4 * d + 255) / 128 * 128;
  std::vector<void*> table[6];
  for (uint64_t t = 0; t < 6; ++t)
    for (uint64_t i = 0; i < (R > C ? R : C); ++i) table[t].push_back((void*)(kBase + (t * DADAM_MAX_ROWS + i) * step + (t + i) % 2 * shift));
  auto in_ = [&](int t) { return (const void* const*)table[t].data(); };
  auto out = [&](int t) { return (void* const*)table[t].data(); };
  auto f = [&](int t) { return (float* const*)table[t].data(); };
  float* norms = (float*)(1ull << 30);
  int rc = -100;
  in_call = true;
  if (name == "norm") rc = dadam_grad_norm(h, in_(0), norms, nullptr);
  if (name == "clip") rc = dadam_clip_grads(h, in_(0), out(1), 1.f, norms, nullptr);
  if (name == "encode") rc = dadam_mx4_encode(h, in_(0), f(1), f(2), out(3), nullptr);
  if (name == "product") rc = dadam_mx4_product(h, slot, in_(5), f(0), 0, nullptr);
  if (name == "add") rc = dadam_mx4_product(h, slot, in_(5), f(0), DADAM_MX4_ADD, nullptr);
  if (name == "gossip") rc = dadam_mx4_gossip(h, slot, in_(5), f(0), f(1), in_(2), out(3), 0.5f, nullptr);
  if (name == "round") rc = dadam_mx4_round(h, slot, in_(0), out(1), f(2), f(3), 0.5f, nullptr);
  in_call = false;
  return rc;
}

static int tensors(std::istringstream& in) {
  uint64_t count, len, end = 0;
  in >> count >> len;
  std::vector<dadam_tensor_desc> ts;
  for (uint64_t k = 0; k < count; ++k, end += len + end % 3) ts.push_back({end, len, 0.f, 0});
  dadam_config cfg{};
  cfg.abi_version = DADAM_ABI_VERSION; cfg.n_rows = cfg.n_cols = 1; cfg.d = end; cfg.n_tensors = (uint32_t)count; cfg.tensors = ts.data();
  cfg.lr = 1e-3f; cfg.accum_s = 1; cfg.beta_vhat = -1.f; cfg.eps = 1e-8f;
  long best[2] = {1L << 40, 1L << 40};
  auto now = [] { return std::chrono::steady_clock::now(); };
  for (int k = 0; k < 5; ++k) {
    dadam_handle* one = nullptr;
    const void* grads = (const void*)kBase;
    const auto t0 = now();
    int rc = dadam_init(&cfg, &one);
    const auto t1 = now();
    if (rc == DADAM_OK) rc = dadam_grad_norm(one, &grads, (float*)(1ull << 30), nullptr);
    const auto t2 = now();
    dadam_destroy(one);
    if (rc != DADAM_OK) return rc;
    best[0] = std::min(best[0], (long)std::chrono::duration_cast<std::chrono::microseconds>(t1 - t0).count());
    best[1] = std::min(best[1], (long)std::chrono::duration_cast<std::chrono::microseconds>(t2 - t1).count());
  }
  note("us " + std::to_string(best[0]) + " " + std::to_string(best[1]));
  return 0;
}

int main() {
  dadam_handle* h = nullptr;
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string what;
    in >> what;
    int rc = -100;
    events.clear();
    if (what == "handle") {
      if (h) dadam_destroy(h);
      h = nullptr;
      dadam_config cfg{};
      in >> R >> C >> d >> cfg.param_dtype >> cfg.grad_dtype >> cfg.lds_limit_bytes;
      const dadam_tensor_desc t = {0, d, 0.f, 0};
      cfg.abi_version = DADAM_ABI_VERSION; cfg.n_rows = R; cfg.n_cols = C; cfg.d = d; cfg.n_tensors = 1; cfg.tensors = &t;
      cfg.lr = 1e-3f; cfg.accum_s = 1; cfg.beta_vhat = -1.f; cfg.eps = 1e-8f;
      rc = dadam_init(&cfg, &h);
    } else if (what == "tensors") {
      rc = tensors(in);
    } else if (what == "topology") {
      rc = topology(h, in);
    } else if (what == "call") {
      rc = call(h, in);
    } else if (what == "capture") {
      in >> capturing;
      rc = 0;
    } else if (what == "shift") {
      in >> shift;
      rc = 0;
    } else if (what == "kernels") {
      for (const auto& k : kernels())
        if (k.second.find("k_mx4_") != std::string::npos || k.second.find("k_clip") != std::string::npos || k.second.find("k_grad_norm") != std::string::npos)
          note("kernel " + k.second);
      rc = 0;
    } else if (what == "memory") {
      in >> until;
      rc = 0;
    } else if (what == "left") {
      rc = (int)until;
    }
    std::cout << line << ": " << rc << (rc < 0 && what != "left" ? std::string(" ") + dadam_last_error(h) : "") << events << "\n";
  }
  if (h) dadam_destroy(h);
  return 0;
}
