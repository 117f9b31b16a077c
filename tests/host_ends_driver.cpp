// What the calls at the ends of an iteration ask of the HIP runtime, without a GPU: the built library on a modelled runtime (this program defines the calls, so the
// library's references resolve here) that says what it was asked for, and refuses launches without a workgroup as the real one does.  Reads commands, a line
// each, and prints one line for each: the command, the call's answer, the launches (kernel, grid x block, bytes of LDS) that it made, behind those of the head's gradient
// the piece's first word, its words and how many of them the launch leaves out.  tests/test_ends_calls.py builds and runs it.
//
//   loss ROWS PARAM_TYPE GRAD_TYPE TOKENS VOCAB WIDTH BEFORE GRADIENT WORKSPACE BIAS   one handle and call; BEFORE elements lie before the head
//   ortho ROWS PARAM_TYPE GRAD_TYPE STEP WORKSPACE ROWSxCOLS ...                   one handle, its matrices, and dadam_orthogonalize or (STEP 1) dadam_ortho_step
//   kernels                                                                            the kernels of these calls that the library has
// WORKSPACE: how many hundredths of the bytes that the information call asks for, at least the least.
#include "dadam.h"
#include "dadam_head.h"
#include <hip/hip_runtime_api.h>
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <map>
#include <sstream>
#include <string>
#include <vector>

static std::string events;
static hipError_t last = hipSuccess;
static std::map<const void*, std::string>& kernels() { static std::map<const void*, std::string> m; return m; }

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
hipError_t hipMalloc(void** p, size_t n) { *p = malloc(n); return hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { memcpy(d, s, n); return hipSuccess; }
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, const void*) { static double array[1024]; *p = array; return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipGetLastError() { const hipError_t e = last; last = hipSuccess; return e; }
struct Configuration {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} static pushed;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) { pushed = {grid, block, lds, stream}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* fn, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t) {
  const std::string& name = kernels()[fn];
  std::ostringstream out;
  out << " | launch " << name << " " << grid.x << "," << grid.y << "," << grid.z << "x" << block.x << " " << lds;
  if (name.find("k_head_dhead") != std::string::npos || name.find("k_head_join") != std::string::npos) {
    const dadam::HeadArgs& a = *(const dadam::HeadArgs*)args[0];
    out << " words " << a.first_word << " " << a.words << " " << a.skip;
  }
  events += out.str();
  const bool fits = grid.x && grid.y && grid.z && block.x && block.x <= 1024 && grid.y <= 65535 && grid.z <= 65535 && (uint64_t)grid.x * block.x <= 0xffffffffull && lds <= 160 * 1024;
  if (!fits) last = hipErrorInvalidConfiguration;
  return last;
}
}

// Buffers of one call: addresses only, nothing is read or written.
static uint64_t next_address = 1ull << 32;
static std::vector<void*> buffers(uint32_t n, uint64_t bytes) {
  std::vector<void*> t;
  for (uint32_t i = 0; i < n; ++i, next_address += (bytes + 511) / 256 * 256) t.push_back((void*)next_address);
  return t;
}
static const void* const* in(const std::vector<void*>& t) { return (const void* const*)t.data(); }
static uint64_t part(uint64_t hundredths, uint64_t least, uint64_t bytes) { return std::max(least, bytes / 100 * hundredths + bytes % 100 * hundredths / 100); }
static dadam_config config(uint32_t rows, uint64_t d, const std::vector<dadam_tensor_desc>& ts, uint32_t pt, uint32_t gt) {
  dadam_config cfg{};
  cfg.abi_version = DADAM_ABI_VERSION; cfg.n_rows = cfg.n_cols = rows; cfg.d = d; cfg.n_tensors = (uint32_t)ts.size(); cfg.tensors = ts.data();
  cfg.param_dtype = pt; cfg.grad_dtype = gt; cfg.lr = 1e-3f; cfg.accum_s = 1; cfg.beta_vhat = -1.f; cfg.eps = 1e-8f;
  return cfg;
}

static int loss(std::istringstream& line, std::string* text) {
  uint32_t rows, pt, gt, tokens, vocab, width, gradient, bias;
  uint64_t before, hundredths;
  line >> rows >> pt >> gt >> tokens >> vocab >> width >> before >> gradient >> hundredths >> bias;
  const uint64_t n = (uint64_t)vocab * width, d = before + n + (bias ? vocab : 0);
  std::vector<dadam_tensor_desc> ts;
  if (before) ts.push_back({0, before, 0.f, 0});
  ts.push_back({before, n, 0.f, 0});
  if (bias) ts.push_back({before + n, vocab, 0.f, 0});
  const dadam_config cfg = config(rows, d, ts, pt, gt);
  dadam_handle* h = nullptr;
  if (const int rc = dadam_init(&cfg, &h)) return rc;
  const dadam_head head = {before ? 1u : 0u, bias ? (uint32_t)ts.size() - 1 : DADAM_HEAD_NO_BIAS, vocab, width};
  dadam_head_info info{};
  int rc = dadam_head_get_info(h, &head, tokens, gradient, &info);
  const uint64_t bytes = part(hundredths, info.least_bytes, info.bytes), vectors = (uint64_t)tokens * width * 4;
  const auto params = buffers(rows, d * 4), hidden = buffers(rows, vectors), targets = buffers(rows, tokens * 4ull), nll = buffers(rows, tokens * 4ull), dhidden = buffers(rows, vectors),
             grads = buffers(rows, d * 4), losses = buffers(1, rows * 4), workspace = buffers(1, bytes);
  if (!rc)
    rc = dadam_head_loss(h, &head, in(params), in(hidden), (const int32_t* const*)targets.data(), tokens, 1.f, DADAM_HEAD_MEAN, (float*)losses[0], (float* const*)nll.data(),
                         gradient ? dhidden.data() : nullptr, gradient ? grads.data() : nullptr, workspace[0], bytes, nullptr);
  *text = dadam_last_error(h);
  dadam_destroy(h);
  return rc;
}

static int ortho(std::istringstream& line, std::string* text) {
  uint32_t rows, pt, gt, step;
  uint64_t hundredths, d = 0;
  line >> rows >> pt >> gt >> step >> hundredths;
  std::vector<dadam_tensor_desc> ts;
  std::vector<dadam_matrix_desc> ms;
  for (std::string shape; line >> shape;) {
    uint32_t r = 0, c = 0;
    sscanf(shape.c_str(), "%ux%u", &r, &c);
    ms.push_back({(uint32_t)ts.size(), r, c, c, 0, 1.f, 0});
    ts.push_back({d, (uint64_t)r * c, 0.f, 0});
    d += (uint64_t)r * c;
  }
  const dadam_config cfg = config(rows, d, ts, pt, gt);
  dadam_handle* h = nullptr;
  if (const int rc = dadam_init(&cfg, &h)) return rc;
  std::vector<int32_t> ptr(rows + 1), col(rows);
  std::vector<float> w(rows, 1.f);
  for (uint32_t i = 0; i < rows; ++i) ptr[i + 1] = (int32_t)i + 1, col[i] = (int32_t)i;
  int rc = dadam_set_topology(h, 0, ptr.data(), col.data(), w.data(), nullptr);
  if (!rc) rc = dadam_set_matrices(h, ms.data(), (uint32_t)ms.size());
  dadam_ortho_info info{};
  if (!rc) rc = dadam_ortho_get_info(h, &info);
  const uint64_t bytes = part(hundredths, info.least_bytes, info.bytes);
  const auto x = buffers(rows, d * 4), out = buffers(rows, d * 4), g = buffers(rows, d * 4), m = buffers(rows, d * 4), v = buffers(rows, d * 4), workspace = buffers(1, bytes);
  if (!rc && step) {
    dadam_buffers b{};
    b.x_src = in(x), b.x_dst = out.data(), b.m_hat = (float* const*)m.data(), b.v_hat = (float* const*)v.data();
    rc = dadam_bind(h, &b);
    if (!rc) rc = dadam_ortho_step(h, 0, in(g), 1, DADAM_FUSE_ACCUM, workspace[0], bytes, nullptr);
  } else if (!rc) {
    rc = dadam_orthogonalize(h, in(g), out.data(), workspace[0], bytes, nullptr);
  }
  *text = dadam_last_error(h);
  dadam_destroy(h);
  return rc;
}

int main() {
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream words(line);
    std::string what, text;
    words >> what;
    events.clear();
    next_address = 1ull << 32;
    int rc = -100;
    if (what == "loss") rc = loss(words, &text);
    if (what == "ortho") rc = ortho(words, &text);
    if (what == "kernels") {
      rc = 0;
      for (const auto& k : kernels())
        if (k.second.find("k_head_") != std::string::npos || k.second.find("k_few_") != std::string::npos || k.second.find("k_ortho_") != std::string::npos) events += " | kernel " + k.second;
    }
    std::cout << line << ": " << rc << (rc < 0 ? " " + text : "") << events << "\n";
  }
  return 0;
}
