// Host side of orthogonalised updates (include/dadam.h, "The ends of an iteration"): the matrices of a layout, the schedule of the iteration, what
// the operands are held times, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <vector>

#include "dadam_checks.h"
#include "dadam_handle.h"
#include "dadam_ortho.h"

namespace dadam {

struct MatrixState {
  // dadam_set_matrices: by size, the largest first
  std::vector<OrthoTask> tasks;
  std::vector<uint32_t> parts[2]; // OrthoTask::parts, with one plane and with two
  std::vector<uint64_t> need[2];  // bytes of workspace of a matrix and a replica, with one plane and with two
  char* memory = nullptr;         // tasks, and the matrix of every tile of each kind
  const OrthoTask* d_tasks[2] = {};
  const uint32_t* d_units[4] = {};  // OrthoTask::gram_units, whole_units, cell_units, small_units
  uint32_t n_units[4] = {};
  uint32_t lone_lds = 0;          // where a workgroup holds each of them: the most that one takes
  // dadam_set_ortho_schedule
  std::vector<float> coefficients{3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f};
};

namespace {

void free_matrices(MatrixState* m) {
  if (!m) return;
  if (m->memory) (void)hipFree(m->memory);
  delete m;
}

MatrixState* state_of(dadam_handle* h) {
  if (!h->matrices) {
    h->matrices = new MatrixState();
    h->free_matrices = free_matrices;
  }
  return h->matrices;
}

uint32_t filled(uint32_t n, uint32_t each) { return (n + each - 1) / each * each; }

uint64_t lower_half(uint64_t n) { return n * (n + 1) / 2; }

// Large tiles: for matrices whose sides they fill up by an eighth more than the small ones at most, if there are enough of them for the chip (256 compute
// units, that hold one each).
bool suits_large(uint32_t n) { return 8 * (uint64_t)filled(n, kLargeEdge) <= 9 * (uint64_t)filled(n, kSmallEdge); }
constexpr uint64_t kEnoughLarge = 256, kComputeUnits = 256;

// X X^T of a matrix whose tiles sum for longer than the chip takes for all small tiles together: in ranges of columns, of as many stages as leave every compute unit the
// same, but eight at least.  (A product of fewer than 32 stages takes no longer than the second launch.)  It depends on the layout alone, so that the workspace's size
// changes no result.
constexpr uint64_t kLongSum = 32, kLeastStages = 8;
uint64_t stages_of(const OrthoTask& t, uint32_t planes) { return (uint64_t)t.Q * planes / 64; }
void split_sums(std::vector<OrthoTask>* tasks, uint32_t planes, uint64_t replicas) {
  uint64_t all = 0, most = 0;
  for (const OrthoTask& t : *tasks)
    if (t.edge == kSmallEdge) all += lower_half(t.P / kSmallEdge) * stages_of(t, planes) * replicas;
  const uint64_t each = std::max(kLeastStages, all / kComputeUnits);
  for (OrthoTask& t : *tasks) {
    if (t.edge != kSmallEdge) continue;
    const uint64_t stages = stages_of(t, planes);
    t.parts = stages < kLongSum ? 1 : (uint32_t)std::max<uint64_t>(1, stages / each);
    most = std::max<uint64_t>(most, t.parts);
  }
  if (most > 1) return;
  for (OrthoTask& t : *tasks) t.parts = 0;
}

constexpr uint32_t kMostMatrices = 65536, kMostSide = 65536;

// Whether two matrices of a tensor share elements.
bool share_elements(const dadam_matrix_desc& one, const dadam_matrix_desc& other) {
  if (one.ld == other.ld) {  // rectangles of rows of ld elements
    auto apart = [](uint64_t p, uint64_t n, uint64_t q, uint64_t m) { return p + n <= q || q + m <= p; };
    return !apart(one.first / one.ld, one.rows, other.first / one.ld, other.rows) && !apart(one.first % one.ld, one.cols, other.first % one.ld, other.cols);
  }
  const dadam_matrix_desc &a = one.rows <= other.rows ? one : other, &b = one.rows <= other.rows ? other : one;
  for (uint64_t r = 0; r < a.rows; ++r) {
    const uint64_t at = a.first + r * a.ld, end = b.first + b.cols, k = at < end ? 0 : (at - end) / b.ld + 1;  // the first row of b that ends behind at
    if (k < b.rows && b.first + k * b.ld < at + a.cols) return true;
  }
  return false;
}

int check_matrices(const dadam_handle* h, const dadam_matrix_desc* m, uint32_t n) {
  std::vector<std::vector<uint32_t>> of_tensor(h->tensors.size());
  for (uint32_t k = 0; k < n; ++k) {
    if (m[k].tensor >= h->tensors.size()) return fail(h, DADAM_EINVAL, "matrix %u: tensor %u out of range", k, m[k].tensor);
    if (m[k].flags) return fail(h, DADAM_EINVAL, "matrix %u: flags must be 0", k);
    if (!std::isfinite(m[k].scale)) return fail(h, DADAM_EINVAL, "matrix %u: scale must be finite", k);
    const uint64_t rows = m[k].rows, cols = m[k].cols, ld = m[k].ld, numel = h->tensors[m[k].tensor].numel;
    if (!rows || !cols || rows > kMostSide || cols > kMostSide) return fail(h, DADAM_EINVAL, "matrix %u: rows and columns must be 1 to %u", k, kMostSide);
    if (ld < cols || m[k].first % ld + cols > ld) return fail(h, DADAM_EINVAL, "matrix %u: its columns do not lie in one row of ld elements", k);
    if (m[k].first >= numel || numel - m[k].first < cols || (rows - 1) > (numel - m[k].first - cols) / ld)
      return fail(h, DADAM_EINVAL, "matrix %u reaches beyond its tensor", k);
    of_tensor[m[k].tensor].push_back(k);
  }
  for (std::vector<uint32_t>& list : of_tensor) {
    auto end = [&](uint32_t k) { return m[k].first + (uint64_t)(m[k].rows - 1) * m[k].ld + m[k].cols; };
    std::sort(list.begin(), list.end(), [&](uint32_t a, uint32_t b) { return m[a].first < m[b].first; });
    for (size_t i = 0; i < list.size(); ++i)
      for (size_t j = i + 1; j < list.size() && m[list[j]].first < end(list[i]); ++j)
        if (share_elements(m[list[i]], m[list[j]])) return fail(h, DADAM_EINVAL, "matrices %u and %u share elements", list[i], list[j]);
  }
  return DADAM_OK;
}

int set_matrices(dadam_handle* h, const dadam_matrix_desc* m, uint32_t n) {
  if (const int rc = check_matrices(h, m, n)) return rc;
  std::unique_ptr<MatrixState, void (*)(MatrixState*)> s(new MatrixState(), free_matrices);
  if (h->matrices) s->coefficients = h->matrices->coefficients;
  // A layout of matrices that each fit a compute unit goes by those (64 x 48 and 48 x 192: 42 us instead of 138).  Beside larger ones they go with those, whose launches
  // they lengthen by little (40 matrices of odd sizes 466 us, the small ones apart 623).
  bool lone = n > 0;
  std::vector<OrthoTask> tasks(n);
  for (uint32_t k = 0; k < n; ++k) {
    OrthoTask& t = tasks[k];
    const dadam_tensor_desc& tensor = h->tensors[m[k].tensor];
    t.first = tensor.offset_elems + m[k].first;
    t.ld = m[k].ld;
    t.tall = m[k].rows > m[k].cols;
    t.p = std::min(m[k].rows, m[k].cols);
    t.q = std::max(m[k].rows, m[k].cols);
    t.edge = suits_large(t.p) && suits_large(t.q) ? kLargeEdge : kSmallEdge;
    lone = lone && lone_lds_bytes(filled(t.p, kLoneEdge), filled(t.q, kLoneEdge)) <= kMostLoneLds;
    t.scale = m[k].scale;
    t.decay = tensor.weight_decay;
  }
  uint64_t large = 0, units[4] = {};
  for (const OrthoTask& t : tasks)
    if (t.edge == kLargeEdge) large += lower_half(filled(t.p, kLargeEdge) / kLargeEdge);
  for (OrthoTask& t : tasks) {
    if (large * h->cfg.n_rows < kEnoughLarge) t.edge = kSmallEdge;
    if (lone) t.edge = kLoneEdge;
    t.P = filled(t.p, t.edge);
    t.Q = filled(t.q, t.edge);
    if (lone) {
      s->lone_lds = std::max(s->lone_lds, (uint32_t)lone_lds_bytes(t.P, t.Q));
      continue;
    }
    units[0] += lower_half(t.P / t.edge);
    units[1] += (uint64_t)(t.P / t.edge) * (t.Q / t.edge);
    units[2] += (uint64_t)(t.P / kOrthoCell) * (t.Q / kOrthoCell);
    units[3] += lower_half(t.P / kSmallEdge);
  }
  if (units[2] >> 31) return fail(h, DADAM_EINVAL, "the matrices have more than 2^31 tiles");
  // by tile and size, the largest first
  std::stable_sort(tasks.begin(), tasks.end(), [](const OrthoTask& a, const OrthoTask& b) {
    return a.edge != b.edge ? a.edge > b.edge : (uint64_t)a.P * a.P * a.Q > (uint64_t)b.P * b.P * b.Q;
  });
  std::vector<uint32_t> of_unit[4];
  for (int kind = 0; kind < 4; ++kind) of_unit[kind].reserve(units[kind]);
  for (uint32_t k = 0; k < n && !lone; ++k) {
    OrthoTask& t = tasks[k];
    t.gram_units = (uint32_t)of_unit[0].size();
    t.whole_units = (uint32_t)of_unit[1].size();
    t.cell_units = (uint32_t)of_unit[2].size();
    t.small_units = (uint32_t)of_unit[3].size();
    of_unit[0].insert(of_unit[0].end(), lower_half(t.P / t.edge), k);
    of_unit[1].insert(of_unit[1].end(), (uint64_t)(t.P / t.edge) * (t.Q / t.edge), k);
    of_unit[2].insert(of_unit[2].end(), (uint64_t)(t.P / kOrthoCell) * (t.Q / kOrthoCell), k);
    of_unit[3].insert(of_unit[3].end(), lower_half(t.P / kSmallEdge), k);
  }
  std::vector<OrthoTask> planes[2] = {tasks, tasks};
  for (uint32_t p = 0; p < 2; ++p) {
    split_sums(&planes[p], p + 1, h->cfg.n_rows);
    uint64_t at = 0;
    for (OrthoTask& t : planes[p]) {
      t.at = at;
      s->parts[p].push_back(t.parts);
      s->need[p].push_back(lone ? 0 : ortho_places(t.P, t.Q, p + 1, t.parts).bytes);
      at += s->need[p].back();
    }
    s->need[p].push_back(at);
  }
  s->tasks = planes[0];
  for (int kind = 0; kind < 4; ++kind) s->n_units[kind] = (uint32_t)of_unit[kind].size();
  if (h->cfg.device != DADAM_DEVICE_NONE && n) {
    DeviceGuard guard(h->cfg.device);
    if (guard.err != hipSuccess) return fail(h, DADAM_EHIP, "hipSetDevice: %s", hipGetErrorString(guard.err));
    std::vector<char> image;
    auto add = [&image](const auto& v) {
      const size_t at = image.size();
      image.resize(at + (v.size() * sizeof(v[0]) + 63) / 64 * 64);
      memcpy(image.data() + at, v.data(), v.size() * sizeof(v[0]));
      return at;
    };
    size_t at[6] = {add(planes[0]), add(planes[1]), add(of_unit[0]), add(of_unit[1]), add(of_unit[2]), add(of_unit[3])};
    hipError_t e = hipMalloc((void**)&s->memory, image.size());
    if (e == hipSuccess) e = hipMemcpy(s->memory, image.data(), image.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return fail(h, DADAM_EHIP, "uploading the matrices failed: %s", hipGetErrorString(e));
    }
    for (int p = 0; p < 2; ++p) s->d_tasks[p] = reinterpret_cast<const OrthoTask*>(s->memory + at[p]);
    for (int kind = 0; kind < 4; ++kind) s->d_units[kind] = reinterpret_cast<const uint32_t*>(s->memory + at[2 + kind]);
    MatrixState* old = h->matrices;
    h->matrices = s.release();
    h->free_matrices = free_matrices;
    free_matrices(old);
    return DADAM_OK;
  }
  if (h->cfg.device != DADAM_DEVICE_NONE && h->matrices) {
    DeviceGuard guard(h->cfg.device);
    free_matrices(h->matrices);
  } else {
    free_matrices(h->matrices);
  }
  h->matrices = s.release();
  h->free_matrices = free_matrices;
  return DADAM_OK;
}

// The largest |f| on [0, limit], by samples close enough for a bound with a margin.
template <typename Fn>
double largest(double limit, Fn f) {
  double most = 0.0;
  constexpr int n = 2048;
  for (int k = 0; k <= n; ++k) most = std::max(most, std::fabs(f(limit * k / n)));
  return 1.01 * most;
}

// What X, A and B of every iteration are held times: the power of two that brings a bound of the spectral norm, and with it of every element, to
// [2^12, 2^13], an eighth of what a half can hold.  X of iteration 0 has Frobenius norm 1.
struct Powers {
  std::vector<int> x, a, b;
};
constexpr double kLargestNorm = 1024.0;
int power_for(double bound) { return 13 - (int)std::ceil(std::log2(std::max(bound, 1e-3))); }
bool find_powers(const std::vector<float>& c, Powers* out) {
  double bound = 1.0;
  for (size_t k = 0; k + 2 < c.size(); k += 3) {
    const double a = c[k], b = c[k + 1], cc = c[k + 2];
    out->x.push_back(power_for(bound));
    out->a.push_back(power_for(bound * bound));
    out->b.push_back(power_for(largest(bound * bound, [&](double s) { return b * s + cc * s * s; })));
    bound = largest(bound, [&](double s) { return a * s + b * s * s * s + cc * s * s * s * s * s; });
    if (!(bound <= kLargestNorm)) return false;
  }
  return true;
}

// Workspace that a call makes good use of.  Beyond it a larger one gains nothing: the matrices go in groups that fill the chip.
constexpr uint64_t kOrthoWorkspace = 1ull << 30;

uint32_t planes_of(uint32_t dtype) { return dtype == DADAM_BF16 ? 1 : 2; }

struct Call {
  const void* const* grads;
  void* const* out;
  OrthoSource source;
  Phase phase;
  Scalars c;
  bool mix;
  uint32_t slot, dtype;  // of the result
  char* workspace;
  uint64_t bytes;
};

// What a launch of so many tiles takes, in the time of a large one: the chip holds 256 large or 512 small ones at a time, and two small ones beside each other take 0.66
// of a large one's time (0.55 with two planes).
double time_of(uint32_t edge, double tiles, uint32_t planes) {
  return edge == kLargeEdge ? std::ceil(tiles / 256) : std::ceil(tiles / 512) * (planes == 1 ? 0.66 : 0.55);
}
// A and B by large tiles, or by small ones where the chip is through with those sooner.
bool gram_by_large(uint32_t edge, double large, double small, uint32_t planes) {
  return edge == kLargeEdge && time_of(kLargeEdge, large, planes) <= time_of(kSmallEdge, small, planes);
}

// Matrices k0 .. that go together, of all replicas in `most` bytes: those whose launches leave the least of the chip idle.
uint32_t end_of_group(const dadam_handle* h, uint32_t planes, uint32_t k0, uint64_t most) {
  const std::vector<OrthoTask>& tasks = h->matrices->tasks;
  const std::vector<uint64_t>& need = h->matrices->need[planes - 1];
  const double R = h->cfg.n_rows, unit = tasks[k0].edge == kLargeEdge ? 256 : 512;
  double gram = 0, small = 0, whole = 0, long_gram = 0, best = 0;
  uint32_t chosen = k0;
  uint64_t bytes = 0;
  for (uint32_t k = k0; k < tasks.size() && tasks[k].edge == tasks[k0].edge && bytes + need[k] <= most / h->cfg.n_rows; ++k) {
    const OrthoTask& t = tasks[k];
    bytes += need[k];
    gram += R * lower_half(t.P / t.edge);
    small += R * lower_half(t.P / kSmallEdge);
    whole += R * (double)(t.P / t.edge) * (t.Q / t.edge);
    long_gram = std::max(long_gram, (double)t.Q / t.P);  // X X^T sums that much longer than the other products
    // the share of the time in which the chip is full, A A and X X^T by the tiles that they go by; a launch begins and ends like half a round of tiles
    const bool by_large = gram_by_large(t.edge, gram, small, planes);
    const double tiles = by_large ? gram : small, slots = by_large ? 256 : 512, idle = (std::ceil(tiles / slots) + 0.5) * slots / tiles;
    const double share = (2 * whole + (1 + long_gram) * gram) / (2 * (std::ceil(whole / unit) + 0.5) * unit + (1 + long_gram) * gram * idle);
    if (share >= best || k + 1 == tasks.size() || tasks[k + 1].edge != t.edge) best = share, chosen = k + 1;  // (all that are left, if there is room for them)
  }
  return chosen;
}

// A matrices-by-replicas rectangle, whole.
int run_group(dadam_handle* h, const Call& call, const Powers& pw, uint32_t k0, uint32_t k1, uint32_t i0, uint32_t replicas, void* stream) {
  const MatrixState& m = *h->matrices;
  const uint32_t planes = planes_of(call.dtype), n = (uint32_t)m.tasks.size();
  OrthoSpan spans[4] = {};
  uint32_t units[4];
  for (int kind = 0; kind < 4; ++kind) {
    auto before = [&](uint32_t k) {
      if (k == n) return m.n_units[kind];
      const OrthoTask& t = m.tasks[k];
      return kind == 0 ? t.gram_units : kind == 1 ? t.whole_units : kind == 2 ? t.cell_units : t.small_units;
    };
    OrthoSpan& s = spans[kind];
    s.tasks = m.d_tasks[planes - 1];
    s.units = m.d_units[kind];
    s.workspace = (uint64_t)(uintptr_t)call.workspace;
    for (uint32_t k = 0; k < k0; ++k) s.before += m.need[planes - 1][k];
    for (uint32_t k = k0; k < k1; ++k) s.stride += m.need[planes - 1][k];
    s.first_unit = before(k0);
    s.n_xcd = h->n_xcds;
    units[kind] = before(k1) - s.first_unit;
  }
  const uint32_t edge = m.tasks[k0].edge, whole_units = units[1];
  const OrthoSpan& whole = spans[1];
  const bool by_large = gram_by_large(edge, units[0] * (double)replicas, units[3] * (double)replicas, planes);
  const uint32_t gram_edge = by_large ? kLargeEdge : kSmallEdge, gram_units = units[by_large ? 0 : 3];
  const OrthoSpan& gram = spans[by_large ? 0 : 3];
  const uint32_t parts = *std::max_element(m.parts[planes - 1].begin() + k0, m.parts[planes - 1].begin() + k1);
  OrthoBeginArgs<kMaxRows> begin;
  memset((void*)&begin, 0, sizeof(begin));
  begin.s = spans[2];
  for (uint32_t r = 0; r < replicas; ++r) {
    begin.grad[r] = call.grads[i0 + r];
    if (call.source == kOrthoGiven) continue;
    begin.m_hat[r] = h->m_hat[i0 + r];
    begin.acc[r] = h->acc[i0 + r];
  }
  begin.c = call.c;
  begin.scale = std::ldexp(1.f, pw.x[0]);
  begin.source = call.source;
  begin.phase = call.phase;
  int e = launch_ortho_norm((int)h->cfg.grad_dtype, begin, planes, units[2], replicas, stream);
  if (!e) e = launch_ortho_begin((int)h->cfg.grad_dtype, begin, planes, units[2], replicas, stream);
  const size_t steps = pw.x.size();
  for (size_t k = 0; k < steps && !e; ++k) {
    const float a = m.coefficients[3 * k], b = m.coefficients[3 * k + 1], c = m.coefficients[3 * k + 2];
    const int x = pw.x[k], pa = pw.a[k], pb = pw.b[k];
    OrthoStepArgs s{};
    s.s = gram;
    s.from = (uint32_t)(k & 1);
    s.to = s.from ^ 1;
    s.fresh = std::ldexp(1.f, pa - 2 * x);
    e = parts > 1 ? launch_ortho_parts(s, planes, parts, gram_units, replicas, stream) : launch_ortho_gram(false, gram_edge, s, planes, gram_units, replicas, stream);
    s.gain = std::ldexp(b, pb - pa);
    s.fresh = std::ldexp(c, pb - 2 * pa);
    if (!e) e = launch_ortho_gram(true, gram_edge, s, planes, gram_units, replicas, stream);
    if (e) break;
    s.s = whole;
    if (k + 1 < steps) {
      s.gain = std::ldexp(a, pw.x[k + 1] - x);
      s.fresh = std::ldexp(1.f, pw.x[k + 1] - x - pb);
      e = launch_ortho_next(edge, s, planes, whole_units, replicas, stream);
      continue;
    }
    OrthoEndArgs<kMaxRows> end;
    memset((void*)&end, 0, sizeof(end));
    end.s = whole;
    end.gain = std::ldexp(a, -x);
    end.fresh = std::ldexp(1.f, -x - pb);
    end.from = s.from;
    end.mix = call.mix;
    for (uint32_t r = 0; r < replicas; ++r) end.out[r] = call.out[i0 + r];
    if (call.mix) {
      for (uint32_t q = 0; q < h->cfg.n_cols; ++q) end.x_src[q] = h->x_src[q];
      const Slot& slot = h->slots[call.slot];
      end.row_ptr = slot.d_row_ptr;
      end.col = slot.d_col;
      end.w = slot.d_w;
      end.first_row = i0;
      end.lr = call.c.lr;
    }
    e = launch_ortho_end((int)call.dtype, edge, end, h->cfg.n_cols, whole_units, replicas, stream);
  }
  return e;
}

// The matrices that a workgroup holds, of all replicas.
int run_lone(dadam_handle* h, const Call& call, const Powers& pw, void* stream) {
  const MatrixState& m = *h->matrices;
  const uint32_t R = h->cfg.n_rows;
  OrthoLoneArgs<kLoneRows, kMaxRows> a;
  memset((void*)&a, 0, sizeof(a));
  a.tasks = m.d_tasks[planes_of(call.dtype) - 1];
  a.n_steps = (uint32_t)pw.x.size();
  a.source = call.source;
  a.phase = call.phase;
  a.c = call.c;
  a.scale = std::ldexp(1.f, pw.x[0]);
  for (uint32_t k = 0; k < a.n_steps; ++k) {
    const int x = pw.x[k], pa = pw.a[k], pb = pw.b[k], next = k + 1 < a.n_steps ? pw.x[k + 1] : 0;
    a.step[k].a_fresh = std::ldexp(1.f, pa - 2 * x);
    a.step[k].b_gain = std::ldexp(m.coefficients[3 * k + 1], pb - pa);
    a.step[k].b_fresh = std::ldexp(m.coefficients[3 * k + 2], pb - 2 * pa);
    a.step[k].x_gain = std::ldexp(m.coefficients[3 * k], next - x);
    a.step[k].x_fresh = std::ldexp(1.f, next - x - pb);
  }
  if (call.mix) {
    for (uint32_t q = 0; q < h->cfg.n_cols; ++q) a.x_src[q] = h->x_src[q];
    const Slot& slot = h->slots[call.slot];
    a.mix = 1;
    a.row_ptr = slot.d_row_ptr;
    a.col = slot.d_col;
    a.w = slot.d_w;
    a.lr = call.c.lr;
  }
  int e = (int)hipSuccess;
  for (uint32_t i = 0; i < R && !e; i += kLoneRows) {
    const uint32_t replicas = std::min<uint32_t>(kLoneRows, R - i);
    a.first_row = i;
    for (uint32_t r = 0; r < replicas; ++r) {
      a.grad[r] = call.grads[i + r];
      a.out[r] = call.out[i + r];
      a.m_hat[r] = call.source == kOrthoGiven ? nullptr : h->m_hat[i + r];
      a.acc[r] = call.source == kOrthoGiven ? nullptr : h->acc[i + r];
    }
    e = launch_ortho_lone((int)h->cfg.grad_dtype, (int)call.dtype, a, call.mix ? h->cfg.n_cols : 1, (uint32_t)m.tasks.size(), replicas, m.lone_lds, stream);
  }
  return e;
}

int check_workspace(const dadam_handle* h, const void* workspace, uint64_t bytes, uint64_t least) {
  if (!workspace && least) return fail(h, DADAM_EINVAL, "workspace is null");
  if ((uintptr_t)workspace & 255u) return fail(h, DADAM_EALIGN, "workspace is not 256-byte aligned");
  if (bytes && ((uintptr_t)workspace >= kHighest || bytes > kHighest - (uintptr_t)workspace)) return fail(h, DADAM_EINVAL, "workspace reaches above address 2^52");
  if (bytes < least) return fail(h, DADAM_EINVAL, "workspace has %llu bytes, %llu are needed", (unsigned long long)bytes, (unsigned long long)least);
  return DADAM_OK;
}

uint64_t least_bytes(const dadam_handle* h, uint32_t planes) {
  const std::vector<uint64_t>& need = h->matrices->need[planes - 1];
  return need.size() < 2 ? 0 : *std::max_element(need.begin(), need.end() - 1);
}

int run(dadam_handle* h, const Call& call, void* stream) {
  Powers pw;
  (void)find_powers(h->matrices->coefficients, &pw);
  const std::vector<uint64_t>& need = h->matrices->need[planes_of(call.dtype) - 1];
  const uint32_t n = (uint32_t)h->matrices->tasks.size(), R = h->cfg.n_rows;
  DeviceGuard guard(h->cfg.device);
  if (guard.err != hipSuccess) return fail(h, DADAM_EHIP, "hipSetDevice: %s", hipGetErrorString(guard.err));
  const bool lone = h->matrices->lone_lds != 0;
  int e = lone ? run_lone(h, call, pw, stream) : (int)hipSuccess;
  for (uint32_t k = 0; k < n && !lone && !e;) {
    uint32_t end = end_of_group(h, planes_of(call.dtype), k, call.bytes);
    if (end > k) {
      e = run_group(h, call, pw, k, end, 0, R, stream);
    } else {  // one matrix, as many replicas as there is room for
      end = k + 1;
      const uint32_t each = (uint32_t)std::min<uint64_t>(R, call.bytes / need[k]);
      for (uint32_t i = 0; i < R && !e; i += each) e = run_group(h, call, pw, k, end, i, std::min(each, R - i), stream);
    }
    k = end;
  }
  if (e != (int)hipSuccess) return fail(h, DADAM_EHIP, "kernel launch failed: %s", hipGetErrorString((hipError_t)e));
  return DADAM_OK;
}

int check_set(const dadam_handle* h) {
  if (!h->matrices || h->matrices->need[0].empty()) return fail(h, DADAM_ESTATE, "no matrices: call dadam_set_matrices first");
  return DADAM_OK;
}

}  // namespace
}  // namespace dadam

extern "C" {

int dadam_set_matrices(dadam_handle* h, const dadam_matrix_desc* matrices, uint32_t n) {
  if (!h) return DADAM_EINVAL;
  if (!matrices && n) return fail(h, DADAM_EINVAL, "matrices is null");
  if (n > kMostMatrices) return fail(h, DADAM_EINVAL, "more than %u matrices", kMostMatrices);
  return guarded(h, [&] { return set_matrices(h, matrices, n); });
}

int dadam_set_ortho_schedule(dadam_handle* h, uint32_t n_steps, const float* coefficients) {
  if (!h) return DADAM_EINVAL;
  if (!coefficients) return fail(h, DADAM_EINVAL, "coefficients is null");
  if (n_steps < 1 || n_steps > DADAM_ORTHO_MAX_STEPS) return fail(h, DADAM_EINVAL, "1 to %u iterations", DADAM_ORTHO_MAX_STEPS);
  return guarded(h, [&] {
    const std::vector<float> c(coefficients, coefficients + 3 * n_steps);
    for (float v : c)
      if (!std::isfinite(v)) return fail(h, DADAM_EINVAL, "coefficients must be finite");
    Powers pw;
    if (!find_powers(c, &pw)) return fail(h, DADAM_EINVAL, "singular values of up to 1 leave the iteration above %g", kLargestNorm);
    state_of(h)->coefficients = c;
    return DADAM_OK;
  });
}

int dadam_ortho_get_info(const dadam_handle* h, dadam_ortho_info* out) {
  if (!h) return DADAM_EINVAL;
  if (!out) return fail(h, DADAM_EINVAL, "out is null");
  if (const int rc = check_set(h)) return rc;
  // the same for both entry points: a step goes by the parameters' type, the operator by the gradients'
  const uint32_t planes = std::max(planes_of(h->cfg.param_dtype), planes_of(h->cfg.grad_dtype));
  out->n_matrices = (uint32_t)h->matrices->tasks.size();
  out->reserved = 0;
  out->least_bytes = least_bytes(h, planes);
  out->bytes = std::max(out->least_bytes, std::min(h->matrices->need[planes - 1].back() * h->cfg.n_rows, kOrthoWorkspace));
  return DADAM_OK;
}

int dadam_orthogonalize(dadam_handle* h, const void* const* in, void* const* out, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!in || !out) return fail(h, DADAM_EINVAL, "in or out is null");
  return guarded(h, [&] {
    int rc = check_set(h);
    if (rc) return rc;
    const uint32_t R = h->cfg.n_rows, dt = h->cfg.grad_dtype;
    const size_t gb = (size_t)h->cfg.d * dtype_bytes(dt);
    rc = check_workspace(h, workspace, workspace_bytes, least_bytes(h, planes_of(dt)));
    const void* const one[1] = {workspace};
    const Table tables[3] = {{in, R, gb, "in", false, -1}, {out, R, gb, "out", true, 0}, {one, workspace ? 1u : 0u, (size_t)workspace_bytes, "workspace", true, -1}};
    if (!rc) rc = check_tables(h, tables, 3);
    if (!rc) rc = check_device(h);
    if (rc) return rc;
    Call call{};
    call.grads = in, call.out = out, call.source = kOrthoGiven, call.phase = kUpdateOnly;
    call.dtype = dt, call.workspace = (char*)workspace, call.bytes = workspace_bytes;
    return run(h, call, hip_stream);
  });
}

int dadam_ortho_step(dadam_handle* h, uint32_t slot, const void* const* grads, uint64_t t, uint32_t flags, void* workspace, uint64_t workspace_bytes,
                     void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (flags & ~(DADAM_FUSE_ACCUM | DADAM_ORTHO_NESTEROV)) return fail(h, DADAM_EINVAL, "unknown flag bits 0x%x", flags);
  return guarded(h, [&] {
    Call call{};
    int rc = prepare_step(h, slot, grads, t, (flags & DADAM_FUSE_ACCUM) != 0, &call.phase, &call.c);
    if (!rc) rc = check_set(h);
    if (!rc) rc = check_workspace(h, workspace, workspace_bytes, least_bytes(h, planes_of(h->cfg.param_dtype)));
    if (rc) return rc;
    const uint32_t R = h->cfg.n_rows, C = h->cfg.n_cols;
    const size_t gb = (size_t)h->cfg.d * dtype_bytes(h->cfg.grad_dtype), xb = (size_t)h->cfg.d * dtype_bytes(h->cfg.param_dtype), sb = (size_t)h->cfg.d * 4;
    const uintptr_t lo = (uintptr_t)workspace, hi = lo + workspace_bytes;
    auto meets = [&](const void* p, size_t bytes) { return p && (uintptr_t)p < hi && lo < (uintptr_t)p + bytes; };
    for (uint32_t i = 0; i < R && !rc; ++i)
      if (meets(grads[i], gb) || meets(h->x_dst[i], xb) || meets(h->m_hat[i], sb) || meets(h->acc[i], sb)) rc = fail(h, DADAM_EALIAS, "workspace overlaps a buffer of row %u", i);
    for (uint32_t c = 0; c < C && !rc; ++c)
      if (meets(h->x_src[c], xb)) rc = fail(h, DADAM_EALIAS, "workspace overlaps x_src[%u]", c);
    if (!rc) rc = check_device(h);
    if (rc) return rc;
    call.grads = grads, call.out = h->x_dst, call.source = flags & DADAM_ORTHO_NESTEROV ? kOrthoNesterov : kOrthoMoment;
    call.mix = true, call.slot = slot, call.dtype = h->cfg.param_dtype, call.workspace = (char*)workspace, call.bytes = workspace_bytes;
    return run(h, call, hip_stream);
  });
}

}  // extern "C"
