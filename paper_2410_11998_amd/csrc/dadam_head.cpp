// Host side of a head's loss (include/dadam.h, "The ends of an iteration"): validation, how the vocabulary and the replicas go in pieces, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "dadam_checks.h"
#include "dadam_handle.h"
#include "dadam_head.h"

namespace dadam {
namespace {

constexpr uint32_t kMostWords = 1u << 24, kMostWidth = 65536, kMostTokens = 1u << 20;

uint32_t filled(uint32_t n, uint32_t each) { return std::max((n + each - 1) / each, 1u) * each; }

uint32_t planes_of(const dadam_handle* h) { return h->cfg.param_dtype == DADAM_BF16 && h->cfg.grad_dtype == DADAM_BF16 ? 1 : 2; }

int check_head(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens) {
  if (!head) return fail(h, DADAM_EINVAL, "head is null");
  if (!head->vocab || head->vocab > kMostWords) return fail(h, DADAM_EINVAL, "vocab must be 1 to %u", kMostWords);
  if (!head->width || head->width > kMostWidth) return fail(h, DADAM_EINVAL, "width must be 1 to %u", kMostWidth);
  if (n_tokens > kMostTokens) return fail(h, DADAM_EINVAL, "n_tokens must be at most %u", kMostTokens);
  if (head->tensor >= h->tensors.size()) return fail(h, DADAM_EINVAL, "the head's tensor %u is out of range", head->tensor);
  if (h->tensors[head->tensor].numel != (uint64_t)head->vocab * head->width) return fail(h, DADAM_EINVAL, "the head's tensor does not have vocab x width elements");
  if (head->bias_tensor == DADAM_HEAD_NO_BIAS) return DADAM_OK;
  if (head->bias_tensor == head->tensor) return fail(h, DADAM_EINVAL, "the head and its bias are the same tensor");  // (of width 1: their gradients would share elements)
  if (head->bias_tensor >= h->tensors.size()) return fail(h, DADAM_EINVAL, "the bias's tensor %u is out of range", head->bias_tensor);
  if (h->tensors[head->bias_tensor].numel != head->vocab) return fail(h, DADAM_EINVAL, "the bias's tensor does not have vocab elements");
  return DADAM_OK;
}

// How a call goes: words of a piece, replicas of a launch, parts of the sums over words.
struct Way {
  HeadShape s;
  uint32_t rows;
  uint64_t each;  // workspace of a replica
};

constexpr uint32_t kSplits = 64;               // at most
constexpr uint64_t kMostOfPiece = 1ull << 27;  // tokens times words of a piece
constexpr uint64_t kMostOfLaunch = 1ull << 37;  // and of a launch, whose threads are counted in 32 bits
constexpr uint64_t kMostKept = 1ull << 31;     // bytes of softmax that a replica may keep
constexpr uint64_t kMostAtOnce = 1ull << 31;   // bytes of workspace for which replicas are taken together
// Workgroups that the chip holds at a time: one large tile a compute unit, two small ones.
uint32_t at_once(uint32_t edge) { return edge == 256 ? 256 : 512; }

bool suits_large(uint32_t n) { return 8 * (uint64_t)filled(n, 256) <= 9 * (uint64_t)filled(n, 128); }

void fill_shape(const dadam_head* head, uint32_t n_tokens, uint32_t planes, uint32_t edge, uint32_t piece, HeadShape* s) {
  s->tokens = n_tokens;
  s->vocab = head->vocab;
  s->width = head->width;
  s->edge = edge;
  s->T = filled(n_tokens, edge);
  s->D = filled(head->width, edge);
  s->K = filled(head->width, 64);
  s->piece = std::min(piece, filled(head->vocab, edge));
  s->slices = filled(head->vocab, edge) / (edge / 2);
  s->keeps = 0;
  s->parts = 1;
  const uint64_t tiles = (uint64_t)(s->T / edge) * (s->D / edge), stages = (uint64_t)s->piece * planes / 64;
  s->splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(std::min<uint64_t>((at_once(edge) + tiles - 1) / tiles, stages / 8), kSplits));
}

Way good_way(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, bool gradient, bool keeps) {
  Way w{};
  const uint32_t planes = planes_of(h), V = head->vocab, R = std::min<uint32_t>(h->cfg.n_rows, kHeadRows);
  const uint64_t large = (uint64_t)(filled(V, 256) / 256) * (filled(n_tokens, 256) / 256) * R;
  const uint32_t edge = suits_large(n_tokens) && suits_large(head->width) && suits_large(V) && large >= 256 ? 256 : 128;
  const uint64_t across = filled(head->width, edge) / edge, down = filled(n_tokens, edge) / edge, all = filled(V, edge);
  uint64_t piece = std::min(all, std::max<uint64_t>(1, kMostOfLaunch / (down * edge) / edge) * edge);
  if (!keeps && gradient) {
    // pieces whose tiles, of the logits and of the head's gradient, are what the chip holds at a time or more
    piece = std::max<uint64_t>(1, at_once(edge) / std::min(across, down)) * edge;
    piece = std::max<uint64_t>(edge, std::min(piece, kMostOfPiece / (down * edge) / edge * edge));
    piece = std::min(piece, all);
  }
  // Replicas together, so that the last workgroups of a launch have company: tiles of one replica's head are 3.1 times what the chip holds (4 x 4096 tokens, 50257
  // words, width 1024), of four 12.3 times.
  fill_shape(head, n_tokens, planes, edge, (uint32_t)piece, &w.s);
  if (gradient && edge == 128) {
    // The head's gradient where its tiles are less than half of what there are compute units, and sum over 32 stages of tokens and more: in parts of eight and more (8824
    // tokens, 3387 words, width 108: 85 us in one, 25 in parts with their sum; 3053 tokens, 4 words, two replicas 69 / 14).
    const uint64_t tiles = R * all / 128 * across, stages = (uint64_t)w.s.T * planes / 64;
    if (2 * tiles <= 256 && stages >= 32) w.s.parts = (uint32_t)std::min<uint64_t>({256 / tiles, stages / 8, kSplits});
  }
  w.rows = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(R, kMostAtOnce / head_places(w.s, planes, gradient).bytes));
  w.s.keeps = keeps;
  w.each = head_places(w.s, planes, gradient).bytes;
  return w;
}

// Whether a replica's softmax is small enough to be kept.
bool may_keep(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, bool gradient) {
  return gradient && (uint64_t)filled(n_tokens, 256) * filled(head->vocab, 256) * 2 * planes_of(h) <= kMostKept;
}

Way least_way(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, bool gradient) {
  Way w{};
  w.rows = 1;
  fill_shape(head, n_tokens, planes_of(h), 128, 128, &w.s);
  w.each = head_places(w.s, planes_of(h), gradient).bytes;
  return w;
}

// Keeping softmax, or in pieces, or with fewer replicas at a time or smaller pieces where the workspace asks for it.
Way way_for(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, bool gradient, uint64_t bytes) {
  Way w{};
  if (may_keep(h, head, n_tokens, gradient)) w = good_way(h, head, n_tokens, gradient, true);
  if (w.rows == 0 || w.each > bytes) w = good_way(h, head, n_tokens, gradient, false);
  if (w.each <= bytes) {
    w.rows = (uint32_t)std::min<uint64_t>(w.rows, bytes / w.each);
    return w;
  }
  const uint32_t planes = planes_of(h);
  uint32_t low = 1, high = std::max(2u, w.s.piece / 128);  // small tiles of a piece: what fits, and what does not or need not
  while (low + 1 < high) {
    const uint32_t middle = (low + high) / 2;
    fill_shape(head, n_tokens, planes, 128, middle * 128, &w.s);
    (head_places(w.s, planes, gradient).bytes <= bytes ? low : high) = middle;
  }
  w.rows = 1;
  fill_shape(head, n_tokens, planes, 128, low * 128, &w.s);
  w.each = head_places(w.s, planes, gradient).bytes;
  return w;
}

// Few tokens: a wavefront sums a hidden vector's gradient over four blocks of words, or more where there are more than kFewItems of those, or as many as make the sums half
// of what is read of the head (57 tokens, 94661 words, width 512, five replicas: 799 / 654 us) if that leaves the chip kFewLeast.
constexpr uint64_t kFewItems = 4096, kFewLeast = 2048;
struct Few {
  FewShape s;
  uint32_t rows;
  uint64_t each;
};
Few few_way(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, bool gradient) {
  Few f{};
  f.s.tokens = n_tokens;
  f.s.vocab = head->vocab;
  f.s.width = head->width;
  f.s.T = filled(n_tokens, 32);
  f.s.D = filled(head->width, kFewColumns);
  f.s.blocks = (head->vocab + kFewWords - 1) / kFewWords;
  const uint64_t rows = std::min<uint32_t>(h->cfg.n_rows, kHeadRows);
  const uint64_t items = (uint64_t)f.s.blocks * (f.s.D / kFewColumns), by_tokens = n_tokens / (2 * dtype_bytes(h->cfg.param_dtype));
  f.s.each = (uint32_t)std::max<uint64_t>({4, (items + kFewItems - 1) / kFewItems, std::min(by_tokens, rows * items / kFewLeast)});
  f.s.ranges = (f.s.blocks + f.s.each - 1) / f.s.each;
  f.each = few_places(f.s, planes_of(h), gradient).bytes;
  f.rows = (uint32_t)std::max<uint64_t>(1, std::min(rows, kMostAtOnce / f.each));
  return f;
}
bool are_few(uint32_t n_tokens) { return n_tokens >= 1 && n_tokens <= kFewTokens; }

int run_few(const dadam_handle* h, const FewArgs& a, bool dhidden, bool gradient, uint32_t rows, void* stream) {
  const int x = (int)h->cfg.param_dtype, g = (int)h->cfg.grad_dtype;
  int e = launch_few_logits(x, g, a, rows, stream);
  if (!e) e = launch_few_losses(a, rows, stream);
  if (!e && gradient) e = launch_few_softmax(x, g, a, rows, stream);
  if (!e && gradient) e = launch_few_gradients(x, g, a, rows, stream);
  if (!e && dhidden) e = launch_few_end(x, g, a, rows, stream);
  return e;
}

// dW of a piece.  What large tiles there are beyond a multiple of what the chip holds go by small ones, if that takes less than one more round of large ones: three rounds
// and 72 small tiles instead of four (50257 words, width 1024).  Whole rows of tiles only, as a launch's words are: where one row of all replicas is more than the chip
// holds (32 replicas, width 2304: 288 tiles), a piece of one row stays whole.
int run_dhead(int x, int g, HeadArgs a, uint32_t rows, void* stream) {
  const uint32_t down = (a.words + a.s.edge - 1) / a.s.edge, tiles_of_word = a.s.D / a.s.edge * rows, tiles = down * tiles_of_word, over = tiles % at_once(a.s.edge);
  const uint32_t all = a.words, first = (tiles - over) / tiles_of_word * a.s.edge;
  if (a.s.parts > 1) return launch_head_dhead_parts(x, g, a, rows, stream);
  if (a.s.edge == 256 && first && over && over <= at_once(256) / 4) {
    a.words = first;
    if (const int e = launch_head_dhead(x, g, 256, a, rows, stream)) return e;
    a.skip = first;
    a.words = all;
    return launch_head_dhead(x, g, 128, a, rows, stream);
  }
  return launch_head_dhead(x, g, a.s.edge, a, rows, stream);
}

int run_rows(const dadam_handle* h, HeadArgs a, bool dhidden, bool dhead, bool dbias, uint32_t rows, void* stream) {
  const int x = (int)h->cfg.param_dtype, g = (int)h->cfg.grad_dtype;
  const bool gradient = dhidden || dhead;
  const uint32_t pieces = (a.s.vocab + a.s.piece - 1) / a.s.piece;
  auto piece = [&](uint32_t k) {
    a.first_word = k * a.s.piece;
    a.words = std::min(a.s.piece, a.s.vocab - a.first_word);
    a.later = k > 0;
  };
  a.groups = planes_of(h) == 2 ? head_most_groups(a) : 0;
  int e = a.groups ? launch_head_most(x, a, rows, stream) : (int)hipSuccess;
  for (uint32_t k = 0; k < pieces && !e; ++k) {
    piece(k);
    e = launch_head_operands(x, g, a, k == 0, rows, stream);
    a.groups = 0;
    if (!e) e = launch_head_logits(x, g, a.s.keeps ? kHeadKeep : kHeadStatistics, a, rows, stream);
  }
  if (!e) e = launch_head_losses(a, rows, stream);
  if (!gradient) return e;
  if (!e && a.s.keeps) e = launch_head_scale(x, g, a, rows, stream);
  for (uint32_t k = 0; k < pieces && !e; ++k) {
    piece(k);
    if (pieces > 1) e = launch_head_operands(x, g, a, false, rows, stream);
    if (!e && !a.s.keeps) e = launch_head_logits(x, g, kHeadGradient, a, rows, stream);
    if (!e && dhead) e = run_dhead(x, g, a, rows, stream);
    if (!e && dbias) e = launch_head_dbias(x, g, a, rows, stream);
    if (!e && dhidden) e = launch_head_dhidden(x, g, a, rows, stream);
  }
  if (!e && dhidden && a.s.tokens) e = launch_head_end(x, g, a, rows, stream);
  return e;
}

}  // namespace
}  // namespace dadam

extern "C" {

int dadam_head_get_info(const dadam_handle* h, const dadam_head* head, uint32_t n_tokens, uint32_t gradient, dadam_head_info* out) {
  if (!h) return DADAM_EINVAL;
  if (!out) return fail(h, DADAM_EINVAL, "out is null");
  if (const int rc = check_head(h, head, n_tokens)) return rc;
  out->least_bytes = least_way(h, head, n_tokens, gradient != 0).each;
  if (are_few(n_tokens)) {
    const Few f = few_way(h, head, n_tokens, gradient != 0);
    out->bytes = std::max(out->least_bytes, f.each * f.rows);
    return DADAM_OK;
  }
  const Way w = good_way(h, head, n_tokens, gradient != 0, may_keep(h, head, n_tokens, gradient != 0));
  out->bytes = std::max(out->least_bytes, w.each * w.rows);
  return DADAM_OK;
}

int dadam_head_loss(dadam_handle* h, const dadam_head* head, const void* const* params, const void* const* hidden, const int32_t* const* targets,
                    uint32_t n_tokens, float scale, uint32_t flags, float* losses, float* const* nll, void* const* dhidden, void* const* grads,
                    void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (!h) return DADAM_EINVAL;
  if (!params || !hidden || !targets) return fail(h, DADAM_EINVAL, "params, hidden or targets is null");
  if (!losses) return fail(h, DADAM_EINVAL, "losses is null");
  if ((uintptr_t)losses & 3u) return fail(h, DADAM_EALIGN, "losses is not 4-byte aligned");
  if (!std::isfinite(scale)) return fail(h, DADAM_EINVAL, "scale must be finite");
  if (flags & ~(DADAM_HEAD_MEAN | DADAM_HEAD_ADD)) return fail(h, DADAM_EINVAL, "unknown flag bits 0x%x", flags);
  return guarded(h, [&] {
    int rc = check_head(h, head, n_tokens);
    if (rc) return rc;
    const uint32_t R = h->cfg.n_rows, xs = (uint32_t)dtype_bytes(h->cfg.param_dtype), gs = (uint32_t)dtype_bytes(h->cfg.grad_dtype);
    const size_t vectors = (size_t)n_tokens * head->width * xs, values = (size_t)n_tokens * 4;
    const bool gradient = dhidden || grads;
    const uint64_t least = least_way(h, head, n_tokens, gradient).each;
    if (!workspace) return fail(h, DADAM_EINVAL, "workspace is null");
    if ((uintptr_t)workspace & 255u) return fail(h, DADAM_EALIGN, "workspace is not 256-byte aligned");
    if (workspace_bytes < least)
      return fail(h, DADAM_EINVAL, "workspace has %llu bytes, %llu are needed", (unsigned long long)workspace_bytes, (unsigned long long)least);
    const void* const one[1] = {workspace};
    const Table tables[7] = {{params, R, (size_t)h->cfg.d * xs, "params", false, -1},
                             {hidden, R, vectors, "hidden", false, -1, xs},
                             {(const void* const*)targets, R, values, "targets", false, -1, 4},
                             {(const void* const*)nll, nll ? R : 0, values, "nll", true, -1, 4},
                             {dhidden, dhidden ? R : 0, vectors, "dhidden", true, -1, xs},
                             {grads, grads ? R : 0, (size_t)h->cfg.d * gs, "grads", true, -1},
                             {one, 1, (size_t)workspace_bytes, "workspace", true, -1}};
    rc = check_tables(h, tables, 7);
    const uintptr_t lo = (uintptr_t)losses, hi = lo + 4 * R;
    for (const Table& t : tables)
      for (uint32_t i = 0; t.bytes && i < t.n && !rc; ++i)
        if (lo < (uintptr_t)t.p[i] + t.bytes && (uintptr_t)t.p[i] < hi) rc = fail(h, DADAM_EALIAS, "losses overlaps %s[%u]", t.name, i);
    if (!rc) rc = check_device(h);
    if (rc) return rc;
    const uint64_t at = h->tensors[head->tensor].offset_elems;
    const bool biased = head->bias_tensor != DADAM_HEAD_NO_BIAS;
    const uint64_t bias_at = biased ? h->tensors[head->bias_tensor].offset_elems : 0;
    auto fill = [&](auto* a, uint32_t i, uint32_t rows) {
      memset((void*)a, 0, sizeof(*a));
      a->workspace = (uint64_t)(uintptr_t)workspace;
      a->losses = losses + i;
      a->scale = scale;
      a->mean = (flags & DADAM_HEAD_MEAN) != 0;
      a->add = (flags & DADAM_HEAD_ADD) != 0;
      for (uint32_t r = 0; r < rows; ++r) {
        HeadRow& row = a->row[r];
        row.head = (uint64_t)(uintptr_t)params[i + r] + at * xs;
        row.bias = biased ? (uint64_t)(uintptr_t)params[i + r] + bias_at * xs : 0;
        row.hidden = (uint64_t)(uintptr_t)hidden[i + r];
        row.target = (uint64_t)(uintptr_t)targets[i + r];
        row.nll = nll ? (uint64_t)(uintptr_t)nll[i + r] : 0;
        row.dhidden = dhidden ? (uint64_t)(uintptr_t)dhidden[i + r] : 0;
        row.dhead = grads ? (uint64_t)(uintptr_t)grads[i + r] + at * gs : 0;
        row.dbias = grads && biased ? (uint64_t)(uintptr_t)grads[i + r] + bias_at * gs : 0;
      }
    };
    DeviceGuard guard(h->cfg.device);
    if (guard.err != hipSuccess) return fail(h, DADAM_EHIP, "hipSetDevice: %s", hipGetErrorString(guard.err));
    int e = (int)hipSuccess;
    const Few few = are_few(n_tokens) ? few_way(h, head, n_tokens, gradient) : Few{};
    if (are_few(n_tokens) && few.each <= workspace_bytes) {
      const uint32_t together = (uint32_t)std::min<uint64_t>(few.rows, workspace_bytes / few.each);
      for (uint32_t i = 0; i < R && !e; i += together) {
        const uint32_t rows = std::min(together, R - i);
        FewArgs a;
        fill(&a, i, rows);
        a.s = few.s;
        a.w = few_places(few.s, planes_of(h), gradient);
        a.stride = few.each;
        e = run_few(h, a, dhidden != nullptr, gradient, rows, hip_stream);
      }
    } else {
      const Way way = way_for(h, head, n_tokens, gradient, workspace_bytes);
      for (uint32_t i = 0; i < R && !e; i += way.rows) {
        const uint32_t rows = std::min(way.rows, R - i);
        HeadArgs a;
        fill(&a, i, rows);
        a.s = way.s;
        a.w = head_places(way.s, planes_of(h), gradient);
        a.stride = way.each;
        a.n_xcd = h->n_xcds;
        a.straight = planes_of(h) == 1 && head->width == way.s.D && at * xs % 16 == 0;
        e = run_rows(h, a, dhidden != nullptr, grads != nullptr, grads && biased, rows, hip_stream);
      }
    }
    if (e != (int)hipSuccess) return fail(h, DADAM_EHIP, "kernel launch failed: %s", hipGetErrorString((hipError_t)e));
    return DADAM_OK;
  });
}

}  // extern "C"
