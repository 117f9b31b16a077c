"""The loss of a language model's head and its gradients on the GPU, through the C ABI, against their statement in 64 bits (oracle/ends_oracle.py, which
also derives how far the roundings may take every element: head_loss_error)."""

import numpy as np
import pytest
import torch

from oracle import ends_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
KINDS = {"f32": (B.DADAM_F32, torch.float32, 2.0 ** -24), "bf16": (B.DADAM_BF16, torch.bfloat16, 2.0 ** -8)}
SENTINEL = 7.0


def host(t):
    return t.detach().float().cpu().numpy()


class Head:
    """Rows with a head (and a bias) in packed vectors, hidden vectors, targets of which some are none, and everything a call writes, filled with SENTINEL."""

    def __init__(self, tokens, vocab, width, kind="f32", grad=None, rows=1, bias=False, seed=0, before=5, spread=1.0, device=0):
        self.tokens, self.vocab, self.width, self.kind, self.grad, self.rows, self.bias = tokens, vocab, width, kind, grad or kind, rows, bias
        sizes = [before, vocab * width] + ([vocab] if bias else []) + [3]
        offsets, at = [], 0
        for n in sizes:
            offsets.append(at)
            at += n + 1                                     # nothing is aligned
        self.d, self.at, self.bias_at = -(-at // 8) * 8, offsets[1], offsets[2]
        self.h = B.dadam_init(rows, rows, self.d, offsets, sizes, KINDS[kind][0], KINDS[self.grad][0], device=device)
        self.head = B.dadam_head(1, 2 if bias else B.DADAM_HEAD_NO_BIAS, vocab, width)
        rng = np.random.default_rng(seed)
        kt, gt = KINDS[kind][1], KINDS[self.grad][1]
        put = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV).to(t)  # noqa: E731
        x = np.full((rows, self.d), np.nan)
        x[:, self.at:self.at + vocab * width] = rng.standard_normal((rows, vocab * width)) * spread / np.sqrt(width)
        if bias:
            x[:, self.bias_at:self.bias_at + vocab] = rng.standard_normal((rows, vocab))
        self.x = put(x, kt)
        self.target = rng.integers(0, vocab, (rows, tokens)).astype(np.int32)
        self.target[rng.random((rows, tokens)) < 0.15] = -1
        hidden = 2 * rng.standard_normal((rows, tokens, width))
        hidden[self.target < 0] = np.nan                    # what takes no part may hold anything
        self.hidden = put(hidden, kt)
        self.y = torch.from_numpy(self.target).to(DEV)
        self.losses = torch.full((rows,), SENTINEL, device=DEV)
        self.nll = torch.full((rows, tokens), SENTINEL, device=DEV)
        self.dhidden = torch.full((rows, tokens, width), SENTINEL, device=DEV, dtype=kt)
        self.g = torch.full((rows, self.d), SENTINEL, device=DEV, dtype=gt)

    def info(self, gradient=True):
        return B.dadam_head_get_info(self.h, self.head, self.tokens, gradient)

    def workspace(self, n_bytes=None, gradient=True):
        w = torch.empty(self.info(gradient).bytes if n_bytes is None else n_bytes, dtype=torch.uint8, device=DEV)
        w.fill_(0xFF)
        return w

    def run(self, flags=B.DADAM_HEAD_MEAN, scale=1.0, gradient=True, nll=True, dhidden=True, grads=True, work=None):
        B.dadam_head_loss(self.h, self.head, self.x, self.hidden.flatten(1), self.y, self.tokens, scale, flags, self.losses, self.nll if nll else None,
                          self.dhidden.flatten(1) if gradient and dhidden else None, self.g if gradient and grads else None,
                          self.workspace(gradient=gradient) if work is None else work, B.current_stream())

    def expected(self, i, scale=1.0, mean=True):
        w = host(self.x[i, self.at:self.at + self.vocab * self.width]).reshape(self.vocab, self.width)
        b = host(self.x[i, self.bias_at:self.bias_at + self.vocab]) if self.bias else None
        r = O.head_loss(host(self.hidden[i]), w, b, self.target[i], scale, mean)
        planes = 1 if self.kind == self.grad == "bf16" else 2
        return r, O.head_loss_error(r, w, b, planes, KINDS[self.kind][2]), O.head_loss_error(r, w, b, planes, KINDS[self.grad][2])

    def check(self, scale=1.0, mean=True, before=None, gradient=True, dhidden=True, grads=True):
        """before: what the gradients held, where they were added to."""
        for i in range(self.rows):
            r, may, may_g = self.expected(i, scale, mean)
            near(self.losses[i], r["loss"], may["loss"], "loss")
            near(self.nll[i], r["nll"], may["nll"], "nll")
            if gradient and dhidden:
                near(self.dhidden[i], r["dhidden"], may["dhidden"], "dhidden")
            g, taken = host(self.g[i]), np.zeros(self.d, dtype=bool)
            parts = {"dhead": (self.at, self.vocab * self.width)} | ({"dbias": (self.bias_at, self.vocab)} if self.bias else {})
            for name, (at, n) in parts.items() if gradient and grads else ():
                old = 0 if before is None else host(before[i, at:at + n]).astype(np.float64)
                off = KINDS[self.grad][2] * np.abs(old)
                near(g[at:at + n], old + r[name].reshape(-1), may_g[name].reshape(-1) + 2 * off, name)
                taken[at:at + n] = True
            left = np.full(self.d, SENTINEL, dtype=np.float32) if before is None else host(before[i])
            assert np.array_equal(g[~taken], left[~taken], equal_nan=True), "gradients of other tensors were written"
            if not (gradient and dhidden):
                assert bool((self.dhidden == SENTINEL).all())

    def close(self):
        B.dadam_destroy(self.h)


def near(got, want, may, what):
    got = (host(got) if hasattr(got, "detach") else got).astype(np.float64)
    off = np.abs(got - want) - may
    assert np.isfinite(got).all() and (off <= 0).all(), f"{what}: off by {np.abs(got - want).max()}, beyond what may be by {off.max()} at {np.argmax(off)}"


SIZES = [(1, 2, 8), (1, 1, 1), (3, 7, 5), (17, 130, 33), (128, 64, 192), (129, 257, 64), (130, 1000, 128), (300, 129, 200), (64, 3001, 72)]


@pytest.mark.parametrize("kind,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_losses_and_gradients(tokens, vocab, width, kind, grad):
    for rows, bias in ((1, False), (3, True)):
        c = Head(tokens, vocab, width, kind, grad, rows, bias, seed=rows)
        c.run()
        c.check()
        c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_sums_added_gradients_and_single_outputs(kind):
    c = Head(40, 150, 70, kind, rows=2, bias=True, seed=5)
    before = torch.randn(c.g.shape, device=DEV).to(c.g.dtype)
    c.g.copy_(before)
    c.run(flags=B.DADAM_HEAD_ADD, scale=-0.5)
    c.check(scale=-0.5, mean=False, before=before)
    for kw in ({"dhidden": False}, {"grads": False}, {"gradient": False}):
        c.g.fill_(SENTINEL)
        c.dhidden.fill_(SENTINEL)
        c.run(**kw)
        c.check(**kw)
    c.losses.fill_(SENTINEL)
    c.nll.fill_(SENTINEL)
    c.run(nll=False, gradient=False)
    assert bool((c.nll == SENTINEL).all())
    near(c.losses, [c.expected(i)[0]["loss"] for i in range(2)], [c.expected(i)[1]["loss"] for i in range(2)], "loss")
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_small_workspaces(kind):
    """Pieces of the vocabulary and replicas one at a time: only the order of sums changes."""
    c = Head(150, 1111, 130, kind, rows=3, bias=True, seed=6)
    least, n = c.info().least_bytes, c.info().bytes
    assert least < n
    for n_bytes in (least, least + (n - least) // 7, n // 3, n - 256):
        if n_bytes < least:
            continue
        c.g.fill_(SENTINEL)
        c.run(work=c.workspace(n_bytes))
        c.check()
    c.g.fill_(SENTINEL)
    c.dhidden.fill_(SENTINEL)
    least = c.info(False).least_bytes
    assert least < c.info(False).bytes
    c.run(work=c.workspace(least), gradient=False)
    c.check(gradient=False)
    c.close()


def test_tokens_without_targets_and_no_tokens():
    c = Head(20, 40, 24, rows=2, seed=7)
    c.target[:] = -1
    c.target[1, 3:6] = 40, 41, 2 ** 31 - 1                  # beyond the vocabulary: none either
    c.y.copy_(torch.from_numpy(c.target))
    c.hidden.fill_(float("inf"))
    c.run()
    assert bool((c.losses == 0).all()) and bool((c.nll == 0).all()) and bool((c.dhidden == 0).all())
    assert bool((c.g[:, c.at:c.at + 40 * 24] == 0).all())
    c.close()
    c = Head(0, 40, 24, rows=2, seed=7)
    c.hidden, c.dhidden = c.hidden.new_zeros(2, 1, 24), c.hidden.new_zeros(2, 1, 24)
    c.y, c.nll = torch.zeros(2, 1, dtype=torch.int32, device=DEV), torch.full((2, 1), SENTINEL, device=DEV)
    c.run()
    assert bool((c.losses == 0).all()) and bool((c.nll == SENTINEL).all()) and bool((c.g[:, c.at:c.at + 40 * 24] == 0).all())
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_far_logits_words_that_cannot_come_and_certain_tokens(kind):
    c = Head(33, 300, 16, kind, bias=True, seed=8, spread=60.0)     # logits of hundreds
    c.x[:, c.bias_at + 1:c.bias_at + 200] = float("-inf")
    c.target[0][(c.target[0] > 0) & (c.target[0] < 200)] = 0
    c.y.copy_(torch.from_numpy(c.target))
    c.run()
    c.check()
    assert bool((c.g[:, c.bias_at + 1:c.bias_at + 200] == 0).all())
    c.close()


def test_a_nan_keeps_to_its_replica():
    c = Head(20, 50, 24, rows=3, seed=9)
    c.x[1, c.at + 7] = float("nan")
    c.run()
    assert bool(torch.isnan(c.losses[1])) and bool(torch.isnan(c.g[1, c.at:c.at + 50 * 24]).any())
    for i in (0, 2):
        r, may, _ = c.expected(i)
        near(c.losses[i], r["loss"], may["loss"], "loss")
        near(c.dhidden[i], r["dhidden"], may["dhidden"], "dhidden")
    c.close()


def test_more_replicas_than_a_launch_takes():
    c = Head(9, 33, 17, rows=40, seed=10)
    c.run()
    c.check()
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_against_differences(kind):
    """In float32 a difference over the loss, 64 bits summed, of single elements of the hidden vectors, the head and the bias."""
    c = Head(24, 60, 20, "f32", rows=1, bias=True, seed=11)
    c.run()
    taken = int(np.flatnonzero(c.target[0] >= 0)[0])
    spots = [(c.x, (0, c.at + 3 * 20 + 4), c.g), (c.x, (0, c.bias_at + 5), c.g), (c.hidden, (0, taken, 7), c.dhidden)]
    for data, spot, gradient in spots:
        slope, old, step, sums = float(gradient[spot]), data[spot].clone(), 2.0 ** -6, []
        for sign in (1, -1):
            data[spot] = old + sign * step
            r, _, _ = c.expected(0)
            sums.append(r["loss"])
        data[spot] = old
        difference = (sums[0] - sums[1]) / (2 * step)
        # third derivatives of the loss are below 1 times the cube of what multiplies the element (at most 10 here)
        assert abs(slope - difference) <= step ** 2 * 1000 / 6 * 0.1 + 1e-6
    c.close()


def test_recorded_into_a_graph():
    c = Head(70, 500, 64, "bf16", rows=2, bias=True, seed=12)
    work = c.workspace()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.run(work=work)
    for k in range(3):
        c.hidden.copy_(torch.randn(c.hidden.shape, device=DEV))
        c.run()
        eager = [t.clone() for t in (c.losses, c.nll, c.dhidden, c.g)]
        for t in (c.losses, c.nll, c.dhidden, c.g):
            t.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (c.losses, c.nll, c.dhidden, c.g)):
            assert torch.equal(a, b)
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [1, 30, 64])
def test_few_tokens_with_a_workspace_for_pieces_only(tokens, kind):
    """Up to 64 tokens have a way of their own, which a workspace of least_bytes does not allow where the vocabulary is long."""
    c = Head(tokens, 20011, 90, kind, rows=2, bias=True, seed=13)
    info = c.info()
    assert info.least_bytes < info.bytes
    for n_bytes in (info.bytes, info.bytes // 2, info.least_bytes):
        if n_bytes < info.least_bytes:
            continue
        c.g.fill_(SENTINEL)
        c.dhidden.fill_(SENTINEL)
        c.run(work=c.workspace(n_bytes))
        c.check()
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("share", [1.0, 0.4])
def test_large_tiles(kind, share):
    """As many words and tokens as make 256 large tiles, with what large tiles leave over; share: of the workspace that a call makes good use of."""
    c = Head(1024, 16400, 256, kind, bias=True, seed=14)
    work = c.workspace(int(c.info().bytes * share))
    c.run(work=work)
    c.check()
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_operands_as_they_lie_and_vectors_of_any_beginning(kind):
    """A head whose rows begin at multiples of 16 bytes and fill whole tiles, and hidden vectors that begin at an odd element."""
    c = Head(200, 384, 128, kind, rows=2, seed=15, before=7)       # (behind 7 elements and a gap of one)
    assert c.at % 8 == 0
    flat = torch.full((2, 200 * 128 + 1), SENTINEL, device=DEV, dtype=c.hidden.dtype)
    flat[:, 1:] = c.hidden.flatten(1)
    out = torch.full((2, 200 * 128 + 1), SENTINEL, device=DEV, dtype=c.hidden.dtype)
    B.dadam_head_loss(c.h, c.head, c.x, [v[1:] for v in flat], c.y, 200, 1.0, B.DADAM_HEAD_MEAN, c.losses, c.nll, [v[1:] for v in out], c.g, c.workspace(), B.current_stream())
    assert bool((out[:, 0] == SENTINEL).all())
    c.dhidden.copy_(out[:, 1:].view(2, 200, 128))
    c.check()
    c.close()


@pytest.mark.parametrize("tokens", [40, 300])
def test_two_calls_at_once_on_streams_of_their_own(tokens):
    """Two replicas' losses by two handles, each with a stream and a workspace."""
    cs = [Head(tokens, 900, 80, "bf16", bias=True, seed=16 + k) for k in range(2)]
    works = [c.workspace() for c in cs]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, w in zip(cs, works):
            with torch.cuda.stream(torch.cuda.Stream()):
                c.run(work=w)
    torch.cuda.synchronize()
    for c in cs:
        c.check()
        c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens,vocab,width", [(3053, 4, 8), (2113, 300, 72), (4096, 129, 130), (70001, 40, 8)])
def test_many_tokens_of_few_words(tokens, vocab, width, kind):
    """The head's gradient in parts of the tokens, written and added to."""
    c = Head(tokens, vocab, width, kind, rows=2, bias=True, seed=17)
    c.run()
    c.check()
    before = torch.randn(c.g.shape, device=DEV).to(c.g.dtype)
    c.g.copy_(before)
    c.run(flags=B.DADAM_HEAD_MEAN | B.DADAM_HEAD_ADD)
    c.check(before=before)
    c.close()
