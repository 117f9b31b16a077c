"""The loss of a language model's head by large tiles, several replicas in a launch (tests/test_ends_calls.py shows which kernels such calls launch), against its
statement in 64 bits (oracle/ends_oracle.py) for some of the replicas."""

import copy

import numpy as np
import pytest
import torch
from test_ends_calls import LOSSES
from test_head_loss import KINDS, SENTINEL, Head, host

from paper_2410_11998_amd import binding as B

pytestmark = pytest.mark.gpu


def check_some(c, replicas, before=None, **kw):
    for i in replicas:
        one = copy.copy(c)
        one.rows, one.target = 1, c.target[i:i + 1]
        one.x, one.hidden, one.losses, one.nll, one.dhidden, one.g = (t[i:i + 1] for t in (c.x, c.hidden, c.losses, c.nll, c.dhidden, c.g))
        one.check(before=None if before is None else before[i:i + 1], **kw)


@pytest.mark.parametrize("kind", KINDS)
def test_a_vocabulary_of_one_row_of_tiles(kind):
    """288 large tiles of the head's gradient in one row of all replicas, 32 more than the chip holds at a time."""
    c = Head(2048, 256, 2304, kind, rows=32, seed=21)
    c.run()
    check_some(c, (0, 17, 31))
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", LOSSES)
def test_losses_by_large_tiles(name, kind):
    (rows, tokens, vocab, width, at, share, gradient), _, _ = LOSSES[name]
    c = Head(tokens, vocab, width, kind, rows=rows, bias=True, seed=24, before=at - 1)
    assert c.at == at
    work = c.workspace(max(c.info(gradient).least_bytes, c.info(gradient).bytes * share // 100))
    c.run(gradient=gradient, work=work)
    some = sorted({0, rows // 2, rows - 1})
    check_some(c, some, gradient=gradient)
    if gradient:
        before = torch.randn(c.g.shape, device=c.g.device).to(c.g.dtype)
        c.g.copy_(before)
        c.run(flags=B.DADAM_HEAD_MEAN | B.DADAM_HEAD_ADD, work=work)
        check_some(c, some[:1], before=before)
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_no_tokens_in_empty_tensors(kind):
    c = Head(0, 40, 24, kind, rows=2, bias=True, seed=7)
    assert c.hidden.data_ptr() == 0
    c.run()
    assert bool((c.losses == 0).all())
    for at, n in ((c.at, 40 * 24), (c.bias_at, 40)):
        assert bool((c.g[:, at:at + n] == 0).all())
        c.g[:, at:at + n] = SENTINEL
    assert bool((c.g == SENTINEL).all())
    c.hidden, c.dhidden = list(c.hidden), list(c.dhidden)
    B.dadam_head_loss(c.h, c.head, c.x, c.hidden, list(c.y), 0, 1.0, 0, c.losses, list(c.nll), c.dhidden, c.g, c.workspace(), B.current_stream())
    assert bool((c.losses == 0).all()) and bool((c.g[:, c.at:c.at + 40 * 24] == 0).all())
    torch.cuda.synchronize()
    c.close()


def lone_token(vocab, width, tokens=65):
    """float32, one token with a target (word 0), and zeros for its hidden vector and the head."""
    c = Head(tokens, vocab, width, "f32", seed=23)
    c.target[:] = -1
    c.target[0, 0] = 0
    c.y.copy_(torch.from_numpy(c.target))
    c.hidden[0, 0] = 0
    head = c.x[0, c.at:c.at + vocab * width].view(vocab, width)
    head.zero_()
    return c, head


def run_within(c, share):
    info = c.info()
    c.run(flags=0, work=c.workspace(info.bytes if share else info.least_bytes))
    return host(c.g[0, c.at:c.at + c.vocab * c.width]).astype(np.float64).reshape(c.vocab, c.width), host(c.dhidden[0, 0]).astype(np.float64)


SHARES = pytest.mark.parametrize("share", [1, 0], ids=["kept", "pieces"])


@SHARES
def test_softmax_is_held_to_a_small_part_of_1(share):
    """Words of probabilities of 2^-38 to 2^-30: their rows of the head's gradient are off by 2^-39 and by what their logits' roundings make of them, 30 * 2^-21 of
    the probability twice."""
    c, head = lone_token(300, 8)
    z = -np.log(2) * np.random.default_rng(1).uniform(30, 38, 300).astype(np.float32)
    z[0] = 0
    c.hidden[0, 0, 0] = 1
    head[:, 0] = torch.from_numpy(z).to(head)
    got, _ = run_within(c, share)
    p = np.exp(z.astype(np.float64))
    p /= p.sum()
    may = 2.0 ** -39 + 60 * 2.0 ** -21 * p
    off = np.abs(got[1:, 0] - p[1:])
    assert (off <= may[1:]).all(), np.max(off / may[1:])
    c.close()


@SHARES
@pytest.mark.parametrize("side", ["hidden", "head"])
def test_operands_are_held_to_a_small_part_of_the_largest(side, share):
    """Elements of 2^-37 to 2^-26 of the largest: held to 2^-39 of it or 2^-22 of themselves; what they are multiplied by is 1/2 to within 2^-20."""
    c, head = lone_token(2, 64)
    rng = np.random.default_rng(2)
    v = (rng.choice([-1, 1], 64) * 2.0 ** -rng.uniform(26, 37, 64)).astype(np.float32)
    v[0] = 1
    if side == "hidden":
        c.hidden[0, 0] = torch.from_numpy(v).to(c.hidden)
    else:
        head[1] = torch.from_numpy(v).to(head)
    dhead, dhidden = run_within(c, share)
    got = dhead[1] if side == "hidden" else dhidden
    may = 0.5 * (2.0 ** -39 + (2.0 ** -22 + 2.0 ** -19 + 2.0 ** -23) * np.abs(v))
    off = np.abs(got - 0.5 * v)
    assert (off <= may).all(), np.max(off / may)
    c.close()
