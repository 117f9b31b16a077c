"""The loss of a language model's head by large tiles, several replicas in a launch (tests/test_ends_calls.py shows which kernels such calls launch), against its
statement in 64 bits (oracle/ends_oracle.py) for some of the replicas."""

import copy

import pytest
import torch
from test_head_loss import KINDS, SENTINEL, Head

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
