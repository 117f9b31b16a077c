"""The loss of a language model's head by large tiles, several replicas in a launch (tests/test_ends_calls.py shows which kernels such calls launch), against its
statement in 64 bits (oracle/ends_oracle.py) for some of the replicas."""

import copy

import pytest
from test_head_loss import KINDS, Head

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
