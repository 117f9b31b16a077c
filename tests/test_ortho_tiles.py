"""Orthogonalised updates by large tiles (tests/test_ends_calls.py shows which kernels these calls launch)."""

import pytest
import torch
from test_ends_calls import LARGE
from test_ortho import DEV, SENTINEL, TYPES, Layout, on_device

from paper_2410_11998_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", LARGE)
def test_large_and_small_tiles_give_the_same_bits(name, kind):
    """A and B by large tiles, and with less workspace by small ones."""
    L = Layout(LARGE[name], kind, rows=4)
    g = on_device(L.random(22), kind)
    mask = torch.from_numpy(L.mask()).to(DEV)
    outs = []
    for n_bytes in (L.info.bytes, L.info.bytes // 5, L.info.least_bytes):
        outs.append(torch.full_like(g, SENTINEL))
        B.dadam_orthogonalize(L.h, g, outs[-1], L.workspace(n_bytes), B.current_stream())
    for o in outs[1:]:
        assert torch.equal(o[:, mask], outs[0][:, mask])
    L.close()
