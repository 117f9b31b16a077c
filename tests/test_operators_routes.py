"""Routes that the rules of the operators around the step can choose, on the GPU: every one against the oracle or, to the bit, against the
calls that say the same.  Tolerances as in tests/test_operators.py."""

import numpy as np
import pytest
import torch

from oracle import operators_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

import harness as H
from test_operators import DEV, EPS, TINY, Case, check_sums, csr_of, host, same, stored_of, stream

pytestmark = pytest.mark.gpu


def lists_of(rows, n):
    """n complete graphs side by side: rows / n rows that share each of n lists."""
    each = rows // n
    col = np.concatenate([np.arange(i // each * each, i // each * each + each) for i in range(rows)])
    return np.arange(0, rows * each + 1, each), col, np.full(rows * each, np.float32(1) / np.float32(each))


@pytest.mark.parametrize("layout", [515, "many", "gaps"])
@pytest.mark.parametrize("rows,lists", [(16, 1), (64, 4), (101, 1)])
def test_handles_with_little_lds_have_the_same_bits(rows, lists, layout):
    """Rounds without room for shared sums, products and gossip of rows that share their list without workgroups that form it."""
    csr = lists_of(rows, lists)
    messages = rows * (272 if rows <= 64 else 136)
    with Case(layout, rows, csr=csr, seed=rows) as c:
        x, copy, total, msg = c.values(0.02), c.values(0.02), c.values(0.02), c.random_messages(rows)
        results = []
        for limit in (0, messages):
            h = B.dadam_init(rows, rows, c.d, c.offsets, c.sizes, lds_limit_bytes=limit)
            B.dadam_set_topology(h, 0, *csr)
            s, k, y = [t.clone() for t in total], [t.clone() for t in copy], [t.clone() for t in x]
            B.dadam_mx4_round(h, 0, y, y, k, s, 0.6, stream())
            results.append(y + k + s)
            torch.cuda.synchronize()
            B.dadam_destroy(h)
        for limit in (0, 1024):
            h = B.dadam_init(rows, rows, c.d, c.offsets, c.sizes, lds_limit_bytes=limit)
            B.dadam_set_topology(h, 0, *csr)
            out, add, s, y = c.values(0.0), [t.clone() for t in total], [t.clone() for t in total], [t.clone() for t in x]
            B.dadam_mx4_product(h, 0, msg, out, 0, stream())
            B.dadam_mx4_product(h, 0, msg, add, B.DADAM_MX4_ADD, stream())
            B.dadam_mx4_gossip(h, 0, msg, s, copy, y, y, 0.6, stream())
            results.append(out + add + s + y)
            torch.cuda.synchronize()
            B.dadam_destroy(h)
        for a, b in ((results[0], results[1]), (results[2], results[3])):
            for p, q in zip(a, b):
                assert same(host(p), host(q))


def test_a_first_call_under_capture_leaves_the_capture_alone():
    """It is refused, and what was recorded before and behind it runs; after a first call outside, calls are recorded."""
    with Case("many", 4, csr=WL.ring(4)) as c:
        g, norms, mark = c.values(0.1), torch.zeros(4, device=DEV), torch.zeros(8, device=DEV)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            mark[:4] += 1
            with pytest.raises(B.DadamError) as e:
                B.dadam_grad_norm(c.h, g, norms, stream())
            mark[4:] += 2
        assert e.value.code == B.DADAM_ESTATE
        for k in range(1, 4):
            graph.replay()
            torch.cuda.synchronize()
            assert mark.tolist() == [k] * 4 + [2 * k] * 4 and not norms.any()
        B.dadam_grad_norm(c.h, g, norms, stream())
        torch.cuda.synchronize()
        want = norms.clone()
        again = torch.cuda.CUDAGraph()
        with torch.cuda.graph(again, stream=side):
            B.dadam_grad_norm(c.h, g, norms, stream())
        for _ in range(3):
            norms.zero_()
            again.replay()
            torch.cuda.synchronize()
            assert torch.equal(norms, want)
