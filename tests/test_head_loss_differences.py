"""Gradients of the head's loss against differences of the loss's statement in 64 bits, where they are large."""

import numpy as np
import pytest
from test_head_loss import Head, host

from oracle import ends_oracle as O

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -14


@pytest.mark.parametrize("kind,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens", [24, 100])
def test_gradients_against_differences(tokens, kind, grad):
    """The elements with the largest gradients, and the target's word and bias of a token: by up to 64 tokens' way and by tiles."""
    vocab, width = 60, 20
    c = Head(tokens, vocab, width, kind, grad, bias=True, seed=25)
    c.run(flags=0)
    w = host(c.x[0, c.at:c.at + vocab * width]).astype(np.float64).reshape(vocab, width)
    bias, hidden = host(c.x[0, c.bias_at:c.bias_at + vocab]).astype(np.float64), np.nan_to_num(host(c.hidden[0]).astype(np.float64))
    _, may, may_g = c.expected(0, mean=False)
    got = {"hidden": host(c.dhidden[0]), "head": host(c.g[0, c.at:c.at + vocab * width]).reshape(vocab, width), "bias": host(c.g[0, c.bias_at:c.bias_at + vocab])}
    bounds, data = {"hidden": may["dhidden"], "head": may_g["dhead"], "bias": may_g["dbias"]}, {"hidden": hidden, "head": w, "bias": bias}
    loss = lambda: O.head_loss(hidden, w, bias, c.target[0], 1.0, False)["loss"]  # noqa: E731
    # a token's loss's third derivative is at most 1 times the cube of what multiplies the element; nothing else of the statement's difference counts beside
    # its roundings, 2^-50 of a loss of some hundreds over 2 steps
    largest = {"hidden": np.abs(w).max(), "head": np.abs(hidden).max(), "bias": 1.0}
    some = int(np.flatnonzero(c.target[0] >= 0)[0])
    spots = {"hidden": [(some, 7)], "head": [(int(c.target[0, some]), 3)], "bias": [(int(c.target[0, some]),)]}
    for name, x in data.items():
        spots[name] += [np.unravel_index(k, x.shape) for k in np.argsort(-np.abs(got[name]), axis=None)[:3]]
        for spot in spots[name]:
            old, sums = x[spot], []
            for sign in (1, -1):
                x[spot] = old + sign * STEP
                sums.append(loss())
            x[spot] = old
            difference = (sums[0] - sums[1]) / (2 * STEP)
            allowed = STEP ** 2 / 6 * tokens * largest[name] ** 3 + 2.0 ** -50 * 1000 / STEP + bounds[name][spot]
            assert abs(got[name][spot] - difference) <= allowed, f"{name} {spot}: {got[name][spot]} and {difference}, may differ by {allowed}"
        top = spots[name][1]
        assert abs(got[name][top]) >= 20 * (allowed - bounds[name][spot] + bounds[name][top]), f"{name}: {got[name][top]} shows nothing beside {allowed}"
    c.close()
