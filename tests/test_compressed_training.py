"""The example of clipped, 4-bit gossip training: it learns as the same run with whole parameters mixed does, and its replicas stay together."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_with_4_bit_gossip_learns_as_exact_mixing_does():
    spec = importlib.util.spec_from_file_location("compressed_training", os.path.join(ROOT, "examples", "compressed_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got, apart = example.train(steps=150)
    exact, apart_exact = example.train(steps=150, exact=True)
    first, last, last_exact = got[0], sum(got[-20:]) / 20, sum(exact[-20:]) / 20
    print("loss", first, "->", last, "exact", last_exact, "apart", apart, apart_exact, flush=True)
    assert abs(first - exact[0]) < 1e-5
    assert last < 0.9 * first and abs(last - last_exact) < 0.05 * first
    assert apart < 0.3
