"""Values of orthogonalised updates on the GPU, both types, to a small multiple of what their operands' bits cost.

The tolerance is three times oracle/ends_oracle.py's orthogonalised_spread (the largest of four draws of the roundings, in the 2-norm: a fifth draw, the library's, differs
from these by what a sum of so many roundings differs from another), half a step of the result's type, and, as held operands that meet a step's middle may round either way,
2^-21 of the result in 32 bits.  test_tolerances_are_small needs no GPU: outputs of zeros, of the other sign, without one of the three products of 32-bit operands or with the
moment in the place of what looks ahead of it are not within them."""

import numpy as np
import pytest
import torch
from test_ends_calls import LARGE
from test_ortho import DEV, SENTINEL, SHAPES, TYPES, Layout, Step, host, on_device, view

from oracle import ends_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

gpu = pytest.mark.gpu
MANY = {**{k: [(170, 230)] + v for k, v in SHAPES.items()},           # (beside the first, small ones go by tiles)
        "long": [(5, 6759), (130, 8200), (2500, 300), (1, 5000)], "fit a compute unit": [(32, 960), (64, 416), (400, 60), (96, 320), (128, 160), (1, 1), (9, 7)]}


def planes_of(shapes, kind):
    """Layouts of matrices that each fit a compute unit are held in two halves whatever the result's type."""
    return 2 if kind == "f32" or shapes is MANY["fit a compute unit"] else 1


def direction_tolerance(u, planes):
    """Rows of few elements have too few roundings for one draw to tell of another: theirs are bounded one by one (3.5e-5 of the result in 32 bits, 9.4e-3 in bfloat16)."""
    spread = 3 * O.orthogonalised_spread(u, planes)
    return max(spread, O.orthogonalised_error_of_a_row(u, planes)) if min(u.shape) == 1 and u.size <= 64 else spread


def tolerance(u, want, planes, kind):
    n = np.linalg.norm(want)
    return direction_tolerance(u, planes) + TYPES[kind][2] * n + 2.0 ** -21 * n


def random_matrix(seed, r, c):
    rng = np.random.default_rng(seed)
    k = max(1, min(r, c) // 4)
    return (rng.standard_normal((r, k)) * 2.0 ** -(np.arange(k) * 6.0 / k) @ rng.standard_normal((k, c)) / np.sqrt(k) + 0.2 * rng.standard_normal((r, c))).astype(np.float32)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", MANY)
def test_tolerances_are_small(name, kind):
    planes = planes_of(MANY[name], kind)
    for shape in MANY[name]:
        r, c = shape[0], shape[1] // (shape[2] if len(shape) > 2 else 1)
        m = random_matrix(1, r, c)
        want = O.orthogonalised(m)
        may, size = tolerance(m, want, planes, kind), np.linalg.norm(want)
        assert may <= (4e-5 if kind == "f32" else 2e-2) * size, (shape, may / size)
        if min(r, c) > 1:
            looked_ahead = O.orthogonalised(0.9 * m + 0.1 * random_matrix(2, r, c))
            assert np.linalg.norm(looked_ahead - want) > may
            if planes == 2 and kind == "f32":
                assert np.linalg.norm(O.orthogonalised_with_roundings(m, 1) - want) > may


def check(L, given, got, kind, planes, every=1):
    for i in range(L.rows):
        for m in L.matrices[i % every::every]:
            a = view(given[i], L.offsets, m)
            want = O.orthogonalised(a)
            off, may = np.linalg.norm(view(got[i], L.offsets, m) - want), tolerance(a, want, planes, kind)
            assert off <= may, f"row {i} matrix {m}: off by {off}, may be {may} (norm {np.linalg.norm(want)})"


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", MANY)
def test_matrices(name, kind):
    L = Layout(MANY[name], kind, rows=2, gap=3)
    assert (L.info.bytes == 0) == (name == "fit a compute unit")
    g = on_device(L.random(31), kind)
    out = torch.full_like(g, SENTINEL)
    B.dadam_orthogonalize(L.h, g, out, L.workspace() if L.info.bytes else (0, 0), B.current_stream())
    check(L, host(g), host(out), kind, planes_of(MANY[name], kind))
    L.close()


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", LARGE)
def test_matrices_by_large_tiles(name, kind):
    """All products by large tiles, and A and B by small ones."""
    L = Layout(LARGE[name], kind, rows=4)
    g = on_device(L.random(32), kind)
    for n_bytes in (L.info.bytes, L.info.bytes // 5):
        out = torch.full_like(g, SENTINEL)
        B.dadam_orthogonalize(L.h, g, out, L.workspace(n_bytes), B.current_stream())
        check(L, host(g), host(out), kind, planes_of(LARGE[name], kind), every=9)
    L.close()


STEPS = {"held": ([(40, 72), (72, 40), (96, 120), (1, 17), (128, 100)], 1), "tiles": ([(170, 230), (40, 72), (131, 65), (96, 288, 3), (1, 17)], 1), "large": (LARGE["512"], 9)}


@gpu
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("kind,grad", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("name", STEPS)
def test_directions_of_steps(name, kind, grad, nesterov):
    """From parameters of zero a step is its direction, to the bits of the parameters' type; then from parameters like those, mixed over a ring, with weight decay."""
    shapes, every = STEPS[name]
    planes = 2 if kind == "f32" or name == "held" else 1
    L = Layout(shapes, kind, rows=4, csr=WL.ring(4), grad=grad, lr=0.5, beta1=0.9, weight_decay=[0.25] * len(shapes))
    S = Step(L, 33, 0.5, 0.9, 1, WL.ring(4), 4, 0.25)
    flags = B.DADAM_FUSE_ACCUM | (B.DADAM_ORTHO_NESTEROV if nesterov else 0)
    be, (rp, col, w) = S.beta, S.csr
    S.bind()
    for turn in range(2):
        if turn:
            S.x.copy_(torch.randn(S.x.shape, generator=torch.Generator().manual_seed(5)).to(S.x) * 0.02)
        else:
            S.x.zero_()
        g = on_device(L.random(34 + turn), grad)
        m0, x0 = S.m.cpu().numpy().astype(np.float64), host(S.x).astype(np.float64)
        B.dadam_ortho_step(L.h, 0, g, turn + 1, flags, L.workspace() if L.info.bytes else (0, 0), B.current_stream())
        x, given = host(S.out), host(g).astype(np.float64)
        for i in range(4):
            for mat in L.matrices[i % every::every]:
                gi, mi = view(given[i], L.offsets, mat), view(m0[i], L.offsets, mat)
                u = be * mi + (1 - be) * gi
                u = be * u + (1 - be) * gi if nesterov else u
                direction = O.orthogonalised(u)
                mixed = sum(float(w[k]) * view(x0[col[k]], L.offsets, mat) for k in range(rp[i], rp[i + 1]))
                size = sum(float(w[k]) * np.abs(view(x0[col[k]], L.offsets, mat)) for k in range(rp[i], rp[i + 1]))
                want = mixed - 0.5 * (mat[5] * direction + 0.25 * view(x0[i], L.offsets, mat))
                # the direction's operands as above; u itself has some four roundings of 2^-24, as orthogonalised_spread's copies of it have
                n = np.linalg.norm
                may = 0.5 * abs(mat[5]) * (direction_tolerance(u, planes) + 2.0 ** -21 * n(direction)) + 8 * 2.0 ** -24 * n(size + np.abs(want)) + TYPES[kind][2] * n(want)
                off = n(view(x[i], L.offsets, mat) - want)
                assert off <= may, f"turn {turn} row {i} matrix {mat}: off by {off}, may be {may} (norm {n(want)})"
    L.close()
