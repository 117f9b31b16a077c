"""Refusals of the head's loss and of orthogonalised updates, on a host-only handle: every call is validated as on a device handle, and one that passes is
refused for want of a device.  Addresses are numbers; nothing is touched."""

import ctypes as C

import numpy as np
import pytest

from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

ROWS, VOCAB, WIDTH, TOKENS = 3, 100, 24, 7
SIZES = [VOCAB * WIDTH, VOCAB, 40 * 30, 200 * 300]
OFFSETS = [0, 2400, 2504, 3704]
D = 63704
HEAD = B.dadam_head(0, 1, VOCAB, WIDTH)
STEP = 1 << 18
NAN = float("nan")


def handle(**kw):
    h = B.dadam_init(ROWS, ROWS, D, OFFSETS, SIZES, device=B.DADAM_DEVICE_NONE, **kw)
    B.dadam_set_topology(h, 0, *WL.ring(ROWS))
    return h


def code(call):
    try:
        call()
    except B.DadamError as e:
        return e.code
    return B.DADAM_OK


def addresses(n, base):
    return [base + k * STEP for k in range(n)]


class Loss:
    """The arguments of a sound call, any of which a test changes."""

    def __init__(self, h):
        self.h, self.head, self.n, self.scale, self.flags = h, HEAD, TOKENS, 1.0, B.DADAM_HEAD_MEAN
        self.params, self.hidden, self.targets, self.nll, self.dhidden, self.grads = (addresses(ROWS, (k + 1) << 24) for k in range(6))
        self.losses = 7 << 24
        self.workspace = (8 << 24, 1 << 22)

    def code(self, **change):
        c = Loss(self.h)
        for k, v in change.items():
            setattr(c, k, v)
        return code(lambda: B.dadam_head_loss(c.h, c.head, c.params, c.hidden, c.targets, c.n, c.scale, c.flags, c.losses, c.nll, c.dhidden, c.grads, c.workspace))


def test_sound_losses_are_refused_for_want_of_a_device_only():
    h = handle()
    c = Loss(h)
    for change in ({}, {"nll": None}, {"dhidden": None}, {"grads": None}, {"dhidden": None, "grads": None}, {"flags": 0}, {"flags": 3}, {"scale": -0.5}, {"n": 0}, {"n": 1},
                   {"head": B.dadam_head(0, B.DADAM_HEAD_NO_BIAS, VOCAB, WIDTH)},
                   {"hidden": [x + 4 for x in c.hidden]}, {"targets": [x + 4 for x in c.targets]}, {"hidden": [c.hidden[0]] * ROWS, "targets": [c.targets[0]] * ROWS}):
        assert c.code(**change) == B.DADAM_ESTATE, change
    B.dadam_destroy(h)


def test_heads_and_scalars():
    h = handle()
    c = Loss(h)
    for head in (B.dadam_head(4, 1, VOCAB, WIDTH), B.dadam_head(0, 4, VOCAB, WIDTH), B.dadam_head(0, 1, VOCAB + 1, WIDTH), B.dadam_head(0, 1, VOCAB, WIDTH + 1), B.dadam_head(0, 0, VOCAB, WIDTH),
                 B.dadam_head(0, 2, VOCAB, WIDTH), B.dadam_head(0, 1, 0, WIDTH), B.dadam_head(0, 1, VOCAB, 0), B.dadam_head(0, 1, 2 ** 24 + 1, WIDTH), B.dadam_head(0, 1, VOCAB, 65537)):
        assert c.code(head=head) == B.DADAM_EINVAL, (head.tensor, head.bias_tensor, head.vocab, head.width)
        assert code(lambda: B.dadam_head_get_info(h, head, TOKENS, True)) == B.DADAM_EINVAL
    assert c.code(n=2 ** 20 + 1) == B.DADAM_EINVAL
    assert code(lambda: B.dadam_head_get_info(h, HEAD, 2 ** 20 + 1, True)) == B.DADAM_EINVAL
    for change in ({"scale": NAN}, {"scale": float("inf")}, {"flags": 4}, {"flags": B.DADAM_FUSE_ACCUM << 8}, {"losses": 0}):
        assert c.code(**change) == B.DADAM_EINVAL, change
    B.dadam_destroy(h)


def test_null_misaligned_and_overlapping_buffers_of_a_loss():
    h = handle()
    c = Loss(h)
    for name in ("params", "hidden", "targets"):
        assert c.code(**{name: None}) == B.DADAM_EINVAL
    for name in ("params", "hidden", "targets", "nll", "dhidden", "grads"):
        good = getattr(c, name)
        assert c.code(**{name: [good[0], 0, good[2]]}) == B.DADAM_EINVAL, name
        assert c.code(**{name: [good[0], good[1] + 2, good[2]]}) == B.DADAM_EALIGN, name
        assert c.code(**{name: [good[0], 2 ** 64 - 64, good[2]]}) != B.DADAM_ESTATE, name
        assert c.code(losses=good[1]) == B.DADAM_EALIAS, name
        assert c.code(workspace=(good[1] // 256 * 256, 1 << 22)) == B.DADAM_EALIAS, name
    for name in ("params", "grads"):
        assert c.code(**{name: [x + 4 for x in getattr(c, name)]}) == B.DADAM_EALIGN
    for written in ("nll", "dhidden", "grads"):
        for other in ("params", "hidden", "targets", "nll", "dhidden", "grads"):
            if other != written:
                assert c.code(**{written: getattr(c, other)}) == B.DADAM_EALIAS, (written, other)
        good = getattr(c, written)
        assert c.code(**{written: [good[0], good[0], good[2]]}) == B.DADAM_EALIAS
    assert c.code(losses=c.losses + 2) == B.DADAM_EALIGN and c.code(losses=c.workspace[0] + 64) == B.DADAM_EALIAS
    B.dadam_destroy(h)


@pytest.mark.parametrize("tokens", [0, 1, 7, 64, 65, 5000])
def test_workspaces_of_a_loss(tokens):
    h = handle()
    c = Loss(h)
    wide = {k: [(40 + 8 * j + i) << 24 for i in range(ROWS)] for j, k in enumerate(("hidden", "dhidden", "targets", "nll"))}
    for gradient in (True, False):
        info = B.dadam_head_get_info(h, HEAD, tokens, gradient)
        assert 0 < info.least_bytes <= info.bytes
        change = dict(wide, n=tokens) if gradient else dict(wide, n=tokens, dhidden=None, grads=None)
        for n_bytes in (info.least_bytes, info.bytes, info.bytes + 77):
            assert c.code(workspace=(1 << 40, n_bytes), **change) == B.DADAM_ESTATE
        assert c.code(workspace=(1 << 40, info.least_bytes - 1), **change) == B.DADAM_EINVAL
        assert c.code(workspace=(0, info.bytes), **change) == B.DADAM_EINVAL
        assert c.code(workspace=((1 << 40) + 128, info.bytes), **change) == B.DADAM_EALIGN
    B.dadam_destroy(h)


GOOD = [(2, 40, 30), (3, 200, 100, 300, 0, 2.0), (3, 200, 100, 300, 100), (3, 200, 100, 300, 200, -1.0)]


def test_matrices():
    h = handle()
    assert code(lambda: B.dadam_ortho_get_info(h)) == B.DADAM_ESTATE
    for bad in ([(4, 2, 2)], [(2, 41, 30)], [(2, 40, 31)], [(2, 0, 30)], [(2, 40, 0)], [(2, 65537, 1, 1)], [(2, 1, 65537)], [(2, 40, 30, 29)], [(2, 40, 30, 30, 1)], [(2, 39, 30, 30, 31)],
                [(2, 1, 1, 1, 1200)], [(2, 1, 1, 1, 2 ** 63)], [(3, 200, 100, 300, 201)], [(2, 40, 30, 30, 0, NAN)], [(2, 40, 30, 30, 0, float("inf"))],
                [(2, 40, 30), (2, 1, 1)], [(3, 200, 100, 300, 0), (3, 200, 100, 300, 99)], [(2, 20, 30), (2, 20, 30, 30, 570)], [(3, 200, 100, 300, 0), (3, 2, 48, 48, 96)],
                [B.dadam_matrix_desc(2, 40, 30, 30, 0, 1.0, 1)]):
        assert code(lambda: B.dadam_set_matrices(h, bad)) == B.DADAM_EINVAL, bad
    B.dadam_set_matrices(h, GOOD)
    info = B.dadam_ortho_get_info(h)
    assert info.n_matrices == 4 and 0 < info.least_bytes <= info.bytes
    assert code(lambda: B.dadam_set_matrices(h, [(4, 2, 2)])) == B.DADAM_EINVAL
    assert B.dadam_ortho_get_info(h).n_matrices == 4                       # a refused set leaves the last one
    B.dadam_set_matrices(h, [(3, 200, 300), (2, 20, 30), (2, 20, 30, 30, 600)])
    B.dadam_set_matrices(h, [])
    assert B.dadam_ortho_get_info(h).n_matrices == 0 and B.dadam_ortho_get_info(h).bytes == 0
    assert B.lib.dadam_set_matrices(h, None, 1) == B.DADAM_EINVAL and B.lib.dadam_set_matrices(h, None, 65537) == B.DADAM_EINVAL
    B.dadam_destroy(h)


def test_schedules():
    h = handle()
    for bad in ([], [(1.0, 0.0, 0.0)] * 17, [(NAN, 0.0, 0.0)], [(1.0, float("inf"), 0.0)], [(2000.0, 0.0, 0.0)], [(40.0, 0.0, 0.0)] * 2):
        assert code(lambda: B.dadam_set_ortho_schedule(h, bad)) == B.DADAM_EINVAL, bad
    for good in ([(1.0, 0.0, 0.0)], [(1.5, -0.5, 0.0)] * 16, [(3.4445, -4.7750, 2.0315)] * 10):
        B.dadam_set_ortho_schedule(h, good)                                 # before and after matrices are registered
        B.dadam_set_matrices(h, GOOD)
    assert B.lib.dadam_set_ortho_schedule(h, 1, None) == B.DADAM_EINVAL
    B.dadam_destroy(h)


def test_null_handles_and_outputs():
    h = handle()
    L = B.lib
    assert L.dadam_set_matrices(None, None, 0) == B.DADAM_EINVAL and L.dadam_set_ortho_schedule(None, 1, (C.c_float * 3)()) == B.DADAM_EINVAL
    assert L.dadam_ortho_get_info(None, C.byref(B.dadam_ortho_info())) == B.DADAM_EINVAL and L.dadam_ortho_get_info(h, None) == B.DADAM_EINVAL
    assert L.dadam_head_get_info(None, C.byref(HEAD), 1, 0, C.byref(B.dadam_head_info())) == B.DADAM_EINVAL
    assert L.dadam_head_get_info(h, None, 1, 0, C.byref(B.dadam_head_info())) == B.DADAM_EINVAL and L.dadam_head_get_info(h, C.byref(HEAD), 1, 0, None) == B.DADAM_EINVAL
    assert L.dadam_orthogonalize(None, None, None, None, 0, None) == B.DADAM_EINVAL and L.dadam_ortho_step(None, 0, None, 1, 0, None, 0, None) == B.DADAM_EINVAL
    assert L.dadam_head_loss(None, C.byref(HEAD), None, None, None, 1, 1.0, 0, None, None, None, None, None, 0, None) == B.DADAM_EINVAL
    B.dadam_destroy(h)


def test_orthogonalised_buffers():
    h = handle()
    work, a, b = (8 << 24, 1 << 24), addresses(ROWS, 1 << 24), addresses(ROWS, 2 << 24)
    call = lambda i=a, o=b, w=work: code(lambda: B.dadam_orthogonalize(h, i, o, w))  # noqa: E731
    assert call() == B.DADAM_ESTATE
    B.dadam_set_matrices(h, GOOD)
    least = B.dadam_ortho_get_info(h).least_bytes
    for good in ({}, {"o": a}, {"w": (8 << 24, least)}, {"o": [b[0], a[1], b[2]]}):
        assert call(**good) == B.DADAM_ESTATE, good
        assert b"host-only" in B.lib.dadam_last_error(h) or b"device" in B.lib.dadam_last_error(h)
    for bad in ({"i": None}, {"o": None}, {"i": [a[0], 0, a[2]]}, {"o": [0, b[1], b[2]]}, {"w": (0, 1 << 24)}, {"w": (8 << 24, least - 1)}, {"w": None}):
        assert call(**bad) == B.DADAM_EINVAL, bad
    for bad in ({"i": [a[0] + 4, a[1], a[2]]}, {"o": [b[0], b[1] + 8, b[2]]}, {"w": ((8 << 24) + 16, 1 << 24)}):
        assert call(**bad) == B.DADAM_EALIGN, bad
    for bad in ({"o": [a[1], a[0], a[2]]}, {"o": [b[0], b[0], b[2]]}, {"o": [a[0] + 16, b[1], b[2]]}, {"w": (a[1], 1 << 24)}, {"w": (b[2], 1 << 24)}):
        assert call(**bad) == B.DADAM_EALIAS, bad
    B.dadam_destroy(h)


def test_steps_of_matrices():
    h = handle(accum_s=2)
    g, work = addresses(ROWS, 1 << 24), (8 << 24, 1 << 24)
    src, dst, m, v, acc = (addresses(ROWS, (k + 2) << 24) for k in range(5))
    call = lambda slot=0, grads=g, t=1, flags=B.DADAM_FUSE_ACCUM, w=work: code(lambda: B.dadam_ortho_step(h, slot, grads, t, flags, w))  # noqa: E731
    assert call() == B.DADAM_ESTATE                                         # nothing is bound
    B.dadam_bind(h, src, dst, m, v, acc)
    assert call() == B.DADAM_ESTATE and b"dadam_set_matrices" in B.lib.dadam_last_error(h)
    B.dadam_set_matrices(h, GOOD)
    for good in ({}, {"flags": 0}, {"flags": B.DADAM_ORTHO_NESTEROV}, {"flags": B.DADAM_ORTHO_NESTEROV | B.DADAM_FUSE_ACCUM, "t": 2}):
        assert call(**good) == B.DADAM_ESTATE and b"device" in B.lib.dadam_last_error(h), good
    for bad in ({"grads": None}, {"t": 0}, {"flags": 2}, {"flags": 16}, {"w": None}, {"w": (8 << 24, 256)}):
        assert call(**bad) == B.DADAM_EINVAL, bad
    for slot in (1, 99):                                                    # no topology there, as dadam_gossip_step says it
        assert call(slot=slot) == B.DADAM_ESTATE and b"slot" in B.lib.dadam_last_error(h)
    assert call(grads=[g[0], g[1] + 4, g[2]]) == B.DADAM_EALIGN and call(w=((8 << 24) + 64, 1 << 24)) == B.DADAM_EALIGN
    for table in (g, src, dst, m, acc):
        assert call(w=(table[1], 1 << 24)) == B.DADAM_EALIAS
    assert call(grads=[g[0], dst[1], g[2]]) == B.DADAM_EALIAS
    B.dadam_bind(h, src, src, m, v, acc)                                    # a ring's rows read each other
    assert call() == B.DADAM_EALIAS
    B.dadam_destroy(h)


def test_the_binding_refuses_other_shapes():
    h = handle()
    with pytest.raises(ValueError):
        B.dadam_set_matrices(h, [(2, 40)])
    with pytest.raises(ValueError):
        B.dadam_set_ortho_schedule(h, [(1.0, 2.0)])
    with pytest.raises(ValueError):
        B.dadam_orthogonalize(h, [1 << 20], [1 << 21], (1 << 24, 1 << 24))
    B.dadam_destroy(h)


def test_a_workspace_grows_with_what_it_holds():
    """Larger layouts and more tokens never ask for less, and a replica's matrix with the sums of its ranges fits."""
    last = 0
    for q in (1, 127, 128, 1000, 4096, 65536):
        h = B.dadam_init(1, 1, 5 * q + (-5 * q) % 8, [0], [5 * q], device=B.DADAM_DEVICE_NONE)
        B.dadam_set_matrices(h, [(0, 5, q)])
        info = B.dadam_ortho_get_info(h)
        assert info.least_bytes == info.bytes >= max(last, 2 * 128 * q * 4 if q > 960 else 0)  # (up to there a compute unit holds it)
        last = info.bytes
        B.dadam_destroy(h)
    h = handle()
    least = [B.dadam_head_get_info(h, HEAD, n, True).least_bytes for n in (0, 1, 100, 1000, 10 ** 5, 2 ** 20)]
    assert least == sorted(least)
    assert np.all([B.dadam_head_get_info(h, HEAD, n, False).least_bytes <= B.dadam_head_get_info(h, HEAD, n, True).least_bytes for n in (1, 100, 5000)])
    B.dadam_destroy(h)


def test_a_head_of_one_column_is_not_its_own_bias():
    """Both gradients would be written to the same elements."""
    h = B.dadam_init(2, 2, 2 * VOCAB, [0, VOCAB], [VOCAB, VOCAB], device=B.DADAM_DEVICE_NONE)
    c = Loss(h)
    for tensor in (0, 1):
        own = B.dadam_head(tensor, tensor, VOCAB, 1)
        assert c.code(head=own) == B.DADAM_EINVAL and b"same tensor" in B.lib.dadam_last_error(h)
        assert code(lambda: B.dadam_head_get_info(h, own, TOKENS, True)) == B.DADAM_EINVAL
        assert c.code(head=B.dadam_head(tensor, 1 - tensor, VOCAB, 1)) == B.DADAM_ESTATE
    B.dadam_destroy(h)


def test_no_tokens_need_no_memory():
    """Buffers of no elements may be null, as empty tensors are, and lie anywhere."""
    h = handle()
    c = Loss(h)
    none = {k: [0] * ROWS for k in ("hidden", "targets", "nll", "dhidden")}
    assert c.code(n=0, **none) == B.DADAM_ESTATE and b"device" in B.lib.dadam_last_error(h)
    for inside in (c.params[1] + 64, c.grads[0] + 64, c.workspace[0] + 64, c.losses + 4):
        assert c.code(n=0, **{k: [inside] * ROWS for k in none}) == B.DADAM_ESTATE, inside
    for k in none:
        assert c.code(**{k: none[k]}) == B.DADAM_EINVAL
    assert c.code(n=0, params=[0] * ROWS, **none) == B.DADAM_EINVAL and c.code(n=0, **dict(none, hidden=None)) == B.DADAM_EINVAL
    B.dadam_destroy(h)


def test_matrices_of_other_row_distances_share_a_tensor_but_no_element():
    """A matrix may lie between another's rows with a distance of its own (of one row: whatever the distance); against a map of the tensor's elements."""
    h = handle()
    apart = [[(3, 200, 100, 300), (3, 1, 100, 100, 100)], [(3, 1, 100, 100, 100), (3, 200, 100, 300)], [(3, 200, 100, 300), (3, 100, 200, 600, 100), (3, 100, 200, 600, 400)]]
    for good in apart:
        B.dadam_set_matrices(h, good)
        assert B.dadam_ortho_get_info(h).n_matrices == len(good)
    rng = np.random.default_rng(3)
    seen = [0, 0]
    for _ in range(3000):
        ms = []
        for _ in range(2):
            ld = int(rng.integers(1, 40))
            cols, rows = int(rng.integers(1, ld + 1)), int(rng.integers(1, 20))
            first = int(rng.integers(0, 40)) * ld + int(rng.integers(0, ld - cols + 1))
            ms.append((2, rows, cols, ld, first))
        reached = [m[4] + (m[1] - 1) * m[3] + m[2] for m in ms]
        if max(reached) > SIZES[2]:
            continue
        taken = [np.zeros(SIZES[2], dtype=bool) for _ in ms]
        for t, (_, rows, cols, ld, first) in zip(taken, ms):
            np.lib.stride_tricks.as_strided(t[first:], (rows, cols), (ld, 1))[:] = True
        shared = bool((taken[0] & taken[1]).any())
        seen[shared] += 1
        assert code(lambda: B.dadam_set_matrices(h, ms)) == (B.DADAM_EINVAL if shared else B.DADAM_OK), (ms, shared)
    assert min(seen) > 300
    B.dadam_destroy(h)


def test_workspaces_that_reach_beyond_memory():
    """More bytes than addresses: the end wraps, and would lie before the buffers that the workspace overlaps."""
    h = handle(accum_s=2)
    B.dadam_set_matrices(h, GOOD)
    g, work = addresses(ROWS, 1 << 24), 8 << 24
    src, dst, m, v, acc = (addresses(ROWS, (k + 2) << 24) for k in range(5))
    B.dadam_bind(h, src, dst, m, v, acc)
    for at, n_bytes in ((1 << 20, 2 ** 64 - 256), (work, 2 ** 64 - 1), (work, 2 ** 64 - work), (1 << 52, 1 << 24), (work, (1 << 52) - work + 1)):
        assert code(lambda: B.dadam_ortho_step(h, 0, g, 1, 0, (at, n_bytes))) == B.DADAM_EINVAL, (at, n_bytes)
        assert code(lambda: B.dadam_orthogonalize(h, g, dst, (at, n_bytes))) == B.DADAM_EINVAL, (at, n_bytes)
        assert Loss(h).code(workspace=(at, n_bytes)) == B.DADAM_EINVAL, (at, n_bytes)
    assert code(lambda: B.dadam_ortho_step(h, 0, g, 1, 0, (work, (1 << 52) - work))) == B.DADAM_ESTATE and b"device" in B.lib.dadam_last_error(h)
    B.dadam_destroy(h)
