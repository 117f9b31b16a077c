"""Refusals of the operators around the step, on a host-only handle: every call is validated as on a device handle, and one that
passes is refused for want of a device.  Addresses are numbers; nothing is touched."""

import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import operators_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 1000
STEP = 1 << 16


class Addresses:
    """Tables of distinct addresses."""

    def __init__(self):
        self.at = 1 << 20

    def __call__(self, n):
        out = []
        for _ in range(n):
            out.append(self.at)
            self.at += STEP
        return out


def handle(rows=3, cols=3, **kw):
    h = B.dadam_init(rows, cols, D, [0], [D], device=B.DADAM_DEVICE_NONE, **kw)
    if rows == cols:
        B.dadam_set_topology(h, 0, *WL.ring(rows))
    else:
        B.dadam_set_topology(h, 0, *WL.node_share_ring())
    return h


CALLS = {
    "norm": (lambda h, t, **k: B.dadam_grad_norm(h, t["grads"], t["norms"]), {"grads": 3}),
    "clip": (lambda h, t, limit=1.0: B.dadam_clip_grads(h, t["grads"], t["out"], limit, t["norms"]), {"grads": 3, "out": 3}),
    "encode": (lambda h, t, **k: B.dadam_mx4_encode(h, t["x"], t["copy_in"], t["copy_out"], t["msg"]),
               {"x": 3, "copy_in": 3, "copy_out": 3, "msg": 3}),
    "product": (lambda h, t, slot=0, flags=0: B.dadam_mx4_product(h, slot, t["msg"], t["out"], flags), {"msg": 3, "out": 3}),
    "gossip": (lambda h, t, slot=0, gamma=0.5: B.dadam_mx4_gossip(h, slot, t["msg"], t["sum"], t["copy"], t["x_src"], t["x_dst"], gamma),
               {"msg": 3, "sum": 3, "copy": 3, "x_src": 3, "x_dst": 3}),
    "round": (lambda h, t, slot=0, gamma=0.5: B.dadam_mx4_round(h, slot, t["x_src"], t["x_dst"], t["copy"], t["sum"], gamma),
              {"x_src": 3, "x_dst": 3, "copy": 3, "sum": 3}),
}
WRITTEN = {"norm": [], "clip": ["out"], "encode": ["copy_out", "msg"], "product": ["out"], "gossip": ["sum", "x_dst"], "round": ["x_dst", "copy", "sum"]}
IN_PLACE = {("clip", "out", "grads"), ("encode", "copy_out", "copy_in"), ("gossip", "x_dst", "x_src"), ("round", "x_dst", "x_src")}


def tables(name):
    new = Addresses()
    t = {k: new(n) for k, n in CALLS[name][1].items()}
    t["norms"] = new(1)[0] + 4
    return t


def code_of(name, t, h=None, **kw):
    own = h is None
    h = h or handle()
    with pytest.raises(B.DadamError) as e:
        CALLS[name][0](h, t, **kw)
    text = B.dadam_last_error(h)
    if own:
        B.dadam_destroy(h)
    assert text
    return e.value.code


@pytest.mark.parametrize("name", CALLS)
def test_a_sound_call_is_refused_for_want_of_a_device_only(name):
    assert code_of(name, tables(name)) == B.DADAM_ESTATE


@pytest.mark.parametrize("name", CALLS)
def test_null_misaligned_and_far_buffers(name):
    for table in CALLS[name][1]:
        for value, code in ((0, B.DADAM_EINVAL), ((1 << 20) + 8, B.DADAM_EALIGN), ((1 << 52) - 16, B.DADAM_EINVAL), (1 << 60, B.DADAM_EINVAL)):
            t = tables(name)
            t[table][1] = value
            assert code_of(name, t) == code, (table, value)


@pytest.mark.parametrize("name", CALLS)
def test_what_is_written_overlaps_nothing_else(name):
    sized = CALLS[name][1]
    for w in WRITTEN[name]:
        for other in sized:
            for shift in (0, 16, -16):
                t = tables(name)
                t[w][2] = t[other][0 if other != w else 1] + shift
                assert code_of(name, t) == B.DADAM_EALIAS, (w, other, shift)
            t = tables(name)
            t[w][1] = t[other][1]
            want = B.DADAM_ESTATE if w == other or (name, w, other) in IN_PLACE else B.DADAM_EALIAS
            assert code_of(name, t) == want, (w, other)


def test_what_is_read_may_coincide():
    t = tables("product")
    t["msg"] = [t["msg"][0]] * 3
    assert code_of("product", t) == B.DADAM_ESTATE
    t = tables("gossip")
    t["copy"][1] = t["copy"][0]
    assert code_of("gossip", t) == B.DADAM_ESTATE


def test_norms():
    for name in ("norm", "clip"):
        t = tables(name)
        t["norms"] = 0
        assert code_of(name, t) == B.DADAM_EINVAL
        t["norms"] = (1 << 24) + 2
        assert code_of(name, t) == B.DADAM_EALIGN
        for table in CALLS[name][1]:
            t = tables(name)
            t["norms"] = t[table][1] + 4 * D - 4
            assert code_of(name, t) == B.DADAM_EALIAS
            t["norms"] = t[table][1] + 4 * D
            assert code_of(name, t) == B.DADAM_ESTATE
            t["norms"] = t[table][1] - 8
            assert code_of(name, t) == B.DADAM_EALIAS


def test_scalars_slots_and_flags():
    for bad in (-1.0, float("nan"), float("inf")):
        assert code_of("clip", tables("clip"), limit=bad) == B.DADAM_EINVAL
    assert code_of("clip", tables("clip"), limit=0.0) == B.DADAM_ESTATE
    for name in ("gossip", "round"):
        for bad in (0.0, -0.5, 1.5, float("nan")):
            assert code_of(name, tables(name), gamma=bad) == B.DADAM_EINVAL
    for name in ("product", "gossip", "round"):
        assert code_of(name, tables(name), slot=16) == B.DADAM_EINVAL
        h = handle()
        assert code_of(name, tables(name), h, slot=1) == B.DADAM_ESTATE and "topology" in B.dadam_last_error(h)
        B.dadam_destroy(h)
    assert code_of("product", tables("product"), flags=2) == B.DADAM_EINVAL


def test_null_tables_and_handles():
    lib, h = B.lib, handle()
    none = C.POINTER(C.c_void_p)()
    some = (C.c_void_p * 3)(*Addresses()(3))
    assert lib.dadam_grad_norm(h, none, 16, None) == B.DADAM_EINVAL
    assert lib.dadam_clip_grads(h, some, none, 1.0, 16, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_encode(h, none, none, none, some, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_encode(h, some, none, none, none, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_product(h, 0, none, some, 0, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_gossip(h, 0, some, some, none, some, some, 0.5, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_round(h, 0, some, some, some, none, 0.5, None) == B.DADAM_EINVAL
    assert lib.dadam_mx4_get_info(h, None) == B.DADAM_EINVAL
    for call in (lambda: lib.dadam_grad_norm(None, some, 16, None), lambda: lib.dadam_clip_grads(None, some, some, 1.0, 16, None),
                 lambda: lib.dadam_mx4_encode(None, some, none, none, some, None), lambda: lib.dadam_mx4_product(None, 0, some, some, 0, None),
                 lambda: lib.dadam_mx4_gossip(None, 0, some, some, some, some, some, 0.5, None),
                 lambda: lib.dadam_mx4_round(None, 0, some, some, some, some, 0.5, None), lambda: lib.dadam_mx4_get_info(None, None)):
        assert call() == B.DADAM_EINVAL
    B.dadam_destroy(h)


def test_a_round_needs_every_replica():
    h = handle(1, 3)
    t = {k: v[:1] for k, v in tables("round").items() if isinstance(v, list)}
    assert code_of("round", t, h) == B.DADAM_ESTATE and "n_cols" in B.dadam_last_error(h)
    B.dadam_destroy(h)


def test_sizes_of_messages():
    for d in (1, 31, 32, 33, 64, 512, 1000, 124439808):
        h = B.dadam_init(1, 1, d, [0], [d], device=B.DADAM_DEVICE_NONE)
        i = B.dadam_mx4_get_info(h)
        assert (i.n_blocks, i.scale_offset, i.bytes) == O.message_size(d)
        B.dadam_destroy(h)


def test_vectors_that_are_too_long_are_refused():
    h = B.dadam_init(1, 1, (1 << 36) + 8, [0], [8], device=B.DADAM_DEVICE_NONE)
    with pytest.raises(B.DadamError) as e:
        B.dadam_grad_norm(h, [1 << 20], 1 << 50)
    assert e.value.code == B.DADAM_EINVAL and "2^36" in str(e.value)
    B.dadam_destroy(h)


def test_the_binding_refuses_short_buffers():
    import torch
    h = handle()
    good, short = [torch.zeros(D) for _ in range(3)], [torch.zeros(D - 1) for _ in range(3)]
    half, norms = [torch.zeros(D, dtype=torch.bfloat16) for _ in range(3)], torch.zeros(3)
    for bad in (short, half, good[:2], torch.zeros(3, D - 1), torch.zeros(2, D), torch.zeros(3, 2 * D)[:, ::2], [torch.zeros(2 * D)[::2]] * 3):
        with pytest.raises(ValueError):
            B.dadam_grad_norm(h, bad, norms)
    with pytest.raises(ValueError):
        B.dadam_grad_norm(h, good, torch.zeros(2))
    with pytest.raises(ValueError):
        B.dadam_mx4_product(h, 0, [torch.zeros(543, dtype=torch.uint8)] * 3, good)       # a message has 544 bytes
    B.dadam_destroy(h)


def test_the_oracle_of_messages():
    """Hand-worked blocks: scale by the largest magnitude, ties to the even code, saturation, signs, a NaN block, a part of a block."""
    x = np.zeros(65, np.float32)
    x[:8] = [4.0, 2.5, -3.5, 0.25, 0.75, 7.0, -0.2, 5.0]     # scale 1: 4, tie to 2, tie to -4, tie to 0, tie to 1, saturates at 6, -0, tie to 4
    x[32] = np.inf
    x[64] = -0.375                                            # 1.5 * 2^-2: scale 2^-4, -6
    m, v = O.encode(x, None, np.ones(65, bool))
    assert list(v[:8]) == [4, 2, -4, 0, 1, 6, 0, 4] and np.isnan(v[32:64]).all() and v[64] == -0.375
    assert list(m[:4]) == [6 + 16 * 4, 14 + 16 * 0, 2 + 16 * 7, 8 + 16 * 6]
    assert list(m[48:]) == [127, 255, 123] and m[32] == 15
    assert np.array_equal(O.decode(m, 65), v, equal_nan=True)


def test_host_code_under_address_and_ub_sanitizers(tmp_path):
    """The host side with its launchers modelled: random layouts and calls, and what tells padding from elements against the tensor
    list, granule by granule."""
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        pytest.skip("clang++ of the ROCm toolchain not available")
    exe, csrc = str(tmp_path / "operators_driver"), os.path.join(ROOT, "paper_2410_11998_amd", "csrc")
    cmd = [clang, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", "/opt/rocm/include", os.path.join(ROOT, "tests", "host_operators_driver.cpp"),
           os.path.join(csrc, "dadam_host.cpp"), os.path.join(csrc, "dadam_operators.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "bad 0" in r.stdout and "ERROR" not in r.stderr, (r.stdout[-500:], r.stderr[-3000:])


def test_tables_made_before_are_of_addresses():
    """What is not an array of 8-byte whole numbers or pointers would be read beyond its end, or as other addresses."""
    from array import array
    h, at = handle(), Addresses()(3)
    for good in (array("Q", at), array("q", at), (C.c_void_p * 3)(*at), (C.c_uint64 * 3)(*at)):
        with pytest.raises(B.DadamError) as e:
            B.dadam_grad_norm(h, good, 1 << 16)
        assert e.value.code == B.DADAM_ESTATE
    for bad in (array("I", at), array("d", at), array("B", [0] * 24), (C.c_uint32 * 3)(*at), (C.c_double * 3)(*at), (C.c_char * 24)()):
        with pytest.raises(ValueError):
            B.dadam_grad_norm(h, bad, 1 << 16)
    B.dadam_destroy(h)


def test_a_handle_by_its_number_and_a_handle_that_is_none():
    """The number that a handle holds names it as well, sizes are checked by it all the same; what dadam_init has not returned, or
    dadam_destroy has freed, is refused before the library is asked."""
    import torch
    h, at = handle(), Addresses()(3)
    with pytest.raises(B.DadamError) as e:
        B.dadam_grad_norm(h.value, at, 1 << 16)
    assert e.value.code == B.DADAM_ESTATE
    with pytest.raises(ValueError):
        B.dadam_grad_norm(h.value, [torch.zeros(D - 1)] * 3, 1 << 16)
    gone = C.c_void_p(h.value)
    B.dadam_destroy(h.value)
    for none in (gone, gone.value, None, C.c_void_p(), 12345):
        for call in (lambda x: B.dadam_grad_norm(x, at, 1 << 16), lambda x: B.dadam_clip_grads(x, at, at, 1.0, 1 << 16),
                     lambda x: B.dadam_mx4_encode(x, at, None, None, at), lambda x: B.dadam_mx4_product(x, 0, at, at),
                     lambda x: B.dadam_mx4_gossip(x, 0, at, at, at, at, at, 0.5), lambda x: B.dadam_mx4_round(x, 0, at, at, at, at, 0.5)):
            with pytest.raises(ValueError):
                call(none)
