"""Compile checks of the kernels around the step (the step's own are in tests/test_host_abi.py)."""

import os
import re
import shutil
import subprocess

import pytest

import asm_checks
from paper_2410_11998_amd import build as bld


def counts(tmp_path):
    """{kernel: (wide stores with the streaming hint, without, wide loads with, without)}"""
    flags = [f for f in bld.FLAGS if f not in ("-shared", "-fPIC")]
    got = {}
    for unit in ("dadam_norm", "dadam_mx4"):
        asm = str(tmp_path / (unit + ".s"))
        subprocess.run([bld.hipcc()] + flags + ["--cuda-device-only", "-S", os.path.join(bld.CSRC, unit + ".hip"), "-o", asm], check=True, capture_output=True,
                       timeout=600)
        hints = asm_checks.streaming_hints(asm)
        plain = subprocess.run(["c++filt"], input="\n".join(hints), capture_output=True, text=True).stdout.splitlines()
        for mangled, name in zip(hints, plain):
            got[re.sub(r"^void |dadam::|\(anonymous namespace\)::", "", name).split("(")[0]] = tuple(hints[mangled])
    return got


def test_streaming_kernels_keep_the_hint_and_others_have_none(tmp_path):
    """The hint is worth 7 to 20 % in both directions (lines that are whole, and lines that are cut) and is metadata that the optimiser may
    drop.  Vectors carry it in every body of a kernel that has it; masks, the addresses of rows, messages (two bytes a lane) and partial sums
    do not, nor do loads of rows that a copying launch finds in the cache."""
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not available")
    found, seen = counts(tmp_path), {}
    for name, (st_hint, st_plain, ld_hint, ld_plain) in found.items():
        kernel, args = re.match(r"(k_\w+)<(.*)>", name).groups()
        args = args.split(", ")
        if kernel == "k_clip_small":                        # rows that fit a workgroup's registers
            hinted = False
        elif kernel in ("k_grad_norm", "k_clip"):
            hinted = args[1] == "true"
        else:                                               # 0 does not stream, 1 does, 2 does on cut lines: lanes apart, no hint
            at = {"k_mx4_encode": 1, "k_mx4_mix": 2, "k_mx4_shared": 2, "k_mx4_products": 1, "k_mx4_copy": 0, "k_mx4_round": 3}[kernel]
            assert args[at] in "012"
            hinted = args[at] == "1"
        seen.setdefault(kernel, set()).add(hinted)
        if kernel == "k_grad_norm":                         # a store of a partial sum, a load of the partial sums
            assert (st_hint, st_plain, ld_hint, ld_plain) == ((0, 1, 16, 1) if hinted else (0, 1, 0, 17)), name
        elif hinted:
            assert st_hint > 0 and st_plain == 0, name
            assert ld_hint == 0 and ld_plain > 0 if kernel == "k_mx4_copy" else ld_plain == 0, name
            stores_only = kernel == "k_mx4_copy" or (kernel in ("k_mx4_mix", "k_mx4_shared", "k_mx4_products") and args[at - 1] == "0")
            assert ld_hint > 0 or stores_only, name
        else:
            assert st_hint == 0 and ld_hint == 0 and st_plain > 0, name
    assert seen == {"k_clip_small": {False}, "k_mx4_copy": {True}, **{k: {False, True} for k in
                    ("k_grad_norm", "k_clip", "k_mx4_encode", "k_mx4_mix", "k_mx4_shared", "k_mx4_products", "k_mx4_round")}}
