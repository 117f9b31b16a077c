"""What the calls around the step ask of the HIP runtime, without a GPU: which kernels they launch, with how much LDS, and when they
allocate (tests/host_calls_driver.cpp, the built library on a modelled runtime)."""

import os
import re
import subprocess

import pytest

from paper_2410_11998_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    clang, rocm = "/opt/rocm/lib/llvm/bin/clang++", "/opt/rocm/lib"
    if not os.path.exists(clang):
        pytest.skip("clang++ of the ROCm toolchain not available")
    exe, libdir = str(tmp_path_factory.mktemp("calls") / "calls_driver"), os.path.dirname(B.LIB_PATH)
    cmd = [clang, "-std=c++17", "-O1", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
           os.path.join(ROOT, "paper_2410_11998_amd", "csrc"), "-I", "/opt/rocm/include", os.path.join(ROOT, "tests", "host_calls_driver.cpp"), "-o", exe, "-L", libdir, "-ldadam", f"-Wl,-rpath,{libdir}",
           f"-Wl,-rpath,{rocm}", f"-Wl,-rpath-link,{rocm}"]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    return exe


def plain_kernel(text):
    return re.sub(r"^void |dadam::|\(anonymous namespace\)::", "", text).split("(")[0]


class Answer:
    """One call: its status, the error's text, bytes allocated, the launches as (kernel, its template arguments, grid, block, LDS), and of products
    and gossip the rows that each launch forms, or (copy, of) pairs."""

    def __init__(self, line):
        head, *events = line.split(": ", 1)[1].split(" | ")
        self.code, _, self.text = head.partition(" ")
        self.code = int(self.code)
        self.mallocs = [int(e.split()[1]) for e in events if e.startswith("malloc")]
        self.rows = [e.split()[1:] for e in events if e.startswith("rows")]
        self.rows = [[tuple(int(v) for v in r.split("<")) if "<" in r else int(r) for r in launch] for launch in self.rows]   # (int refuses a "!")
        self.kernels = {plain_kernel(e[len("kernel "):]) for e in events if e.startswith("kernel")}
        self.us = [int(v) for e in events if e.startswith("us") for v in e.split()[1:]]
        self.launches = []
        for e in events:
            m = re.match(r"launch (?:void )?(?:dadam::\(anonymous namespace\)::)?(\w+)<(.*)>\(.*\) (\d+)x(\d+) (\d+)$", e)
            if m:
                args = m.group(2).replace("dadam::(anonymous namespace)::", "").split(", ")
                self.launches.append((m.group(1), args) + tuple(int(m.group(k)) for k in (3, 4, 5)))
            else:
                assert not e.startswith("launch"), e


def ask(exe, *commands, **env):
    r = subprocess.run([exe], input="\n".join(commands) + "\n", capture_output=True, text=True, timeout=600, env={**os.environ, **env})
    assert r.returncode == 0, (r.stdout[-500:], r.stderr[-2000:])
    plain = subprocess.run(["c++filt"], input=r.stdout, capture_output=True, text=True, timeout=60).stdout.splitlines()
    assert len(plain) == len(commands), r.stdout
    return [Answer(x) for x in plain]


SHARED_SUM_LDS = 8192     # four parts of a unit's sum


@pytest.mark.parametrize("d", [4096, 1_000_000])
@pytest.mark.parametrize("rows,lists", [(16, 4), (16, 1), (64, 4), (64, 64), (101, 1), (160, 4), (160, 1), (128, 2)])
def test_rounds_keep_to_the_handles_lds(driver, rows, lists, d):
    """A round whose messages fit goes without the shared sums' room where that is too much, and one whose messages do not fit is refused
    before anything is launched.  The messages of a unit of every row: 272 bytes a row up to four rows a wavefront, 136 beyond."""
    each = max(-(-rows // 16), min(3, rows) if rows * d * 24 > 512 << 20 else 0)
    messages = rows * (272 if each <= 4 else 136)
    for limit in (0, 16384, messages, messages - 1, 65536, 1024):
        *_, a = ask(driver, f"handle {rows} {rows} {d} 0 0 {limit}", f"topology 0 lists {lists}", "call round 0")
        if 0 < limit < messages:
            assert a.code == B.DADAM_EINVAL and not a.launches and "dadam_mx4_gossip" in a.text, (limit, a.text)
            continue
        assert a.code == 0 and [x[0] for x in a.launches] == ["k_mx4_round"]
        lds = a.launches[0][4]
        assert messages <= lds <= (limit or 160 << 10), limit
        if limit in (0, 65536) and lists <= 4 and rows // lists >= 12:
            assert lds > messages


@pytest.mark.parametrize("d", [4096, 1_000_000])
@pytest.mark.parametrize("name", ["product", "add", "gossip"])
def test_shared_sums_keep_to_the_handles_lds(driver, name, d):
    """Workgroups that form a sum together hold its parts in 8 KB of LDS; a handle with less has a wavefront form every sum."""
    for limit in (0, SHARED_SUM_LDS, SHARED_SUM_LDS - 1, 1024):
        *_, a = ask(driver, f"handle 32 32 {d} 0 0 {limit}", "topology 0 lists 1", f"call {name} 0")
        assert a.code == 0 and a.launches
        shared = any(x[0] == "k_mx4_shared" for x in a.launches)
        assert not shared or not 0 < limit < SHARED_SUM_LDS
        assert shared or limit or (name != "gossip" and d > 786432)


NAMES = ["norm", "clip", "encode", "product", "add", "gossip", "round"]


@pytest.mark.parametrize("name", NAMES)
def test_a_first_call_under_capture_is_refused_before_it_allocates(driver, name):
    """An allocation would end the caller's capture.  Once a call has been made, all of them can be recorded."""
    answers = ask(driver, "handle 4 4 5000 0 0 0", "topology 0 ring", "capture 1", f"call {name} 0", "capture 0", f"call {name} 0",
                  "capture 1", *(f"call {n} 0" for n in NAMES))
    first, second, recorded = answers[3], answers[5], answers[7:]
    assert first.code == B.DADAM_ESTATE and "captur" in first.text and not first.mallocs and not first.launches
    assert second.code == 0 and second.mallocs and second.launches
    for a in recorded:
        assert a.code == 0 and a.launches and not a.mallocs


def listed_bytes(rows, degree):
    """What the step's kernels read of a slot without loops: row_ptr, col and w; lengths, columns and weights by row, and the rows' order."""
    entries = rows * degree
    return sum(-(-4 * n // 256) * 256 for n in (rows + 1, entries, entries, rows, entries, entries, rows))


@pytest.mark.parametrize("rows", [3, 32, 160])
def test_topologies_of_programs_without_messages_hold_the_steps_lists_only(driver, rows):
    """What the messages' kernels read of a slot is made on a handle's first call of theirs, for every slot that is set, and from then on by
    dadam_set_topology: no call but the first allocates."""
    a = ask(driver, f"handle {rows} {rows} 5000 0 0 0", "topology 0 ring", "topology 3 ring", "topology 0 ring", f"call norm 0", "topology 7 ring",
            "topology 3 ring", *(f"call {n} {s}" for n in NAMES for s in (0, 3, 7)), "capture 1", *(f"call {n} {s}" for n in NAMES for s in (0, 3, 7)))
    for k in (1, 2, 3):
        assert a[k].code == 0 and a[k].mallocs == [listed_bytes(rows, 3)]
    assert a[4].code == 0 and len(a[4].mallocs) == 1
    for k in (5, 6):
        assert a[k].code == 0 and a[k].mallocs[0] == listed_bytes(rows, 3) and len(a[k].mallocs) == 2
    for x in a[7:7 + 3 * len(NAMES)] + a[8 + 3 * len(NAMES):]:
        assert x.code == 0 and x.launches and not x.mallocs, x.text


@pytest.mark.parametrize("name", NAMES)
def test_calls_without_host_memory_launch_nothing_and_can_be_made_again(driver, name):
    """Every allocation of host memory of a handle's first and second call fails once.  The large product copies rows that share their list."""
    begin = ["handle 8 8 13000000 0 0 0", "topology 0 lists 2"]
    for first in (True, False):
        k = failed = 0
        while True:
            k += 1
            *_, got, left, _, again = ask(driver, *begin, *([] if first else ["call encode 0"]), f"memory {k}", f"call {name} 0", "left", "memory 0", f"call {name} 0")
            assert again.code == 0 and again.launches
            if left.code > 0:
                break
            failed += 1
            assert got.code == B.DADAM_EINVAL and "host memory" in got.text and not got.launches, (k, got.text)
        assert got.code == 0 and (failed or not first)


@pytest.mark.parametrize("rows,d,per_row", [(1, 8_500_001, 256), (3, 2_100_003, 65), (7, 1_000_000, 31), (5, 100_003, 4), (160, 70_001, 1), (1, 32_768, 1),
                                            (1, 32_769, 2)])
def test_workgroups_that_share_a_norm(driver, rows, d, per_row):
    *_, a = ask(driver, f"handle {rows} {rows} {d} 0 0 0", "call norm 0")
    assert a.code == 0 and [(x[0], x[2], x[3]) for x in a.launches] == [("k_grad_norm", rows * per_row, 1024)]


# d and rows to either side of the rules' limits
@pytest.mark.parametrize("rows,lists,d", [(8, 1, 1_000_003), (8, 2, 13_000_007), (16, 2, 1_000_000), (24, 2, 800_017), (32, 8, 786_432), (32, 8, 786_433 - 1024),
                                          (100, 1, 4096), (160, 2, 4096), (160, 1, 786_432), (160, 40, 700_000), (20, 5, 5_200_000), (97, 1, 1_100_000),
                                          (160, 160, 4096), (97, 97, 4096), (96, 96, 100), (12, 12, 9_000_000)])
def test_every_row_is_formed_once(driver, rows, lists, d):
    """Over the launches of a product or of gossip every row comes up once: formed, with the list of that row, or copied from a row of the same
    list that was formed before."""
    *_, store, add, gossip, round_ = ask(driver, f"handle {rows} {rows} {d} 0 0 0", f"topology 0 lists {lists}",
                                         *(f"call {n} 0" for n in ("product", "add", "gossip", "round")))
    streams, shared, large = rows * d * 24 > 512 << 20, rows >= 4 * lists, d > 1535 * 512
    each = rows // lists
    for name, a in (("product", store), ("add", add), ("gossip", gossip)):
        assert a.code == 0 and len(a.rows) == len(a.launches)
        formed = [r for launch in a.rows for r in launch if isinstance(r, int)]
        copied = [r for launch in a.rows for r in launch if not isinstance(r, int)]
        assert sorted(formed + [r[0] for r in copied]) == list(range(rows))
        assert all(of in formed and of // each == row // each for row, of in copied)
        kernels = [x[0] for x in a.launches]
        copies = name == "product" and shared and large and rows * d >= 10 ** 8
        if copies:
            assert kernels == ["k_mx4_mix"] * -(-lists // 96) + ["k_mx4_copy"] * -(-len(copied) // 96) and len(formed) == lists
        else:
            want = "k_mx4_mix" if not shared else "k_mx4_products" if name != "gossip" and large else "k_mx4_shared"
            assert set(kernels) == {want} and not copied
        long_block = rows > 16
        for x, launch in zip(a.launches, a.rows):
            assert len(launch) <= (96 if long_block else 16)
            hints = int([v for v in x[1] if v not in ("TF32", "TBF16")][0 if x[0] == "k_mx4_copy" else 1])
            assert hints == (1 if streams else 0)
    assert [x[0] for x in round_.launches] == ["k_mx4_round"]


def test_every_kernel_of_these_calls_is_reached_and_every_call_has_one(driver):
    """Handles of both types, from one row to 160, that stream or not, on and off a line, with lists of their own and shared ones."""
    script, names = ["kernels"], ["norm", "clip", "encode", "product", "add", "gossip", "round"]
    for rows in (1, 2, 8, 16, 17, 24, 40, 64, 70, 100, 128, 160):
        for d in (4096, 50_000, 1_000_000, 25_000_000 // rows + 5, 110_000_000 // rows + 5):
            for kind in (0, 1):
                script += [f"handle {rows} {rows} {d} {kind} {kind} 0"]
                for topology in ("lists 1", "ring"):
                    script += [f"topology 0 {topology}" if topology != "ring" or rows > 2 else f"topology 0 lists {rows}"]
                    for shift in (0, 16):
                        script += [f"shift {shift}"] + [f"call {n} 0" for n in names]
    answers = ask(driver, *script)
    reached = set()
    for command, a in zip(script, answers):
        assert a.code == 0 and (a.launches or not command.startswith("call")), (command, a.text)
        reached |= {f"{x[0]}<{', '.join(x[1])}>" for x in a.launches}
    assert reached == answers[0].kernels, (sorted(answers[0].kernels - reached), sorted(reached - answers[0].kernels))


def test_a_first_call_on_many_short_tensors_takes_no_longer_than_the_handle(driver):
    """Telling padding from elements goes by words of 32, not element by element: 40000 tensors of 500 elements, host time of the first call
    against dadam_init's on the same layout (twice that by elements)."""
    (a,) = ask(driver, "tensors 40000 500")
    assert a.code == 0 and a.us[1] < a.us[0], a.us


def test_lists_under_address_and_ub_sanitizers(tmp_path):
    """What launches are given of matrices whose rows share lists or do not, against the matrix (tests/host_lists_driver.cpp)."""
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        pytest.skip("clang++ of the ROCm toolchain not available")
    exe, csrc = str(tmp_path / "lists_driver"), os.path.join(ROOT, "paper_2410_11998_amd", "csrc")
    cmd = [clang, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", "/opt/rocm/include", os.path.join(ROOT, "tests", "host_lists_driver.cpp"),
           os.path.join(csrc, "dadam_host.cpp"), os.path.join(csrc, "dadam_operators.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and " bad 0" in r.stdout and "ERROR" not in r.stderr, (r.stdout[-500:], r.stderr[-3000:])
    assert int(r.stdout.split()[1]) > 4000
