"""Which kernels the calls at the ends of an iteration launch, over how much, without a GPU (tests/host_ends_driver.cpp, the built library on a modelled
runtime that refuses what the real one refuses)."""

import os
import random
import re
import subprocess

import pytest

from paper_2410_11998_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"f32": B.DADAM_F32, "bf16": B.DADAM_BF16}


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    clang, rocm = "/opt/rocm/lib/llvm/bin/clang++", "/opt/rocm/lib"
    if not os.path.exists(clang):
        pytest.skip("clang++ of the ROCm toolchain not available")
    exe, libdir = str(tmp_path_factory.mktemp("ends") / "ends_driver"), os.path.dirname(B.LIB_PATH)
    cmd = [clang, "-std=c++17", "-O1", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
           os.path.join(ROOT, "paper_2410_11998_amd", "csrc"), "-I", "/opt/rocm/include", os.path.join(ROOT, "tests", "host_ends_driver.cpp"), "-o", exe, "-L", libdir, "-ldadam", f"-Wl,-rpath,{libdir}",
           f"-Wl,-rpath,{rocm}", f"-Wl,-rpath-link,{rocm}"]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    return exe


def plain_kernel(text):
    return re.sub(r"^(void|int) |dadam::|\(anonymous namespace\)::", "", text).split("(")[0]


class Launch:
    """A kernel, its template arguments, grid, and of the head's gradient (the piece's first word, its words, how many of them are left out)."""

    def __init__(self, text):
        m = re.match(r"launch (?:void |int )?(?:dadam::\(anonymous namespace\)::)?(\w+)(?:<(.*)>)?\(.*\) (\d+),(\d+),(\d+)x(\d+) (\d+)(?: words (\d+) (\d+) (\d+))?$", text)
        assert m, text
        self.kernel, self.args = m.group(1), (m.group(2) or "").replace("dadam::(anonymous namespace)::", "").replace("Types<F32, F32>", "two").replace(
            "Types<B16, B16>", "one").replace("Types<B16, F32>", "two").replace("Types<F32, B16>", "two").replace(" ", "").split(",")
        self.grid, self.threads, self.lds = tuple(int(m.group(k)) for k in (3, 4, 5)), int(m.group(6)), int(m.group(7))
        self.words = tuple(int(m.group(k)) for k in (8, 9, 10)) if m.group(8) else None


class Answer:
    def __init__(self, line):
        head, *events = line.split(": ", 1)[1].split(" | ")
        self.code, _, self.text = head.partition(" ")
        self.code, self.launches = int(self.code), [Launch(e) for e in events if e.startswith("launch")]
        self.kernels = {plain_kernel(e[len("kernel "):]) for e in events if e.startswith("kernel")}
        self.reached = {plain_kernel(e[len("launch "):]) for e in events if e.startswith("launch")}

    def of(self, kernel):
        return [x for x in self.launches if x.kernel == kernel]


def ask(exe, commands):
    r = subprocess.run([exe], input="\n".join(commands) + "\n", capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout[-500:], r.stderr[-2000:])
    plain = subprocess.run(["c++filt"], input=r.stdout, capture_output=True, text=True, timeout=60).stdout.splitlines()
    assert len(plain) == len(commands), r.stdout[-500:]
    return [Answer(x) for x in plain]


def loss(rows, kind, tokens, vocab, width, grad=None, before=0, gradient=True, share=100, bias=False):
    return f"loss {rows} {TYPES[kind]} {TYPES[grad or kind]} {tokens} {vocab} {width} {before} {int(gradient)} {share} {int(bias)}"


def check_head_gradient(a, rows, vocab, width, what):
    """No launch without a workgroup, and every word's row of the head's gradient is in exactly one launch of each group of replicas."""
    assert a.code == 0, (what, a.code, a.text)
    reached, groups = 0, 0
    for x in a.of("k_head_dhead"):
        edge = int(x.args[2])
        first, words, skip = x.words
        across, (tiles, _, z) = -(-width // edge), x.grid
        assert tiles == -(-(words - skip) // edge) * across and skip < words, what
        if first + skip == 0:
            assert reached in (0, vocab), what               # the last group's are whole
            reached, groups = 0, groups + z
        assert first + skip == reached, what
        reached = first + words
    if a.of("k_head_dhead"):
        assert reached == vocab and groups == rows, what


SIZES = [(32, "bf16", 2048, 256, 2304), (32, "f32", 2048, 256, 2304), (32, "bf16", 2048, 256, 2560), (32, "f32", 2048, 200, 2400), (17, "bf16", 4096, 256, 4096), (20, "bf16", 4096, 256, 4096),
         (2, "bf16", 1024, 8448, 1024), (4, "bf16", 4096, 50257, 1024), (1, "f32", 2048, 50257, 1024), (40, "bf16", 2048, 300, 2304)]


@pytest.mark.parametrize("rows,kind,tokens,vocab,width", SIZES)
def test_the_heads_gradient_of_large_tiles(driver, rows, kind, tokens, vocab, width):
    """What large tiles there are beyond whole rounds of the chip go by small ones: all words once, whole and in pieces of the vocabulary."""
    shares = (100, 60, 30, 10, 1)
    for share, a in zip(shares, ask(driver, [loss(rows, kind, tokens, vocab, width, share=s) for s in shares])):
        check_head_gradient(a, rows, vocab, width, (share,))


def test_every_launch_of_a_loss_has_workgroups(driver):
    rows, widths, vocabs, tokens = (1, 3, 8, 17, 20, 31, 32, 33), (8, 256, 1024, 2304, 2560, 4096, 4352), (2, 200, 256, 300, 512, 5000), (0, 1, 64, 65, 777, 2048, 4096, 16384)
    calls = [(r, kind, t, v, w) for r in rows for kind in TYPES for t in tokens for v in vocabs for w in widths]
    for c, a in zip(calls, ask(driver, [loss(*c) for c in calls])):
        check_head_gradient(a, c[0], c[3], c[4], c)


def ortho(rows, kind, shapes, step=False, grad=None, share=100):
    return f"ortho {rows} {TYPES[kind]} {TYPES[grad or kind]} {int(step)} {share} " + " ".join(f"{r}x{c}" for r, c in shapes)


# 256 large tiles of X X^T in four replicas, of matrices that fill them or nearly
LARGE = {"256": [(256, 256)] * 64, "512": [(512, 512)] * 8 + [(500, 512)] * 7 + [(512, 498)] * 6 + [(250, 256)]}


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", LARGE)
def test_tiles_of_matrices_go_by_the_workspace(driver, name, kind, step):
    """A and B by large tiles with the workspace that is asked for and by small ones with less, X by large ones with either: what tests/test_ortho_tiles.py compares."""
    for share, edge in ((100, "256"), (20, "128"), (0, "128")):
        a, = ask(driver, [ortho(4, kind, LARGE[name], step, share=share)])
        assert a.code == 0 and {x.args[1] for x in a.of("k_ortho_gram")} == {edge}
        assert {x.args[1] for x in a.of("k_ortho_next")} == {x.args[2] for x in a.of("k_ortho_end")} == {"256"}


# (replicas, tokens, words, width, where the head begins, hundredths of the workspace that is asked for, with gradients), and the modes of k_head_logits (0: statistics, 1:
# exponentials kept, 2: the logits' gradient) and edges of the head's gradient that go with them
LOSSES = {
    "value": ((32, 512, 1000, 250, 6, 100, False), {"0"}, set()),
    "value of a few replicas at a time": ((32, 512, 1000, 250, 6, 30, False), {"0"}, set()),
    "pieces": ((1, 1024, 20000, 1024, 6, 90, True), {"0", "2"}, {"256"}),
    "pieces of a head as it lies": ((1, 1024, 20000, 1024, 8, 90, True), {"0", "2"}, {"256"}),
    "a head as it lies": ((4, 512, 8448, 256, 8, 100, True), {"1"}, {"256"}),
    "a remainder by small tiles": ((2, 1000, 8440, 1000, 6, 100, True), {"1"}, {"256", "128"}),
}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("name", LOSSES)
def test_losses_by_large_tiles(driver, name, kind):
    """What tests/test_head_loss_tiles.py compares goes by the kernels that it is about."""
    (rows, tokens, vocab, width, before, share, gradient), modes, edges = LOSSES[name]
    a, = ask(driver, [loss(rows, kind, tokens, vocab, width, before=before, gradient=gradient, share=share)])
    check_head_gradient(a, rows, vocab, width, name)
    assert {x.args[2] for x in a.of("k_head_logits")} == {"256"} and {x.args[4] for x in a.of("k_head_logits")} == modes
    assert {x.args[2] for x in a.of("k_head_dhead")} == edges and {x.args[1] for x in a.of("k_head_dhidden")} == ({"256"} if gradient else set())
    straight = kind == "bf16" and before == 8
    assert a.of("k_head_operands")[0].grid[1] == (1 if straight else 2)        # hidden vectors only, or the head's as well
    assert len({x.words[0] for x in a.of("k_head_dhead")}) == (2 if "pieces" in name else 1 if gradient else 0)


def test_every_kernel_is_reached(driver):
    """By calls of every size, type, workspace and number of replicas, drawn once, and those above in every pair of types."""
    rng = random.Random(1)
    calls = [loss(rows, kind, tokens, vocab, width, grad, before, gradient, share) for (rows, tokens, vocab, width, before, share, gradient), _, _ in LOSSES.values() for kind in TYPES for grad in TYPES]

    def log(low, high):
        return int(2 ** rng.uniform(low, high))

    for _ in range(600):
        rows, tokens, vocab, width = rng.choice([1, 2, 4, 8, 17, 32, 40]), log(0, 14), log(0, 17), log(1, 12)
        if rng.random() < 0.4:
            tokens, vocab, width = rng.choice([1024, 2048, 4096]), rng.choice([50257, 8448, 20000]), rng.choice([256, 512, 1024])
        calls.append(loss(rows, rng.choice(list(TYPES)), tokens, vocab, width, rng.choice(list(TYPES)), rng.choice([6, 8]), rng.random() < 0.8, rng.choice([100, 100, 60, 30, 1]), rng.random() < 0.5))
    for _ in range(250):
        rows, n, kind = rng.choice([1, 2, 4, 17, 20, 70]), rng.choice([3, 20, 60]), rng.random()
        if kind < 0.7:
            shapes = [(log(0, 5 if kind < 0.3 else 10), log(0, 6 if kind < 0.3 else 11)) for _ in range(n)]
        else:
            shapes = [(512, 512)] * rng.choice([5, 22, 64]) if kind < 0.9 else [(100, 60000), (64, 64)]
        calls.append(ortho(rows, rng.choice(list(TYPES)), shapes, rng.random() < 0.5, rng.choice(list(TYPES)), rng.choice([100, 20, 0])))
    there, *answers = ask(driver, ["kernels"] + calls)
    assert all(a.code == 0 for a in answers) and len(there.kernels) > 150
    reached = set().union(*(a.reached for a in answers))
    assert reached == there.kernels, there.kernels - reached
