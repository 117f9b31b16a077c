"""The operators around the step on the GPU, through the C ABI, against the double-precision statement of them in
oracle/operators_oracle.py: gradient norms and clipping, 4-bit messages, products with them, the gossip update, the round in one pass.

Tolerances.  eps = 2^-24 is half a unit in the last place of float32, 2^-8 a whole one of bfloat16.
* norm: sums in 64 bits, one rounding to float32: 2 eps of the norm.
* clipped gradient: the norm's rounding, a quotient's and a product's: 4 eps of the element, a bfloat16 rounding more.
* message, and the copy that it moves: whole numbers, a float32 difference and a float32 sum of the oracle's own: the same bits.
* sum: n products folded in with n roundings, one more onto the old sum: (n + 2) eps of the magnitudes that make it up.
* x: gamma times the sum's and the difference's error, one rounding of float32, one of bfloat16."""

import numpy as np
import pytest
import torch

from oracle import operators_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

import harness as H

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 2.0 ** -24
TINY = 2.0 ** -149
ODD = [s for _, s in WL.odd_shapes()]


def layout_of(kind):
    """(offsets, sizes, d)"""
    if isinstance(kind, int):
        return [0], [kind], kind
    if kind == "odd":                       # packed to multiples of 8
        L = WL.pack(WL.odd_shapes())
        return list(L.offsets), list(L.numels), L.d
    if kind == "many":                      # most granules cut, over several workgroups
        L = WL.pack([("t%d" % k, (1 + (k * 97) % 700,)) for k in range(300)])
        return list(L.offsets), list(L.numels), L.d
    if kind == "empty":                     # no tensor has an element
        return [0, 40], [0, 0], 100
    if kind == "gaps":                      # odd beginnings, whole granules of padding, an empty tensor, an end that is no multiple of 4
        return [3, 70, 701, 5000, 5000, 9001], [60, 500, 1024, 0, 2049, 1002], 10007
    raise ValueError(kind)


LAYOUTS = [1, 2, 31, 33, 255, 512, 515, 4096, 100003, "odd", "many", "gaps", "empty"]


def stored_of(layout):
    offsets, sizes, d = layout
    m = np.zeros(d, dtype=bool)
    for o, n in zip(offsets, sizes):
        m[int(o):int(o + n)] = True
    return m


class Case:
    """Rows of random values with NaN in the padding, and a handle."""

    def __init__(self, layout, rows, cols=None, kind="f32", csr=None, seed=1, device=0):
        self.offsets, self.sizes, self.d = layout_of(layout)
        self.stored = stored_of((self.offsets, self.sizes, self.d))
        self.rows, self.cols, self.kind = rows, cols or rows, kind
        self.h = B.dadam_init(rows, self.cols, self.d, self.offsets, self.sizes, H.ABI_DT[kind], H.ABI_DT[kind], device=device)
        if csr is not None:
            B.dadam_set_topology(self.h, 0, *csr)
        self.csr = csr
        self.rng = np.random.default_rng(seed)
        self.info = B.dadam_mx4_get_info(self.h)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        torch.cuda.synchronize()
        B.dadam_destroy(self.h)

    def values(self, std, kind="f32", count=None):
        """Device tensors [count][d] of the type, in allocations of their own, padding NaN."""
        out = []
        for _ in range(count or self.rows):
            v = (self.rng.standard_normal(self.d) * std).astype(np.float32)
            t = torch.from_numpy(v).to(DEV).to(H.TORCH_DT[kind])
            t[torch.from_numpy(~self.stored).to(DEV)] = float("nan")
            out.append(t)
        return out

    def messages(self, count):
        return [torch.full((self.info.bytes,), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(count)]

    def random_messages(self, count):
        """Codes at random, padding 0 as an encoder leaves it, scales around 2^-8 with the smallest among them."""
        n, at = self.info.n_blocks, self.info.scale_offset
        out = []
        for _ in range(count):
            nibble = np.zeros(n * 32, dtype=np.uint8)
            nibble[:self.d][self.stored] = self.rng.integers(0, 16, int(self.stored.sum()))
            scale = self.rng.integers(112, 124, n)
            scale[self.rng.random(n) < 0.02] = 0
            m = np.zeros(self.info.bytes, dtype=np.uint8)
            m[:at] = nibble[0::2] + 16 * nibble[1::2]
            m[at:at + n] = scale
            out.append(torch.from_numpy(m).to(DEV))
        return out

    def padding_is_untouched(self, tensors):
        for t in tensors:
            assert torch.isnan(t[torch.from_numpy(~self.stored).to(DEV)]).all(), "padding was written"


def host(t):
    return t.float().cpu().numpy()


def same(a, b):
    return np.array_equal(np.asarray(a, dtype=np.float32), np.asarray(b, dtype=np.float32), equal_nan=True)


def stream():
    return B.current_stream()


def graph_of(rows, kind):
    return {"ring": WL.ring, "exp": WL.static_exponential, "complete": WL.complete, "identity": WL.identity}[kind](rows)


# ---------------------------------------------------------------------------------------------
# norms and clipping
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_norm_and_clipping(layout, kind):
    for rows in (1, 5):
        with Case(layout, rows, kind=kind, seed=rows) as c:
            g = c.values(0.1, kind)
            g = [t * (0.2 + k) for k, t in enumerate(g)]
            norms = torch.full((rows,), -1.0, device=DEV)
            B.dadam_grad_norm(c.h, g, norms, stream())
            want = [O.grad_norm(host(t), c.stored) for t in g]
            assert np.all(np.abs(norms.cpu().numpy() - want) <= 2 * EPS * np.asarray(want)), (layout, rows)
            limit = float(np.float32(np.median(want) * 0.7))
            out = c.values(1.0, kind)
            again = torch.full((rows,), -1.0, device=DEV)
            B.dadam_clip_grads(c.h, g, out, limit, again, stream())
            inplace = [t.clone() for t in g]
            B.dadam_clip_grads(c.h, inplace, inplace, limit, again, stream())
            assert torch.equal(norms, again)
            for t, o, p in zip(g, out, inplace):
                n, ref = O.clip(host(t), c.stored, limit)
                got = host(o)
                if n <= limit:
                    assert same(got[c.stored], host(t)[c.stored])
                bound = np.abs(ref) * (4 * EPS + (2.0 ** -8 if kind == "bf16" else 0)) + TINY
                assert np.all((np.abs(got - ref) <= bound)[c.stored])
                assert same(host(p), np.where(c.stored, got, np.nan))
            c.padding_is_untouched(out + inplace)


def test_a_norm_on_the_limit_leaves_the_gradient_alone():
    with Case(4, 1) as c:
        g = [torch.tensor([3.0, 0.0, 0.0, -4.0], device=DEV)]
        norms = torch.zeros(1, device=DEV)
        for limit, want in ((5.0, [3, 0, 0, -4]), (2.5, [1.5, 0, 0, -2]), (0.0, [0, 0, 0, 0])):
            out = [torch.full((4,), 9.0, device=DEV)]
            B.dadam_clip_grads(c.h, g, out, limit, norms, stream())
            assert norms.item() == 5.0 and out[0].tolist() == want


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norms_of_values_whose_squares_leave_float32(kind):
    """Squares are taken in 64 bits: neither 1e30 nor 1e-30 is lost, and no infinity comes of a norm that float32 holds."""
    for v in (1e30, 1e-30, 1e-38):
        with Case(1000, 2, kind=kind) as c:
            g = [torch.full((1000,), v, device=DEV).to(H.TORCH_DT[kind]) for _ in range(2)]
            norms = torch.zeros(2, device=DEV)
            out = c.values(1.0, kind)
            B.dadam_clip_grads(c.h, g, out, 0.0, norms, stream())
            want = float(g[0][0]) * np.sqrt(1000.0)
            assert np.all(np.abs(norms.cpu().numpy() - want) <= 2 * EPS * want + TINY)
            assert all((o == 0).all() for o in out)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norms_of_infinities_and_nans(kind):
    """Each row keeps to itself: infinite, NaN, zero, ordinary."""
    with Case("odd", 4, kind=kind) as c:
        g = c.values(0.1, kind)
        at = int(np.flatnonzero(c.stored)[-1])
        g[0][at] = float("-inf")
        g[1][at] = float("nan")
        g[2][torch.from_numpy(c.stored).to(DEV)] = 0
        norms = torch.zeros(4, device=DEV)
        out = c.values(1.0, kind)
        B.dadam_clip_grads(c.h, g, out, 0.25, norms, stream())
        n = norms.cpu().numpy()
        assert n[0] == np.inf and np.isnan(n[1]) and n[2] == 0 and np.isfinite(n[3])
        first = host(out[0])[c.stored]
        assert np.isnan(first[-1]) and np.all(first[:-1] == 0)
        assert np.isnan(host(out[1])[c.stored]).all() and np.all(host(out[2])[c.stored] == 0)
        assert abs(O.grad_norm(host(out[3]), c.stored) - 0.25) <= 0.25 * 2.0 ** -7
        c.padding_is_untouched(out)


def test_norms_of_many_rows_and_in_a_fixed_order():
    """160 rows on the long argument block; the same call gives the same bits, whichever workgroup is last."""
    with Case(70001, 160) as c:
        g = c.values(0.1)
        norms = [torch.zeros(160, device=DEV) for _ in range(6)]
        for n in norms:
            B.dadam_grad_norm(c.h, g, n, stream())
        want = np.asarray([O.grad_norm(host(t), c.stored) for t in g])
        assert np.all(np.abs(norms[0].cpu().numpy() - want) <= 2 * EPS * want)
        assert all(torch.equal(n, norms[0]) for n in norms)


# ---------------------------------------------------------------------------------------------
# messages
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_messages(layout, kind):
    """Codes, scales and copies bit for bit, with a copy, without one, in place, and without moving it; what fills a message up stays."""
    for rows in (1, 17):
        with Case(layout, rows, kind=kind, seed=3 * rows) as c:
            x, before = c.values(0.02, kind), c.values(0.02)
            at, n = c.info.scale_offset, c.info.n_blocks
            for copy, behind in ((None, "new"), (before, "new"), (before, "same"), (before, None), (None, None)):
                msg = c.messages(rows)
                copy = copy if behind != "same" else [t.clone() for t in copy]
                out = copy if behind == "same" else c.values(1.0) if behind else None
                B.dadam_mx4_encode(c.h, x, copy, out, msg, stream())
                for i in range(rows):
                    want, values = O.encode(host(x[i]), None if copy is None else host(before[i]), c.stored)
                    got = msg[i].cpu().numpy()
                    assert np.array_equal(got[:at + n], want), (rows, i)
                    assert np.all(got[at + n:] == 0xA5)
                    if out is not None:
                        moved = values.astype(np.float32) if copy is None else host(before[i]) + values.astype(np.float32)
                        assert same(host(out[i])[c.stored], moved[c.stored])
                if out is not None:
                    c.padding_is_untouched(out)


def test_every_rounding_of_the_4_bit_type():
    """All magnitudes and the middles between them, one unit in the last place to either side, both signs, over the range of scales."""
    points = np.concatenate([O.GRID, (O.GRID[1:] + O.GRID[:-1]) / 2, [5.0, 5.5, 6.5, 7.0, 7.9]]).astype(np.float32)
    near = np.concatenate([points, np.nextafter(points, np.float32(100)), np.nextafter(points[1:], np.float32(0))])
    near = np.concatenate([near, -near])
    blocks = []
    for e in (-149, -140, -130, -127, -126, -125, -124, -120, -60, -3, 0, 1, 60, 120, 124, 125):
        for lead in (4.0, 5.9, 6.0, 7.9):             # the element that sets the block's scale
            for k in range(0, len(near), 31):
                b = np.zeros(32, dtype=np.float32)
                v = near[k:k + 31]
                b[:len(v)] = v
                b[31] = lead
                with np.errstate(all="ignore"):
                    blocks.append(np.ldexp(b.astype(np.float64), e).astype(np.float32))
    blocks = [b for b in blocks if np.isfinite(b).all()] + [np.zeros(32, np.float32), np.full(32, -0.0, np.float32)]
    x = np.concatenate(blocks)
    with Case(len(x), 1) as c:
        msg, values = c.messages(1), c.values(1.0)
        B.dadam_mx4_encode(c.h, [torch.from_numpy(x).to(DEV)], None, values, msg, stream())
        want, ref = O.encode(x, None, c.stored)
        got = msg[0].cpu().numpy()[:len(want)]
        bad = np.flatnonzero(got != want)
        assert bad.size == 0, (bad[:5], got[bad[:5]], want[bad[:5]])
        assert same(host(values[0]), ref)


def test_messages_of_infinities_and_nans():
    """A block with one of them is NaN as a whole, its neighbours are not; also where the copy has it, or the difference overflows."""
    with Case(32 * 6, 1) as c:
        x, copy = np.ones(192, np.float32), np.zeros(192, np.float32)
        x[5], x[40], copy[70], x[100], copy[100] = np.inf, np.nan, -np.inf, 3e38, -3e38
        x[160] = 3.4e38
        msg, behind = c.messages(1), c.values(1.0)
        B.dadam_mx4_encode(c.h, [torch.from_numpy(x).to(DEV)], [torch.from_numpy(copy).to(DEV)], behind, msg, stream())
        want, values = O.encode(x, copy, c.stored)
        assert np.array_equal(msg[0].cpu().numpy()[:len(want)], want) and list(want[96:102]) == [255, 255, 255, 255, 125, 252]
        got = host(behind[0])
        assert np.isnan(got[:128]).all() and np.isfinite(got[128:]).all()
        assert same(got[128:], values[128:])


# ---------------------------------------------------------------------------------------------
# products and gossip
# ---------------------------------------------------------------------------------------------

GRAPHS = [(1, 3, "share"), (1, 1, "identity"), (5, 5, "ring"), (16, 16, "exp"), (17, 17, "complete"), (100, 100, "exp"), (3, 40, "rect"),
          (97, 160, "rect"), (40, 40, "complete"), (16, 16, "aer"), (120, 120, "aer")]


def csr_of(rows, cols, kind, seed=5):
    if kind == "share":
        return WL.node_share_ring()
    if kind == "rect":                      # rows of different lengths and unequal weights
        rng = np.random.default_rng(seed)
        ptr, col, w = [0], [], []
        for i in range(rows):
            n = int(rng.integers(1, min(cols, 90) + 1))
            col += list(rng.permutation(cols)[:n])
            p = rng.random(n) + 0.1
            w += list((p / p.sum()).astype(np.float32))
            ptr.append(len(col))
        return np.asarray(ptr, np.int32), np.asarray(col, np.int32), np.asarray(w, np.float32)
    return WL.aer(rows // 4, 1) if kind == "aer" else graph_of(rows, kind)


def check_sums(c, msg, csr, old, got, where):
    """The sums against the oracle's; returns (sums in 64 bits, their bound)."""
    mixed, size = O.product([m.cpu().numpy() for m in msg], *csr, c.d)
    sums, bounds = [], []
    for i in range(c.rows):
        n = int(csr[0][i + 1] - csr[0][i])
        base = host(old[i]).astype(np.float64) if old is not None else 0.0
        ref, bound = base + mixed[i], (n + 2) * EPS * (size[i] + np.abs(base)) + (n + 2) * TINY
        assert np.all((np.abs(host(got[i]) - ref) <= bound)[c.stored]), (where, i)
        sums.append(ref)
        bounds.append(bound)
    return sums, bounds


@pytest.mark.parametrize("layout", [1, 33, 515, "odd", "many", "gaps", "empty", 40961])
@pytest.mark.parametrize("graph", GRAPHS)
def test_products_and_gossip(graph, layout):
    rows, cols, kind = graph
    csr = csr_of(rows, cols, kind)
    for xt in ("f32", "bf16"):
        with Case(layout, rows, cols, xt, csr, seed=11) as c:
            msg = c.random_messages(cols)
            out = c.values(1.0)
            B.dadam_mx4_product(c.h, 0, msg, out, 0, stream())
            check_sums(c, msg, csr, None, out, "store")
            c.padding_is_untouched(out)
            old = c.values(0.02)
            add = [t.clone() for t in old]
            B.dadam_mx4_product(c.h, 0, msg, add, B.DADAM_MX4_ADD, stream())
            sums, bounds = check_sums(c, msg, csr, old, add, "add")
            total, copy, x, behind = [t.clone() for t in old], c.values(0.02), c.values(0.02, xt), c.values(1.0, xt)
            B.dadam_mx4_gossip(c.h, 0, msg, total, copy, x, behind, 0.3, stream())
            for i in range(rows):
                assert same(host(total[i]), host(add[i]))          # the same sums, to the bit
                a, s, v = host(copy[i]).astype(np.float64), sums[i], host(x[i]).astype(np.float64)
                ref = v + float(np.float32(0.3)) * (s - a)
                bound = 0.3 * (bounds[i] + EPS * (np.abs(s) + np.abs(a))) + EPS * (np.abs(ref) + bounds[i]) + TINY
                bound = bound * 1.01 + (2.0 ** -8 * np.abs(ref) if xt == "bf16" else 0)
                assert np.all((np.abs(host(behind[i]) - ref) <= bound)[c.stored]), i
            c.padding_is_untouched(add + total + behind)
            inplace, again = [t.clone() for t in x], [t.clone() for t in old]
            B.dadam_mx4_gossip(c.h, 0, msg, again, copy, inplace, inplace, 0.3, stream())
            for i in range(rows):
                assert same(host(inplace[i]), host(behind[i])) and same(host(again[i]), host(total[i]))


def test_a_message_that_stands_for_nan_reaches_its_readers_only():
    """Rows that do not list a source are not touched by what it holds, whole block or not."""
    n = 24
    csr = WL.static_exponential(n)
    with Case("odd", n, n, "f32", csr) as c:
        msg = c.random_messages(n)
        msg[7][c.info.scale_offset + 1] = 255
        out = c.values(1.0)
        B.dadam_mx4_product(c.h, 0, msg, out, 0, stream())
        hit = np.zeros(c.d, dtype=bool)
        hit[32:64] = True
        for i in range(n):
            reads = 7 in csr[1][csr[0][i]:csr[0][i + 1]]
            got = np.isnan(host(out[i])[c.stored])
            assert np.array_equal(got, (hit & reads)[c.stored]), i


def test_decoding_is_the_product_with_the_identity():
    with Case("many", 3, csr=WL.identity(3)) as c:
        x, values, msg, out = c.values(0.02), c.values(1.0), c.messages(3), c.values(1.0)
        B.dadam_mx4_encode(c.h, x, None, values, msg, stream())
        B.dadam_mx4_product(c.h, 0, msg, out, 0, stream())
        for a, b in zip(values, out):
            assert same(host(a), host(b))


# ---------------------------------------------------------------------------------------------
# the round in one pass
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,graph", [(1, "identity"), (2, "ring"), (5, "ring"), (16, "exp"), (17, "exp"), (32, "complete"), (33, "exp"), (64, "exp"),
                                        (65, "ring"), (96, "complete"), (160, "ring")])
def test_round_is_encoding_and_gossip(rows, graph, kind):
    """The same bits as the two calls, over layouts with every kind of edge, to new parameters and in place, three rounds on."""
    csr = graph_of(rows, graph)
    for layout in (1, 515, "many", "gaps", 20000):
        with Case(layout, rows, kind=kind, csr=csr, seed=rows) as c:
            x, copy, total = c.values(0.02, kind), c.values(0.02), c.values(0.02)
            two = [[t.clone() for t in v] for v in (x, copy, total)]
            one = [[t.clone() for t in v] for v in (x, copy, total)]
            msg = c.messages(rows)
            for k in range(3):
                behind = one[0] if k == 1 else c.values(1.0, kind)
                B.dadam_mx4_encode(c.h, two[0], two[1], two[1], msg, stream())
                B.dadam_mx4_gossip(c.h, 0, msg, two[2], two[1], two[0], two[0], 0.6, stream())
                B.dadam_mx4_round(c.h, 0, one[0], behind, one[1], one[2], 0.6, stream())
                one[0] = behind
                for a, b in zip(one, two):
                    for i in range(rows):
                        assert same(host(a[i]), host(b[i])), (layout, k, i)
            c.padding_is_untouched(one[0] + one[1] + one[2])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_workers_by_themselves_do_what_all_replicas_in_one_handle_do(kind):
    """Six workers on a ring, each with a handle of one row and three messages (its own and the two it receives), against one handle of six
    rows: the same bits after four rounds, x, copies and sums."""
    n = 6
    with Case("many", n, kind=kind, csr=WL.ring(n), seed=9) as c:
        x, copy, total = c.values(0.02, kind), c.values(0.02), c.values(0.02)
        alone = [[t.clone() for t in v] for v in (x, copy, total)]
        handles, msg = [], c.messages(n)
        for _ in range(n):
            h = B.dadam_init(1, 3, c.d, c.offsets, c.sizes, H.ABI_DT[kind], H.ABI_DT[kind])
            B.dadam_set_topology(h, 0, *WL.node_share_ring())
            handles.append(h)
        for _ in range(4):
            B.dadam_mx4_round(c.h, 0, x, x, copy, total, 0.5, stream())
            for i, h in enumerate(handles):
                B.dadam_mx4_encode(h, alone[0][i:i + 1], alone[1][i:i + 1], alone[1][i:i + 1], msg[i:i + 1], stream())
            for i, h in enumerate(handles):
                received = [msg[i], msg[(i - 1) % n], msg[(i + 1) % n]]
                B.dadam_mx4_gossip(h, 0, received, alone[2][i:i + 1], alone[1][i:i + 1], alone[0][i:i + 1], alone[0][i:i + 1], 0.5, stream())
        torch.cuda.synchronize()
        for a, b in zip((x, copy, total), alone):
            for i in range(n):
                assert same(host(a[i]), host(b[i])), i
        for h in handles:
            B.dadam_destroy(h)


def test_replicas_agree_and_their_mean_stays():
    """Rounds alone bring replicas together although 4 bits are sent, and their mean moves by rounding only."""
    n, d = 8, 6000
    with Case(d, n, csr=WL.ring(n)) as c:
        x = c.values(1.0)
        mean = torch.stack(x).double().mean(0)
        copy = [torch.zeros(d, device=DEV) for _ in range(n)]
        total = [torch.zeros(d, device=DEV) for _ in range(n)]
        spread = lambda: float((torch.stack(x).double() - torch.stack(x).double().mean(0)).norm())  # noqa: E731
        at_first = spread()
        for _ in range(150):
            B.dadam_mx4_round(c.h, 0, x, x, copy, total, 0.5, stream())
        assert spread() < 1e-3 * at_first
        assert float((torch.stack(x).double().mean(0) - mean).abs().max()) < 1e-4


@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,graph", [(1, "identity"), (3, "ring"), (16, "exp"), (17, "complete"), (40, "ring"), (60, "complete"), (70, "ring")])
def test_layouts_that_stream(rows, graph, kind, shift):
    """23 million elements and more in all: accesses carry the streaming hint and the halves of a wavefront lie apart.  Long and short
    tensors, gaps inside and at the ends of the blocks of such halves, an end that is no multiple of 32.  Every call against the oracle
    on one row, the round against the two calls on every row.  shift: bytes by which buffers miss the beginning of a line."""
    each = 23_500_000 // rows
    offsets, sizes, at, rng = [], [], 5, np.random.default_rng(rows)
    while at < each:
        n = int(rng.choice([1, 700, 32768 * 3 + 17, 16384, 400_000]))
        n = min(n, each - at)
        offsets.append(at)
        sizes.append(n)
        at += n + int(rng.choice([0, 0, 3, 40, 2000]))
    d = at + 3
    stored = stored_of((offsets, sizes, d))
    pad = torch.from_numpy(~stored).to(DEV)
    csr = graph_of(rows, graph)
    h = B.dadam_init(rows, rows, d, offsets, sizes, H.ABI_DT[kind], H.ABI_DT[kind])
    assert B.dadam_get_plan_info(h).streaming == 1
    B.dadam_set_topology(h, 0, *csr)
    info = B.dadam_mx4_get_info(h)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows)

    def values(std, dtype=torch.float32):
        out = []
        for _ in range(rows):
            room = torch.empty(d + 16, dtype=dtype, device=DEV)
            t = room[shift // room.element_size():][:d]
            t.copy_(torch.randn(d, generator=gen, device=DEV) * std)
            t[pad] = float("nan")
            out.append(t)
        return out

    def copies(tensors):
        out = values(1.0, tensors[0].dtype)
        for a, b in zip(out, tensors):
            a.copy_(b)
        return out
    xt = H.TORCH_DT[kind]
    x, copy, total = values(0.02, xt), values(0.02), values(0.02)
    norms, clipped = torch.zeros(rows, device=DEV), values(1.0, xt)
    B.dadam_clip_grads(h, x, clipped, 1.0, norms, stream())
    msg = [torch.zeros(info.bytes, dtype=torch.uint8, device=DEV) for _ in range(rows)]
    moved, mixed, again, behind = values(1.0), copies(total), copies(total), values(1.0, xt)
    B.dadam_mx4_encode(h, x, copy, moved, msg, stream())
    B.dadam_mx4_gossip(h, 0, msg, mixed, moved, x, behind, 0.4, stream())
    out = values(1.0)
    B.dadam_mx4_product(h, 0, msg, out, 0, stream())
    added = copies(total)
    B.dadam_mx4_product(h, 0, msg, added, B.DADAM_MX4_ADD, stream())
    one = [copies(copy), values(1.0, xt)]
    B.dadam_mx4_round(h, 0, x, one[1], one[0], again, 0.4, stream())
    torch.cuda.synchronize()
    for i in range(rows):
        for a, b in ((one[0][i], moved[i]), (one[1][i], behind[i]), (again[i], mixed[i]), (added[i], mixed[i])):
            assert torch.equal(a.nan_to_num(nan=7.0), b.nan_to_num(nan=7.0)), i
    for t in clipped + moved + mixed + behind + out:
        assert torch.isnan(t[pad]).all() and not torch.isnan(t[~pad]).any()
    i = rows // 2
    xs, hs = host(x[i]), host(copy[i])
    want, sent = O.encode(xs, hs, stored)
    assert np.array_equal(msg[i].cpu().numpy()[:len(want)], want)
    assert same(host(moved[i])[stored], (hs + sent.astype(np.float32))[stored])
    n, scaled = O.clip(xs, stored, 1.0)
    assert abs(float(norms[i]) - n) <= 2 * EPS * n
    assert np.all((np.abs(host(clipped[i]) - scaled) <= np.abs(scaled) * (4 * EPS + (2.0 ** -8 if kind == "bf16" else 0)) + TINY)[stored])
    entries = [int(c) for c in csr[1][csr[0][i]:csr[0][i + 1]]]
    terms = [float(np.float32(1.0 / len(entries))) * O.decode(msg[c].cpu().numpy(), d) for c in entries]
    ref, size, k = sum(terms), sum(np.abs(v) for v in terms), len(entries)
    assert np.all((np.abs(host(out[i]) - ref) <= (k + 2) * EPS * size + (k + 2) * TINY)[stored])
    base = host(total[i]).astype(np.float64)
    assert np.all((np.abs(host(mixed[i]) - (base + ref)) <= (k + 2) * EPS * (size + np.abs(base)) + (k + 2) * TINY)[stored])
    s, c, v = host(mixed[i]).astype(np.float64), host(moved[i]).astype(np.float64), xs.astype(np.float64)
    ref = v + float(np.float32(0.4)) * (s - c)
    bound = 0.41 * EPS * (np.abs(s) + np.abs(c)) + 1.01 * EPS * np.abs(ref) + TINY + (2.0 ** -8 * np.abs(ref) if kind == "bf16" else 0)
    assert np.all((np.abs(host(behind[i]) - ref) <= bound)[stored])
    B.dadam_destroy(h)


def test_large_products_whose_rows_share_their_sums():
    """1e8 elements and more in all rows: one row of every list is formed and the others are copies of it.  Two loops of the alternating
    exponential ring and two nodes by themselves, 20 rows, gaps and odd ends; every row against the oracle's sum of its list."""
    rows, d = 20, 5_200_007
    offsets, sizes = [0, 1_000_003, 3_000_100], [1_000_000, 1_999_777, d - 3_000_103]
    stored = stored_of((offsets, sizes, d))
    pad = torch.from_numpy(~stored).to(DEV)
    csr = WL.aer(rows // 4, 0)
    h = B.dadam_init(rows, rows, d, offsets, sizes, B.DADAM_F32, B.DADAM_F32)
    B.dadam_set_topology(h, 0, *csr)
    info = B.dadam_mx4_get_info(h)
    msg = []
    for r in range(rows):
        m = torch.zeros(info.bytes, dtype=torch.uint8, device=DEV)
        x = torch.randn(d, device=DEV) * 0.02
        x[pad] = float("nan")
        one = B.dadam_init(1, 1, d, offsets, sizes, B.DADAM_F32, B.DADAM_F32)
        B.dadam_mx4_encode(one, [x], None, None, [m], stream())
        torch.cuda.synchronize()
        B.dadam_destroy(one)
        msg.append(m)
    out = torch.full((rows, d + 1), float("nan"), device=DEV)       # an even number of elements: every other row misses a line, all are aligned
    B.dadam_mx4_product(h, 0, msg, out, 0, stream())
    torch.cuda.synchronize()
    values = [O.decode(m.cpu().numpy(), d).astype(np.float32).astype(np.float64) for m in msg]
    for i in range(rows):
        entries = [int(c) for c in csr[1][csr[0][i]:csr[0][i + 1]]]
        terms = [float(np.float32(1.0 / len(entries))) * values[c] for c in entries]
        bound = (len(entries) + 2) * EPS * sum(np.abs(v) for v in terms) + (len(entries) + 2) * TINY
        got = host(out[i])
        assert np.all((np.abs(got[:d] - sum(terms)) <= bound)[stored]), i
        assert np.isnan(got[:d][~stored]).all() and np.isnan(got[d])
    B.dadam_destroy(h)


# ---------------------------------------------------------------------------------------------
# streams, graphs, other places
# ---------------------------------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    """All calls on a side stream, recorded once and replayed between eager work; every replay against the eager result."""
    n = 6
    csr = WL.ring(n)
    with Case("many", n, csr=csr) as c:
        def fresh():
            c.rng = np.random.default_rng(4)
            return c.values(0.1), c.values(0.02), c.values(0.02), c.values(0.02)
        norms, out, msg = torch.zeros(n, device=DEV), c.values(1.0), c.messages(n)

        def calls(g, x, copy, total):
            s = stream()
            B.dadam_clip_grads(c.h, g, out, 1.0, norms, s)
            B.dadam_mx4_round(c.h, 0, x, x, copy, total, 0.5, s)
            B.dadam_mx4_encode(c.h, x, copy, copy, msg, s)
            B.dadam_mx4_gossip(c.h, 0, msg, total, copy, x, x, 0.5, s)

        eager, recorded = fresh(), fresh()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        kept = []
        with torch.cuda.stream(side):
            for _ in range(3):
                calls(*eager)
                kept.append([t.clone() for v in (eager[1], eager[2], eager[3], out, [norms]) for t in v])
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls(*recorded)
        for want in kept:
            graph.replay()
            torch.cuda.synchronize()
            got = [t for v in (recorded[1], recorded[2], recorded[3], out, [norms]) for t in v]
            for a, b in zip(got, want):
                assert same(host(a), host(b))
            (torch.ones(1 << 20, device=DEV) * 2).sum().item()


def test_buffers_that_are_not_on_a_gpu_are_refused():
    with Case(100, 1, csr=WL.identity(1)) as c:
        on, off, norms = torch.zeros(1, 100, device=DEV), torch.zeros(1, 100), torch.zeros(1, device=DEV)
        for bad in (off, [off[0]]):
            with pytest.raises(ValueError, match="not on a GPU"):
                B.dadam_grad_norm(c.h, bad, norms)
        with pytest.raises(ValueError, match="not on a GPU"):
            B.dadam_grad_norm(c.h, on, off[0, :1])
        with pytest.raises(ValueError, match="not on a GPU"):
            B.dadam_mx4_round(c.h, 0, on, on, on.clone(), off, 0.5)


def test_rows_of_one_tensor():
    """A tensor whose rows are the buffers, some of them apart."""
    with Case(1000, 3, csr=WL.identity(3)) as c:
        big = torch.randn(3, 1024, device=DEV)
        rows = [big[k, :1000].clone() for k in range(3)]
        a, b = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV)
        B.dadam_grad_norm(c.h, big, a, stream())
        B.dadam_grad_norm(c.h, rows, b, stream())
        assert torch.equal(a, b)


def test_vectors_whose_offsets_pass_32_bits():
    """2^31 and a few elements in bfloat16: bytes and elements past 2^32 and 2^31; the values behind the mark count and are written."""
    d = (1 << 31) + 1027
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    h = B.dadam_init(1, 1, d, [0], [d], B.DADAM_BF16, B.DADAM_BF16)
    B.dadam_set_topology(h, 0, *WL.identity(1))
    tail = 4096
    g = torch.zeros(d, dtype=torch.bfloat16, device=DEV)
    g[-tail:] = torch.randn(tail, device=DEV).to(torch.bfloat16)
    norms = torch.zeros(1, device=DEV)
    B.dadam_clip_grads(h, [g], [g], 1.0, norms, stream())
    info = B.dadam_mx4_get_info(h)
    want = float(g[-tail:].double().norm())
    assert abs(want - 1.0) < 2.0 ** -7 and norms.item() > 10
    msg = torch.zeros(info.bytes, dtype=torch.uint8, device=DEV)
    copy, total = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    B.dadam_mx4_encode(h, [g], [copy], [copy], [msg], stream())
    ref, values = O.encode(host(g[-1027:]), None, np.ones(1027, bool))      # blocks begin at the mark
    assert same(host(copy[-1027:]), values)
    assert np.array_equal(msg[info.scale_offset:info.scale_offset + info.n_blocks][-33:].cpu().numpy(), ref[33 * 16:])
    B.dadam_mx4_product(h, 0, [msg], [total], 0, stream())
    assert torch.equal(total, copy)
    x = torch.zeros(d, dtype=torch.bfloat16, device=DEV)
    x[-5:] = 1
    B.dadam_mx4_round(h, 0, [g], [x], [copy], [total], 1.0, stream())
    B.dadam_mx4_gossip(h, 0, [msg], [total], [copy], [x], [x], 1.0, stream())
    torch.cuda.synchronize()
    assert not (x[-5:] == 1).any() and torch.isfinite(x[-tail:].float()).all()
    B.dadam_destroy(h)
