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


# ---------------------------------------------------------------------------------------------
# norms of rows that many workgroups share
# ---------------------------------------------------------------------------------------------

def workgroups_of_a_row(d, rows):
    """Sixteen wavefronts a workgroup, four granules of 512 elements a wavefront and more, 256 workgroups in all."""
    return max(1, min(-(-(-(-d // 512)) // 64), 256 // rows))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout,rows,least", [(8_500_001, 1, 256), (2_100_003, 3, 64), (1_000_000, 7, 31), (100_003, 5, 4), ("many", 2, 2)])
def test_norms_that_many_workgroups_share_are_the_same_every_time(layout, rows, least, kind):
    """Whichever workgroup of a row is last adds the same partial sums in the same order: 24 calls, norms alone and clipping, under load or
    not, the same bits, and within 2 eps of the oracle's."""
    with Case(layout, rows, kind=kind, seed=rows) as c:
        assert workgroups_of_a_row(c.d, rows) >= least >= 2
        g = [t * (0.2 + k) for k, t in enumerate(c.values(0.1, kind))]
        out = c.values(1.0, kind)
        norms = [torch.full((rows,), -1.0, device=DEV) for _ in range(24)]
        noise = torch.randn(1 << 22, device=DEV)
        for k, n in enumerate(norms):
            if k % 3 == 1:
                noise = noise * 1.0001
            if k % 2:
                B.dadam_clip_grads(c.h, g, out, 1e-3, n, stream())
            else:
                B.dadam_grad_norm(c.h, g, n, stream())
        want = np.asarray([O.grad_norm(host(t), c.stored) for t in g])
        assert np.all(np.abs(norms[0].cpu().numpy() - want) <= 2 * EPS * want)
        assert all(torch.equal(n, norms[0]) for n in norms)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 4, 40])
def test_clipping_in_place_where_handles_stream(rows, kind):
    """Gaps inside and between the halves of a wavefront's block: the same bits in place and to other buffers, padding untouched, rows
    below the limit left alone."""
    each = 23_000_000 // rows
    offsets, sizes, at, rng = [], [], 3, np.random.default_rng(rows)
    while at < each:
        n = min(int(rng.choice([1, 900, 32768 + 11, 300_000])), each - at)
        offsets.append(at)
        sizes.append(n)
        at += n + int(rng.choice([0, 2, 50, 1500]))
    d = at + 5
    stored = torch.from_numpy(stored_of((offsets, sizes, d))).to(DEV)
    h = B.dadam_init(rows, rows, d, offsets, sizes, H.ABI_DT[kind], H.ABI_DT[kind])
    assert B.dadam_get_plan_info(h).streaming == 1
    g = []
    for k in range(rows):
        t = (torch.randn(d, device=DEV) * (0.1 if k % 3 else 1e-6)).to(H.TORCH_DT[kind])
        t[~stored] = float("nan")
        g.append(t)
    out, inplace = [torch.full_like(t, float("nan")) for t in g], [t.clone() for t in g]
    a, b = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    B.dadam_clip_grads(h, g, out, 1.0, a, stream())
    B.dadam_clip_grads(h, inplace, inplace, 1.0, b, stream())
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    for k in range(rows):
        n = float(g[k][stored].double().norm())
        assert abs(float(a[k]) - n) <= 3 * EPS * n       # the oracle's own sum is in 64 bits too
        assert torch.equal(inplace[k].nan_to_num(nan=7.0), out[k].nan_to_num(nan=7.0))
        assert torch.isnan(inplace[k][~stored]).all() and not torch.isnan(inplace[k][stored]).any()
        if k % 3 == 0:
            assert torch.equal(inplace[k][stored], g[k][stored])
        else:
            ref = g[k].double() / n
            bound = ref.abs() * (4 * EPS + (2.0 ** -8 if kind == "bf16" else 0)) + TINY
            assert bool(((inplace[k].double() - ref).abs() <= bound)[stored].all())
    B.dadam_destroy(h)


# ---------------------------------------------------------------------------------------------
# parameters of one type, gradients of the other
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", [1000, 70001, "gaps"])
@pytest.mark.parametrize("param,grad", [("f32", "bf16"), ("bf16", "f32")])
def test_handles_with_two_types(param, grad, layout):
    """Norms and clipping go by the gradients' type, messages, gossip and rounds by the parameters': the bits of handles of one type."""
    n, csr = 3, WL.ring(3)
    with Case(layout, n, kind=param, csr=csr) as p, Case(layout, n, kind=grad, csr=csr) as q:
        h = B.dadam_init(n, n, p.d, p.offsets, p.sizes, H.ABI_DT[param], H.ABI_DT[grad])
        B.dadam_set_topology(h, 0, *csr)
        g, x, copy, total, msg = q.values(0.1, grad), p.values(0.02, param), p.values(0.02), p.values(0.02), p.random_messages(n)
        results = []
        for hg, hp in ((h, h), (q.h, p.h)):
            norms, again, out = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), [torch.zeros_like(t) for t in g]
            B.dadam_grad_norm(hg, g, norms, stream())
            B.dadam_clip_grads(hg, g, out, 0.5, again, stream())
            sent, moved = p.messages(n), [torch.zeros_like(t) for t in copy]
            B.dadam_mx4_encode(hp, x, copy, moved, sent, stream())
            s, y = [t.clone() for t in total], [torch.zeros_like(t) for t in x]
            B.dadam_mx4_gossip(hp, 0, msg, s, copy, x, y, 0.6, stream())
            k, r, z = [t.clone() for t in copy], [t.clone() for t in total], [torch.zeros_like(t) for t in x]
            B.dadam_mx4_round(hp, 0, x, z, k, r, 0.6, stream())
            results.append([norms, again] + out + moved + s + y + k + r + z + sent)
        torch.cuda.synchronize()
        B.dadam_destroy(h)
        for a, b in zip(*results):
            assert same(host(a), host(b))


# ---------------------------------------------------------------------------------------------
# rows that share lists
# ---------------------------------------------------------------------------------------------

def unequal_lists(rows, n):
    """Rows in turn of n lists of all sources that differ in their weights, and a last row of its own."""
    rng = np.random.default_rng(n)
    w = rng.random((n + 1, rows)) + 0.2
    w = (w / w.sum(1, keepdims=True)).astype(np.float32)
    pick = [i % n for i in range(rows - 1)] + [n]
    return np.arange(0, rows * rows + 1, rows), np.tile(np.arange(rows), rows), w[pick].reshape(-1)


SHARED = [(32, 2, "lists"), (48, 3, "lists"), (64, 4, "lists"), (96, 4, "lists"), (128, 4, "lists"), (160, 2, "lists"), (97, 1, "lists"), (101, 1, "lists"),
          (127, 1, "lists"), (20, 2, "unequal"), (65, 3, "unequal"), (113, 3, "unequal")]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,lists", SHARED + [(97, 0, "ring"), (112, 0, "ring"), (128, 0, "exp")])
def test_rounds_of_every_shape(rows, n, lists, kind):
    """One to four lists whose sums the wavefronts form together, a list of one row among them, and rounds of 97 to 128 rows: the bits of
    encoding and gossip, two rounds on."""
    csr = {"lists": lists_of, "unequal": unequal_lists}[lists](rows, n) if n else csr_of(rows, rows, lists)
    for layout in (1, 515, "gaps", 3000):
        with Case(layout, rows, kind=kind, csr=csr, seed=rows) as c:
            x, copy, total = c.values(0.02, kind), c.values(0.02), c.values(0.02)
            two = [[t.clone() for t in v] for v in (x, copy, total)]
            one = [[t.clone() for t in v] for v in (x, copy, total)]
            msg = c.messages(rows)
            for k in range(2):
                behind = one[0] if k else c.values(1.0, kind)
                B.dadam_mx4_encode(c.h, two[0], two[1], two[1], msg, stream())
                B.dadam_mx4_gossip(c.h, 0, msg, two[2], two[1], two[0], two[0], 0.6, stream())
                B.dadam_mx4_round(c.h, 0, one[0], behind, one[1], one[2], 0.6, stream())
                one[0] = behind
                for a, b in zip(one, two):
                    for i in range(rows):
                        assert same(host(a[i]), host(b[i])), (layout, k, i)
            c.padding_is_untouched(one[0] + one[1] + one[2])


@pytest.mark.parametrize("rows,n,lists", SHARED)
def test_products_and_gossip_of_shared_lists(rows, n, lists):
    """By workgroups that form a sum together: against the oracle, and gossip's sums against the product's."""
    csr = {"lists": lists_of, "unequal": unequal_lists}[lists](rows, n)
    for layout in (33, "gaps"):
        with Case(layout, rows, csr=csr, seed=rows) as c:
            msg, old = c.random_messages(rows), c.values(0.02)
            out, add, total, x = c.values(1.0), [t.clone() for t in old], [t.clone() for t in old], c.values(0.02)
            B.dadam_mx4_product(c.h, 0, msg, out, 0, stream())
            check_sums(c, msg, csr, None, out, "store")
            B.dadam_mx4_product(c.h, 0, msg, add, B.DADAM_MX4_ADD, stream())
            check_sums(c, msg, csr, old, add, "add")
            B.dadam_mx4_gossip(c.h, 0, msg, total, [t.clone() for t in old], x, x, 0.6, stream())
            for a, b in zip(add, total):
                assert same(host(a), host(b))
            c.padding_is_untouched(out + add + total + x)


@pytest.mark.parametrize("rows,n,d", [(8, 1, 1_000_003), (16, 2, 1_000_000), (24, 2, 800_017)])
def test_products_of_shared_lists_that_do_not_stream(rows, n, d):
    """1536 granules and more, up to 22 million elements in all: a wavefront takes a unit of all rows, stored and added."""
    csr = lists_of(rows, n)
    with Case(d, rows, csr=csr, seed=rows) as c:
        assert B.dadam_get_plan_info(c.h).streaming == 0 and d >= 1536 * 512
        msg, old = c.random_messages(rows), c.values(0.02)
        out, add = c.values(1.0), [t.clone() for t in old]
        B.dadam_mx4_product(c.h, 0, msg, out, 0, stream())
        B.dadam_mx4_product(c.h, 0, msg, add, B.DADAM_MX4_ADD, stream())
        values = [O.decode(m.cpu().numpy(), d) for m in msg]
        for i in range(rows):
            entries = [int(k) for k in csr[1][csr[0][i]:csr[0][i + 1]]]
            if i == entries[0]:
                w = float(csr[2][csr[0][i]])
                ref, size = w * sum(values[k] for k in entries), w * sum(np.abs(values[k]) for k in entries)
            k = len(entries) + 2
            assert np.all(np.abs(host(out[i]) - ref) <= k * EPS * size + k * TINY), i
            base = host(old[i]).astype(np.float64)
            assert np.all(np.abs(host(add[i]) - (base + ref)) <= k * EPS * (size + np.abs(base)) + k * TINY), i


@pytest.mark.parametrize("rows,n", [(8, 1), (8, 2)])
def test_large_products_of_few_rows_copy_their_first(rows, n):
    """1e8 elements in all rows, up to sixteen rows: the first row of every list against the oracle, the others its copies; adding to zeros
    gives the same values by wavefronts that form the sums themselves."""
    d, csr = 13_000_007, lists_of(rows, n)
    offsets, sizes = [2, 5_000_001], [4_000_000, d - 5_000_001]
    stored = stored_of((offsets, sizes, d))
    pad = torch.from_numpy(~stored).to(DEV)
    h = B.dadam_init(rows, rows, d, offsets, sizes)
    B.dadam_set_topology(h, 0, *csr)
    info = B.dadam_mx4_get_info(h)
    x = []
    for _ in range(rows):
        t = torch.randn(d, device=DEV) * 0.02
        t[pad] = float("nan")
        x.append(t)
    msg = [torch.zeros(info.bytes, dtype=torch.uint8, device=DEV) for _ in range(rows)]
    B.dadam_mx4_encode(h, x, None, None, msg, stream())
    out, add = [torch.full((d,), float("nan"), device=DEV) for _ in range(rows)], [torch.zeros(d, device=DEV) for _ in range(rows)]
    B.dadam_mx4_product(h, 0, msg, out, 0, stream())
    B.dadam_mx4_product(h, 0, msg, add, B.DADAM_MX4_ADD, stream())
    torch.cuda.synchronize()
    each = rows // n
    for i in range(rows):
        first = i // each * each
        assert torch.isnan(out[i][pad]).all() and not add[i][pad].any()
        assert torch.equal(out[i][~pad], out[first][~pad]) and torch.equal(out[i][~pad], add[i][~pad])
        if i == first:
            terms = [float(csr[2][0]) * O.decode(m.cpu().numpy(), d) for m in msg[first:first + each]]
            bound = (each + 2) * EPS * sum(np.abs(v) for v in terms) + (each + 2) * TINY
            assert np.all((np.abs(host(out[i]) - sum(terms)) <= bound)[stored])
    B.dadam_destroy(h)


@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,graph", [(100, "exp"), (112, "complete"), (127, "complete"), (128, "ring"), (150, "ring"), (160, "complete")])
def test_streaming_rounds_of_many_rows(rows, graph, kind, shift):
    """97 rows and more where handles stream, eight and ten rows a wavefront: the bits of encoding and gossip.  Gaps, odd ends, rows on
    and off a line."""
    each = 23_000_000 // rows
    offsets, sizes, at, rng = [], [], 7, np.random.default_rng(rows)
    while at < each:
        n = min(int(rng.choice([1, 700, 16384 + 5, 60_000])), each - at)
        offsets.append(at)
        sizes.append(n)
        at += n + int(rng.choice([0, 3, 40, 1000]))
    d = at + 3
    pad = torch.from_numpy(~stored_of((offsets, sizes, d))).to(DEV)
    h = B.dadam_init(rows, rows, d, offsets, sizes, H.ABI_DT[kind], H.ABI_DT[kind])
    assert B.dadam_get_plan_info(h).streaming == 1
    B.dadam_set_topology(h, 0, *csr_of(rows, rows, graph))
    info = B.dadam_mx4_get_info(h)

    def values(dtype=torch.float32):
        t = (torch.randn(rows, -(-d // 64) * 64 + 64, device=DEV) * 0.02).to(dtype)
        t = t[:, shift // t.element_size():][:, :d]
        t[:, pad] = float("nan")
        return t

    def copied(t):
        room = torch.empty(rows, t.stride(0), dtype=t.dtype, device=DEV)[:, shift // t.element_size():][:, :d]
        room.copy_(t)
        return room
    x, copy, total = values(H.TORCH_DT[kind]), values(), values()
    y, k, s, z = copied(x), copied(copy), copied(total), copied(x)
    msg = torch.zeros(rows, info.bytes, dtype=torch.uint8, device=DEV)
    B.dadam_mx4_round(h, 0, x, z, k, s, 0.4, stream())
    B.dadam_mx4_encode(h, x, copy, copy, msg, stream())
    B.dadam_mx4_gossip(h, 0, msg, total, copy, x, y, 0.4, stream())
    torch.cuda.synchronize()
    for a, b in ((z, y), (k, copy), (s, total)):
        assert torch.equal(a.nan_to_num(nan=7.0), b.nan_to_num(nan=7.0))
        assert torch.isnan(a[:, pad]).all() and not torch.isnan(a[:, ~pad]).any()
    B.dadam_destroy(h)


# ---------------------------------------------------------------------------------------------
# matrices that change
# ---------------------------------------------------------------------------------------------

def test_a_sum_for_every_matrix_where_matrices_change():
    """One-peer exponential graph on 8 replicas, a slot a phase, 150 rounds: gossip with the round's slot on that slot's sum, its messages added
    to the other sums too.  Every sum stays W copy, replicas agree and their mean stays, also where they start apart from copies at 0.
    Two of the slots are set after the handle's first call.
    Bounds: a round's rounding of a sum is 4 eps of what it is made of (two products), of a copy 1 eps, twice in W copy; magnitudes below 8."""
    n, phases, rounds = 8, 3, 150
    with Case("many", n, csr=WL.one_peer_exponential(n, 0), seed=2) as c:
        stored = torch.from_numpy(c.stored).to(DEV)
        x = [t.nan_to_num(nan=0.0) for t in c.values(1.0)]
        start = torch.stack(x).double()
        copy = [torch.zeros(c.d, device=DEV) for _ in range(n)]
        sums = [[torch.zeros(c.d, device=DEV) for _ in range(n)] for _ in range(phases)]
        msg, norms = c.messages(n), torch.zeros(n, device=DEV)
        B.dadam_grad_norm(c.h, x, norms, stream())
        for p in range(1, phases):
            B.dadam_set_topology(c.h, p, *WL.one_peer_exponential(n, p))
        for k in range(rounds):
            B.dadam_mx4_encode(c.h, x, copy, copy, msg, stream())
            for p in range(phases):
                if p != k % phases:
                    B.dadam_mx4_product(c.h, p, msg, sums[p], B.DADAM_MX4_ADD, stream())
            B.dadam_mx4_gossip(c.h, k % phases, msg, sums[k % phases], copy, x, x, 0.5, stream())
        torch.cuda.synchronize()
        h = torch.stack(copy).double()
        assert float(h.abs().max()) < 8
        for p in range(phases):
            ptr, col, w = WL.one_peer_exponential(n, p)
            for i in range(n):
                want = sum(float(w[e]) * h[int(col[e])] for e in range(ptr[i], ptr[i + 1]))
                assert float((sums[p][i].double() - want).abs()[stored].max()) <= rounds * 6 * EPS * 8, (p, i)
        spread = lambda t: float((t - t.mean(0))[:, stored].norm())  # noqa: E731
        assert spread(torch.stack(x).double()) < 1e-2 * spread(start)
        assert float((torch.stack(x).double().mean(0) - start.mean(0)).abs()[stored].max()) < 1e-4
