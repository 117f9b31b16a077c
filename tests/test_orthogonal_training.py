"""The example of training with the head's loss and orthogonalised steps: that it runs, and its gradients."""

import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from oracle import ends_oracle as O
from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 2.0 ** -24


def example():
    spec = importlib.util.spec_from_file_location("orthogonal_training", os.path.join(ROOT, "examples", "orthogonal_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("adam", [False, True])
def test_it_runs(adam):
    losses = example().train(replicas=4, steps=7, adam=adam, say=lambda line: print(line, flush=True))
    assert len(losses) == 7 and all(math.isfinite(v) for v in losses)
    assert abs(losses[0] - math.log(64)) < 0.1          # small parameters: every word is as likely


def test_gradients_are_those_of_the_whole_loss():
    ex = example()
    t = ex.Trainer(replicas=3, seed=4)
    tokens = next(t.data)
    got = t.gradients(tokens).cpu().double()
    for i in range(3):
        flat = t.x[i].cpu().double().requires_grad_()
        p = ex.views(flat, t.layout)
        hidden = ex.hidden_vectors(flat, t.layout, tokens[i][:, :-1].cpu())
        loss = torch.nn.functional.cross_entropy(hidden @ p["words"].T + p["bias"], tokens[i][:, -1].cpu())
        loss.backward()
        # Sums of at most 384 float32 products, three deep, of factors that are themselves rounded: in the 2-norm below 1000 half steps of the gradient.
        assert abs(float(t.losses[i]) - float(loss.detach())) <= 1e-5
        off = float((got[i] - flat.grad).norm())
        assert off <= 1000 * EPS * float(flat.grad.norm()), f"replica {i}: off by {off} of {float(flat.grad.norm())}"
    t.close()


def test_a_run_of_all_calls_on_a_stream_and_in_a_graph():
    """Loss, clip, the matrices' step and everything else's: eagerly on a stream of its own and replayed, bit for bit; and against the statement in 64 bits."""
    rows, vocab, width, tokens = 4, 130, 72, 33
    shapes = [("words", (vocab, width)), ("bias", (vocab,)), ("w", (width, 200))]
    layout = WL.pack(shapes, align_elems=32)
    h = B.dadam_init(rows, rows, layout.d, layout.offsets, layout.numels, lr=0.01)
    B.dadam_set_topology(h, 0, *WL.ring(rows))
    B.dadam_set_matrices(h, [(2, width, 200)])
    head = B.dadam_head(0, 1, vocab, width)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    new = lambda *s, std=1.0: std * torch.randn(*s, generator=gen, device="cuda:0")  # noqa: E731
    x0, m0, v0 = new(rows, layout.d, std=0.1), new(rows, layout.d, std=1e-3), new(rows, layout.d, std=1e-3).square()
    hidden = new(rows, tokens, width)
    targets = torch.randint(-1, vocab, (rows, tokens), generator=gen, device="cuda:0", dtype=torch.int32)
    rest = new(rows, layout.d, std=1e-2)                # the gradients of everything before the head
    x, out, m, v = x0.clone(), torch.zeros_like(x0), m0.clone(), v0.clone()
    grads, losses, norms = torch.zeros_like(x0), torch.zeros(rows, device="cuda:0"), torch.zeros(rows, device="cuda:0")
    dhidden = torch.zeros_like(hidden)
    work = torch.empty(max(B.dadam_head_get_info(h, head, tokens, True).bytes, B.dadam_ortho_get_info(h).bytes), dtype=torch.uint8, device="cuda:0")
    B.dadam_bind(h, list(x), list(out), list(m), list(v))
    g = list(grads)

    def iteration():
        s = B.current_stream()
        grads.copy_(rest)
        B.dadam_head_loss(h, head, x, hidden.flatten(1), targets, tokens, 1.0, B.DADAM_HEAD_MEAN | B.DADAM_HEAD_ADD, losses, None, dhidden.flatten(1), grads, work, s)
        B.dadam_clip_grads(h, grads, grads, 1.0, norms, s)
        B.dadam_ortho_step(h, 0, g, 1, B.DADAM_FUSE_ACCUM, work, s)
        B.dadam_gossip_step_range(h, 0, g, 1, B.DADAM_FUSE_ACCUM, 0, 2, s)

    def again():
        for a, b in ((m, m0), (v, v0)):
            a.copy_(b)
        for a in (out, dhidden, losses, norms):
            a.fill_(7.0)
        work.fill_(0xFF)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again()
        iteration()
    torch.cuda.synchronize()
    eager = [a.clone() for a in (out, m, v, dhidden, losses, norms, grads)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        iteration()
    for _ in range(3):
        again()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (out, m, v, dhidden, losses, norms, grads)):
            assert torch.equal(a, b)

    spans = [(int(o), int(o) + int(n)) for o, n in zip(layout.offsets, layout.numels)]
    xs, ms, beta = x0.cpu().numpy().astype(np.float64), m0.cpu().numpy(), float(np.float32(0.9))
    rp, col, w = WL.ring(rows)
    for i in range(rows):
        r = O.head_loss(hidden[i].cpu().numpy(), xs[i, slice(*spans[0])].reshape(vocab, width), xs[i, slice(*spans[1])], targets[i].cpu().numpy(), 1.0, True)
        total = rest[i].cpu().numpy().astype(np.float64)
        total[slice(*spans[0])] += r["dhead"].reshape(-1)
        total[slice(*spans[1])] += r["dbias"]
        norm = np.sqrt(sum(np.square(total[a:b]).sum() for a, b in spans))
        assert abs(float(losses[i]) - r["loss"]) <= 1e-5 * r["loss"] and abs(float(norms[i]) - norm) <= 1e-5 * norm
        matrix = slice(*spans[2])
        u = beta * ms[i, matrix] + (1 - beta) * total[matrix] * min(1.0, 1.0 / norm)
        o = O.orthogonalised(u.reshape(width, 200)).reshape(-1)
        want = sum(float(w[k]) * xs[col[k], matrix] for k in range(rp[i], rp[i + 1])) - 0.01 * o
        # the direction by its own bound and by 900 (the steepest slope of five iterations) times what u was rounded: a norm, a factor, two products, a sum
        off = 0.01 * (O.orthogonalised_error(u.reshape(width, 200), 2) + 900 * 1e-5) + 8 * EPS * np.linalg.norm(want)
        assert np.linalg.norm(out[i, matrix].cpu().numpy() - want) <= off
    B.dadam_destroy(h)
