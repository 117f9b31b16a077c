"""Decentralized training over a slow network: clipped gradients, the Adam step, gossip in 4 bits.

    python examples/compressed_training.py [--replicas 8] [--steps 200] [--exact]

Replicas of a small language model on one GPU, every one with data of its own, on a ring.  One iteration is

    dadam_clip_grads      every replica's gradient by its own norm
    dadam_gossip_step     the Adam step of every replica for itself (the identity as mixing matrix)
    dadam_mx4_round       what the replicas would send each other, as 4-bit differences, and the gossip update from it

--exact mixes whole parameters in the step instead (the ring as mixing matrix), for comparison.  Prints the loss, how far the
replicas are apart and the bytes a replica sends an iteration.  Where a process holds one replica, dadam_mx4_encode gives the
message to send and dadam_mx4_gossip takes those received.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_11998_amd import binding as B  # noqa: E402
from paper_2410_11998_amd import workloads as WL  # noqa: E402

VOCAB, WIDTH, CONTEXT, BATCH = 64, 48, 8, 128
SHAPES = [("embed", (VOCAB, WIDTH)), ("w1", (CONTEXT * WIDTH, 4 * WIDTH)), ("b1", (4 * WIDTH,)), ("w2", (4 * WIDTH, VOCAB)), ("b2", (VOCAB,))]
IDENTITY, RING = 0, 1


def model_loss(flat, layout, tokens):
    """Next-token loss of a feed-forward language model whose parameters are views of one packed vector."""
    p = {n: flat[int(o):int(o) + int(k)].view(s) for (n, s), o, k in zip(SHAPES, layout.offsets, layout.numels)}
    h = torch.tanh(p["embed"][tokens[:, :-1]].flatten(1) @ p["w1"] + p["b1"])
    return torch.nn.functional.cross_entropy(h @ p["w2"] + p["b2"], tokens[:, -1])


def batches(replicas, device, gen):
    """Text of a random first-order process; replica i sees its words shifted half of the time, so no two have the same data."""
    table = torch.softmax(3 * torch.randn(VOCAB, VOCAB, generator=gen, device=device), dim=1)
    while True:
        out = []
        for i in range(replicas):
            t = [torch.randint(0, VOCAB, (BATCH,), generator=gen, device=device)]
            for _ in range(CONTEXT):
                t.append(torch.multinomial(table[t[-1]], 1, generator=gen)[:, 0])
            t = torch.stack(t, dim=1)
            t[:BATCH // 2] = (t[:BATCH // 2] + i) % VOCAB
            out.append(t)
        yield out


def train(replicas=8, steps=200, exact=False, seed=0, gamma=0.5, max_norm=0.4, say=print):
    device = torch.device("cuda:0")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    layout = WL.pack(SHAPES, align_elems=32)        # no block of a message belongs to two tensors
    d = layout.d
    h = B.dadam_init(replicas, replicas, d, layout.offsets, layout.numels, lr=3e-3)
    B.dadam_set_topology(h, IDENTITY, *WL.identity(replicas))
    B.dadam_set_topology(h, RING, *WL.ring(replicas))
    x = torch.zeros(replicas, d, device=device)
    for o, n in zip(layout.offsets, layout.numels):
        x[:, int(o):int(o) + int(n)] = 0.05 * torch.randn(int(n), generator=gen, device=device)
    stepped, m, v = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    B.dadam_bind(h, list(x), list(stepped), list(m), list(v))
    copy, total = x.clone(), x.clone()              # everybody knows the common start
    norms = torch.zeros(replicas, device=device)
    data, losses = batches(replicas, device, gen), []
    for t in range(1, steps + 1):
        grads, loss = torch.zeros_like(x), 0.0
        for i, tokens in enumerate(next(data)):
            flat = x[i].detach().requires_grad_()
            value = model_loss(flat, layout, tokens)
            value.backward()
            grads[i] = flat.grad
            loss += float(value.detach()) / replicas
        stream = B.current_stream()
        B.dadam_clip_grads(h, grads, grads, max_norm, norms, stream)
        if exact:
            B.dadam_gossip_step(h, RING, list(grads), t, B.DADAM_FUSE_ACCUM, stream)
            x.copy_(stepped)
        else:
            B.dadam_gossip_step(h, IDENTITY, list(grads), t, B.DADAM_FUSE_ACCUM, stream)
            B.dadam_mx4_round(h, RING, stepped, x, copy, total, gamma, stream)
        losses.append(loss)
        if t % 50 == 0 or t == steps:
            apart = float((x - x.mean(0)).norm() / x.norm())
            say("step %4d  loss %.4f  apart %.2e  largest gradient norm %.2f" % (t, loss, apart, float(norms.max())))
    sent = 4 * d if exact else B.dadam_mx4_get_info(h).bytes
    say("a replica sends %d bytes to each neighbour an iteration (%.2f bits an element)" % (sent, 8 * sent / d))
    torch.cuda.synchronize()
    B.dadam_destroy(h)
    return losses, float((x - x.mean(0)).norm() / x.norm())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--replicas", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--exact", action="store_true")
    a = ap.parse_args()
    train(a.replicas, a.steps, a.exact)
