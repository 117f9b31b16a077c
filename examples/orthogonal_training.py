"""Decentralized training of a small language model whose matrices step along orthogonalised momenta.

    python examples/orthogonal_training.py [--replicas 8] [--steps 200] [--adam]

Replicas on one GPU, every one with data of its own, on a ring.  The words' vectors are the output matrix too.  One iteration is

    torch                    hidden vectors of every replica's batch
    dadam_head_loss          the loss of all replicas, its gradient into the packed gradients (dW, dbias) and to the hidden vectors
    torch                    backward from there
    dadam_clip_grads         every replica's gradient by its own norm
    dadam_ortho_step         the hidden layers' matrices, mixed and stepped along their orthogonalised first moments
    dadam_gossip_step_range  everything else, by Adam

--adam steps everything by Adam, for comparison.  Prints the loss and how far the replicas are apart.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_11998_amd import binding as B  # noqa: E402
from paper_2410_11998_amd import workloads as WL  # noqa: E402

VOCAB, WIDTH, INNER, CONTEXT, BATCH = 64, 48, 192, 8, 128
SHAPES = [("words", (VOCAB, WIDTH)), ("bias", (VOCAB,)), ("b1", (INNER,)), ("w1", (CONTEXT * WIDTH, INNER)), ("w2", (INNER, WIDTH))]
BY_ADAM, MATRICES = (0, 3), (3, 4)                  # tensors
RING = 0


def views(flat, layout):
    return {n: flat[int(o):int(o) + int(k)].view(s) for (n, s), o, k in zip(SHAPES, layout.offsets, layout.numels)}


def hidden_vectors(flat, layout, tokens):
    p = views(flat, layout)
    return torch.tanh(p["words"][tokens].flatten(1) @ p["w1"] + p["b1"]) @ p["w2"]


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


class Trainer:
    def __init__(self, replicas=8, seed=0, lr=3e-3):
        device = torch.device("cuda:0")
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        self.layout = WL.pack(SHAPES, align_elems=32)
        d = self.layout.d
        self.h = B.dadam_init(replicas, replicas, d, self.layout.offsets, self.layout.numels, lr=lr)
        B.dadam_set_topology(self.h, RING, *WL.ring(replicas))
        B.dadam_set_matrices(self.h, [(k, *SHAPES[k][1], SHAPES[k][1][1], 0, 0.2 * max(SHAPES[k][1]) ** 0.5) for k in MATRICES])
        self.head = B.dadam_head(0, 1, VOCAB, WIDTH)
        x = torch.zeros(replicas, d, device=device)
        for o, n in zip(self.layout.offsets, self.layout.numels):
            x[:, int(o):int(o) + int(n)] = 0.05 * torch.randn(int(n), generator=self.gen, device=device)
        self.x, self.stepped, m, v = x, torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
        self.bound = [list(t) for t in (m, v)]
        B.dadam_bind(self.h, list(self.x), list(self.stepped), *self.bound)
        n = max(B.dadam_head_get_info(self.h, self.head, BATCH, True).bytes, B.dadam_ortho_get_info(self.h).bytes)
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)
        self.norms, self.losses = torch.zeros(replicas, device=device), torch.zeros(replicas, device=device)
        self.data = batches(replicas, device, self.gen)

    def gradients(self, tokens):
        """(replicas, d) gradients of every replica's own mean loss, which is left in self.losses."""
        flats = [row.detach().requires_grad_() for row in self.x]
        hidden = [hidden_vectors(f, self.layout, t[:, :-1]) for f, t in zip(flats, tokens)]
        targets = [t[:, -1].to(torch.int32) for t in tokens]
        grads, dhidden = torch.zeros_like(self.x), [torch.empty_like(v) for v in hidden]
        B.dadam_head_loss(self.h, self.head, self.x, [v.detach() for v in hidden], targets, BATCH, 1.0, B.DADAM_HEAD_MEAN, self.losses, None, dhidden, grads, self.workspace,
                          B.current_stream())
        for v, dv in zip(hidden, dhidden):
            v.backward(dv)
        for g, f in zip(grads, flats):
            g += f.grad                             # the words' gradient as inputs beside the one as outputs
        return grads

    def step(self, grads, t, adam=False, max_norm=1.0):
        stream, g = B.current_stream(), list(grads)
        B.dadam_clip_grads(self.h, grads, grads, max_norm, self.norms, stream)
        if adam:
            B.dadam_gossip_step(self.h, RING, g, t, B.DADAM_FUSE_ACCUM, stream)
        else:
            B.dadam_ortho_step(self.h, RING, g, t, B.DADAM_FUSE_ACCUM | B.DADAM_ORTHO_NESTEROV, self.workspace, stream)
            B.dadam_gossip_step_range(self.h, RING, g, t, B.DADAM_FUSE_ACCUM, *BY_ADAM, stream)
        B.dadam_swap_x(self.h)
        self.x, self.stepped = self.stepped, self.x

    def close(self):
        torch.cuda.synchronize()
        B.dadam_destroy(self.h)


def train(replicas=8, steps=200, adam=False, seed=0, say=print):
    trainer, losses = Trainer(replicas, seed), []
    for t in range(1, steps + 1):
        grads = trainer.gradients(next(trainer.data))
        losses.append(float(trainer.losses.mean()))
        trainer.step(grads, t, adam)
        if t % 50 == 0 or t == steps:
            x = trainer.x
            say("step %4d  loss %.4f  apart %.2e  largest gradient norm %.2f" % (t, losses[-1], float((x - x.mean(0)).norm() / x.norm()), float(trainer.norms.max())))
    trainer.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--replicas", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--adam", action="store_true")
    a = ap.parse_args()
    train(a.replicas, a.steps, a.adam)
