"""The ends of an iteration where elements' numbers pass 32 bits: matrices and heads that lie that far in the packed vector, and a head that is that long."""

import pytest
import torch

from paper_2410_11998_amd import binding as B
from paper_2410_11998_amd import workloads as WL

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FAR = 2 ** 32 + 64
KINDS = {"f32": (B.DADAM_F32, torch.float32), "bf16": (B.DADAM_BF16, torch.bfloat16)}


def normal(seed, *shape, std=1.0):
    return std * torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def handle(before, sizes, kind):
    """(handle, where the tensors begin, elements): tensors of these sizes behind one of `before` elements."""
    offsets, at = [], before
    for n in sizes:
        offsets.append(at)
        at += -(-n // 8) * 8
    return B.dadam_init(1, 1, at, [0] + offsets, [before] + sizes, KINDS[kind][0], KINDS[kind][0], lr=0.1), offsets, at


@pytest.mark.parametrize("shape", [(60, 48), (300, 200)], ids=["held", "tiles"])
def test_matrices_far_in_the_vector(shape):
    r, c = shape
    got = []
    for before in (64, FAR):
        h, (at,), d = handle(before, [r * c], "bf16")
        B.dadam_set_topology(h, 0, *WL.identity(1))
        B.dadam_set_matrices(h, [(1, r, c)])
        g, out = torch.zeros(1, d, device=DEV, dtype=torch.bfloat16), torch.zeros(1, d, device=DEV, dtype=torch.bfloat16)
        g[0, at:at + r * c] = normal(1, r * c).to(g)
        work = torch.empty(max(256, B.dadam_ortho_get_info(h).bytes), dtype=torch.uint8, device=DEV)
        B.dadam_orthogonalize(h, g, out, work, B.current_stream())
        alone = out[0, at:at + r * c].clone()
        x, m, v = torch.zeros_like(g), torch.zeros(1, d, device=DEV), torch.zeros(1, d, device=DEV)
        x[0, at:at + r * c] = normal(2, r * c).to(x)
        B.dadam_bind(h, list(x), list(out), list(m), list(v))
        B.dadam_ortho_step(h, 0, g, 1, B.DADAM_FUSE_ACCUM, work, B.current_stream())
        got.append((alone, out[0, at:at + r * c].clone(), m[0, at:at + r * c].clone()))
        assert bool((got[-1][2] != 0).all()) and not m[0, :64].any() and not out[0, :64].any()
        B.dadam_destroy(h)
    for near, far in zip(*got):
        assert torch.equal(near, far)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [7, 90])
def test_heads_far_in_the_vector(tokens, kind):
    vocab, width, got = 300, 128, []
    kt = KINDS[kind][1]
    for before in (64, FAR):
        h, (at, bias_at), d = handle(before, [vocab * width, vocab], kind)
        head = B.dadam_head(1, 2, vocab, width)
        x, g = torch.zeros(1, d, device=DEV, dtype=kt), torch.zeros(1, d, device=DEV, dtype=kt)
        x[0, at:at + vocab * width] = normal(3, vocab * width, std=0.1).to(kt)
        x[0, bias_at:bias_at + vocab] = normal(4, vocab).to(kt)
        hidden, dhidden = normal(5, 1, tokens, width).to(kt), torch.zeros(1, tokens, width, device=DEV, dtype=kt)
        y = torch.arange(tokens, device=DEV, dtype=torch.int32)[None] * 3
        loss, nll = torch.zeros(1, device=DEV), torch.zeros(1, tokens, device=DEV)
        work = torch.empty(B.dadam_head_get_info(h, head, tokens, True).bytes, dtype=torch.uint8, device=DEV)
        B.dadam_head_loss(h, head, x, hidden.flatten(1), y, tokens, 1.0, B.DADAM_HEAD_MEAN, loss, nll, dhidden.flatten(1), g, work, B.current_stream())
        got.append((loss, nll, dhidden, g[0, at:at + vocab * width].clone(), g[0, bias_at:bias_at + vocab].clone()))
        assert bool((got[-1][3] != 0).any()) and not g[0, :64].any()
        B.dadam_destroy(h)
        del x, g
    for near, far in zip(*got):
        assert torch.equal(near, far)


@pytest.mark.parametrize("kind,vocab", [("bf16", 2 ** 23 + 77), ("f32", 2 ** 23 - 1001)])
@pytest.mark.parametrize("tokens", [5, 70])
def test_a_head_of_more_than_32_bits_of_elements(tokens, kind, vocab):
    """Against products in 64 bits, some words at a time; targets among the first and the last words.  Of gradients the norm of what they are off over all words:
    logits of at most 4 are off by 2^-18, softmax by as much and by half a step of what holds it, results by half a step of their type."""
    width, kt, half = 520, KINDS[kind][1], 2.0 ** -24 if kind == "f32" else 2.0 ** -8
    h, (at,), d = handle(8, [vocab * width], kind)
    assert vocab * width > 2 ** 32
    head = B.dadam_head(1, B.DADAM_HEAD_NO_BIAS, vocab, width)
    x, g = torch.zeros(1, d, device=DEV, dtype=kt), torch.zeros(1, d, device=DEV, dtype=kt)
    words = x[0, at:at + vocab * width].view(vocab, width)
    for k, part in enumerate(words.split(2 ** 20)):
        part.copy_(normal(6 + k, *part.shape, std=0.03))
    hidden, dhidden = normal(5, 1, tokens, width).to(kt), torch.zeros(1, tokens, width, device=DEV, dtype=kt)
    y = torch.randint(0, 1000, (1, tokens), device=DEV, dtype=torch.int32)
    y[0, ::2] = vocab - 1 - y[0, ::2]
    loss, nll = torch.zeros(1, device=DEV), torch.zeros(1, tokens, device=DEV)
    work = torch.empty(B.dadam_head_get_info(h, head, tokens, True).bytes, dtype=torch.uint8, device=DEV)
    B.dadam_head_loss(h, head, x, hidden.flatten(1), y, tokens, 1.0, 0, loss, nll, dhidden.flatten(1), g, work, B.current_stream())
    u = hidden[0].double()
    total, hit = torch.zeros(tokens, dtype=torch.float64, device=DEV), (u * words[y[0].long()].double()).sum(1)
    for part in words.split(2 ** 18):
        total += (u @ part.double().t()).exp().sum(1)
    want = total.log() - hit
    assert float((nll[0].double() - want).abs().max()) <= 2.0 ** -16 and abs(float(loss[0]) - float(want.sum())) <= tokens * 2.0 ** -16
    into, off, size, first = torch.zeros(tokens, width, dtype=torch.float64, device=DEV), 0.0, 0.0, 0
    gradient = g[0, at:at + vocab * width].view(vocab, width)
    for part, got in zip(words.split(2 ** 18), gradient.split(2 ** 18)):
        p = (u @ part.double().t()).exp() / total[:, None]
        mine = (y[0] >= first) & (y[0] < first + len(part))
        p[mine, y[0, mine].long() - first] -= 1
        into += p @ part.double()
        exact = p.t() @ u
        off += float((got.double() - exact).square().sum())
        size += float(exact.square().sum())
        first += len(part)
    # one rounding of softmax (bfloat16: half a step of it and of the kept half), one of the result; 2^-16 for the logits; a word's softmax is 2^-23 of 1, held to 2^-39
    may = 2 * half + 2.0 ** -16 + (0 if tokens <= 64 else 2.0 ** -39 * (vocab * tokens) ** 0.5 * float(u.norm(dim=1).max()) / size ** 0.5)
    assert off ** 0.5 <= may * size ** 0.5, (off ** 0.5, size ** 0.5, may)
    assert float((dhidden[0].double() - into).norm()) <= may * float(into.norm())
    for k in (0, vocab - 1, int(y[0, 0]), int(y[0, 1])):
        assert bool((gradient[k] != 0).any())
    B.dadam_destroy(h)
