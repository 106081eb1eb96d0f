"""The operators together: one training example through all of them, against the same model in plain torch."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    from paper_2512_13728_gb300 import build

    build.build()
    import distill_gpt

    return distill_gpt


def plain_logits(m, W, table, norms, tokens):
    """The model of the example in float64."""
    b, t = tokens.shape
    d = m.dim // m.heads
    freq = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    ang = torch.arange(t, device="cuda").double()[:, None] * freq
    cos, sin = ang.cos()[None, :, None], ang.sin()[None, :, None]

    def rms(x, eps):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)

    def rotate(x):
        a, c = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - c * sin, c * cos + a * sin], -1)

    x = table[tokens] * m.scale
    mask = torch.full((t, t), -math.inf, device="cuda", dtype=torch.float64).triu(1)
    eps = torch.finfo(torch.bfloat16).eps  # torch's own for rms_norm of bf16
    for i in range(m.blocks):
        wq, wk, wv, wo, w1, w2 = W[6 * i:6 * i + 6]
        y = rms(x, eps)
        q, k, v = ((y @ w).view(b, t, m.heads, d) for w in (wq, wk, wv))
        q, k = rotate(rms(q, 1e-6) * norms[2 * i]), rotate(rms(k, 1e-6) * norms[2 * i + 1])
        s = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(d) + mask
        x = x + torch.einsum("bhqk,bkhd->bqhd", s.softmax(-1), v).reshape(b, t, m.dim) @ wo
        x = x + torch.nn.functional.gelu(rms(x, eps) @ w1) @ w2
    return rms(x, eps).view(b * t, m.dim) @ table.t()


def test_gradients_of_one_step(example):
    """Loss and every gradient against float64 autograd; the example's products round to bf16 (2^-8 each, a
    dozen deep, at random), hence 3% of a gradient's norm."""
    m = example.GPT(vocab=211, dim=64, heads=2, blocks=2, batch=3, tokens=29, seed=5)
    g = torch.Generator(device="cuda").manual_seed(1)
    text = torch.randint(0, 211, (3, 29), generator=g, device="cuda")
    ids = torch.rand(87, 211, generator=g, device="cuda").topk(9, 1).indices
    t = torch.randn(87, 9, generator=g, device="cuda") * 3
    w = torch.rand(87, generator=g, device="cuda") / 87
    with torch.no_grad():  # one set of weights on both sides
        for p in (m.table, *m.norms):
            p.copy_(p.to(torch.bfloat16))
    logits, x0 = m.logits(text)
    loss = example.Distill.apply(logits, ids, t, 2.0, w)
    loss.backward()
    m.embed.gradient(text, x0.grad, m.scale, out=m.table.grad, accumulate=True)

    W = [x.detach().double().requires_grad_() for x in m.W]
    table, norms = m.table.detach().double().requires_grad_(), [n.detach().double().requires_grad_() for n in m.norms]
    z = plain_logits(m, W, table, norms, text) / 2.0
    lp = torch.log_softmax(t.double() / 2.0, 1)
    want = (w.double() * 4.0 * (lp.exp() * (lp - torch.log_softmax(z, 1).gather(1, ids))).sum(1)).sum()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 0.01 * float(want.detach())
    for got, ref in zip((*m.G, m.table.grad, *(n.grad for n in m.norms)), (*W, table, *norms)):
        assert float((got.double() - ref.grad).norm()) <= 0.03 * float(ref.grad.norm())


def test_training_lowers_the_loss(example):
    losses = example.train(steps=40, log=None)
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5])
