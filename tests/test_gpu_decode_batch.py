"""The decode batch of examples/decode_batch.py against plain float32 torch on the uncompressed weights (MI355X).

Bound: on its way through a layer a value is rounded to bf16 12 times (two norms, three of q, k and v, the attention
weights and output, the MLP's product, two sums, and the products' inputs), each by at most 2^-9 of its size in the
mean, and errors only add: 2 layers * 12 * 2^-9 = 0.047 of the output's norm."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
BOUND = 2 * 12 * 2.0**-9


class Plain:
    """The same layers in float32, each sequence on its own, over all of its tokens at once."""

    def __init__(self, decoder):
        self.d = decoder

    def run(self, x):
        """x [tokens, hidden]: outputs of all tokens."""
        d, n = self.d, x.shape[0]
        x = x.float()
        half = d.dim // 2
        angle = torch.arange(n, device=x.device)[:, None, None] * 500000.0 ** (-torch.arange(half, device=x.device) / half)

        def norm(t, w):
            return t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * w.float()

        def rotate(t):
            a, b = t[..., :half], t[..., half:]
            return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)

        hidden = torch.ones(n, n, device=x.device).triu(1).bool()
        for layer in d.layers:
            w = {name: t.float() for name, t in layer.plain.items()}
            a = norm(x, layer.norm1)
            q, k, v = (torch.matmul(a, w[t].t().contiguous()).view(n, -1, d.dim) for t in ("q", "k", "v"))
            q, k = rotate(q), rotate(k)
            out = torch.empty_like(q)
            for h in range(d.heads):
                g = h // (d.heads // d.kv_heads)
                s = torch.matmul(q[:, h], k[:, g].t().contiguous()) / d.dim**0.5
                out[:, h] = torch.matmul(torch.softmax(s.masked_fill(hidden, float("-inf")), -1), v[:, g].contiguous())
            x = x + torch.matmul(out.reshape(n, -1), w["o"].t().contiguous())
            a = norm(x, layer.norm2)
            mlp = torch.nn.functional.silu(torch.matmul(a, w["gate"].t().contiguous()))
            mlp = mlp * torch.matmul(a, w["up"].t().contiguous())
            x = x + torch.matmul(mlp, w["down"].t().contiguous())
        return x


def far(a, b):
    return float((a - b).norm() / b.norm())


def make(batch, capacity):
    import decode_batch as ex
    d = ex.Decoder(layers=2, hidden=512, inter=1024, heads=4, kv_heads=2, dim=128, plain=True)
    caches = [ex.Cache(batch, capacity, 2, 128) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    return ex, d, caches, lambda n: torch.randn((n, 512), generator=g, device="cuda").bfloat16()


def test_against_plain():
    batch, prompt, steps = 3, 150, 9
    _, d, caches, embed = make(batch, 16)
    shared, plain = embed(prompt), Plain(d)
    y = d.prefill(shared)
    assert far(y, plain.run(shared)) <= BOUND
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    tokens = [embed(batch) for _ in range(steps)]
    outs = [d.step(t, caches, lens, prompt + i) for i, t in enumerate(tokens)]
    assert lens.tolist() == [steps] * batch
    for b in range(batch):
        want = plain.run(torch.cat([shared] + [t[b:b + 1] for t in tokens]))[prompt:]
        assert far(torch.stack([o[b] for o in outs]), want) <= BOUND


def test_eviction_keeps_the_heaviest():
    batch, capacity, keep, recent = 2, 24, 10, 4
    ex, d, caches, embed = make(batch, capacity)
    spares = [ex.Cache(batch, capacity, 2, 128) for _ in range(2)]
    d.prefill(embed(40))
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for i in range(capacity):
        d.step(embed(batch), caches, lens, 40 + i)
    old, gathered = caches[1].k.clone(), caches[1].weights.clone()
    assert (gathered > 0).all()
    caches, spares, lens = d.evict(caches, spares, lens, keep, recent)
    assert lens.tolist() == [keep] * batch
    for b in range(batch):
        for h in range(2):
            w = gathered[b, h, :capacity - recent]
            best = torch.sort(torch.sort(w, descending=True, stable=True).indices[:keep - recent]).values.tolist()
            best += list(range(capacity - recent, capacity))
            assert torch.equal(caches[1].k[b, :keep, h], old[b, best, h])
            assert torch.equal(caches[1].weights[b, h, :keep], gathered[b, h, best])
    y = d.step(embed(batch), caches, lens, 40 + capacity)
    assert y.isfinite().all() and lens.tolist() == [keep + 1] * batch
