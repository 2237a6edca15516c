"""A decode batch over compressed weights: a prompt that all sequences share, their own caches, and eviction from them.

The prompt is run once (products by DeviceTensor.gemm, causal attention over its own keys); its keys and values become
the prefix of every sequence. Each step then takes one token of each sequence through the layers: the norm with the
residual's addition, q, k and v in one call, attention over the prefix and the own cache, the output product, the norm
again, the MLP. When the own caches are full, the newest tokens and those that gathered most attention stay.

Weights and embeddings are random (the shapes are those of an 8B model's layers); the tokens mean nothing.

    python examples/decode_batch.py --layers 2 --batch 16 --prompt 2048 --steps 64 --cache 256 --keep 128 --recent 32
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2502_00922_amd as hl  # noqa: E402
from gen import random_bf16  # noqa: E402

EPS = 1e-5


class Layer:
    """One decoder layer: its matrices as containers on the device, its norms' weights."""

    NAMES = ("q", "k", "v", "o", "gate", "up", "down")

    def __init__(self, hidden, inter, heads, kv_heads, dim, seed, plain=False):
        shapes = {"q": (heads * dim, hidden), "k": (kv_heads * dim, hidden), "v": (kv_heads * dim, hidden),
                  "o": (hidden, heads * dim), "gate": (inter, hidden), "up": (inter, hidden), "down": (hidden, inter)}
        self.plain = {}
        for i, name in enumerate(self.NAMES):
            w = random_bf16(shapes[name], seed=seed * 10 + i)
            setattr(self, name, hl.DeviceTensor(hl.encode(w)))
            if plain:
                self.plain[name] = torch.from_numpy(w.view(np.int16)).view(torch.bfloat16).cuda()
        g = torch.Generator().manual_seed(seed)
        self.norm1, self.norm2 = ((1 + 0.1 * torch.randn(hidden, generator=g)).bfloat16().cuda() for _ in range(2))


class Cache:
    """The own keys and values of every sequence of one layer, and the attention that each key has gathered."""

    def __init__(self, batch, capacity, kv_heads, dim):
        self.k = torch.zeros((batch, capacity, kv_heads, dim), dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.weights = torch.zeros((batch, kv_heads, capacity), device="cuda")


def rotate(x, positions, base=500000.0):
    """Rotary position embedding of x [..., heads, dim] in float32, rounded to bf16; positions: [...]."""
    half = x.shape[-1] // 2
    angle = positions[..., None, None] * base ** (-torch.arange(half, device=x.device) / half)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).bfloat16()


class Decoder:
    def __init__(self, layers=2, hidden=4096, inter=14336, heads=32, kv_heads=8, dim=128, plain=False):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.layers = [Layer(hidden, inter, heads, kv_heads, dim, seed=100 + i, plain=plain) for i in range(layers)]
        self.prefix = []

    def split(self, q, k, v, shape, positions):
        """The products' float32 rows as rotated queries and keys, and values, in bf16."""
        q, k, v = (t.view(*shape, -1, self.dim) for t in (q, k, v))
        return rotate(q, positions), rotate(k, positions), v.bfloat16()

    def prefill(self, x):
        """Runs a prompt x [tokens, hidden] bf16; its keys and values are the prefix from then on."""
        n = x.shape[0]
        positions = torch.arange(n, device=x.device, dtype=torch.float32)
        lens = torch.tensor([n], dtype=torch.int32, device=x.device)
        self.prefix, delta = [], None
        for layer in self.layers:
            a, x = self.norm(delta, x, layer.norm1)
            q, k, v = self.split(layer.q.gemm(a), layer.k.gemm(a), layer.v.gemm(a), (n,), positions)
            out = hl.prefix_attention(q[None].contiguous(), k[None], v[None], lens).out
            self.prefix.append((k.contiguous(), v))
            a, x = self.norm(layer.o.gemm(out.view(n, -1)), x, layer.norm2)
            h = torch.nn.functional.silu(layer.gate.gemm(a)) * layer.up.gemm(a)
            delta = layer.down.gemm(h.bfloat16())
        return x.float() + delta

    @staticmethod
    def norm(delta, x, weight):
        """The norm of x + delta, and that sum (x without a delta)."""
        if delta is None:
            return hl.rms_norm(x, weight, eps=EPS).out, x
        r = hl.rms_norm(delta, weight, residual=x, eps=EPS)
        return r.out, r.sum

    def step(self, x, caches, lens, position):
        """One token of every sequence, x [batch, hidden] bf16, at this position; lens counts the tokens in the caches
        without it, and afterwards with it."""
        batch = x.shape[0]
        positions = torch.full((batch,), float(position), device=x.device)
        rows, slots = torch.arange(batch, device=x.device), lens.long()
        lens += 1
        delta = None
        for layer, cache, (pk, pv) in zip(self.layers, caches, self.prefix):
            a, x = self.norm(delta, x, layer.norm1)
            q, k, v = self.split(*hl.gemv_multi([layer.q, layer.k, layer.v], a), (batch,), positions)
            cache.k[rows, slots], cache.v[rows, slots] = k, v
            out = hl.prefix_attention(q.view(batch, 1, self.heads, self.dim), cache.k, cache.v, lens, prefix_k=pk,
                                      prefix_v=pv, weights=cache.weights, weights_out=cache.weights).out
            a, x = self.norm(layer.o.gemv(out.view(batch, -1)), x, layer.norm2)
            gate, up = hl.gemv_multi([layer.gate, layer.up], a)
            delta = layer.down.gemv((torch.nn.functional.silu(gate) * up).bfloat16())
        return x.float() + delta

    @staticmethod
    def evict(caches, spares, lens, keep, recent):
        """Moves what is kept of every layer's cache to its spare; gives the caches, the spares and the new lengths."""
        new = lens
        for cache, spare in zip(caches, spares):
            r = hl.cache_evict(cache.k, cache.v, cache.weights, lens, keep=keep, recent=recent, k_out=spare.k,
                               v_out=spare.v)
            spare.weights.zero_()
            spare.weights[:, :, :keep] = r.weights
            new = r.lens
        return spares, caches, new


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 2), ("hidden", 4096), ("inter", 14336), ("heads", 32), ("kv-heads", 8), ("dim", 128),
                        ("batch", 16), ("prompt", 2048), ("steps", 64), ("cache", 256), ("keep", 128), ("recent", 32)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    if a.steps < 1 or a.prompt < 1 or a.cache < 1:
        p.error("steps, prompt and cache must be at least 1")
    if a.steps > a.cache and (a.keep < 1 or not 0 <= a.recent <= a.keep < a.cache):
        p.error("an eviction has to leave room: 0 <= recent <= keep < cache, and keep at least 1")
    d = Decoder(a.layers, a.hidden, a.inter, a.heads, a.kv_heads, a.dim)
    g = torch.Generator(device="cuda").manual_seed(0)
    embed = lambda n: torch.randn((n, a.hidden), generator=g, device="cuda").bfloat16()  # noqa: E731
    d.prefill(embed(a.prompt))
    caches, spares = ([Cache(a.batch, a.cache, a.kv_heads, a.dim) for _ in range(a.layers)] for _ in range(2))
    lens = torch.zeros(a.batch, dtype=torch.int32, device="cuda")
    held = evictions = 0
    torch.cuda.synchronize()
    start = time.perf_counter()
    for s in range(a.steps):
        if held == a.cache:
            caches, spares, lens = d.evict(caches, spares, lens, a.keep, a.recent)
            held, evictions = a.keep, evictions + 1
        y = d.step(embed(a.batch), caches, lens, a.prompt + s)
        held += 1
    torch.cuda.synchronize()
    t = time.perf_counter() - start
    print(f"{a.steps} steps of {a.batch} sequences through {a.layers} layers on a prompt of {a.prompt}: "
          f"{1e3 * t / a.steps:.3f} ms a step, {evictions} evictions, outputs finite: {bool(y.isfinite().all())}")


if __name__ == "__main__":
    main()
