"""A decode batch over compressed weights: a prompt that all sequences share, their own caches, and eviction from them.

The prompt is run once (products by DeviceTensor.gemm, causal attention over its own keys); its keys and values become
the prefix of every sequence. Each step then takes one token of each sequence through the layers: the norm with the
residual's addition, q, k and v in one call, attention over the prefix and the own cache, the output product, the norm
again, the MLP. When the own caches are full, the newest tokens and those that gathered most attention stay.

With --cache-bits 4 the prefix and the own caches are held in 4-bit rows: each step rounds its keys and values into them,
attends over them, and an eviction moves them, as they are. With --vocab a matrix of 4-bit codes gives the logits of a
step's outputs, a token of each row is drawn from them, and its row of the same matrix is the next step's input.

Weights and embeddings are random (the shapes are those of an 8B model's layers); the tokens mean nothing.

    python examples/decode_batch.py --layers 2 --batch 16 --prompt 2048 --steps 64 --cache 256 --keep 128 --recent 32
    python examples/decode_batch.py --cache-bits 4 --vocab 32000 --temperature 0.8 --top-k 50 --top-p 0.95
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
    """The own keys and values of every sequence of one layer (bf16, or 4-bit rows), and the attention that each key has
    gathered."""

    def __init__(self, batch, capacity, kv_heads, dim, bits=16):
        if bits == 16:
            self.k = torch.zeros((batch, capacity, kv_heads, dim), dtype=torch.bfloat16, device="cuda")
        else:
            # a key head's rows next to each other: they are shorter than a line of memory
            row = hl.cache4_row_bytes(dim)
            self.k = torch.zeros((batch, kv_heads, capacity, row), dtype=torch.uint8, device="cuda").transpose(1, 2)
        self.v = torch.zeros_like(self.k)
        self.weights = torch.zeros((batch, kv_heads, capacity), device="cuda")


def rotate(x, positions, base=500000.0):
    """Rotary position embedding of x [..., heads, dim] in float32, rounded to bf16; positions: [...]."""
    half = x.shape[-1] // 2
    angle = positions[..., None, None] * base ** (-torch.arange(half, device=x.device) / half)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).bfloat16()


class Head:
    """A vocabulary's rows, a 4-bit code each column and a bf16 scale for 64 (128, 32) of them: the tokens' inputs, and the
    products that give their logits."""

    def __init__(self, vocab, hidden, seed=0):
        group = next((n for n in (64, 128, 32) if hidden % n == 0), None)
        if group is None:
            raise ValueError("a vocabulary's columns come in groups of 32")
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.codes = torch.randint(0, 256, (vocab, hidden // 2), generator=g, device="cuda", dtype=torch.uint8)
        self.scales = (0.2 + 0.1 * torch.rand((vocab, hidden // group), generator=g, device="cuda")).bfloat16()
        self.norm = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")

    def embed(self, tokens):
        codes = self.codes[tokens.long()]
        steps = torch.stack([codes & 15, codes >> 4], -1).flatten(1).float() - 8
        scales = self.scales[tokens.long()].float()
        return (steps.unflatten(1, (scales.shape[1], -1)) * scales[..., None]).flatten(1).bfloat16()

    def next(self, y, uniforms, **settings):
        """A token of each row of y [batch, hidden], a step's float32 outputs, and the logarithm of its probability."""
        x = hl.rms_norm(y, self.norm, eps=EPS, out_dtype=torch.bfloat16).out
        logits = hl.gemv4(self.codes, self.scales, x) * y.shape[1] ** -0.5
        return hl.sample(logits, uniforms, **settings)


class Decoder:
    def __init__(self, layers=2, hidden=4096, inter=14336, heads=32, kv_heads=8, dim=128, plain=False, bits=16):
        self.heads, self.kv_heads, self.dim, self.bits = heads, kv_heads, dim, bits
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
            if self.bits == 4:
                cache = Cache(1, n, self.kv_heads, self.dim, bits=4)
                hl.cache_write4(k[None], v[None], cache.k, cache.v)
                self.prefix.append((cache.k[0], cache.v[0]))
            else:
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
        attend = hl.prefix_attention4 if self.bits == 4 else hl.prefix_attention
        delta = None
        for layer, cache, (pk, pv) in zip(self.layers, caches, self.prefix):
            a, x = self.norm(delta, x, layer.norm1)
            q, k, v = self.split(*hl.gemv_multi([layer.q, layer.k, layer.v], a), (batch,), positions)
            if self.bits == 4:
                hl.cache_write4(k[:, None], v[:, None], cache.k, cache.v, lens)
            else:
                cache.k[rows, slots], cache.v[rows, slots] = k, v
            out = attend(q.view(batch, 1, self.heads, self.dim), cache.k, cache.v, lens, prefix_k=pk, prefix_v=pv,
                         weights=cache.weights, weights_out=cache.weights).out
            a, x = self.norm(layer.o.gemv(out.view(batch, -1)), x, layer.norm2)
            gate, up = hl.gemv_multi([layer.gate, layer.up], a)
            delta = layer.down.gemv((torch.nn.functional.silu(gate) * up).bfloat16())
        return x.float() + delta

    @staticmethod
    def evict(caches, spares, lens, keep, recent):
        """Moves what is kept of every layer's cache to its spare; gives the caches, the spares and the new lengths."""
        new = lens
        for cache, spare in zip(caches, spares):
            # 4-bit rows move like rows of 16-bit columns
            k, v, k_out, v_out = (t.view(torch.int16) if t.dtype == torch.uint8 else t
                                  for t in (cache.k, cache.v, spare.k, spare.v))
            r = hl.cache_evict(k, v, cache.weights, lens, keep=keep, recent=recent, k_out=k_out, v_out=v_out)
            spare.weights.zero_()
            spare.weights[:, :, :keep] = r.weights
            new = r.lens
        return spares, caches, new


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 2), ("hidden", 4096), ("inter", 14336), ("heads", 32), ("kv-heads", 8), ("dim", 128),
                        ("batch", 16), ("prompt", 2048), ("steps", 64), ("cache", 256), ("keep", 128), ("recent", 32),
                        ("vocab", 0), ("top-k", 0)):
        p.add_argument("--" + name, type=int, default=value)
    for name, value in (("temperature", 1.0), ("top-p", 1.0), ("min-p", 0.0)):
        p.add_argument("--" + name, type=float, default=value)
    p.add_argument("--cache-bits", type=int, default=16, choices=(4, 16))
    a = p.parse_args()
    if a.steps < 1 or a.prompt < 1 or a.cache < 1:
        p.error("steps, prompt and cache must be at least 1")
    if a.steps > a.cache and (a.keep < 1 or not 0 <= a.recent <= a.keep < a.cache):
        p.error("an eviction has to leave room: 0 <= recent <= keep < cache, and keep at least 1")
    if a.vocab < 0 or a.vocab >= 1 << 20 or (a.vocab and a.hidden % 32):
        p.error("vocab must be below 2^20, and its rows' columns a multiple of 32")
    if a.cache_bits == 4 and (a.dim % 32 or a.dim > 256):
        p.error("with cache-bits 4, dim must be a multiple of 32, at most 256")
    d = Decoder(a.layers, a.hidden, a.inter, a.heads, a.kv_heads, a.dim, bits=a.cache_bits)
    g = torch.Generator(device="cuda").manual_seed(0)
    embed = lambda n: torch.randn((n, a.hidden), generator=g, device="cuda").bfloat16()  # noqa: E731
    d.prefill(embed(a.prompt))
    head = Head(a.vocab, a.hidden) if a.vocab else None
    uniforms = torch.rand((a.steps, a.batch), generator=g, device="cuda")
    settings = {"temperature": a.temperature, "top_k": a.top_k, "top_p": a.top_p, "min_p": a.min_p}
    caches, spares = ([Cache(a.batch, a.cache, a.kv_heads, a.dim, a.cache_bits) for _ in range(a.layers)] for _ in range(2))
    lens = torch.zeros(a.batch, dtype=torch.int32, device="cuda")
    x, drawn = embed(a.batch), []
    held = evictions = 0
    torch.cuda.synchronize()
    start = time.perf_counter()
    for s in range(a.steps):
        if held == a.cache:
            caches, spares, lens = d.evict(caches, spares, lens, a.keep, a.recent)
            held, evictions = a.keep, evictions + 1
        y = d.step(x, caches, lens, a.prompt + s)
        held += 1
        if head is None:
            x = embed(a.batch)
        else:
            drawn.append(head.next(y, uniforms[s], **settings))
            x = head.embed(drawn[-1].tokens)
    torch.cuda.synchronize()
    t = time.perf_counter() - start
    print(f"{a.steps} steps of {a.batch} sequences through {a.layers} layers on a prompt of {a.prompt}: "
          f"{1e3 * t / a.steps:.3f} ms a step, {evictions} evictions, outputs finite: {bool(y.isfinite().all())}")
    if drawn:
        print(f"tokens of the first sequence: {' '.join(str(int(r.tokens[0])) for r in drawn[:16])}, mean log probability "
              f"{float(torch.stack([r.logprobs for r in drawn]).mean()):.3f}")


if __name__ == "__main__":
    main()
