"""examples/decode_batch.py with its caches in 4 bits and tokens of a 4-bit vocabulary (MI355X)."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2502_00922_amd as hl
from rows4 import rows_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def make(batch, capacity):
    import decode_batch as ex
    d = ex.Decoder(layers=2, hidden=512, inter=1024, heads=4, kv_heads=2, dim=128, bits=4)
    caches, spares = ([ex.Cache(batch, capacity, 2, 128, bits=4) for _ in range(2)] for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    return ex, d, caches, spares, lambda n: torch.randn((n, 512), generator=g, device="cuda").bfloat16()


def test_steps_and_eviction():
    batch, capacity, keep, recent = 2, 24, 10, 4
    _, d, caches, spares, embed = make(batch, capacity)
    d.prefill(embed(40))
    assert [t.shape for layer in d.prefix for t in layer] == [(40, 2, 80)] * 4
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for i in range(capacity):
        before = caches[1].k.clone()
        y = d.step(embed(batch), caches, lens, 40 + i)
        assert y.isfinite().all() and lens.tolist() == [i + 1] * batch
        before[:, i] = caches[1].k[:, i]
        assert torch.equal(caches[1].k, before)  # one slot written
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


def test_first_layer_rows_are_those_of_its_keys_and_values():
    _, d, caches, _, embed = make(3, 8)
    prompt, x = embed(20), embed(3)
    d.prefill(prompt)
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    d.step(x, caches, lens, 20)
    layer = d.layers[0]
    a, _ = d.norm(None, x, layer.norm1)
    at = torch.full((3,), 20.0, device="cuda")
    _, k, v = d.split(*hl.gemv_multi([layer.q, layer.k, layer.v], a), (3,), at)
    assert torch.equal(caches[0].k[:, 0].cpu(), rows_of(k)) and torch.equal(caches[0].v[:, 0].cpu(), rows_of(v))


def test_tokens():
    import decode_batch as ex
    head = ex.Head(1000, 512)
    rows = head.embed(torch.tensor([3, 999], device="cuda"))
    one = head.next(rows.float(), torch.zeros(2, device="cuda"), temperature=0.0)
    assert one.tokens.tolist() == [3, 999]  # no row is nearer to a row than itself
    drawn = head.next(torch.randn((5, 512), device="cuda"), torch.rand(5, device="cuda"), top_p=0.9)
    assert ((0 <= drawn.tokens) & (drawn.tokens < 1000)).all() and (drawn.logprobs <= 0).all()


@pytest.mark.parametrize("args", ["--cache-bits 4", "--vocab 500 --top-k 20", "--cache-bits 4 --vocab 1000 --temperature 0.7"])
def test_command(args):
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_batch.py"), "--hidden", "512", "--inter", "1024",
                        "--heads", "4", "--kv-heads", "2", "--batch", "3", "--prompt", "50", "--steps", "20", "--cache", "16",
                        "--keep", "8", "--recent", "2", *args.split()], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-500:]
    assert "1 evictions" in r.stdout or "2 evictions" in r.stdout
    assert "outputs finite: True" in r.stdout and ("tokens of" in r.stdout) == ("vocab" in args)
