"""A decode step's 4-bit operators after each other, as a serving loop calls them (MI355X): rows written to the caches,
attention over them that gathers weights, an eviction of the rows as they are, a product with 4-bit weights, a token.

The attention's results are held against the definition in 64 bits on the very rows, with the bounds that
test_gpu_prefix_attention4 derives; rows, evictions and tokens are equal."""
import pytest
import torch

import paper_2502_00922_amd as hl
import test_gpu_gemv4 as products
import test_gpu_prefix_attention4 as attention
import test_gpu_sample as sampling
from rows4 import rows_of

pytestmark = pytest.mark.gpu
BATCH, HEADS, KV, DIM, CAPACITY, PREFIX, VOCAB = 3, 8, 2, 96, 40, 70, 4001


class Loop:
    """What a loop holds from step to step, all of it allocated once."""

    def __init__(self, dtype, seed=0):
        self.dtype = dtype
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        row = hl.cache4_row_bytes(DIM)
        self.prefix = self.empty(1, PREFIX, row)
        hl.cache_write4(*(self.rand(1, PREFIX, KV, DIM) for _ in range(2)), *self.prefix)
        self.cache, self.spare = (self.empty(BATCH, CAPACITY, row) for _ in range(2))
        self.weights = torch.zeros((BATCH, KV, CAPACITY), device="cuda")
        self.lens = torch.zeros(BATCH, dtype=torch.int32, device="cuda")
        self.q = self.rand(BATCH, 1, HEADS, DIM)
        self.k, self.v = (self.rand(BATCH, 1, KV, DIM) for _ in range(2))
        self.u = torch.rand(BATCH, generator=self.g, device="cuda")
        self.head = products.make(VOCAB, HEADS * DIM, 1, 32, dtype)

    def empty(self, batch, tokens, row):
        return [torch.zeros((batch, tokens, KV, row), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def rand(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").to(self.dtype)

    def new_inputs(self):
        for t in (self.q, self.k, self.v):
            t.copy_(self.rand(*t.shape))
        self.u.copy_(torch.rand(BATCH, generator=self.g, device="cuda"))

    def step(self):
        self.lens += 1
        hl.cache_write4(self.k, self.v, *self.cache, self.lens)
        a = hl.prefix_attention4(self.q, *self.cache, self.lens, prefix_k=self.prefix[0][0], prefix_v=self.prefix[1][0],
                                 weights=self.weights, weights_out=self.weights)
        logits = hl.gemv4(self.head["codes"], self.head["scales"], a.out.view(BATCH, -1), self.head["bases"])
        return a.out, logits, hl.sample(logits, self.u, temperature=0.9, top_k=50, top_p=0.9)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_against_the_definition(dtype):
    t = Loop(dtype)
    keep, recent = 12, 3
    want = [torch.zeros_like(c).cpu() for c in t.cache]
    for step in range(CAPACITY + 5):
        n = int(t.lens[0])
        if n == CAPACITY:
            r = hl.cache_evict(*(c.view(torch.int16) for c in t.cache), t.weights, t.lens, keep=keep, recent=recent,
                               k_out=t.spare[0].view(torch.int16), v_out=t.spare[1].view(torch.int16))
            for b in range(BATCH):
                for h in range(KV):
                    w = t.weights[b, h, :CAPACITY - recent]
                    at = torch.sort(torch.sort(w, descending=True, stable=True).indices[:keep - recent]).values.tolist()
                    at += list(range(CAPACITY - recent, CAPACITY))
                    assert r.slots[b, h].tolist() == at
                    for c in want:
                        c[b, :keep, h] = c[b, at, h]
            t.cache, t.spare, t.lens = t.spare, t.cache, r.lens
            t.weights.zero_()
            t.weights[:, :, :keep] = r.weights
            n = keep
        t.new_inputs()
        before = t.weights.clone()
        out, logits, drawn = t.step()
        for c, x in zip(want, (t.k, t.v)):
            c[:, n] = rows_of(x)[:, 0]
        for c, w in zip(t.cache, want):
            assert torch.equal(c[:, :n + 1].cpu(), w[:, :n + 1])
        c = {"q": t.q, "k": t.cache[0], "v": t.cache[1], "lens": t.lens, "prefix_k": t.prefix[0][0], "prefix_v": t.prefix[1][0]}
        if step % 4 == 0:
            again = attention.check(c)
            assert torch.equal(again.out, out)
            gathered = hl.prefix_attention4(**c, weights=before).weights
            assert torch.equal(gathered, t.weights)
            x = {**t.head, "x": out.view(BATCH, -1)}
            assert torch.equal(products.check(x), logits)
        same = sampling.check(logits, t.u, temperature=0.9, top_k=50, top_p=0.9)
        assert torch.equal(same.tokens, drawn.tokens)
    assert t.lens.tolist() == [keep + 5] * BATCH


def test_captured_step():
    # a graph's steps and eager ones, in turn, on two loops of the same inputs
    t, plain = Loop(torch.bfloat16), Loop(torch.bfloat16)
    for x in (t, plain):
        x.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = t.step()
    for i in range(8):
        t.new_inputs()
        plain.new_inputs()
        if i % 3 == 2:
            got = t.step()
        else:
            graph.replay()
            got = held
        torch.cuda.synchronize()
        out, logits, drawn = plain.step()
        assert torch.equal(got[0], out) and torch.equal(got[1], logits)
        assert torch.equal(got[2].tokens, drawn.tokens) and torch.equal(got[2].logprobs, drawn.logprobs)
        assert torch.equal(t.weights, plain.weights) and torch.equal(t.lens, plain.lens)
        assert all(torch.equal(a, b) for a, b in zip(t.cache, plain.cache))


def test_graphs_that_share_workspaces():
    # two graphs of one workspace each for attention and sampling, replayed after each other
    loops = [Loop(torch.bfloat16, seed=i) for i in range(2)]
    work, draw = (torch.empty(1 << 23, dtype=torch.uint8, device="cuda") for _ in range(2))

    def run(t):
        a = hl.prefix_attention4(t.q, *t.cache, t.lens, prefix_k=t.prefix[0][0], prefix_v=t.prefix[1][0], workspace=work)
        logits = hl.gemv4(t.head["codes"], t.head["scales"], a.out.view(BATCH, -1), t.head["bases"])
        return a.out, hl.sample(logits, t.u, top_p=0.9, workspace=draw).tokens

    graphs = []
    for t in loops:
        for _ in range(5):
            t.step()
        run(t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run(t)
        graphs.append((graph, held))
    for _ in range(3):
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for t, (_, (out, tokens)) in zip(loops, graphs):
            want = run(t)
            assert torch.equal(out, want[0]) and torch.equal(tokens, want[1])
            t.new_inputs()
