"""sample against the definition in 64 bits, row by row (MI355X). Tokens are equal; logprobs are float32 roundings of a
sum of weights with 43 bits: 2^-24 of them and 2^-38 of the sum."""
import math

import numpy as np
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def plain(x, u, temperature=1.0, k=0, p=1.0, least=0.0):
    """(token, logprob, kept tokens) of one row x, float64 on the CPU."""
    x = np.where(np.isnan(x), -np.inf, x)
    if x.max() == -np.inf:
        return -1, -math.inf, np.array([])
    if not temperature > 0:
        return int(np.argmax(x)), 0.0, np.array([np.argmax(x)])
    with np.errstate(all="ignore"):
        w = np.where(x == x.max(), 1.0, np.exp((x - x.max()) / temperature))
    order = np.lexsort((np.arange(x.size), -x))
    if 0 < k < x.size:
        order = order[:k]
    order = order[w[order] >= 2.0**-40]
    if p < 1:
        sums = np.cumsum(w[order])
        order = order[:int(np.searchsorted(sums, p * sums[-1])) + 1]
    kept = np.sort(order[(w[order] >= min(least, 1.0)) | (np.arange(order.size) == 0)])
    sums = np.cumsum(w[kept])
    i = min(int(np.searchsorted(sums, max(u, 0.0) * sums[-1], side="right")), kept.size - 1)
    return int(kept[i]), float(np.log(w[kept[i]] / sums[-1])), kept


def check(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    rows = logits.shape[0]
    r = hl.sample(logits, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    at = lambda t, i: float(t[i]) if torch.is_tensor(t) else float(np.float32(t))  # noqa: E731
    x, uniforms = logits.double().cpu().numpy(), u.double().cpu().numpy()
    got, logprobs = r.tokens.cpu().tolist(), r.logprobs.double().cpu().tolist()
    for i in range(rows):
        token, logprob, _ = plain(x[i], uniforms[i], at(temperature, i), int(at(top_k, i)), at(top_p, i), at(min_p, i))
        assert got[i] == token, (i, got[i], token)
        assert logprobs[i] == logprob or abs(logprobs[i] - logprob) <= 2.0**-24 * abs(logprob) + 2.0**-38, (i, logprobs[i], logprob)
    return r


def make(rows, vocab, dtype=torch.float32, size=2.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (size * torch.randn((rows, vocab), generator=g, device="cuda")).to(dtype)
    return x, torch.rand((rows,), generator=g, device="cuda")


VOCABS = [1, 2, 3, 7, 64, 255, 1000, 4097, 8191, 8192, 8193, 32000, 50257, 65537, 131072]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_whole_distribution(dtype, vocab):
    check(*make(5, vocab, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 50, 8192, 20001, 70000])
@pytest.mark.parametrize("settings", [
    dict(top_k=1), dict(top_k=2), dict(top_k=50), dict(top_k=1000), dict(top_p=0.9), dict(top_p=0.1), dict(top_p=0.0),
    dict(min_p=0.1), dict(min_p=1.0), dict(top_k=40, top_p=0.7), dict(top_k=300, top_p=0.99, min_p=0.02, temperature=0.7),
    dict(temperature=0.0), dict(temperature=0.01), dict(temperature=30.0, top_p=0.5), dict(temperature=1e-30, top_p=0.5)])
def test_settings(dtype, vocab, settings):
    check(*make(4, vocab, dtype, seed=vocab), **settings)


# borders in steps of their own, and in one: top_k above what a list holds, top_p near and far from it, min_p between
@pytest.mark.parametrize("settings", [
    dict(top_k=3000), dict(top_k=3000, top_p=0.8), dict(top_k=3000, top_p=0.999), dict(top_k=3000, top_p=1.0 - 2.0**-24),
    dict(top_k=2000, top_p=0.8, min_p=0.05), dict(top_k=2000, min_p=0.001), dict(top_p=0.9, min_p=0.001),
    dict(top_p=0.5, min_p=0.001), dict(top_p=0.999, min_p=0.001), dict(top_k=1025, top_p=0.95), dict(top_k=1024, top_p=0.95)])
@pytest.mark.parametrize("size", [0.3, 2.0, 5.0])
@pytest.mark.parametrize("vocab,dtype", [(9000, torch.float32), (150000, torch.float32), (40000, torch.bfloat16)])
def test_borders(settings, size, vocab, dtype):
    check(*make(3, vocab, dtype, size=size, seed=7), **settings)


def test_many_rows():
    x, u = make(700, 3000)
    check(x, u, top_p=0.9)


def test_settings_of_each_row():
    rows = 64
    x, u = make(rows, 5000, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(5)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device="cuda")[  # noqa: E731
        torch.randint(0, len(values), (rows,), generator=g, device="cuda")]
    check(x, u, temperature=pick([0.0, 0.5, 1.0, 2.0], torch.float32), top_k=pick([0, 1, 10, 5000, 6000, -3], torch.int32),
          top_p=pick([1.0, 0.9, 0.3, 0.0], torch.float32), min_p=pick([0.0, 0.05, 0.5], torch.float32))


def test_settings_that_are_no_numbers():
    # in a tensor, which the host does not see: no filter, and the greatest logit for a temperature
    x, u = make(4, 300)
    nan = torch.full((4,), math.nan, device="cuda")
    want = hl.sample(x, u)
    got = hl.sample(x, u, top_p=nan, min_p=nan)
    assert torch.equal(got.tokens, want.tokens) and torch.equal(got.logprobs, want.logprobs)
    assert torch.equal(hl.sample(x, u, temperature=nan).tokens.long(), x.argmax(1))
    assert torch.equal(hl.sample(x, u, temperature=-nan.new_ones(4)).tokens.long(), x.argmax(1))


@pytest.mark.parametrize("settings", [dict(), dict(top_k=5), dict(top_k=700), dict(top_p=0.5), dict(top_k=600, top_p=0.5)])
@pytest.mark.parametrize("vocab", [1000, 20000])
def test_equal_logits(settings, vocab):
    # the lowest indexes of equal ones come first
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(0, 3, (6, vocab), generator=g, device="cuda").float()
    x[4], x[5] = 0.0, -0.0
    x[5, ::2] = 0.0
    u = torch.tensor([0.0, 0.3, 0.6, 0.999, 0.5, 0.5], device="cuda")
    check(x, u, **settings)


@pytest.mark.parametrize("vocab", [10, 9000])
def test_sums_that_meet_the_goal_exactly(vocab):
    # two (of four) equal tokens hold half of the weight: the border belongs to them
    x = torch.full((4, vocab), -math.inf, device="cuda")
    x[:, [1, 3, 5, 8]] = 2.0
    u = torch.tensor([0.0, 0.25, 0.5, 0.75], device="cuda")
    r = check(x, u)
    assert r.tokens.tolist() == [1, 3, 5, 8]
    r = check(x, u, top_p=0.5)
    assert r.tokens.tolist() == [1, 1, 3, 3]


def test_uniforms_at_and_past_the_ends():
    x = torch.zeros((6, 100), device="cuda")
    u = torch.tensor([0.0, 1.0 - 2.0**-24, 1.0, 2.0, -1.0, math.nan], device="cuda")
    assert hl.sample(x, u).tokens.tolist() == [0, 99, 99, 99, 0, 0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [500, 12345])
def test_masked(dtype, vocab):
    x, u = make(8, vocab, dtype)
    x[0, 10:], x[1, :-1], x[2, 1:] = -math.inf, -math.inf, -math.inf
    x[3], x[4] = -math.inf, torch.finfo(dtype).min
    x[5, 5:] = torch.finfo(dtype).min
    x[6], x[7, ::2] = math.nan, math.nan
    r = check(x, u, top_p=0.9)
    assert r.tokens[3] == -1 and r.tokens[6] == -1 and r.logprobs[3] == -math.inf
    check(x, u, top_k=20)
    check(x, u)
    check(x, u, temperature=0.0)


@pytest.mark.parametrize("vocab", [500, 12345])
def test_infinite_logits(vocab):
    x, u = make(4, vocab)
    x[:, [7, 90, 400]] = math.inf
    r = check(x, u, top_p=0.99)
    assert all(t in (7, 90, 400) for t in r.tokens.tolist())
    check(x, u, top_k=2)
    check(x, u, temperature=0.0)


def test_light_tokens_are_never_drawn():
    # weights 2^-39 and 2^-41 of the greatest, and u below either's share
    x = torch.full((2, 64), -math.inf, device="cuda")
    x[0, 50], x[0, 3] = 0.0, -39 * math.log(2)
    x[1, 50], x[1, 3] = 0.0, -41 * math.log(2)
    u = torch.zeros(2, device="cuda")
    assert hl.sample(x, u).tokens.tolist() == [3, 50]


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart(dtype):
    big, u = make(7, 3001, dtype)
    for first, last in ((0, 3001), (1, 3000), (3, 2999), (5, 1030)):
        part = big[::2, first:last]
        check(part, u[::2].contiguous(), top_k=30)


def test_one_row_as_a_vector():
    x, u = make(1, 700)
    assert torch.equal(hl.sample(x[0], u).tokens, hl.sample(x, u).tokens)


def test_frequencies():
    # evenly spaced uniforms give every token its share of the draws
    w = torch.tensor([0.5, 0.25, 0.125, 0.0625, 0.0625], device="cuda")
    n = 40000
    u = (torch.arange(n, device="cuda") + 0.5) / n
    r = hl.sample(w.log().expand(n, 5).contiguous(), u)
    assert torch.equal(torch.bincount(r.tokens.long(), minlength=5).cpu(), (w * n).long().cpu())


def test_captured():
    x, u = make(3, 40000)
    hl.sample(x, u, top_p=0.8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hl.sample(x, u, top_p=0.8)
    for i in range(4):
        x.mul_(0.7)
        u.copy_(torch.rand(3, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = check(x, u, top_p=0.8)
        assert torch.equal(held.tokens, eager.tokens) and torch.equal(held.logprobs, eager.logprobs)


def test_two_streams_at_once():
    cases = [make(16, 60000, seed=i) for i in range(2)]
    want = [hl.sample(x, u, top_k=100, top_p=0.9).tokens for x, u in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [hl.sample(x, u, top_k=100, top_p=0.9, stream=s).tokens for (x, u), s in zip(cases, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_far_rows():
    # rows whose offsets pass 32 bits
    big = torch.empty((1 << 30) + (1 << 28) + 1000, device="cuda")
    x = big.as_strided((3, 1000), ((1 << 29) + (1 << 27), 1))
    near, u = make(3, 1000)
    x.copy_(near)
    assert torch.equal(hl.sample(x, u).tokens, hl.sample(near, u).tokens)
