"""sample where many light tokens stand beside a far heavier one (MI355X).

A weight is a whole number of 2^-43 of the greatest, its rounding 2^-44, and what it is rounded from is off by 2^-44.3 of it:
the powers of two of a distance z = 64 (l - max) log2(e) / T in float64, |z| <= 2560 with two roundings of 2^-53 (2^-46.9 of
the weight), the table's (2^-52), and a polynomial of degree 4 in |x| ln 2 / 64 <= 0.00542 (0.00542^5 / 120 = 2^-44.5). So a
weight is off by 2^-43 of the greatest at most, a sum of n by n * 2^-43, and a token is that of exact numbers but where u
times the total is within n * 2^-42 of where another begins. The logprob's total is off by n * 2^-43 of at least 1."""
import math

import numpy as np
import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu


def compare(x, u, **settings):
    """x: one row of float64 logits that float32 holds; u: draws from it. Gives how many draws are told apart."""
    rows = torch.from_numpy(x).float().cuda().expand(len(u), -1).contiguous()
    r = hl.sample(rows, torch.from_numpy(u).cuda(), **settings)
    w = np.exp((x - x.max()).astype(np.longdouble))
    ends = np.cumsum(w)
    target = u.astype(np.longdouble) * ends[-1]
    want = np.searchsorted(ends, target, side="right")
    margin = np.longdouble(len(x) * 2.0**-42)
    begins = np.concatenate([[np.longdouble(0)], ends])
    near = np.minimum(np.abs(target - begins[want]), np.abs(ends[want] - target)) <= margin
    got = r.tokens.cpu().numpy()
    assert (got[~near] == want[~near]).all()
    # those near a border are one of the tokens there
    assert (target >= begins[got] - margin).all() and (target <= ends[got] + margin).all()
    logprob = np.log(w / ends[-1]).astype(np.float64)[got]
    err = np.abs(r.logprobs.double().cpu().numpy() - logprob)
    assert (err <= 2.0**-24 * np.abs(logprob) + len(x) * 2.0**-43 + 2.0**-40).all(), err.max()
    return int((~near).sum())


@pytest.mark.parametrize("vocab", [5000, 131072])
@pytest.mark.parametrize("light", [-8.0, -16.0, -18.0, -24.0])
def test_equal_light_tokens(vocab, light):
    x = np.full(vocab, light)
    x[-1] = 0.0
    share = (vocab - 1) * math.exp(light) / (1 + (vocab - 1) * math.exp(light))
    u = ((np.arange(500) + 0.5) / 500 * share).astype(np.float32)
    told = compare(x, u)
    # draws are spread over tokens of weight w evenly, and all but 2 margins of w are told apart (131072 at -16: 2^-24 of
    # 2^-23.1, so 47 in a hundred)
    assert told >= 0.9 * 500 * (1 - 2 * vocab * 2.0**-42 / math.exp(light))


def test_mixed_light_tokens():
    g = np.random.default_rng(3)
    x = (-14 + 2 * g.standard_normal(100000)).astype(np.float32).astype(np.float64)
    x[70000] = 0.0
    u = np.concatenate([g.random(200), 0.2 * g.random(300)]).astype(np.float32)
    assert compare(x, u) > 200
