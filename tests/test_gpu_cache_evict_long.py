"""cache_evict of caches whose weights do not stay in a block's registers (above 65536 slots), which are read again for each
digit (MI355X): exact, as in test_gpu_cache_evict."""
import pytest
import torch

import paper_2502_00922_amd as hl
from test_gpu_cache_evict import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [65535, 65536, 65537, 70001, 131072, 200003])
@pytest.mark.parametrize("keep,recent", [(1, 0), (1000, 100), (60000, 1), (65000, 65000)])
def test_sizes(cap, keep, recent):
    k, v, w = make(2, cap, 2, 8, seed=cap)
    lens = torch.tensor([cap, cap - 700], dtype=torch.int32, device="cuda")
    check(k, v, w, lens, keep, recent)


@pytest.mark.parametrize("kind", ["equal", "few values", "special", "near", "mostly NaN"])
def test_ties_and_special_weights(kind):
    cap = 140000
    k, v, w = make(2, cap, 1, 8, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    pick = lambda values: torch.tensor(values, device="cuda")[  # noqa: E731
        torch.randint(len(values), w.shape, generator=g, device="cuda")]
    if kind == "equal":
        w[...] = 0.25
    elif kind == "few values":
        w = pick([0.5, 0.25, 0.25, 1.0])
    elif kind == "special":
        w = pick([float("nan"), float("inf"), -float("inf"), 1.0, -0.0, 0.0, -1e-40])
    elif kind == "near":  # differ in the last bits alone
        w = (torch.randint(0, 1000, w.shape, generator=g, device="cuda").int() + 0x3F800000).view(torch.float32)
    else:  # fewer numbers than are kept
        w = torch.where(w < 0.9, torch.full_like(w, float("nan")), w)
    lens = torch.tensor([cap, 66001], dtype=torch.int32, device="cuda")
    for keep, recent in ((66000, 0), (30000, 30), (100, 1)):
        check(k, v, w.contiguous(), lens, keep, recent)


def test_mixed_lengths():
    # short and long sequences of one call
    k, v, w = make(5, 80000, 2, 16, seed=7)
    lens = torch.tensor([80000, 0, 500, 65536, 70000], dtype=torch.int32, device="cuda")
    r = check(k, v, w, lens, 400, 60)
    assert r.lens.tolist() == [400, 0, 400, 400, 400]
    assert isinstance(r, hl.EvictResult)
