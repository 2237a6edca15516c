"""prefix_attention where its rules take the forms that small calls do not: items of 128 rows (which need 4096 units of
128 keys on 256 compute units) and rows of many parts (MI355X). The bounds are those of test_gpu_prefix_attention; the
definition is computed in 64 bits on the GPU here."""
import math

import pytest
import torch

import paper_2502_00922_amd as hl
import test_gpu_prefix_attention as small

pytestmark = pytest.mark.gpu


def reference(c, scale=None):
    q = c["q"].double()
    batch, queries, heads, dim = q.shape
    scale = 1 / math.sqrt(dim) if scale is None else scale
    kv_heads = (c["k"] if "k" in c else c["prefix_k"]).shape[-2]
    share, cap = heads // kv_heads, c["k"].shape[1] if "k" in c else 0
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.zeros((batch, queries, heads), dtype=torch.float64, device="cuda")
    weights = torch.zeros((batch, kv_heads, cap), dtype=torch.float64, device="cuda")
    none, most = torch.zeros((0, dim), dtype=torch.float64, device="cuda"), 0.0
    for h in range(kv_heads):
        at = slice(h * share, (h + 1) * share)
        pk, pv = (c[x][:, h].double() if "prefix_k" in c else none for x in ("prefix_k", "prefix_v"))
        for b in range(batch):
            n = min(max(int(c["lens"][b]), 0), cap) if cap else 0
            ok, ov = (c[x][b, :n, h].double() if cap else none for x in ("k", "v"))
            keys, values = torch.cat([pk, ok]), torch.cat([pv, ov])
            rows = q[b, :, at].reshape(-1, dim)
            token = torch.arange(queries, device="cuda").repeat_interleave(share)[:, None]
            hidden = torch.arange(len(keys), device="cuda")[None] >= len(pk) + n - (queries - 1 - token)
            hidden &= torch.arange(len(keys), device="cuda")[None] >= len(pk)
            s = (rows @ keys.T.contiguous() * scale).masked_fill(hidden, -math.inf)
            most = max(most, float((rows.abs() @ keys.abs().T.contiguous()).max()) * abs(scale))
            p = torch.softmax(s, 1).nan_to_num(0.0)
            out[b, :, at] = (p @ values).view(queries, share, dim)
            size[b, :, at] = (p @ values.abs()).view(queries, share, dim)
            lse[b, :, at] = torch.logsumexp(s, 1).view(queries, share)
            weights[b, h, :n] = p[:, len(pk):].sum(0)
    return out.cpu(), lse.cpu(), weights.cpu(), size.cpu(), most


@pytest.fixture(autouse=True)
def quick(monkeypatch):
    monkeypatch.setattr(small, "reference", reference)


@pytest.mark.parametrize("dtype,batch,queries,heads,kv_heads,dim,prefix,own,lens", [
    (torch.bfloat16, 65, 1, 64, 64, 64, 8192, 33, None),       # shared rows alone are wide
    (torch.float16, 130, 1, 32, 32, 128, 8160, 20, None),      # two items a head, of 128 rows and 2
    (torch.bfloat16, 2, 65, 64, 64, 128, 0, 4113, [4113, 64]),  # own rows; the second sequence's first token sees none
    (torch.float16, 1, 100, 64, 32, 80, 8192, 150, [150]),     # both, columns that are not a power of two
    (torch.bfloat16, 3, 33, 128, 32, 40, 3600, 333, [333, 0, 200])])
def test_128_rows(dtype, batch, queries, heads, kv_heads, dim, prefix, own, lens):
    small.check(small.make(dtype, batch, queries, heads, kv_heads, dim, prefix, own, lens))


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_128_rows_later_tokens_do_not_reach_earlier_ones(bad):
    c = small.make(torch.bfloat16, 1, 65, 32, 32, 128, 16384, 130, [130])
    want = hl.prefix_attention(**c)
    c["v"][0, 100:] = bad  # tokens 35 and later see these
    got = hl.prefix_attention(**c)
    assert torch.equal(got.out[0, :35], want.out[0, :35])
    assert not got.out[0, 35:].isfinite().any()


@pytest.mark.parametrize("dtype", small.TYPES)
@pytest.mark.parametrize("shape", [(2, 1, 4, 2, 64, 9000, 300), (9, 1, 8, 2, 256, 6000, 33), (16, 1, 32, 8, 128, 4101, 40),
                                   (3, 1, 16, 4, 80, 5000, 2600), (1, 5, 4, 1, 128, 0, 20000)])
def test_many_parts(dtype, shape):
    small.check(small.make(dtype, *shape))
