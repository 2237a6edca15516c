"""cache_write4 and cache_read4 (MI355X): rows byte for byte as the definition gives them, and their values to one
rounding."""
import pytest
import torch

import paper_2502_00922_amd as hl
from rows4 import random_rows, row_bytes, rows_of, values

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
FILL = 0xA5


def rand(shape, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(shape, generator=g, device="cuda") * torch.exp(2 * torch.randn(shape[-1], generator=g, device="cuda"))
    return t.to(dtype)


def caches(batch, capacity, heads, dim):
    return [torch.full((batch, capacity, heads, row_bytes(dim)), FILL, dtype=torch.uint8, device="cuda") for _ in range(2)]


def check(k, v, ck, cv, lens):
    """The caches after a write: the new tokens' rows in their slots, every other byte as it was."""
    hl.cache_write4(k, v, ck, cv, lens)
    batch, tokens = k.shape[:2]
    for x, cache in ((k, ck), (v, cv)):
        want = torch.full(cache.shape, FILL, dtype=torch.uint8)
        rows = rows_of(x)
        for b in range(batch):
            for i in range(tokens):
                slot = i if lens is None else int(lens[b]) - tokens + i
                if 0 <= slot < cache.shape[1]:
                    want[b, slot] = rows[b, i]
        assert torch.equal(cache.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("batch,tokens,heads", [(1, 1, 1), (3, 5, 2), (2, 67, 3)])
def test_rows(dtype, dim, batch, tokens, heads):
    k, v = rand((batch, tokens, heads, dim), dtype), rand((batch, tokens, heads, dim), dtype, 1)
    ck, cv = caches(batch, tokens + 3, heads, dim)
    lens = torch.arange(tokens, tokens + batch, dtype=torch.int32, device="cuda")
    check(k, v, ck, cv, lens)


@pytest.mark.parametrize("lens", [[4, 0, -7, 9], [12, 13, 100, 2**31 - 1], None, [1, 2, 3, -(2**31)]])
def test_slots_outside_the_cache_are_left_out(lens):
    k, v = rand((4, 4, 2, 64), torch.bfloat16), rand((4, 4, 2, 64), torch.bfloat16, 1)
    ck, cv = caches(4, 12, 2, 64)
    check(k, v, ck, cv, None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))


def test_more_tokens_than_the_cache_has_slots():
    k, v = rand((2, 9, 1, 32), torch.float16), rand((2, 9, 1, 32), torch.float16, 1)
    ck, cv = caches(2, 4, 1, 32)
    check(k, v, ck, cv, torch.tensor([4, 9], dtype=torch.int32, device="cuda"))
    ck, cv = caches(2, 4, 1, 32)
    check(k, v, ck, cv, None)


def test_ties_and_steps():
    # with a base and a scale of whole numbers, columns on every tie and next to it
    x = torch.zeros((1, 16, 1, 32), dtype=torch.bfloat16, device="cuda")
    for i in range(16):
        scale = 2.0 ** (i - 8)
        t = torch.arange(32, dtype=torch.float32) / 2 - 8
        t[31] = 7
        x[0, i, 0] = t * scale
    for sign in (1, -1):
        ck, cv = caches(1, 16, 1, 32)
        check(sign * x, -sign * x, ck, cv, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_columns_far_apart_in_size(dtype):
    # differences that float32 rounds
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((4, 512, 2, 64), generator=g, device="cuda")
    x *= 2.0 ** torch.randint(-24, 8, x.shape, generator=g, device="cuda")
    ck, cv = caches(4, 512, 2, 64)
    check(x.to(dtype), (-x).to(dtype), ck, cv, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_tiny_and_huge_columns(dtype):
    info = torch.finfo(dtype)
    x = torch.zeros((1, 8, 1, 64), dtype=dtype, device="cuda")
    x[0, 0] = 3.125
    x[0, 1, 0, ::3] = info.tiny
    x[0, 2, 0, ::2] = info.tiny * info.eps  # the least number there is
    x[0, 3, 0, ::5] = info.max
    x[0, 3, 0, 1::5] = -info.max
    x[0, 4] = -info.max
    x[0, 5] = 100 + torch.arange(64, device="cuda").to(dtype) / 4
    x[0, 6] = -info.tiny
    x[0, 7, 0, 40] = 1.0
    ck, cv = caches(1, 8, 1, 64)
    check(x, x.flip(-1).contiguous(), ck, cv, None)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_group_with_infinity_or_nan_is_nan(bad):
    x = rand((1, 3, 1, 96), torch.bfloat16)
    x[0, 1, 0, 45] = bad
    ck, cv = caches(1, 3, 1, 96)
    check(x, x.clone(), ck, cv, None)
    got = hl.cache_read4(ck, 96, torch.float32)
    assert got[0, 1, 0, 32:64].isnan().all() and got[0, [0, 2]].isfinite().all()
    assert got[0, 1, 0, :32].isfinite().all() and got[0, 1, 0, 64:].isfinite().all()


def test_strides():
    # caches by heads, inputs out of one packed product, and caches that are a part of a larger one
    packed = rand((2, 6, 5 * 128), torch.bfloat16)
    k, v = packed[..., 128:384].unflatten(-1, (2, 128)), packed[..., 384:].unflatten(-1, (2, 128))
    ck, cv = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in caches(2, 9, 2, 128))
    check(k, v, ck, cv, torch.tensor([6, 9], dtype=torch.int32, device="cuda"))
    big = torch.full((2, 9, 4, 160), FILL, dtype=torch.uint8, device="cuda")
    ck, cv = big[..., 1:3, :80], big[..., 2:4, 80:]
    check(k, v, ck, cv, torch.tensor([9, 7], dtype=torch.int32, device="cuda"))
    assert (big[:, :, 0] == FILL).all() and (big[:, :, 3, :80] == FILL).all()
    k = rand((1, 1, 2, 128), torch.bfloat16).expand(2, 6, 2, 128)  # one token everywhere
    check(k, v, *caches(2, 9, 2, 128), None)


@pytest.mark.parametrize("dtype,step", [(torch.float32, 2.0**-24), (torch.bfloat16, 2.0**-8 + 2.0**-24),
                                        (torch.float16, 2.0**-11 + 2.0**-24)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
def test_read(dtype, step, dim):
    # one rounding in float32 and one more to 16 bits
    g = torch.Generator(device="cuda").manual_seed(dim)
    rows = random_rows((2, 33, 3), dim, g)
    got, want = hl.cache_read4(rows, dim, dtype), values(rows, dim)
    assert got.dtype == dtype and got.shape == want.shape
    err = (got.double().cpu() - want).abs()
    assert (err <= step * want.abs() + 2.0**-25).all()
    part = rows.transpose(0, 1)[5:20, :, 1:]  # [15, 2, 2, bytes] of other strides
    assert torch.equal(hl.cache_read4(part, dim, dtype), hl.cache_read4(part.contiguous(), dim, dtype))
    out = torch.zeros((33, 3, dim), dtype=dtype, device="cuda")
    assert hl.cache_read4(rows[1], dim, out=out) is out and torch.equal(out, got[1])


def test_default_type():
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = random_rows((3, 1), 64, g)
    assert hl.cache_read4(rows, 64).dtype == torch.bfloat16


def test_captured():
    # a graph's write goes by the lengths at each replay
    k, v = rand((2, 1, 2, 64), torch.bfloat16), rand((2, 1, 2, 64), torch.bfloat16, 1)
    ck, cv = caches(2, 5, 2, 64)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    hl.cache_write4(k, v, ck, cv, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens += 1
        hl.cache_write4(k, v, ck, cv, lens)
        read = hl.cache_read4(ck, 64)
    want_k, want_v = rows_of(k), rows_of(v)
    for n in range(1, 5):
        k.copy_(k.flip(-1))
        graph.replay()
        torch.cuda.synchronize()
        want_k = rows_of(k)
        assert torch.equal(ck[:, n - 1].cpu(), want_k[:, 0]) and torch.equal(cv[:, n - 1].cpu(), want_v[:, 0])
        assert (ck[:, n:] == FILL).all()
        assert torch.equal(read, hl.cache_read4(ck, 64))


def test_far_offsets():
    # a cache whose rows lie past 32 bits
    stride = 48 * 1024 * 1024
    big = torch.empty(100 * stride + 48, dtype=torch.uint8, device="cuda")
    cache = big.as_strided((1, 100, 1, 48), (0, stride, 48, 1))
    k = rand((1, 100, 1, 64), torch.bfloat16)
    near, other = caches(1, 100, 1, 64)
    hl.cache_write4(k, k, cache, other)
    hl.cache_write4(k, k, near, other)
    assert torch.equal(cache, near) and torch.equal(hl.cache_read4(cache, 64), hl.cache_read4(near, 64))
