"""4-bit cache rows in plain numpy and torch on the CPU, for the tests: what a row stands for, and what a row of given
values is."""
import numpy as np
import torch


def row_bytes(dim):
    return -(-(dim // 2 + dim // 8) // 16) * 16


def places(dim):
    """(byte, shift) of each column's code."""
    d = np.arange(dim)
    return d % 32 // 2 * (dim // 32) + d // 32, d % 2 * 4


def parts(rows, dim):
    """(codes, scale, base) [.., dim] in float64 of rows, a uint8 tensor."""
    r = rows.cpu().numpy()
    byte, shift = places(dim)
    codes = (r[..., byte] >> shift & 15).astype(np.float64)
    pairs = np.ascontiguousarray(r[..., dim // 2:dim // 2 + dim // 8]).view(np.uint16).astype(np.uint32) << 16
    pairs = pairs.view(np.float32).astype(np.float64).repeat(32, axis=-1).reshape(*r.shape[:-1], dim // 32, 2, 32)
    scale, base = (pairs[..., i, :].reshape(*r.shape[:-1], dim) for i in (0, 1))
    return tuple(torch.from_numpy(t) for t in (codes, scale, base))


def values(rows, dim):
    codes, scale, base = parts(rows, dim)
    return base + scale * (codes - 8)


def to_bf16(x):
    """float32 numbers rounded to bfloat16, ties to even, as bits (NaN: 0x7FC0)."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + (b >> 16 & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def rows_of(x):
    """The rows of x [.., dim], a bf16 or f16 tensor, from the definition."""
    dim = x.shape[-1]
    t = x.float().cpu().numpy().reshape(*x.shape[:-1], dim // 32, 32)
    out = np.zeros((*x.shape[:-1], row_bytes(dim)), dtype=np.uint8)
    with np.errstate(all="ignore"):
        low, high = t.min(-1), t.max(-1)
        f = np.float32
        base = (to_bf16((f(7) * low + f(8) * high) / f(15)).astype(np.uint32) << 16).view(f)
        scale = (to_bf16(np.maximum((high - base) / f(7), (base - low) / f(8))).astype(np.uint32) << 16).view(f)
        good = np.isfinite(t).all(-1) & np.isfinite(base) & np.isfinite(scale)
        q = (t.astype(np.float64) - base.astype(np.float64)[..., None]) / scale.astype(np.float64)[..., None]
        steps = np.clip(np.rint(q), -8, 7)
        codes = np.where((good & (scale > 0))[..., None], steps + 8, 8).astype(np.uint8).reshape(*x.shape[:-1], dim)
    byte, shift = places(dim)
    for d in range(dim):
        out[..., byte[d]] |= codes[..., d] << np.uint8(shift[d])
    pairs = np.stack([np.where(good, to_bf16(scale), 0x7FC0), np.where(good, to_bf16(base), 0x7FC0)], -1)
    out[..., dim // 2:dim // 2 + dim // 8] = np.ascontiguousarray(pairs.astype(np.uint16)).view(np.uint8).reshape(
        *x.shape[:-1], dim // 8)
    return torch.from_numpy(out)


def random_rows(shape, dim, g, scale=0.3, base=0.4):
    """Rows [*shape, bytes] of random codes, on the GPU; g: a generator there."""
    t = torch.randint(0, 256, (*shape, row_bytes(dim)), generator=g, device="cuda", dtype=torch.uint8)
    pairs = torch.empty((*shape, dim // 32, 2), dtype=torch.bfloat16, device="cuda")
    pairs[..., 0] = scale * (0.5 + torch.rand((*shape, dim // 32), generator=g, device="cuda"))
    pairs[..., 1] = base * torch.randn((*shape, dim // 32), generator=g, device="cuda")
    t[..., dim // 2:dim // 2 + dim // 8] = pairs.flatten(-2).view(torch.uint8)
    t[..., dim // 2 + dim // 8:] = 0
    return t
