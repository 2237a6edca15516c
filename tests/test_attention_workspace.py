"""The workspace of prefix_attention (no GPU, which plans for 256 compute units): its size is what the call's parts need, and
every part that any lengths lead to has its place in it. The partition of the keys among blocks is restated in Python."""
import ctypes
import random

import pytest

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
A, MIB = 0x10000, 1 << 20
UNIT, LEAST_WIDE, MANY_UNITS, BLOCKS = 128, 2, 8, 512
SOLO, SOLO_MANY, LEAST = 768, 1024, 512


def size(batch, queries, heads, kv_heads, dim, prefix, own, weights=False):
    def kv(n):
        row = kv_heads * dim
        return hl.KeysValues(A, A, n, n * row, row, dim, n * row, row, dim)
    a = hl.AttentionShape(hl.HL_BF16, batch, queries, heads, kv_heads, dim, 0.1, kv(prefix), kv(own))
    return hl.lib().hl_attention_workspace_bytes(ctypes.byref(a), int(weights))


def units(keys):
    return -(-keys // UNIT)


class Plan:
    """What the host decides: the rows of items, the blocks, and how many parts of each line have a place."""

    def __init__(self, batch, queries, heads, kv_heads, dim, prefix, own):
        self.batch, self.kv_heads, self.prefix, self.own = batch, kv_heads, prefix, own
        share = heads // kv_heads
        rows = {"prefix": batch * queries * share, "own": queries * share}
        r = 2 if max(rows.values()) > 64 and dim <= 128 else 1
        while True:
            self.wide = {s: n > 16 for s, n in rows.items()}
            self.held = {s: 64 * r if self.wide[s] else 16 for s in rows}
            self.tiles = {s: -(-rows[s] // self.held[s]) for s in rows}
            self.items = {"prefix": kv_heads * self.tiles["prefix"] if prefix else 0,
                          "own": batch * kv_heads * self.tiles["own"] if own else 0}
            self.units = {"prefix": self.items["prefix"] * units(prefix), "own": self.items["own"] * units(own)}
            wide_units = sum(self.units[s] for s in rows if self.wide[s])
            if r == 1 or wide_units >= MANY_UNITS * BLOCKS:
                break
            r = 1
        narrow_units = sum(self.units.values()) - wide_units
        self.blocks = min(BLOCKS, max(16, (wide_units // LEAST_WIDE + narrow_units + 15) // 8 * 8))
        self.solo = rows["own"] <= 16 and prefix + own <= (SOLO_MANY if batch * kv_heads * 2 >= 256 else SOLO)
        self.places = {}
        for wide, n in ((True, wide_units), (False, narrow_units)):
            self.places[wide] = self.blocks + sum(self.items[s] for s in rows if self.wide[s] == wide) if n else 0
        self.part_rows = {True: max((self.held[s] for s in rows if self.wide[s]), default=0),
                          False: min(16, max((rows[s] for s in rows if not self.wide[s]), default=0))}
        self.columns = 64 if dim <= 64 else 128 if dim <= 128 else 256

    def bytes(self):
        n = 0
        for wide in (True, False) if not self.solo else ():
            for floats in (self.columns, 2):
                n += -(-self.places[wide] * self.part_rows[wide] * floats * 4 // 256) * 256
        return max(n, LEAST)

    def parts(self, lens):
        """(line, place) of every part, for these lengths of the own caches."""
        line = {True: [], False: []}  # units' item numbers, in the line's order
        for wide in line:
            item = 0
            if self.wide["prefix"] == wide:
                for _ in range(self.items["prefix"]):
                    line[wide] += [item] * units(self.prefix)
                    item += 1
            if self.wide["own"] == wide and self.own:
                for n in lens:
                    for _ in range(self.kv_heads * self.tiles["own"]):
                        line[wide] += [item] * units(n)
                        item += 1
        total = {wide: len(u) for wide, u in line.items()}
        w = 0
        if total[True]:
            w = self.blocks * total[True] // (total[True] + total[False]) if total[False] else self.blocks
            w = min(w, -(-total[True] // LEAST_WIDE))
            w = max(min(-(-w // 8) * 8, self.blocks - (8 if total[False] else 0)), 8)
        out = []
        for wide, blocks in ((True, w), (False, self.blocks - w)):
            takers = min(blocks, total[wide])
            for k in range(takers):
                mine = line[wide][k * total[wide] // takers:(k + 1) * total[wide] // takers]
                out += [(wide, k + item) for item in sorted(set(mine))]
        return out


SHAPES = [(16, 1, 32, 8, 128, 8192, 1024), (256, 1, 32, 8, 128, 8192, 1024), (300, 1, 32, 8, 128, 8192, 0),
          (40, 1, 32, 8, 128, 0, 2000), (3, 1, 16, 2, 64, 0, 1500), (4, 256, 32, 8, 128, 4096, 512),
          (2, 64, 8, 8, 128, 0, 3000), (5, 3, 32, 32, 128, 1777, 777), (9, 20, 8, 2, 80, 40, 1200),
          (1, 40, 8, 1, 256, 900, 300), (2, 10, 8, 2, 64, 0, 90), (64, 2, 64, 8, 256, 16384, 300)]


@pytest.mark.parametrize("shape", SHAPES)
def test_every_part_has_its_own_place(shape):
    plan, rng = Plan(*shape), random.Random(1)
    assert size(*shape) == plan.bytes()
    batch, own = shape[0], shape[6]
    full = [[own] * batch, [0] * batch, [1] * batch, [own] + [0] * (batch - 1), [0] * (batch - 1) + [own]]
    for lens in full + [[rng.randint(0, own) for _ in range(batch)] for _ in range(3)]:
        parts = plan.parts(lens)
        assert len(set(parts)) == len(parts)
        assert all(place < plan.places[wide] for wide, place in parts)


def test_small_where_few_parts_can_be():
    # decode batches on a shared prefix: wide parts for the prefix alone, narrow ones for the sequences
    assert size(256, 1, 32, 8, 128, 8192, 1024) < 48 * MIB
    assert size(4096, 1, 32, 8, 128, 8192, 1024) < 192 * MIB
    assert size(4096, 1, 32, 8, 128, 8192, 0) < 100 * MIB
    # a block a sequence and key head has no parts; the weights need its scores
    assert size(1024, 1, 32, 8, 128, 500, 200) == LEAST
    assert size(1024, 1, 32, 8, 128, 500, 200, True) == 4 * 1024 * 32 * 224


def test_never_nothing():
    for shape in ((1, 1, 1, 1, 8, 0, 0), (2, 40, 8, 2, 64, 0, 0), (1, 1, 4, 4, 64, 1, 0)):
        assert size(*shape) == LEAST
