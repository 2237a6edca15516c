"""sample's settings as numbers past what the library's types hold (no GPU: a library that notes what it is given)."""
import math
import struct

import pytest

hl = pytest.importorskip("paper_2502_00922_amd.hufflm")
from test_operator4_arguments import gpus, sample_args  # noqa: E402, F401

MOST = (2 - 2.0**-23) * 2.0**127  # of float32


@pytest.mark.parametrize("given,held", [
    (dict(top_k=math.inf), dict(top_k=0x7FFFFFFF)), (dict(top_k=1 << 40), dict(top_k=0x7FFFFFFF)), (dict(top_k=7), dict(top_k=7)),
    (dict(temperature=1e39), dict(temperature=MOST)), (dict(temperature=math.inf), dict(temperature=math.inf)),
    (dict(top_p=1e300), dict(top_p=MOST)), (dict(top_p=0.5, min_p=0.25), dict(top_p=0.5, min_p=0.25))])
def test_what_the_library_gets(gpus, monkeypatch, given, held):  # noqa: F811
    seen = []
    monkeypatch.setattr(hl._torch.lib, "hl_sample", lambda settings, *a: seen.append(settings) or 0, raising=False)
    hl.sample(**{**sample_args(), **dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **given})
    numbers = dict(zip(("temperature", "top_k", "top_p", "min_p"), struct.unpack("=4Qfiff", seen[0])[4:]))
    assert numbers == {**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **held}
