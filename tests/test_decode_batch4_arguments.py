"""examples/decode_batch.py refuses, before it touches a GPU, what its 4-bit operators do not take (no GPU)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("args,what", [
    ("--cache-bits 8", "cache-bits"), ("--cache-bits 4 --dim 80", "dim"), ("--cache-bits 4 --dim 512", "dim"),
    ("--vocab -1", "vocab"), ("--vocab 1048576", "vocab"), ("--vocab 100 --hidden 520", "vocab")])
def test_refused(args, what):
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_batch.py"), *args.split()],
                       capture_output=True, text=True, env={**os.environ, "HIP_VISIBLE_DEVICES": "-1"}, timeout=300)
    assert r.returncode == 2 and what in r.stderr.splitlines()[-1], r.stderr[-500:]
