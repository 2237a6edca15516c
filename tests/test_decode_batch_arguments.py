"""examples/decode_batch.py refuses, before it touches a GPU, sizes with which a step would write past a cache's end (no GPU)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# an eviction that leaves no room for the next token; no token kept; sizes of nothing
@pytest.mark.parametrize("args,what", [
    ("--cache 64 --keep 64 --steps 65", "cache"), ("--cache 64 --keep 100 --steps 65", "cache"), ("--cache 0", "cache"),
    ("--keep 16 --recent 17 --steps 300", "recent"), ("--recent -1 --steps 300", "recent"),
    ("--keep 0 --recent 0 --steps 300", "keep"), ("--steps 0", "steps"), ("--prompt 0", "prompt")])
def test_refused(args, what):
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_batch.py"), *args.split()],
                       capture_output=True, text=True, env={**os.environ, "HIP_VISIBLE_DEVICES": "-1"}, timeout=300)
    assert r.returncode == 2 and what in r.stderr.splitlines()[-1], r.stderr[-500:]
