"""Calls of the paged KV4 entry points that are easily got wrong: results that must not depend on which shapes a process ran before."""
import hashlib
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2410_05265_b200 import binding

import paged_ref as ref
from test_gpu_paged import i32

pytestmark = pytest.mark.gpu
D = 128


# (sequences, tokens of each, query heads, KV heads), own steps but for the last: the shared memory of the first two differs by 3.6 KB, and with the larger one
# three CTAs fit an SM, with the smaller one four
SHAPES = {"smaller": (500, 300, 8, 2), "larger": (800, 250, 8, 2), "static": (60, 3000, 32, 8)}


def digest(names):
    """Outputs of decode calls of these shapes, in this order, as one hash each."""
    ctx, seen = binding.Context(), []
    for name in names:
        B, n, Hq, Hkv = SHAPES[name]
        lengths = [n - (37 * b) % (n // 2) for b in range(B)]
        cache = ref.make_cache(lengths, Hq, Hkv, 16, "head" if name == "static" else "vector", seed=B)
        out = ctx.attn_kv4_paged(cache, ref.queries(B, Hq), i32(list(range(B + 1))), 1, 1 / math.sqrt(D), ctx.attn_kv4_paged_workspace(cache, B, 1))
        ctx.check()
        seen.append(name + " " + hashlib.sha256(out.view(torch.int16).cpu().numpy().tobytes()).hexdigest())
    return sorted(seen)


def test_results_do_not_depend_on_what_ran_before():
    """The same calls in another order, in processes of their own: the same bits. (How many workers share the keys follows from the call alone.)"""
    here = os.path.dirname(os.path.abspath(__file__))
    runs = []
    for order in ("smaller larger static", "static larger smaller"):
        code = f"import test_gpu_paged_calls as t; print('\\n'.join(t.digest('{order}'.split())))"
        env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here), os.environ.get("PYTHONPATH", "")]))
        r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        runs.append(r.stdout.split("\n"))
    assert len(runs[0]) == 4 and runs[0] == runs[1]
