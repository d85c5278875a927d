"""Calls of the paged KV4 entry points that are easily got wrong: row ranges outside the queries, and results that must not depend on which
shapes a process ran before."""
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
D, DEV = 128, "cuda"
PQ_ERR_SHAPE = 2


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.check()
    c.close()


@pytest.mark.parametrize("max_new", [1, 3])
@pytest.mark.parametrize("n_seqs", [3, 700])
@pytest.mark.parametrize("begin", [[0, 1, 5], [-1, 0, 1], [2, 1, 2], [3, 4, 5], [0, 0, -1], [0, 2**31 - 1, 3], [-2**31, 2**31 - 1, 3]])
def test_rows_outside_the_queries_are_reported_in_a_step_of_single_tokens_too(ctx, begin, n_seqs, max_new):
    """Whatever bound the caller gives; the rows of sequences that are in order are computed, the others left out. With one worker to a pair (few
    sequences) and in equal stretches (many)."""
    lengths = [20, 40] + [100] * (n_seqs - 2)
    cache = ref.make_cache(lengths[:2], 4, 2, 16, seed=8, width=8)
    extra = n_seqs - 2  # sequences without rows behind the two
    pg = cache.pages
    table = torch.cat((pg.table, torch.zeros((extra, pg.max_pages), dtype=torch.int32, device=DEV)))
    cache = binding.KV4PagedCache(binding.Pages(table, i32(lengths), pg.free_list, pg.n_free, 16), cache.prefix_k, cache.prefix_v, cache.codes, 4, s_k=cache.s_k,
                                  s_v=cache.s_v)
    q = ref.queries(4, 4)
    ws = ctx.attn_kv4_paged_workspace(cache, 4, max_new)
    out = torch.full((4, 4, D), 9.0, dtype=torch.bfloat16, device=DEV)
    ctx.attn_kv4_paged(cache, q, i32(begin + [begin[-1]] * extra), max_new, 0.1, ws, out=out)
    assert ctx.check_status() == PQ_ERR_SHAPE
    good = [(b, begin[b]) for b in range(2) if begin[b + 1] - begin[b] == 1 and 0 <= begin[b] < 4]
    want, tol = torch.full(out.shape, 9.0, dtype=torch.float64, device=DEV), torch.zeros(out.shape, dtype=torch.float64, device=DEV)
    for b, r in good:
        w, t = ref.attention(cache, q[r: r + 1], [0] * (b + 1) + [1] * (n_seqs - b), lengths[: b + 1] + [0] * (n_seqs - b - 1), 0.1)
        want[r], tol[r] = w[0], t[0]
    assert ((out.double() - want).abs() <= tol).all()


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
