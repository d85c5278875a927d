"""Calls of the paged KV4 entry points that are easily got wrong: row ranges outside the queries, one row appended in place, ids that are none given back, host
threads with a context each, and results that must not depend on which shapes a process ran before."""
import ctypes
import hashlib
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2410_05265_b200 import binding

import paged_ref as ref
from test_gpu_paged import gains, heads, i32, pages_of, positions

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


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_one_row_is_appended_in_place(ctx, steps):
    """The stride of a single row says nothing: the query heads may stay where the projection wrote them, as with several rows."""
    Hq, Hkv = 4, 2
    (gq, gk), pos, slot = gains(1), positions(1, 1, 5), torch.tensor([3], device=DEV)
    qkv = heads(1, Hq + 2 * Hkv, 6).view(1, -1)
    a, b = (ref.make_cache([20], Hq, Hkv, 32, steps, seed=1) for _ in range(2))
    q = ctx.qk_norm_rope_kv4_paged_append(a, qkv, gq, gk, 1e-5, pos, slot, 500000.0)
    rest = qkv[:, Hq * D:].clone()
    ctx.qk_norm_rope_kv4_paged_append(b, qkv, gq, gk, 1e-5, pos, slot, 500000.0, q_out=qkv[:, : Hq * D].unflatten(1, (Hq, D)))
    ctx.check()
    assert torch.equal(qkv[:, : Hq * D].view(1, Hq, D), q) and torch.equal(qkv[:, Hq * D:], rest)
    assert torch.equal(a.codes, b.codes) and (steps == "head" or torch.equal(a.steps, b.steps))


@pytest.mark.parametrize("n_pages", [12, 5000])
@pytest.mark.parametrize("bad", [-1, 10**6, "n_pages"])
def test_release_gives_no_ids_back_that_are_none(ctx, bad, n_pages):
    """A page id outside the pool in the table of an ended request: nothing changes and it is reported, as with a length that is none. Ids of requests that
    go on, and entries behind an ended one's pages, are not looked at. One CTA and a cluster of them."""
    bad = n_pages if bad == "n_pages" else bad
    free = [2, 4] + [9] * (n_pages - 2)
    for table, done, refused in (([[3, bad, -1], [0, -1, -1]], [1, 1], True), ([[3, 1, -1], [bad, -1, -1]], [1, 1], True), ([[3, bad, -1], [0, -1, -1]], [0, 1], False),
                                 ([[3, 1, bad], [0, bad, -1]], [1, 1], False)):
        pg = pages_of(table, [20, 16], free, 2, 16)
        ctx.page_release(pg, i32(done))
        if refused:
            assert ctx.check_status() == PQ_ERR_SHAPE
            assert pg.length.tolist() == [20, 16] and pg.n_free.tolist() == [2] and pg.free_list.tolist() == free
        else:
            back = ([3, 1] if done[0] else []) + [0]
            ctx.check()
            assert pg.length.tolist() == [0 if d else n for d, n in zip(done, [20, 16])] and pg.n_free.tolist() == [2 + len(back)]
            assert pg.free_list.tolist() == [2, 4] + back + free[2 + len(back):]


def test_host_threads_with_a_context_each_do_not_disturb_one_another():
    """Plans and releases of batches whose shared memory differs and is above what a kernel gets by itself, from four host threads at once, each on a stream of its
    own: all are launched. (The library is called directly, so that the threads meet in it.)"""
    lib, page, n_calls, seen = binding.load_library(), 16, 10000, {}

    def serve(B):
        c, stream = binding.Context(), torch.cuda.Stream()
        with torch.cuda.stream(stream):
            z = lambda n, dtype=torch.int32: torch.zeros(n, dtype=dtype, device=DEV)
            pg = binding.Pages(z(2 * B).view(B, 2), z(B), torch.arange(B, dtype=torch.int32, device=DEV), i32([B]), page)
            n_new, done, out = z(B), z(B), [z(B + 1), z(4, torch.int64), z(4), z(B), z(1)]
            n_new[0] = 1
            torch.cuda.synchronize()
            at, ref_pages, s = [t.data_ptr() for t in out], ctypes.byref(pg.struct), stream.cuda_stream
            statuses = set()
            for _ in range(n_calls):
                statuses.add(lib.pq_page_plan(c.h, ref_pages, n_new.data_ptr(), 0, 4, *at, s))
                statuses.add(lib.pq_page_release(c.h, ref_pages, done.data_ptr(), at[3], at[4], s))
            statuses.add(c.check_status())
            seen[B] = statuses
        c.close()

    threads = [threading.Thread(target=serve, args=(B,)) for B in (4200, 5000, 7000, 8192)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert seen == {B: {0} for B in (4200, 5000, 7000, 8192)}


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
