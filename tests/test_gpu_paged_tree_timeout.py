"""Waits of the attention of drafted trees that run out: with a limit of a few clocks they do so at ever other places. The kernel winds down and reports it, and the next call
gives what it always gives. (Short limits take the kernel's polling form.)"""
import pytest
import torch

import masked_ref as ref
import paged_ref
from paper_2410_05265_b200 import binding

from test_gpu_paged_tree import begins, i32, see

pytestmark = pytest.mark.gpu
PQ_ERR_TIMEOUT = 6
# lengths, drafts: one item, items of one key tile, items that workers share, several items to a sequence and head
CASES = {"one": ([700], [9]), "short": ([40 + i for i in range(90)], [1 + i % 30 for i in range(90)]), "shared": ([9000, 300], [20, 5]), "wide": ([900, 128, 2000], [128, 100, 33])}


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.set_wait_limit(0)
    c.check()
    c.close()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("name", list(CASES))
def test_waits_that_run_out(ctx, name, steps):
    lengths, new = CASES[name]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps=steps, seed=5)
    begin, trees = begins(new), see(new, 3)
    n = begin[-1]
    q, mask, qb = paged_ref.queries(n + 1, 8, seed=5), ref.words_of(trees, 4, n + 1), i32(begin)
    ws = ctx.attn_kv4_paged_tree_workspace(cache, n + 1, max(new))
    out = torch.empty_like(q)

    def attend(limit):
        ctx.set_wait_limit(limit)
        out.fill_(7.0)
        ctx.attn_kv4_paged_tree(cache, q, qb, max(new), mask, 128**-0.5, ws, out=out)
        ctx.set_wait_limit(0)
        status = ctx.check_status()
        assert ctx.check_status() == 0  # reading the status word clears it
        assert (out[n:] == 7.0).all()
        return status

    assert attend(0) == 0
    good = out[:n].clone()
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    seen = []
    for limit in (1, 16, 100, 300, 1000, 2000, 5000, 16000):
        for _ in range(4):
            seen.append(attend(limit))
            assert seen[-1] in (0, PQ_ERR_TIMEOUT)
            # what is not reported is right (the polling form may have other columns than the usual one)
            assert seen[-1] == PQ_ERR_TIMEOUT or torch.all((out[:n].double() - want[:n]).abs() <= tol[:n])
            assert attend(0) == 0 and torch.equal(out[:n], good)
    assert PQ_ERR_TIMEOUT in seen[:8], "no limit of a few clocks ran out"
