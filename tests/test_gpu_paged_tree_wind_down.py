"""How long the attention of drafted trees takes to wind down when a wait runs out: no wait of the way out has a bound of its own. The default bound is 2^31 clocks, 1.1 s
at the highest clock; a call that gives up is to end within a tenth of that (its own waits are some microseconds)."""
import pytest
import torch

import masked_ref as ref
import paged_ref
from paper_2410_05265_b200 import binding

from test_gpu_paged_tree import begins, i32, see
from test_gpu_paged_tree_timeout import CASES, PQ_ERR_TIMEOUT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.set_wait_limit(0)
    c.check()
    c.close()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("name", list(CASES) + ["three tiles and four"])
def test_a_call_that_gives_up_ends_soon(ctx, name, steps):
    """Wherever the wait runs out, also after the last copy has been asked for, when the ring of copies has been gone round once or more."""
    lengths, new = ([384, 512, 500], [20, 9, 30]) if name == "three tiles and four" else CASES[name]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps=steps, seed=5)
    begin, most = begins(new), max(new)
    q, mask, qb = paged_ref.queries(begin[-1], 8, seed=5), ref.words_of(see(new, 3), 4, begin[-1]), i32(begin)
    ws = ctx.attn_kv4_paged_tree_workspace(cache, begin[-1], most)
    out, gave_up = torch.empty_like(q), 0
    run = lambda: ctx.attn_kv4_paged_tree(cache, q, qb, most, mask, 128**-0.5, ws, out=out)
    run()
    assert ctx.check_status() == 0
    for limit in [50, 200, 400] + list(range(600, 12000, 200)):
        ctx.set_wait_limit(limit)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        run()
        b.record()
        ctx.set_wait_limit(0)
        status = ctx.check_status()
        assert status in (0, PQ_ERR_TIMEOUT)
        assert a.elapsed_time(b) < 110.0, f"limit {limit}: {a.elapsed_time(b)} ms"
        gave_up += status == PQ_ERR_TIMEOUT
    assert gave_up > 0
