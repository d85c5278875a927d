"""A refused pq_page_keep and the moves that follow it in a step that nobody looks at in between: no sequence's cache changes."""
import pytest
import torch

import paged_ref
from paper_2410_05265_b200 import binding

from test_gpu_paged_tree import begins, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def spoil(cache, how, lengths, n_kept):
    pg = cache.pages
    if how == "count above the rows":
        n_kept[1] = 21
    if how == "negative count":
        n_kept[1] = -1
    if how == "fewer tokens than rows":
        pg.length[1] = 19
    if how == "full list":
        pg.n_free.fill_(pg.n_pages)
    if how == "id that is none":
        pg.table[1, paged_ref.up(lengths[1], pg.page) - 1] = pg.n_pages


SPOILT = ["count above the rows", "negative count", "fewer tokens than rows", "full list", "id that is none"]


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("B", [3, 4200])
@pytest.mark.parametrize("how", SPOILT)
def test_moves_after_a_refusal_change_nothing(ctx, how, B, captured, steps):
    """One sequence, the list or an id stops the call; the other sequences' counts are fine and their accepted rows lie behind others."""
    lengths, new = [90 + b % 40 for b in range(B)], [20] * B
    cache = paged_ref.make_cache(lengths, 2, 1, 16, steps=steps, seed=B)
    begin = i32(begins(new))
    kept = i32([x for _ in range(B) for x in [0, 3, 7, 19] + [-1] * 16])
    counts = [4] * B
    spoil(cache, how, lengths, counts)
    n_kept, pg = i32(counts), cache.pages
    state = lambda: [t.clone() for t in (pg.table, pg.length, pg.free_list, pg.n_free, cache.codes) + (() if cache.steps is None else (cache.steps,))]

    def step():
        ctx.page_keep(pg, begin, n_kept)
        for _ in range(2):  # two layers' worth
            ctx.kv4_paged_keep(cache, begin, kept, n_kept)

    if captured:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                step()
        torch.cuda.synchronize()
    before = state()
    graph.replay() if captured else step()
    assert ctx.check_status() == 2
    assert all(torch.equal(a, b) for a, b in zip(before, state()))
    assert torch.all(n_kept == -1)


def test_the_step_after_a_refused_one(ctx):
    """Counts that are put right serve the same lengths, and the moves follow again."""
    cache = paged_ref.make_cache([50, 60], 2, 1, 16, seed=1)
    begin, kept, n_kept, pg = i32([0, 20, 40]), i32([0, 5, 9] + [-1] * 17 + [0, 1, 19] + [-1] * 17), i32([3, 21]), cache.pages
    ctx.page_keep(pg, begin, n_kept)
    ctx.kv4_paged_keep(cache, begin, kept, n_kept)
    assert ctx.check_status() == 2 and pg.length.tolist() == [50, 60]
    table = pg.table.tolist()
    at = lambda b, c: cache.codes[table[b][c // 16], :, :, c % 16]
    want = [at(0, 30 + r).clone() for r in (0, 5, 9)], [at(1, 40 + r).clone() for r in (0, 1, 19)]
    n_kept.fill_(3)
    ctx.page_keep(pg, begin, n_kept)
    ctx.kv4_paged_keep(cache, begin, kept, n_kept)
    assert ctx.check_status() == 0 and pg.length.tolist() == [33, 43] and n_kept.tolist() == [3, 3]
    for i in range(3):
        assert torch.equal(at(0, 30 + i), want[0][i]) and torch.equal(at(1, 40 + i), want[1][i])
