"""Drafted trees behind a first cached key that draws nearly all of the weight (an attention sink that nobody has put into the prefix): the other keys' weights keep their
bits, judged by the row itself."""
import pytest
import torch

import masked_ref as ref
from paper_2410_05265_b200 import binding

import first_keys
from test_gpu_paged_tree import begins, i32, see

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


# lengths, rows, window, n_sink, heads
SHAPES = [([1000], [20], 0, 0, 8, 2), ([9000, 700], [9, 33], 0, 0, 8, 2), ([130, 257, 100], [20, 1, 5], 0, 0, 4, 1), ([2500, 900], [20, 40], 700, 4, 8, 2),
          ([300, 90], [20, 9], 500, 4, 6, 2), ([3000], [100], 400, 140, 8, 1), ([600], [64], 1000, 0, 8, 2), ([500 + 9 * b for b in range(60)], [16] * 60, 0, 0, 16, 2)]


@pytest.mark.parametrize("n_prefix", [0, 3])
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", [3.0, 12.3, 18.4, 21.7, 24.0, 26.0, 30.0])
@pytest.mark.parametrize("lengths,new,window,n_sink,Hq,Hkv", SHAPES)
def test_a_first_key_that_draws_nearly_all_of_the_weight(ctx, lengths, new, window, n_sink, Hq, Hkv, above, steps, n_prefix):
    where = 3 if n_sink else 0
    cache = first_keys.make(lengths, Hq, Hkv, steps, n_prefix, above, where)
    begin, trees = begins(new), see(new, 3)
    q, N = first_keys.ones(begin[-1], Hq), begin[-1]
    want, tol = first_keys.bounds(cache, q, begin, lengths, above, where, window, n_sink, trees)
    ws = ctx.attn_kv4_paged_tree_workspace(cache, N, max(new))
    out = ctx.attn_kv4_paged_tree(cache, q, i32(begin), max(new), ref.words_of(trees, 4, N), first_keys.LN2, ws, window=window, n_sink=n_sink, max_len=max(lengths))
    assert ctx.check_status() == 0
    first_keys.assert_within(out, want, tol, N)


def test_several_first_keys_share_the_weight(ctx):
    """Four of them, with equal scores."""
    lengths, new, above = [1500], [20], 24.0
    for steps in ("head", "vector"):
        cache = first_keys.make(lengths, 8, 2, steps, 0, above, 0, n=4)
        begin, trees = begins(new), see(new, 3)
        q = first_keys.ones(20, 8)
        want, tol = first_keys.bounds(cache, q, begin, lengths, above, 0, 0, 0, trees, n=4)
        ws = ctx.attn_kv4_paged_tree_workspace(cache, 20, 20)
        out = ctx.attn_kv4_paged_tree(cache, q, i32(begin), 20, ref.words_of(trees, 1, 20), first_keys.LN2, ws)
        assert ctx.check_status() == 0
        first_keys.assert_within(out, want, tol, 20)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", [20.0, 26.0])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [([2900], [40], 8, 2), ([5000, 1700], [100, 30], 5, 1), ([1500] * 40, [30] * 40, 8, 2)])
def test_several_tiles_of_first_keys(ctx, lengths, new, Hq, Hkv, above, steps):
    """Some of them begin a worker's share of an item: what sets the reference there is the heavy key's tile, and others follow."""
    window, n_sink, where = 300, 900, 3
    cache = first_keys.make(lengths, Hq, Hkv, steps, 0, above, where)
    begin, trees = begins(new), see(new, 3)
    q, N = first_keys.ones(begin[-1], Hq), begin[-1]
    want, tol = first_keys.bounds(cache, q, begin, lengths, above, where, window, n_sink, trees)
    ws = ctx.attn_kv4_paged_tree_workspace(cache, N, max(new))
    out = ctx.attn_kv4_paged_tree(cache, q, i32(begin), max(new), ref.words_of(trees, 4, N), first_keys.LN2, ws, window=window, n_sink=n_sink, max_len=max(lengths))
    assert ctx.check_status() == 0
    first_keys.assert_within(out, want, tol, N)
