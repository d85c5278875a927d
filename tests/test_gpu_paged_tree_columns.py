"""Attention of drafted trees in each of its forms (32, 64 and 128 columns): the calls are given bounds with which the rule takes that form, checked against the rule itself."""
import random

import pytest
import torch

import first_keys
import masked_ref as ref
import paged_ref
import tree_form
from paper_2410_05265_b200 import binding

from test_gpu_paged_tree import begins, i32, see

pytestmark = pytest.mark.gpu
COLUMNS = pytest.mark.parametrize("columns", [32, 64, 128])
STEPS = pytest.mark.parametrize("steps", ["head", "vector"])
PQ_ERR_TIMEOUT = 6


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.set_wait_limit(0)
    c.check()
    c.close()


class Call:
    """A call of the form wanted: bounds, and sequences without rows behind the others where only they lead there."""

    def __init__(self, columns, lengths, new, Hq, Hkv, steps, n_prefix, window=0, n_sink=0):
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        found = tree_form.call_for(columns, steps == "vector", n_prefix, len(lengths), Hkv, Hq // Hkv, max(new), max(lengths), window, n_sink, sms)
        assert found is not None, "no bounds lead to this form"
        self.max_new, self.max_len, more = found
        self.lengths, self.new = list(lengths) + [1] * more, list(new) + [0] * more
        self.begin, self.width = begins(self.new), paged_ref.up(max(self.max_len, max(lengths)), 16) + 2
        self.window, self.n_sink = window, n_sink

    def cache(self, Hq, Hkv, steps, n_prefix, seed=0, page=16):
        return paged_ref.make_cache(self.lengths, Hq, Hkv, page, steps=steps, n_prefix=n_prefix, seed=seed, width=self.width)

    def run(self, ctx, cache, q, trees, sm=128**-0.5, out=None):
        N = q.shape[0]
        ws = ctx.attn_kv4_paged_tree_workspace(cache, N, self.max_new)
        return ctx.attn_kv4_paged_tree(cache, q, i32(self.begin), self.max_new, ref.words_of(trees, 4, N), sm, ws, window=self.window, n_sink=self.n_sink,
                                       max_len=self.max_len, out=out)


def check(ctx, columns, lengths, trees, Hq=8, Hkv=2, steps="head", n_prefix=4, window=0, n_sink=0, seed=0, page=16, hide=True):
    new = [len(t) for t in trees]
    call = Call(columns, lengths, new, Hq, Hkv, steps, n_prefix, window, n_sink)
    cache = call.cache(Hq, Hkv, steps, n_prefix, seed, page)
    live = call.begin[-1]
    q, trees = paged_ref.queries(live + 3, Hq, seed=seed), trees + [[]] * (len(call.new) - len(new))
    want, tol = ref.attention(cache, q, call.begin, call.lengths, 128**-0.5, window, n_sink, trees)
    if hide:
        ref.hide_unseen_pages(cache, call.begin, call.lengths, window, n_sink, trees)
    out = call.run(ctx, cache, q, trees, out=torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"))
    assert ctx.check_status() == 0
    assert torch.all(out[live:] == 7.0)
    err = (out[:live].double() - want[:live]).abs()
    assert torch.all(err <= tol[:live]), (err - tol[:live]).max()


@COLUMNS
@STEPS
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (3, 1), (5, 1), (12, 2), (7, 1), (16, 2)])
def test_head_ratios(ctx, Hq, Hkv, steps, columns):
    check(ctx, columns, [170, 20, 400], see([20, 20, 7], 4), Hq=Hq, Hkv=Hkv, steps=steps)


# With 64 prefixed keys a form of 64 columns shares its SM with no other CTA and is not taken for trees of any size tried.
@STEPS
@pytest.mark.parametrize("columns,n_prefix", [(c, n) for c in (32, 64, 128) for n in (0, 1, 11, 12)] + [(32, 17), (128, 17), (32, 64), (128, 64)])
def test_prefixes(ctx, columns, n_prefix, steps):
    check(ctx, columns, [300, 9, 130], see([20, 9, 16], 3), n_prefix=n_prefix, steps=steps)


def test_a_prefix_beside_which_64_columns_still_share_an_sm(ctx):
    check(ctx, 64, [300, 9, 130], see([20, 9, 16], 3), n_prefix=24)


@COLUMNS
@STEPS
@pytest.mark.parametrize("window,n_sink", [(128, 0), (129, 4), (200, 17), (300, 140), (150, 300)])
def test_windows(ctx, window, n_sink, steps, columns):
    check(ctx, columns, [500, 41, 700, 1530], see([40, 40, 1, 30], 5), window=window, n_sink=n_sink, steps=steps)


@COLUMNS
@STEPS
def test_pages_and_long_items(ctx, steps, columns):
    """Items that workers share, behind caches on every size of page."""
    for page in (16, 32, 64, 128):
        check(ctx, columns, [3300, 100, 129], see([9, 8, 1], 3), steps=steps, page=page, hide=False)
    check(ctx, columns, [6000, 2500], see([33, 20], 3), steps=steps, n_prefix=0, hide=False)


@COLUMNS
@STEPS
def test_masks_of_the_callers_own(ctx, steps, columns):
    rng, new = random.Random(5), [50, 33, 9]
    masks = [[[rng.random() < 0.4 for _ in range(n)] for _ in range(n)] for n in new]
    check(ctx, columns, [300, 40, 9], masks, steps=steps)
    check(ctx, columns, [900, 333, 200], masks, steps=steps, window=130, n_sink=3, hide=False)


@COLUMNS
@STEPS
@pytest.mark.parametrize("n_prefix", [0, 4])
def test_fewer_cached_keys_than_drafts(ctx, n_prefix, steps, columns):
    check(ctx, columns, [3, 0, 40], see([5, 4, 40], 2), n_prefix=n_prefix, steps=steps)


@COLUMNS
@STEPS
def test_scores_of_every_size(ctx, steps, columns):
    """References that move again and again."""
    lengths, new = [900, 300], [24, 24]
    call = Call(columns, lengths, new, 8, 2, steps, 4)
    cache = paged_ref.make_cache(call.lengths, 8, 2, 16, steps=steps, seed=8, step_range=(0.0, 2.0), width=call.width)
    q = paged_ref.queries(48, 8, seed=8, scale=6.0)
    q[3], q[9, 3] = 0.0, 2.0**-133
    q[5] *= 2.0**-100
    q[7, :2] *= 2.0**5
    trees = see(call.new, 4)
    want, tol = ref.attention(cache, q, call.begin, call.lengths, 128**-0.5, trees=trees)
    out = call.run(ctx, cache, q, trees)
    assert ctx.check_status() == 0
    assert torch.all((out.double() - want).abs() <= tol)


@COLUMNS
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 0.0])
def test_a_draft_without_numbers_stays_in_its_branch(ctx, bad, columns):
    lengths, new = [300, 104], [40, 40]
    call = Call(columns, lengths, new, 8, 2, "vector", 4)
    cache, q, trees = call.cache(8, 2, "vector", 4, seed=5), paged_ref.queries(80, 8, seed=5), see(call.new, 3, seed=5)
    want, tol = ref.attention(cache, q, call.begin, call.lengths, 128**-0.5, trees=trees)
    table, spoilt = cache.pages.table.tolist(), ((0, 2), (1, 38))
    for b, u in spoilt:
        c = lengths[b] - 40 + u
        cache.steps[table[b][c // 16], :, :, c % 16] = bad
    out = call.run(ctx, cache, q, trees)
    apart = torch.tensor([not row[u] for b, u in spoilt for row in trees[b]], device="cuda")
    assert 0 < apart.sum() < 80
    assert torch.all((out.double() - want).abs()[apart] <= tol[apart])
    if bad != bad:
        assert torch.all(out[~apart].isnan())
    assert ctx.check_status() == 0


@COLUMNS
@STEPS
@pytest.mark.parametrize("above", [12.3, 24.0, 30.0])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (300, 4), (300, 400)])
def test_a_first_key_that_draws_nearly_all_of_the_weight(ctx, window, n_sink, above, steps, columns):
    lengths, new = [1000, 130, 60], [20, 20, 9]
    call = Call(columns, lengths, new, 8, 2, steps, 3, window, n_sink)
    cache = first_keys.make(call.lengths, 8, 2, steps, 3, above, 0, width=call.width)
    q, trees = first_keys.ones(49, 8), see(call.new, 3)
    want, tol = first_keys.bounds(cache, q, call.begin, call.lengths, above, 0, window, n_sink, trees)
    out = call.run(ctx, cache, q, trees, sm=first_keys.LN2)
    assert ctx.check_status() == 0
    first_keys.assert_within(out, want, tol, 49)


@COLUMNS
@STEPS
def test_repeatable(ctx, steps, columns):
    call = Call(columns, [3000, 800, 100], [9, 20, 1], 8, 2, steps, 4)
    cache, q, trees = call.cache(8, 2, steps, 4, seed=11), paged_ref.queries(30, 8, seed=11), see(call.new, 3)
    first = call.run(ctx, cache, q, trees).clone()
    for _ in range(8):
        assert torch.equal(call.run(ctx, cache, q, trees), first)
    assert ctx.check_status() == 0


@COLUMNS
@STEPS
def test_waits_that_run_out(ctx, steps, columns):
    """Limits of 16384 clocks and more take the usual forms. Queries of a worker's third item, and scores of its second item's prefix, are waited for while an item goes on:
    some ten microseconds and more behind long caches, whose items every worker has several of."""
    B, n = 120, {32: 8, 64: 16, 128: 32}[columns]  # 960 items
    call = Call(columns, [2000 + 7 * b for b in range(B)], [n] * B, 32, 8, steps, 4)
    cache, q, trees = call.cache(32, 8, steps, 4, seed=5), paged_ref.queries(B * n, 32, seed=5), see(call.new, 3)
    qb, mask, ws = i32(call.begin), ref.words_of(trees, 4, B * n), ctx.attn_kv4_paged_tree_workspace(cache, B * n, call.max_new)
    out, seen = torch.empty_like(q), []

    def attend(limit):
        ctx.set_wait_limit(limit)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        ctx.attn_kv4_paged_tree(cache, q, qb, call.max_new, mask, 128**-0.5, ws, max_len=call.max_len, out=out)
        b.record()
        ctx.set_wait_limit(0)
        status = ctx.check_status()
        assert a.elapsed_time(b) < 110.0  # a tenth of the default bound
        return status

    assert attend(0) == 0
    good = out.clone()
    for limit in (16384, 17000, 20000, 25000, 30000, 40000, 60000, 100000, 200000):
        for _ in range(3):
            seen.append(attend(limit))
            assert seen[-1] in (0, PQ_ERR_TIMEOUT)
            assert seen[-1] == PQ_ERR_TIMEOUT or torch.equal(out, good)
            assert attend(0) == 0 and torch.equal(out, good)
    assert PQ_ERR_TIMEOUT in seen, "no limit ran out"
