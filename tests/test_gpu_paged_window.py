"""Attention of the paged KV4 cache through a sliding window with first keys that stay visible, against its definition in 64 bits."""
import random

import pytest
import torch

import masked_ref as ref
import paged_ref
from paper_2410_05265_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def begins(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def call(ctx, cache, q, begin, new, window, n_sink, max_len=0, out=None):
    N = q.shape[0]
    ws = ctx.attn_kv4_paged_workspace(cache, N, max(new))
    return ctx.attn_kv4_paged_window(cache, q, torch.tensor(begin, dtype=torch.int32, device="cuda"), max(new), window, 128**-0.5, ws, n_sink=n_sink,
                                     max_len=max_len, out=out)


def check(ctx, lengths, new, window, n_sink, Hq=8, Hkv=2, page=16, steps="head", n_prefix=4, pad=2, seed=0, hide=True, max_len=0):
    cache = paged_ref.make_cache(lengths, Hq, Hkv, page, steps=steps, n_prefix=n_prefix, seed=seed)
    begin = begins(new)
    q = paged_ref.queries(begin[-1] + pad, Hq, seed=seed)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, window, n_sink)
    if hide:
        ref.hide_unseen_pages(cache, begin, lengths, window, n_sink)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    call(ctx, cache, q, begin, new, window, n_sink, max_len=max_len, out=out)
    assert ctx.check_status() == 0
    live = begin[-1]
    assert torch.all(out[live:] == 7.0)
    err = (out[:live].double() - want[:live]).abs()
    assert torch.all(err <= tol[:live]), (err - tol[:live]).max()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (2, 1), (15, 0), (16, 4), (17, 16), (31, 17), (100, 0), (128, 4), (129, 33), (257, 130), (1000, 0)])
def test_single_tokens(ctx, window, n_sink, steps):
    check(ctx, [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 300, 513, 700], [1] * 13, window, n_sink, steps=steps)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (5, 3), (64, 0), (127, 4), (128, 0), (129, 130), (200, 17), (300, 300)])
def test_prompts_chunks_and_single_tokens(ctx, window, n_sink, steps):
    """Prompts, chunks behind cached keys and single tokens in one ragged batch; a sequence without rows among them."""
    check(ctx, [150, 3, 400, 64, 333, 700], [150, 2, 1, 0, 70, 300], window, n_sink, steps=steps)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (10, 2), (7, 1), (16, 2)])
@pytest.mark.parametrize("n_prefix", [0, 4, 17])
def test_head_ratios_and_prefixes(ctx, Hq, Hkv, n_prefix):
    check(ctx, [260, 390], [200, 1], 70, 5, Hq=Hq, Hkv=Hkv, n_prefix=n_prefix, page=32)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("steps", ["head", "vector"])
def test_pages(ctx, page, steps):
    check(ctx, [1000, 900, 513], [1, 130, 2], 200, 20, page=page, steps=steps)


@pytest.mark.parametrize("max_len", [0, 9000])
def test_long_single_tokens_in_stretches_and_in_clusters(ctx, max_len):
    check(ctx, [9000, 40, 8999], [1, 1, 1], 4000, 4, max_len=max_len, hide=False)
    check(ctx, [9000], [1], 8000, 100, max_len=max_len, hide=False, steps="vector")
    check(ctx, [3000 + 17 * i for i in range(40)], [1] * 40, 1500, 0, Hq=8, Hkv=8, max_len=max_len, hide=False)


def test_a_long_chunk(ctx):
    """An item's window begins in a later key tile than its sequence's; several workers share items."""
    check(ctx, [5000], [300], 1500, 4, hide=False)
    check(ctx, [2100, 1500], [600, 500], 700, 0, Hq=2, Hkv=2, steps="vector", page=64, hide=False)


def test_no_prefix_and_fewer_cached_keys_than_rows(ctx):
    """Rows at places before the first cached key see nothing; their outputs are zeros. Both this and plain attention report nothing of it."""
    lengths, new = [3, 40], [5, 40]
    cache = paged_ref.make_cache(lengths, 4, 2, 16, n_prefix=0, seed=3)
    begin = begins(new)
    q = paged_ref.queries(begin[-1], 4, seed=3)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, 2, 0)
    out = call(ctx, cache, q, begin, new, 2, 0)
    assert ctx.check_status() == 0
    assert torch.all(out[:2] == 0) and torch.all((out.double() - want).abs() <= tol)


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_a_window_of_the_capacity_is_the_plain_call_bit_for_bit(ctx, steps):
    lengths, new = [700, 300, 5], [1, 130, 5]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps=steps, seed=5)
    begin = begins(new)
    q = paged_ref.queries(begin[-1], 8, seed=5)
    ws = ctx.attn_kv4_paged_workspace(cache, q.shape[0], max(new))
    plain = ctx.attn_kv4_paged(cache, q, torch.tensor(begin, dtype=torch.int32, device="cuda"), max(new), 128**-0.5, ws)
    for window in (cache.pages.max_pages * 16, 2**31 - 1):
        assert torch.equal(plain, call(ctx, cache, q, begin, new, window, 2**31 - 1))
    # a window that merely covers the lengths takes the other kernels: the same to the tolerance of both
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5)
    assert torch.all((call(ctx, cache, q, begin, new, 701, 0).double() - want).abs() <= tol)
    assert ctx.check_status() == 0


def test_a_prefixed_key_that_outweighs_the_cached_ones(ctx):
    """Its value is zero, so that the output is what the others weigh: they keep their bits, in whichever tile a row's window begins."""
    for steps in ("head", "vector"):
        lengths, new = [900, 500], [300, 1]
        cache = paged_ref.make_cache(lengths, 4, 1, 16, steps=steps, n_prefix=1, seed=7)
        begin = begins(new)
        q = paged_ref.queries(begin[-1], 4, seed=7)
        q[..., 0] = 8.0
        cache.prefix_k.zero_()
        cache.prefix_k[..., 0] = 28.0  # 8 x 28 / 11.3 = 19.8: 28 octaves
        cache.prefix_v.zero_()
        want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, 200, 0)
        # the bound relative to the row itself: weights keep 2^-11 of their own
        out = call(ctx, cache, q, begin, new, 200, 0)
        scale = want.abs().amax(-1, keepdim=True)
        off = 2 * (2.0**-11 + 2.0**-14) * 40 + 2.0**-7  # weights' errors against sums in which values cancel to a fortieth, and the rounding
        assert torch.all((out.double() - want).abs() <= off * scale)
    assert ctx.check_status() == 0


def test_rows_strides_and_output_over_the_queries(ctx):
    lengths, new = [500, 300], [1, 40]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, seed=9)
    begin = begins(new)
    wide = paged_ref.queries(begin[-1], 12, seed=9)
    q = wide[:, :8]
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, 90, 3)
    assert torch.all((call(ctx, cache, q, begin, new, 90, 3).double() - want).abs() <= tol)
    dense = q.contiguous()
    call(ctx, cache, dense, begin, new, 90, 3, out=dense)
    assert torch.all((dense.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


def test_repeatable_and_captured(ctx):
    """Every run gives the same bits, also replayed with other inputs and lengths in the same buffers."""
    rng = random.Random(3)
    lengths, new = [3000, 800, 100], [1, 200, 1]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps="vector", seed=11)
    begin = begins(new)
    q = paged_ref.queries(begin[-1], 8, seed=11)
    qb = torch.tensor(begin, dtype=torch.int32, device="cuda")
    ws, out = ctx.attn_kv4_paged_workspace(cache, q.shape[0], 200), torch.zeros_like(q)
    run = lambda: ctx.attn_kv4_paged_window(cache, q, qb, 200, 500, 128**-0.5, ws, n_sink=4, out=out)
    first = run().clone()
    for _ in range(5):
        assert torch.equal(run(), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            run()
    torch.cuda.synchronize()
    for _ in range(3):
        q.copy_(paged_ref.queries(begin[-1], 8, seed=rng.randint(20, 99)))
        now = [rng.randint(1000, 3000), rng.randint(200, 800), rng.randint(1, 100)]
        cache.pages.length.copy_(torch.tensor(now, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want, tol = ref.attention(cache, q, begin, now, 128**-0.5, 500, 4)
        assert torch.all((out.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


def test_an_id_that_is_none_inside_the_window_is_reported(ctx):
    cache = paged_ref.make_cache([300], 8, 2, 16, seed=13)
    q = paged_ref.queries(1, 8)
    cache.pages.table[0, 17] = cache.pages.n_pages
    call(ctx, cache, q, [0, 1], [1], 20, 0)
    assert ctx.check_status() == 2
    call(ctx, cache, q, [0, 1], [1], 12, 0)  # keys 288 .. 299 lie on the page behind it
    assert ctx.check_status() == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 0.0])
def test_a_key_without_numbers_leaves_with_the_window(ctx, bad):
    """Own steps that are no number, of a cached key: rows whose window has left it keep their results, and so do the rows before it."""
    lengths, begin, window = [400], [0, 300], 60
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps="vector", seed=5)
    q = paged_ref.queries(300, 8, seed=5)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, window, 4)
    table, at = cache.pages.table.tolist(), 250
    cache.steps[table[0][at // 16], :, :, at % 16] = bad
    out = call(ctx, cache, q, begin, [300], window, 4)
    place = torch.arange(300, device="cuda") + 100
    sees = (place >= at) & (place < at + window)
    assert torch.all((out.double() - want).abs()[~sees] <= tol[~sees])
    if bad != bad:
        assert torch.all(out[sees].isnan())
    assert ctx.check_status() == 0
