"""Windowed attention beside a first key that draws nearly all of the weight: the other keys' weights keep their bits, judged by the row itself."""
import pytest
import torch

import masked_ref as ref
import paged_ref
from paper_2410_05265_b200 import binding

import first_keys
from test_gpu_paged_tree import begins, i32

pytestmark = pytest.mark.gpu
ABOVE = [3.0, 12.3, 18.4, 21.7, 24.0, 26.0, 30.0]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def attend(ctx, cache, begin, new, window, n_sink, max_len=0):
    q = first_keys.ones(begin[-1], cache.Hq)
    ws = ctx.attn_kv4_paged_workspace(cache, begin[-1], max(new))
    out = ctx.attn_kv4_paged_window(cache, q, i32(begin), max(new), window, first_keys.LN2, ws, n_sink=n_sink, max_len=max_len)
    assert ctx.check_status() == 0
    return q, out


# lengths, rows, window, n_sink, heads: keys that stay visible behind and inside the window, windows that still reach the cache's first key
@pytest.mark.parametrize("n_prefix", [0, 3])
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", ABOVE)
@pytest.mark.parametrize("lengths,new,window,n_sink,Hq,Hkv", [
    ([1000], [200], 300, 4, 8, 2), ([2500, 130], [40, 130], 700, 4, 8, 1), ([700], [300], 650, 0, 8, 2), ([100, 257], [100, 20], 240, 0, 4, 1),
    ([1300], [300], 200, 140, 6, 2), ([600], [600], 5000, 4, 8, 2), ([300 + 20 * b for b in range(12)], [60] * 12, 150, 300, 8, 2)])
def test_prompts_and_chunks(ctx, lengths, new, window, n_sink, Hq, Hkv, above, steps, n_prefix):
    where = 3 if n_sink else 0
    cache = first_keys.make(lengths, Hq, Hkv, steps, n_prefix, above, where, width=400)  # (6400 tokens: no window of these is the plain call)
    begin = begins(new)
    q, out = attend(ctx, cache, begin, new, window, n_sink)
    want, tol = first_keys.bounds(cache, q, begin, lengths, above, where, window, n_sink, near_prefix=True)
    first_keys.assert_within(out, want, tol, begin[-1])


# one token to a sequence: one cluster, clusters of sixteen, equal stretches; first keys in one block and in several, windows that reach into their group and past them
@pytest.mark.parametrize("n_prefix", [0, 3])
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", ABOVE)
@pytest.mark.parametrize("lengths,window,n_sink,Hq,Hkv,max_len", [
    ([1000], 300, 4, 8, 2, 0), ([6000], 5000, 4, 8, 1, 6000), ([9000, 40, 700], 1000, 20, 16, 2, 9000), ([300 + 70 * b for b in range(50)], 900, 4, 8, 4, 0),
    ([20, 35, 50, 64, 65, 33], 30, 5, 6, 2, 0), ([2500] * 30, 600, 200, 8, 8, 2500)])
def test_single_tokens(ctx, lengths, window, n_sink, Hq, Hkv, max_len, above, steps, n_prefix):
    cache = first_keys.make(lengths, Hq, Hkv, steps, n_prefix, above, 3, width=600)
    begin, new = list(range(len(lengths) + 1)), [1] * len(lengths)
    q, out = attend(ctx, cache, begin, new, window, n_sink, max_len)
    want, tol = first_keys.bounds(cache, q, begin, lengths, above, 3, window, n_sink, near_keys=n_sink, code8=True)
    first_keys.assert_within(out, want, tol, begin[-1])


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_windows_and_first_keys_of_every_alignment(ctx, steps):
    """Every length from one token on under windows and first keys that end inside groups and blocks; ordinary scores."""
    lengths = list(range(1, 150))
    for window, n_sink in ((7, 1), (16, 16), (33, 15), (50, 33), (64, 70), (100, 3)):
        cache = paged_ref.make_cache(lengths, 4, 2, 16, steps=steps, seed=window)
        begin, q = list(range(150)), paged_ref.queries(149, 4, seed=n_sink)
        want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, window, n_sink)
        ref.hide_unseen_pages(cache, begin, lengths, window, n_sink)
        ws = ctx.attn_kv4_paged_workspace(cache, 149, 1)
        out = ctx.attn_kv4_paged_window(cache, q, i32(begin), 1, window, 128**-0.5, ws, n_sink=n_sink)
        assert ctx.check_status() == 0
        assert torch.all((out.double() - want).abs() <= tol)
