"""Windowed attention beside a first key that draws nearly all of the weight: the other keys' weights keep their bits, judged by the row itself."""
import pytest
import torch

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

