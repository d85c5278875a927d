"""Attention over the paged cache where one key outweighs the others: value steps at the two ends of their range in one sequence. Scores are set exactly: queries
and keys have their first dim only, a key's score in log2 units is minus its step."""
import math

import pytest
import torch

from paper_2410_05265_b200 import binding

import paged_ref as ref
from test_gpu_paged import i32

pytestmark = pytest.mark.gpu
D, DEV = 128, "cuda"
LN2 = math.log(2.0)


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.check()
    c.close()


def cache_of(lengths, Hq, Hkv, steps, n_prefix, width=None):
    """Key codes -1 in dim 0 and 0 elsewhere, random value codes."""
    c = ref.make_cache(lengths, Hq, Hkv, 16, steps, n_prefix, seed=len(lengths) + Hq, width=width)
    c.codes[:, :, 0] = 0
    c.codes[:, :, 0, :, 0] = 0x0F
    return c


def set_key(cache, b, j, key_step=None, value_step=None, key_code=None, value_codes=None):
    page, k = cache.pages.table[b, j // 16].long(), j % 16
    if key_step is not None:
        cache.steps[page, :, 0, k] = key_step
    if value_step is not None:
        cache.steps[page, :, 1, k] = value_step
    if key_code is not None:
        cache.codes[page, :, 0, k, 0] = key_code
    if value_codes is not None:
        cache.codes[page, :, 1, k] = value_codes


def attend(ctx, cache, new, max_len=0):
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    q = torch.zeros((begin[-1], cache.Hq, D), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    ws = ctx.attn_kv4_paged_workspace(cache, begin[-1], max(new))
    out = ctx.attn_kv4_paged(cache, q, i32(begin), max(new), LN2, ws, max_len=max_len)
    ctx.check()
    return q, begin, out


SHAPES = [([1000], [1], 8, 2), ([40000, 700, 9000, 33], [1] * 4, 16, 2), ([300 + 7 * i for i in range(90)], [1] * 90, 8, 4), ([1000], [100], 8, 2),
          ([9000, 400, 300], [40, 400, 1], 8, 1), ([20000], [3], 6, 2)]


@pytest.mark.parametrize("n_prefix", [0, 3])
@pytest.mark.parametrize("gap", [-7.0, 0.0, 30.0])
@pytest.mark.parametrize("where", [0.0, 0.4, 1.0])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", SHAPES)
def test_value_steps_at_both_ends_of_their_range(ctx, lengths, new, Hq, Hkv, where, gap, n_prefix):
    """One value of step 2^60 among values of step 2^-60 whose scores lie `gap` log2 units above its own: they add nothing to the numerator, but the denominator is
    theirs as much as the one's. Bounds of ref.attention."""
    cache = cache_of(lengths, Hq, Hkv, "vector", n_prefix)
    cache.steps[:, :, 1] = 2.0**-60
    cache.steps[:, :, 0] = max(-gap, 2.0**-60)
    if n_prefix:
        cache.prefix_k.zero_(), cache.prefix_k[..., 0].fill_(-6.0)
    for b, n in enumerate(lengths):
        set_key(cache, b, int(where * (n - 1)), key_step=max(gap, 2.0**-60), value_step=2.0**60)
    q, begin, out = attend(ctx, cache, new)
    want, tol = ref.attention(cache, q, begin, lengths, LN2)
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}"
