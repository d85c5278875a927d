"""Attention over the paged cache where one key outweighs the others: value steps at the two ends of their range in one sequence, and a key that draws
nearly all of the weight and whose value is small (what the prefixed tokens are). Scores are set exactly: queries and keys have their first dim only, a
key's score in log2 units is minus its step."""
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


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", [3.0, 12.3, 18.4, 21.7, 23.4, 30.0])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [([1000], [1], 8, 2), ([9000, 700], [1, 1], 16, 2), ([700], [300], 8, 2), ([9000, 200, 40], [40, 200, 1], 8, 1),
                                                ([130, 2, 129], [130, 2, 129], 4, 4)])
@pytest.mark.parametrize("n_prefix", [1, 20])
def test_a_prefixed_key_that_draws_nearly_all_of_the_weight(ctx, lengths, new, Hq, Hkv, n_prefix, above, steps):
    """Its value is zero and its score `above` log2 units over all others, which are equal: what comes out is theirs, times 2^-above.

    With p the softmax in 64 bits, a relative error e of the weights moves the quotient by at most e (sum p |v| + |out|): e is 2^-11 for the rounding to fp16, where the
    cached keys' weights are normal numbers, and 2^-20 for the exponent. The other prefixed keys share the large one's reference, of whose weight theirs are rounded to
    multiples of 2^-24 (it is 1 at most): each is off by 2^-25 of its p at most. The single-token kernel multiplies with code + 8 and takes 8 sum(p) off, in fp32 sums
    of equal terms: each of the 16 products of a step and the sum so far is off by 2^-23 of 8 p per key, 17 x 8 x 2^-23 sum(p) of the largest step in all.
    The store rounds by 2^-8."""
    cache = cache_of(lengths, Hq, Hkv, steps, n_prefix)
    if steps == "vector":
        cache.steps[:, :, 0] = 2.0**-60
    else:
        cache.codes[:, :, 0] = 0
    cache.prefix_k.zero_(), cache.prefix_v[:, 0].zero_()
    cache.prefix_k[:, 0, 0] = above
    q, begin, out = attend(ctx, cache, new)
    want, _ = ref.attention(cache, q, begin, lengths, LN2)
    tol = torch.zeros_like(want)
    for b, n_keys in enumerate(lengths):
        ids = cache.pages.table[b, : ref.up(n_keys, 16)].long()
        step = cache.steps[ids].double()[..., None] if steps == "vector" else torch.stack((cache.s_k, cache.s_v), 1).double()[None, :, :, None, None]
        v = (ref.unpack(cache.codes[ids]).double() * step)[:, :, 1].permute(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n_keys]
        v = torch.cat((cache.prefix_v.double(), v), 1).abs()
        unit = cache.steps[:, :, 1].max().double() if steps == "vector" else cache.s_v.max().double()
        for t in range(new[b]):
            seen = n_keys - new[b] + t + 1
            p = 1.0 / (2.0 ** float(cache.prefix_k[0, 0, 0]) + n_prefix - 1 + seen)  # of each key but the one
            r = begin[b] + t
            a = (p * v[:, : n_prefix + seen].sum(1))[:, None].expand(-1, Hq // Hkv, -1).reshape(Hq, D)
            near = 2.0**-25 * 2.0 ** float(cache.prefix_k[0, 0, 0]) * p * cache.prefix_v.double().abs().sum(1)
            tol[r] = near[:, None].expand(-1, Hq // Hkv, -1).reshape(Hq, D) + (2.0**-11 + 2.0**-20) * (a + want[r].abs()) + 17 * 8 * 2.0**-23 * seen * p * unit + want[r].abs() * 2.0**-8 + 2.0**-125
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}; worst {float(((out.double() - want).abs() / tol).max())} of the tolerance"


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("step", [-60, -45, -20, 60])
@pytest.mark.parametrize("above", [0.0, 15.0])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [([1000], [1], 8, 2), ([700], [300], 8, 2), ([9000, 200, 40], [40, 200, 1], 8, 1)])
def test_values_of_any_step_beside_a_prefix_without_values(ctx, lengths, new, Hq, Hkv, above, step, steps):
    """The prefixed keys' values are zero, the cached ones' steps at the ends of their range: what comes out is theirs alone, in their own size. Bounds of
    ref.attention, whose largest |v| is a cached one, times the share of the weights that the cached keys have."""
    cache = cache_of(lengths, Hq, Hkv, steps, 2)
    if steps == "vector":
        cache.steps[:, :, 0], cache.steps[:, :, 1] = 2.0**-60, 2.0**step
    else:
        cache.codes[:, :, 0] = 0
        cache.s_v.fill_(2.0**step)
    cache.prefix_k.zero_(), cache.prefix_v.zero_()
    cache.prefix_k[:, :, 0] = above
    q, begin, out = attend(ctx, cache, new)
    want, tol = ref.attention(cache, q, begin, lengths, LN2)
    for b, n_keys in enumerate(lengths):
        for t in range(new[b]):
            r, seen = begin[b] + t, n_keys - new[b] + t + 1
            share = seen / (seen + 2 * 2.0**above)
            whole = want[r].abs() * 2.0**-8 + 2.0**-125
            tol[r] = whole + (tol[r] - whole) * share
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}; worst {float(((out.double() - want).abs() / tol).max())} of the tolerance"


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [([1000, 40], [1, 1], 8, 2), ([700 + 13 * i for i in range(90)], [1] * 90, 8, 4), ([700, 300, 64], [300, 1, 64], 6, 2)])
def test_infinities_and_nan_stay_in_their_row_and_head(ctx, lengths, new, Hq, Hkv, steps):
    """Queries that are not finite, and steps and prefix keys that no row sees because they lie behind a sequence, leave every other row and head as it is, bit for bit."""
    cache = ref.make_cache(lengths, Hq, Hkv, 16, steps, seed=3)
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    q = ref.queries(begin[-1], Hq)
    ws = ctx.attn_kv4_paged_workspace(cache, begin[-1], max(new))
    want = ctx.attn_kv4_paged(cache, q, i32(begin), max(new), 1 / math.sqrt(D), ws)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    for r, h, value in ((0, 1, math.nan), (begin[-1] - 1, Hq - 1, math.inf), (begin[-1] // 2, 0, -math.inf), (begin[-1] // 2, 2, math.nan)):
        q[r, h, (r + h) % D] = value
        bad[r, h] = True
    if steps == "vector":
        for b, n in enumerate(lengths):
            if n % 16:
                cache.steps[cache.pages.table[b, n // 16].long(), :, :, n % 16:] = math.nan
    out = ctx.attn_kv4_paged(cache, q, i32(begin), max(new), 1 / math.sqrt(D), ws)
    ctx.check()
    assert torch.equal(out[~bad], want[~bad])
    assert out[bad].isnan().any(-1).all()
