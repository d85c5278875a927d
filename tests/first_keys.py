"""A first cached key that draws nearly all of the weight and whose value is zero, over a cache whose other scores are zero: what comes out is the other keys' mean, times their
small share. Shared by the tests of windowed attention and of drafted trees."""
import math

import torch

import masked_ref as ref
import paged_ref
from test_gpu_paged_weights import cache_of, set_key

LN2 = math.log(2.0)


def make(lengths, Hq, Hkv, steps, n_prefix, above, where, n=1, width=None):
    """Scores of zero in log2 units; key `where` of every sequence, and the n - 1 behind it, `above` of them (7 s_k, or 7 steps), with value codes of zero."""
    cache = cache_of(lengths, Hq, Hkv, steps, n_prefix, width)
    if steps == "vector":
        cache.steps[:, :, 0] = 2.0**-60
    else:
        cache.codes[:, :, 0] = 0
        cache.s_k.fill_(above / 7)
    if n_prefix:
        cache.prefix_k.zero_()
    for b in range(len(lengths)):
        for j in range(where, min(where + n, lengths[b])):
            set_key(cache, b, j, key_step=above / 7 if steps == "vector" else None, key_code=7, value_codes=0)
    return cache


def ones(rows, Hq):
    q = torch.zeros((rows, Hq, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    return q


def bounds(cache, q, begin, lengths, above, where, window=0, n_sink=0, trees=None, n=1, near_keys=128, near=2.0**-38, near_prefix=False, code8=False):
    """(outputs in 64 bits, tolerance).

    A relative error e of the weights moves the quotient by at most e (sum p |v| + |out|), p the softmax in 64 bits: e is 2^-11 for a weight's rounding to fp16 and 2^-17 for
    its exponent (a score of at most 32 is a product of three factors rounded to fp32 and a difference: 4 x 2^-24 x 32 ln 2, and 2^-22 of 2^x). The keys that share the
    heavy key's tile, the first `near_keys` ones, may be rounded against its reference instead, in multiples of 2^-24: each off by 2^-25 of it, `near` of the heavy key's
    weight where the reference lies 13 octaves below that (times its value's step, which the exponents carry); with `near_prefix` so may the prefixed ones.
    With `code8` (single tokens) the keys but the heavy ones are multiplied as code + 8 and 8 sum(p) is taken off, in fp32 sums of equal terms: each of the 16 products of a
    step and the sum so far is off by 2^-23 of 8 p per key. The store rounds by 2^-8."""
    want, _ = ref.attention(cache, q, begin, lengths, LN2, window, n_sink, trees)
    tol, pages, G = torch.zeros_like(want), cache.pages, cache.Hq // cache.Hkv
    table = pages.table.tolist()
    for b, n_keys in enumerate(lengths):
        rows = begin[b + 1] - begin[b]
        c = torch.arange(n_keys)
        at = torch.tensor([table[b][j // pages.page] * pages.page + j % pages.page for j in range(n_keys)], dtype=torch.int64, device=want.device)
        page, inside = at // pages.page, at % pages.page
        codes = paged_ref.unpack(cache.codes[page, :, 1, inside]).double().abs()  # [keys, Hkv, 128]
        unit = (cache.steps[page, :, 1, inside] if cache.steps is not None else cache.s_v[None].expand(n_keys, -1)).double()[..., None]
        pre = cache.prefix_v.double().abs().sum(1) if cache.n_prefix else 0.0
        heavy = (c >= where) & (c < where + n)
        for t in range(rows):
            see = ref.visible(n_keys, rows, t, window, n_sink, trees[b] if trees else None)
            others, top = int((see & ~heavy).sum()) + cache.n_prefix, int((see & heavy).sum())
            if others + top == 0:
                continue
            p = 1.0 / (top * 2.0**above + others)  # of each key but the heavy ones
            seen = see.to(want.device)
            a = p * ((codes * unit)[seen].sum(0) + pre)
            here = torch.zeros_like(a)
            if top:
                step = unit[(see & heavy).to(want.device)].amax(0)
                here = near * 2.0**above * p * step * (codes[seen & (torch.arange(n_keys, device=want.device) < near_keys)].sum(0) + (pre if near_prefix else 0.0))
            wide = lambda x: x[:, None].expand(-1, G, -1).reshape(cache.Hq, 128)
            r = begin[b] + t
            if code8:
                here = here + 17 * 8 * 2.0**-23 * others * p * unit.max()
            tol[r] = (2.0**-11 + 2.0**-17) * (wide(a) + want[r].abs()) + wide(here) + want[r].abs() * 2.0**-8 + 2.0**-125
    return want, tol


def assert_within(out, want, tol, rows):
    err = (out[:rows].double() - want[:rows]).abs()
    bad = ~(err <= tol[:rows])
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}; worst {float((err / tol[:rows])[bad].max())} of the tolerance"
