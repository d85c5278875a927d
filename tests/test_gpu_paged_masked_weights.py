"""Windowed attention and attention of drafted trees where one key outweighs the others and where steps lie at the ends of their range: what test_gpu_paged_weights.py asks of
the plain call, through a window and in every form of the trees' kernel. Scores are set exactly: queries and keys have their first dim only, a key's score in log2 units is
minus its step."""
import math

import pytest
import torch

import masked_ref as ref
import paged_ref
import tree_form
from paper_2410_05265_b200 import binding

from test_gpu_paged_tree import begins, i32, see
from test_gpu_paged_weights import cache_of, set_key

pytestmark = pytest.mark.gpu
LN2 = math.log(2.0)


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.check()
    c.close()


class Windowed:
    """Lengths, rows, heads, window, first keys that stay visible."""

    def __init__(self, lengths, new, Hq, Hkv, window, n_sink):
        self.lengths, self.new, self.Hq, self.Hkv, self.window, self.n_sink, self.trees = lengths, new, Hq, Hkv, window, n_sink, None
        self.width = 5000  # 80000 tokens: no window of these is the plain call
        self.begin = begins(new)

    def plan(self, steps, n_prefix):
        pass

    def run(self, ctx, cache, q, sm):
        ws = ctx.attn_kv4_paged_workspace(cache, q.shape[0], max(self.new))
        return ctx.attn_kv4_paged_window(cache, q, i32(self.begin), max(self.new), self.window, sm, ws, n_sink=self.n_sink)


class Tree(Windowed):
    def __init__(self, columns, lengths, new, Hq, Hkv, window=0, n_sink=0):
        super().__init__(lengths, new, Hq, Hkv, window, n_sink)
        self.columns, self.first = columns, (lengths, new)

    def plan(self, steps, n_prefix):
        lengths, new = self.first
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        self.max_new, self.max_len, more = tree_form.call_for(self.columns, steps == "vector", n_prefix, len(lengths), self.Hkv, self.Hq // self.Hkv, max(new), max(lengths),
                                                              self.window, self.n_sink, sms)
        self.lengths, self.new = lengths + [1] * more, new + [0] * more
        self.begin, self.trees = begins(self.new), see(self.new, 3)

    def run(self, ctx, cache, q, sm):
        N = q.shape[0]
        ws = ctx.attn_kv4_paged_tree_workspace(cache, N, self.max_new)
        return ctx.attn_kv4_paged_tree(cache, q, i32(self.begin), self.max_new, ref.words_of(self.trees, 4, N), sm, ws, window=self.window, n_sink=self.n_sink,
                                       max_len=self.max_len)


WINDOWED = [Windowed([1000], [1], 8, 2, 300, 4), Windowed([20000, 700, 9000, 33], [1] * 4, 16, 2, 12000, 0), Windowed([300 + 7 * i for i in range(90)], [1] * 90, 8, 4, 200, 20),
            Windowed([1000], [100], 8, 2, 400, 4), Windowed([3000, 400, 300], [40, 400, 1], 8, 1, 600, 0)]
TREES = [t for c in (32, 64, 128) for t in (Tree(c, [1000, 130], [20, 9], 8, 2), Tree(c, [9000], [12], 6, 2), Tree(c, [1500, 60], [24, 40], 8, 1, 500, 4))]
NAMES = [f"window{i}" for i in range(len(WINDOWED))] + [f"tree{t.columns}-{i % 3}" for i, t in enumerate(TREES)]
CALLS = pytest.mark.parametrize("call", WINDOWED + TREES, ids=NAMES)


def ones(call):
    q = torch.zeros((call.begin[-1], call.Hq, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    return q


def live(call):
    return [(b, n) for b, (n, rows) in enumerate(zip(call.lengths, call.new)) if rows > 0]


def within(ctx, out, want, tol):
    assert ctx.check_status() == 0
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}; worst {float(((out.double() - want).abs() / tol)[bad].max())} of the tolerance"


@pytest.mark.parametrize("n_prefix", [0, 3])
@pytest.mark.parametrize("gap", [-7.0, 0.0, 30.0])
@pytest.mark.parametrize("back", [0, 2, 150])
@CALLS
def test_value_steps_at_both_ends_of_their_range(ctx, call, back, gap, n_prefix):
    """One value of step 2^60, `back` keys before the last (or the first key), among values of step 2^-60 whose scores lie `gap` log2 units above its own: they add nothing to
    the numerator, but the denominator is theirs as much as the one's. Bounds of ref.attention."""
    call.plan("vector", n_prefix)
    cache = cache_of(call.lengths, call.Hq, call.Hkv, "vector", n_prefix, call.width)
    cache.steps[:, :, 1] = 2.0**-60
    cache.steps[:, :, 0] = max(-gap, 2.0**-60)
    if n_prefix:
        cache.prefix_k.zero_(), cache.prefix_k[..., 0].fill_(-6.0)
    for b, n in live(call):
        set_key(cache, b, max(0, n - 1 - back), key_step=max(gap, 2.0**-60), value_step=2.0**60)
    q = ones(call)
    want, tol = ref.attention(cache, q, call.begin, call.lengths, LN2, call.window, call.n_sink, call.trees)
    within(ctx, call.run(ctx, cache, q, LN2), want, tol)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("step", [-60, -45, -20, 60])
@pytest.mark.parametrize("above", [0.0, 15.0])
@CALLS
def test_values_of_any_step_beside_a_prefix_without_values(ctx, call, above, step, steps):
    """The prefixed keys' values are zero, the cached ones' steps at the ends of their range: what comes out is theirs alone, in their own size. Bounds of ref.attention,
    whose largest |v| is a cached one, times the share of the weights that the cached keys have."""
    call.plan(steps, 2)
    cache = cache_of(call.lengths, call.Hq, call.Hkv, steps, 2, call.width)
    if steps == "vector":
        cache.steps[:, :, 0], cache.steps[:, :, 1] = 2.0**-60, 2.0**step
    else:
        cache.codes[:, :, 0] = 0
        cache.s_v.fill_(2.0**step)
    cache.prefix_k.zero_(), cache.prefix_v.zero_()
    cache.prefix_k[:, :, 0] = above
    q = ones(call)
    want, tol = ref.attention(cache, q, call.begin, call.lengths, LN2, call.window, call.n_sink, call.trees)
    for b, n_keys in live(call):
        for t in range(call.new[b]):
            r = call.begin[b] + t
            seen = int(ref.visible(n_keys, call.new[b], t, call.window, call.n_sink, call.trees[b] if call.trees else None).sum())
            whole = want[r].abs() * 2.0**-8 + 2.0**-125
            tol[r] = whole + (tol[r] - whole) * seen / (seen + 2 * 2.0**above)
    within(ctx, call.run(ctx, cache, q, LN2), want, tol)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("above", [3.0, 12.3, 21.7, 30.0])
@pytest.mark.parametrize("n_prefix", [1, 20])
@CALLS
def test_a_prefixed_key_that_draws_nearly_all_of_the_weight(ctx, call, n_prefix, above, steps):
    """Its value is zero and its score `above` log2 units over all others, which are equal: what comes out is theirs, times 2^-above.

    With p the softmax in 64 bits, a relative error e of the weights moves the quotient by at most e (sum p |v| + |out|): e is 2^-11 for the rounding to fp16 and 2^-20 for the
    exponent. The other prefixed keys share the large one's reference where they are weighed in fp16 (prompts): each is off by 2^-25 of its p at most. Single tokens multiply
    with code + 8 and take 8 sum(p) off, in fp32 sums of equal terms: 17 x 8 x 2^-23 sum(p) of the largest step in all. The store rounds by 2^-8."""
    if isinstance(call, Tree) and call.columns == 64 and n_prefix == 20 and steps == "vector":
        return  # 64 columns are not taken beside a prefix so long
    call.plan(steps, n_prefix)
    cache = cache_of(call.lengths, call.Hq, call.Hkv, steps, n_prefix, call.width)
    if steps == "vector":
        cache.steps[:, :, 0] = 2.0**-60
    else:
        cache.codes[:, :, 0] = 0
    cache.prefix_k.zero_(), cache.prefix_v[:, 0].zero_()
    cache.prefix_k[:, 0, 0] = above
    q, G = ones(call), call.Hq // call.Hkv
    want, _ = ref.attention(cache, q, call.begin, call.lengths, LN2, call.window, call.n_sink, call.trees)
    tol, table, top = torch.zeros_like(want), cache.pages.table.tolist(), 2.0 ** float(cache.prefix_k[0, 0, 0])
    pre = cache.prefix_v.double().abs().sum(1)
    unit = float(cache.steps[:, :, 1].max()) if steps == "vector" else float(cache.s_v.max())
    for b, n_keys in live(call):
        at = torch.tensor([table[b][j // 16] * 16 + j % 16 for j in range(n_keys)], dtype=torch.int64, device="cuda")
        own = cache.steps[at // 16, :, 1, at % 16] if steps == "vector" else cache.s_v[None].expand(n_keys, -1)
        v = paged_ref.unpack(cache.codes[at // 16, :, 1, at % 16]).double().abs() * own.double()[..., None]  # [keys, Hkv, 128]
        for t in range(call.new[b]):
            see_t = ref.visible(n_keys, call.new[b], t, call.window, call.n_sink, call.trees[b] if call.trees else None)
            p = 1.0 / (top + n_prefix - 1 + int(see_t.sum()))  # of each key but the one
            wide = lambda x: x[:, None].expand(-1, G, -1).reshape(call.Hq, 128)
            r = call.begin[b] + t
            a = wide(p * (v[see_t.cuda()].sum(0) + pre))
            tol[r] = wide(2.0**-25 * top * p * pre) + (2.0**-11 + 2.0**-20) * (a + want[r].abs()) + 17 * 8 * 2.0**-23 * int(see_t.sum()) * p * unit + want[r].abs() * 2.0**-8 + 2.0**-125
    within(ctx, call.run(ctx, cache, q, LN2), want, tol)


@pytest.mark.parametrize("steps", ["head", "vector"])
@CALLS
def test_infinities_and_nan_stay_in_their_row_and_head(ctx, call, steps):
    """Queries that are not finite, and steps of keys that no row sees because they lie behind a sequence, leave every other row and head as it is, bit for bit."""
    call.plan(steps, 4)
    cache = paged_ref.make_cache(call.lengths, call.Hq, call.Hkv, 16, steps, seed=3, width=call.width)
    N, sm = call.begin[-1], 128**-0.5
    q = paged_ref.queries(N, call.Hq)
    want = call.run(ctx, cache, q, sm)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for r, h, value in ((0, 1, math.nan), (N - 1, call.Hq - 1, math.inf), (N // 2, 0, -math.inf), (N // 2, 2, math.nan)):
        q[r, h, (r + h) % 128] = value
        bad[r, h] = True
    if steps == "vector":
        for b, n in live(call):
            if n % 16:
                cache.steps[cache.pages.table[b, n // 16].long(), :, :, n % 16:] = math.nan
    out = call.run(ctx, cache, q, sm)
    assert ctx.check_status() == 0
    assert torch.equal(out[~bad], want[~bad])
    assert out[bad].isnan().any(-1).all()
