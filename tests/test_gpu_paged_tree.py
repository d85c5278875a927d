"""Drafted trees over the paged KV4 cache: plan, attention, acceptance, pages and moves, against their definitions."""
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


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def begins(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def trees_of(new, width, seed, roots=1):
    rng = random.Random(seed)
    return [ref.random_tree(rng, n, width, roots) for n in new]


def call(ctx, cache, q, begin, max_new, mask, window=0, n_sink=0, max_len=0, out=None):
    ws = ctx.attn_kv4_paged_tree_workspace(cache, q.shape[0], max_new)
    return ctx.attn_kv4_paged_tree(cache, q, i32(begin), max_new, mask, 128**-0.5, ws, window=window, n_sink=n_sink, max_len=max_len, out=out)


def check(ctx, lengths, trees, Hq=8, Hkv=2, page=16, steps="head", n_prefix=4, pad=2, seed=0, window=0, n_sink=0, words=None, hide=True, max_len=0, sm=128**-0.5):
    """trees: what the rows of every sequence see of one another."""
    new = [len(s) for s in trees]
    cache = paged_ref.make_cache(lengths, Hq, Hkv, page, steps=steps, n_prefix=n_prefix, seed=seed)
    begin = begins(new)
    q = paged_ref.queries(begin[-1] + pad, Hq, seed=seed)
    mask = ref.words_of(trees, words or paged_ref.up(max(new), 32), begin[-1] + pad)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, window, n_sink, trees)
    if hide:
        ref.hide_unseen_pages(cache, begin, lengths, window, n_sink, trees)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    call(ctx, cache, q, begin, max(new), mask, window, n_sink, max_len, out)
    assert ctx.check_status() == 0
    live = begin[-1]
    assert torch.all(out[live:] == 7.0)
    err = (out[:live].double() - want[:live]).abs()
    assert torch.all(err <= tol[:live]), (err - tol[:live]).max()


def see(new, width, seed=0, roots=1):
    return [ref.ancestors(p) for p in trees_of(new, width, seed, roots)]


# ---- attention -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("new,lengths", [([2], [2]), ([3], [130]), ([7, 1, 5], [500, 300, 5]), ([16], [1000]), ([33, 64], [129, 700]), ([128], [128]), ([127, 128, 65], [200, 384, 1030]),
                                         ([1, 1], [40, 300])])
@pytest.mark.parametrize("width", [1, 4, 200])
def test_trees(ctx, new, lengths, width, steps):
    check(ctx, lengths, see(new, width), steps=steps)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 2), (3, 1), (5, 1), (12, 2), (7, 1), (16, 2)])
@pytest.mark.parametrize("n", [2, 17, 40, 100])
def test_head_ratios(ctx, Hq, Hkv, n):
    check(ctx, [n + 150, n], see([n, n], 5), Hq=Hq, Hkv=Hkv)


@pytest.mark.parametrize("n_prefix", [0, 1, 16, 17, 64])
@pytest.mark.parametrize("steps", ["head", "vector"])
def test_prefixes(ctx, n_prefix, steps):
    check(ctx, [300, 9], see([20, 9], 3), n_prefix=n_prefix, steps=steps)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages_that_end_inside_a_tile_and_inside_the_tree(ctx, page):
    check(ctx, [120 + 37, 250], see([37, 9], 4), page=page)
    check(ctx, [page, page + 1, 3 * page - 1], see([10, 10, 10], 4), page=page, steps="vector")


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("window,n_sink", [(40, 0), (64, 4), (129, 17), (300, 140)])
def test_windows(ctx, window, n_sink, steps):
    check(ctx, [500, 41, 700, 330], see([40, 40, 1, 5], 5), window=window, n_sink=n_sink, steps=steps)
    check(ctx, [1500], see([30], 1), window=window, n_sink=n_sink, steps=steps, page=64)


def test_forests_and_masks_of_the_callers_own(ctx):
    """Several roots; rows that see rows behind them; rows whose mask is empty see themselves; bits past the rows say nothing."""
    check(ctx, [200, 140], see([20, 12], 3, roots=6))
    rng = random.Random(5)
    any_mask = [[[rng.random() < 0.4 for _ in range(n)] for _ in range(n)] for n in (50, 9)]
    check(ctx, [300, 9], any_mask, words=4)
    check(ctx, [300, 9], any_mask, n_prefix=0, steps="vector")
    new, lengths = [9, 3], [100, 3]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, n_prefix=0)
    begin, q = begins(new), paged_ref.queries(12, 8)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=[[[False] * n for _ in range(n)] for n in new])
    for bits in ([0], [-1 << 9]):  # (the second sequence's rows have three bits: bits 9 on are past them, too)
        out = call(ctx, cache, q, begin, 9, i32([bits] * 12))
        assert torch.all((out.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


def test_a_chain_is_causal_attention(ctx):
    lengths, new = [777, 64, 300], [31, 64, 2]
    for steps in ("head", "vector"):
        cache = paged_ref.make_cache(lengths, 8, 2, 16, steps=steps, seed=4)
        begin, q = begins(new), paged_ref.queries(97, 8, seed=4)
        want, tol = paged_ref.attention(cache, q, begin, lengths, 128**-0.5)
        out = call(ctx, cache, q, begin, 64, ref.words_of(see(new, 1), 2, 97))
        assert torch.all((out.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_long_caches_that_workers_share(ctx, steps):
    check(ctx, [6000], see([9], 3), steps=steps, hide=False)
    check(ctx, [3000, 100, 2500], see([33, 8, 1], 3), steps=steps, Hq=16, Hkv=4, hide=False, max_len=3000)


def test_many_sequences(ctx):
    new = [1 + (7 * b) % 9 for b in range(90)]
    check(ctx, [n + (53 * b) % 400 for b, n in enumerate(new)], see(new, 3), hide=False)


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_scores_of_every_size(ctx, steps):
    """Large scores (the reference moves again and again, tile by tile), queries of zeros, of the smallest and of large numbers."""
    lengths, new = [900, 300], [24, 24]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps=steps, seed=8, step_range=(0.0, 2.0))
    begin, q = begins(new), paged_ref.queries(48, 8, seed=8, scale=6.0)
    q[3] = 0.0
    q[5] *= 2.0**-100
    q[7, :2] *= 2.0**5
    q[9, 3] = 2.0**-133
    trees = see(new, 4)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    out = call(ctx, cache, q, begin, 24, ref.words_of(trees, 1, 48))
    assert ctx.check_status() == 0
    assert torch.all((out.double() - want).abs() <= tol)


def test_a_prefixed_key_that_outweighs_the_cached_ones(ctx):
    """Its value is zero: the output is what the other weights keep of their bits."""
    for steps in ("head", "vector"):
        lengths, new = [700, 20], [20, 20]
        cache = paged_ref.make_cache(lengths, 4, 1, 16, steps=steps, n_prefix=1, seed=7)
        begin, q = begins(new), paged_ref.queries(40, 4, seed=7)
        q[..., 0] = 8.0
        cache.prefix_k.zero_()
        cache.prefix_k[..., 0] = 28.0  # 28 octaves above the others
        cache.prefix_v.zero_()
        trees = see(new, 3)
        want, _ = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
        out = call(ctx, cache, q, begin, 20, ref.words_of(trees, 1, 40))
        scale = want.abs().amax(-1, keepdim=True)
        assert torch.all((out.double() - want).abs() <= (2 * (2.0**-11 + 2.0**-14) * 40 + 2.0**-7) * scale)
    assert ctx.check_status() == 0


def test_queries_that_are_not_finite_stay_in_their_row_and_head(ctx):
    lengths, new = [400, 300], [20, 6]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, seed=2)
    begin, q = begins(new), paged_ref.queries(26, 8, seed=2)
    trees = see(new, 3)
    mask = ref.words_of(trees, 1, 26)
    clean = call(ctx, cache, q, begin, 20, mask)
    q[4, 2], q[21, 7, 5] = float("nan"), float("inf")
    out = call(ctx, cache, q, begin, 20, mask)
    same = torch.ones((26, 8), dtype=torch.bool, device="cuda")
    same[4, 2] = same[21, 7] = False
    assert torch.equal(out[same], clean[same])
    assert ctx.check_status() == 0


def test_sequences_that_do_not_fit_are_left_out_and_reported(ctx):
    lengths, new = [100, 100, 100], [5, 40, 6]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, seed=6)
    begin, q = begins(new), paged_ref.queries(51, 8, seed=6)
    trees = see(new, 3)
    mask = ref.words_of(trees, 2, 51)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
    ws = ctx.attn_kv4_paged_tree_workspace(cache, 51, 39)
    ctx.attn_kv4_paged_tree(cache, q, i32(begin), 39, mask, 128**-0.5, ws, out=out)  # the second has more rows than max_new says
    assert ctx.check_status() == 2
    assert torch.all(out[5:45] == 3.0)
    for lo, hi in ((0, 5), (45, 51)):
        assert torch.all((out[lo:hi].double() - want[lo:hi]).abs() <= tol[lo:hi])
    cache.pages.table[0, 2] = -1
    call(ctx, cache, q, begin, 40, mask)
    assert ctx.check_status() == 2


def test_repeatable_captured_and_on_another_stream(ctx):
    rng = random.Random(3)
    lengths, new = [3000, 800, 100], [9, 20, 1]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps="vector", seed=11)
    begin, q = begins(new), paged_ref.queries(30, 8, seed=11)
    qb, mask = i32(begin), ref.words_of(see(new, 3), 1, 30)
    ws, out = ctx.attn_kv4_paged_tree_workspace(cache, 30, 20), torch.zeros_like(q)
    run = lambda: ctx.attn_kv4_paged_tree(cache, q, qb, 20, mask, 128**-0.5, ws, out=out)
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
    assert torch.equal(out, first)
    for k in range(3):
        q.copy_(paged_ref.queries(30, 8, seed=rng.randint(20, 99)))
        now = [rng.randint(1000, 3000), rng.randint(200, 800), rng.randint(1, 100)]
        cache.pages.length.copy_(i32(now))
        trees = see(new, 2 + k, seed=k)
        mask.copy_(ref.words_of(trees, 1, 30))
        g.replay()
        torch.cuda.synchronize()
        want, tol = ref.attention(cache, q, begin, now, 128**-0.5, trees=trees)
        assert torch.all((out.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


# ---- plan ----------------------------------------------------------------------------------------------------
def pages_of(lengths, page=16, width=300):
    B = len(lengths)
    return binding.Pages(torch.zeros((B, width), dtype=torch.int32, device="cuda"), i32(lengths), i32([0]), i32([0]), page)


@pytest.mark.parametrize("new,words", [([1], 1), ([5, 0, 3], 1), ([32], 1), ([33, 1], 2), ([128, 64, 127, 0], 4), ([100], 4), ([7] * 300, 1)])
@pytest.mark.parametrize("width,roots", [(1, 1), (4, 1), (200, 1), (3, 5)])
def test_tree_plan(ctx, new, words, width, roots):
    rng = random.Random(len(new) + width)
    parents = [ref.random_tree(rng, n, width, roots) for n in new]
    lengths = [n + rng.randint(0, 3000) for n in new]
    begin, pad = begins(new), 6
    N = begin[-1] + pad
    parent = i32([p for t in parents for p in t] + [55] * pad)
    mask, pos = ctx.tree_plan(pages_of(lengths), parent, i32(begin), words=words, pos0=4)
    trees = [ref.ancestors(p) for p in parents]
    assert torch.equal(mask, ref.words_of(trees, words, N))
    assert pos.tolist() == [4 + l - len(s) + sum(row) - 1 for l, s in zip(lengths, trees) for row in s] + [0] * pad
    assert ctx.check_status() == 0


def test_tree_plan_reports(ctx):
    parent, begin = i32([-1, 0, 5, 1, -1, 0, -2, 1]), i32([0, 4, 8])
    mask, pos = ctx.tree_plan(pages_of([10, 9]), parent, begin, words=1)
    assert ctx.check_status() == 2
    assert mask[:, 0].tolist() == [1, 3, 4, 11, 1, 3, 4, 11] and pos.tolist() == [6, 7, 6, 8, 5, 6, 5, 7]  # a parent out of range is none
    mask, pos = ctx.tree_plan(pages_of([3, 9]), i32([-1, 0, 1, 2] * 2), begin, words=1)  # fewer cached tokens than drafts
    assert ctx.check_status() == 2
    assert mask[:, 0].tolist() == [0] * 4 + [1, 3, 7, 15] and pos.tolist() == [0] * 4 + [5, 6, 7, 8]
    for bad in ([0, 40, 8], [0, 4, 9], [-1, 4, 8]):
        mask, pos = torch.full((8, 1), 9, dtype=torch.int32, device="cuda"), torch.full((8,), 9, dtype=torch.int32, device="cuda")
        ctx.tree_plan(pages_of([30, 30]), i32([-1, 0, 1, 2] * 2), i32(bad), out=(mask, pos))
        assert ctx.check_status() == 2
    big = i32([-1] + list(range(39)))
    mask = torch.full((40, 1), 9, dtype=torch.int32, device="cuda")
    ctx.tree_plan(pages_of([100]), big, i32([0, 40]), out=(mask, torch.zeros(40, dtype=torch.int32, device="cuda")))  # more rows than bits
    assert ctx.check_status() == 2 and torch.all(mask == 9)


# ---- acceptance ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("new", [[1], [26], [5, 0, 3, 128, 127], [64] * 40, [9] * 300])
@pytest.mark.parametrize("vocab", [2, 5, 100000])
def test_tree_accept(ctx, new, vocab):
    """Small vocabularies: long paths, and siblings with the same token (the first is taken)."""
    rng = random.Random(sum(new) + vocab)
    parents = [ref.random_tree(rng, n, rng.choice([1, 3, 9]), rng.choice([1, 1, 2])) for n in new]
    N, pad = sum(new), 3
    draft, target = ([rng.randrange(vocab) for _ in range(N + pad)] for _ in range(2))
    begin = begins(new)
    kept, n_kept, nxt = ctx.tree_accept(i32(begin), i32([p for t in parents for p in t] + [0] * pad), i32(draft), i32(target))
    want = [ref.accept(p, draft[a: a + len(p)], target[a: a + len(p)]) for p, a in zip(parents, begin)]
    assert n_kept.tolist() == [len(p) for p, _ in want] and nxt.tolist() == [c for _, c in want]
    assert kept.tolist() == [x for (p, _), n in zip(want, new) for x in p + [-1] * (n - len(p))] + [-1] * pad
    assert ctx.check_status() == 0


def test_a_chain_of_128_is_accepted_whole(ctx):
    kept, n_kept, nxt = ctx.tree_accept(i32([0, 128]), i32([-1] + list(range(127))), i32(list(range(128))), i32(list(range(1, 129))))
    assert kept.tolist() == list(range(128)) and n_kept.tolist() == [128] and nxt.tolist() == [128]


def test_tree_accept_reports(ctx):
    one = i32([0] * 4)
    kept, n_kept, _ = ctx.tree_accept(i32([0, 4]), i32([-1, 3, 0, 9]), one, one)
    assert ctx.check_status() == 2 and kept.tolist() == [0, 2, -1, -1] and n_kept.tolist() == [2]
    for bad in ([0, 5], [3, 1], [-2, 1]):
        _, n_kept, nxt = ctx.tree_accept(i32(bad), i32([-1, 0, 0, 0]), one, one)
        assert ctx.check_status() == 2 and n_kept.tolist() == [0] and nxt.tolist() == [-1]
    many = i32([0] * 129)
    _, n_kept, _ = ctx.tree_accept(i32([0, 129]), i32([-1] + [0] * 128), many, many)
    assert ctx.check_status() == 2 and n_kept.tolist() == [0]


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("new", [[5], [40, 0, 7, 33], [20] * 600])
def test_page_keep(ctx, page, new):
    rng = random.Random(page + len(new))
    lengths = [n + rng.randint(0, 50) for n in new]
    n_kept = [rng.randint(0, n) for n in new]
    cache = paged_ref.make_cache(lengths, 1, 1, page, seed=1)
    pg = cache.pages
    table, free, n_free = pg.table.tolist(), pg.free_list.tolist(), int(pg.n_free)
    after = [l - n + k for l, n, k in zip(lengths, new, n_kept)]
    back = [i for b in range(len(new)) for i in table[b][paged_ref.up(after[b], page): paged_ref.up(lengths[b], page)]]
    len_out, n_free_out = torch.zeros_like(pg.length), torch.zeros_like(pg.n_free)
    ctx.page_keep(pg, i32(begins(new)), i32(n_kept), len_out=len_out, n_free_out=n_free_out)
    assert pg.length.tolist() == lengths and int(pg.n_free) == n_free
    ctx.page_keep(pg, i32(begins(new)), i32(n_kept))
    assert pg.length.tolist() == after == len_out.tolist() and int(pg.n_free) == n_free + len(back) == int(n_free_out)
    assert pg.free_list.tolist()[: n_free + len(back)] == free[:n_free] + back and pg.table.tolist() == table
    assert ctx.check_status() == 0


@pytest.mark.parametrize("n_kept,new,spoil", [([3, 6], [5, 5], None), ([-1, 2], [5, 5], None), ([1, 1], [5, 60], None), ([0, 0], [40, 40], "id"), ([0, 0], [40, 40], "full")])
def test_page_keep_changes_nothing_where_it_cannot(ctx, n_kept, new, spoil):
    cache = paged_ref.make_cache([50, 50], 1, 1, 16, seed=1)
    pg = cache.pages
    if spoil == "id":
        pg.table[1, 2] = pg.n_pages
    if spoil == "full":
        pg.n_free.fill_(pg.n_pages)
    before = pg.length.tolist(), int(pg.n_free), pg.free_list.tolist()
    ctx.page_keep(pg, i32(begins(new)), i32(n_kept))
    assert ctx.check_status() == 2
    assert (pg.length.tolist(), int(pg.n_free), pg.free_list.tolist()) == before


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_kv4_paged_keep(ctx, page, steps):
    """Paths whose rows move onto one another's places, any order, the same row twice; every other vector of the cache keeps its bits."""
    new, lengths = [40, 128, 0, 7, 1, 9], [100, 128, 20, 300, 1, 30]
    kept = [[0, 1, 2, 5, 6, 30, 39], list(range(64, 128)), [], [6, 5, 4, 3, 2, 1, 0], [0], [3, 3, 0, 8]]
    cache = paged_ref.make_cache(lengths, 6, 3, page, steps=steps, seed=3)
    pg = cache.pages
    table = pg.table.tolist()
    slot = lambda b, c: table[b][c // page] * page + c % page
    flat = lambda t: t.transpose(2, 3).transpose(1, 2).flatten(0, 1)  # [slots, Hkv, 2, ..]
    codes = flat(cache.codes).clone()
    own = flat(cache.steps).clone() if cache.steps is not None else None
    want, want_own = codes.clone(), own.clone() if own is not None else None
    live = torch.ones(codes.shape[0], dtype=torch.bool, device="cuda")
    for b, (l, n, rows) in enumerate(zip(lengths, new, kept)):
        base = l - n
        for i, f in enumerate(rows):
            want[slot(b, base + i)] = codes[slot(b, base + f)]
            if own is not None:
                want_own[slot(b, base + i)] = own[slot(b, base + f)]
        for c in range(base + len(rows), l):
            live[slot(b, c)] = False  # undefined
    begin = begins(new)
    n_kept = [len(r) for r in kept]
    rows = [x for r, n in zip(kept, new) for x in r + [-1] * (n - len(r))]
    ctx.page_keep(pg, i32(begin), i32(n_kept))
    ctx.kv4_paged_keep(cache, i32(begin), i32(rows), i32(n_kept))
    assert ctx.check_status() == 0
    assert torch.equal(flat(cache.codes)[live], want[live])
    if own is not None:
        assert torch.equal(flat(cache.steps)[live], want_own[live])


def test_kv4_paged_keep_reports(ctx):
    cache = paged_ref.make_cache([40, 40], 2, 1, 16, seed=3)
    before = cache.codes.clone()
    begin = i32([0, 20, 40])
    rows = lambda *r: i32([x for k in r for x in list(k) + [-1] * (20 - len(k))])
    cache.pages.length.copy_(i32([22, 22]))
    for kept, n_kept in ((rows([0, 20], [0, 1]), [2, 2]), (rows([0, -5], [0, 1]), [2, 2]), (rows([0, 1], [0, 1]), [2, 21]), (rows([0, 1], [0, 1]), [2, -1])):
        ctx.kv4_paged_keep(cache, begin, kept, i32(n_kept))
        assert ctx.check_status() == 2 and torch.equal(cache.codes, before)
    cache.pages.table[0, 2] = -1  # places 32 .. 47 of the first sequence
    ctx.kv4_paged_keep(cache, begin, rows([0, 15], [0, 1]), i32([2, 2]))
    assert ctx.check_status() == 2 and torch.equal(cache.codes, before)


# ---- together ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("captured", [False, True])
def test_a_drafted_step_leaves_the_cache_of_plain_decoding(ctx, steps, captured):
    """Steps of drafts as a server runs them: plan, append, attention, acceptance, pages, moves. After each the cache holds what single steps with the accepted
    tokens alone write, and an accepted row's attention is what such a step computes."""
    Hq, Hkv, page, B, theta, sm = 8, 2, 16, 3, 1e4, 128**-0.5
    rng = random.Random(17)
    lengths, new = [30, 100, 15], [12, 5, 20]
    make = lambda: paged_ref.make_cache(lengths, Hq, Hkv, page, steps=steps, seed=21, extra_pages=40, width=24)
    cache, plain = make(), make()
    N = sum(new) + 3
    rows = lambda: torch.empty((N,), dtype=torch.int32, device="cuda")
    q_begin, slot, pos = torch.empty((B + 1,), dtype=torch.int32, device="cuda"), torch.empty((N,), dtype=torch.int64, device="cuda"), rows()
    parent, draft, target, mask, tree_pos, kept = rows(), rows(), rows(), torch.empty((N, 1), dtype=torch.int32, device="cuda"), rows(), rows()
    n_kept, nxt = torch.empty((B,), dtype=torch.int32, device="cuda"), torch.empty((B,), dtype=torch.int32, device="cuda")
    n_new = i32(new)
    qkv = torch.empty((N, (Hq + 2 * Hkv) * 128), dtype=torch.bfloat16, device="cuda")
    q, out = torch.zeros((N, Hq, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((N, Hq, 128), dtype=torch.bfloat16, device="cuda")
    ws = ctx.attn_kv4_paged_tree_workspace(cache, N, 20)

    def step():
        ctx.page_plan(cache.pages, n_new, pos0=4, out=(q_begin, slot, pos))
        ctx.tree_plan(cache.pages, parent, q_begin, pos0=4, out=(mask, tree_pos))
        ctx.qk_norm_rope_kv4_paged_append(cache, qkv, None, None, 0.0, tree_pos, slot, theta, q_out=q)
        ctx.attn_kv4_paged_tree(cache, q, q_begin, 20, mask, sm, ws, out=out)
        ctx.tree_accept(q_begin, parent, draft, target, out=(kept, n_kept, nxt))
        ctx.page_keep(cache.pages, q_begin, n_kept)
        ctx.kv4_paged_keep(cache, q_begin, kept, n_kept)

    graph = None
    if captured:
        state = [t.clone() for t in (cache.pages.table, cache.pages.length, cache.pages.free_list, cache.pages.n_free, cache.codes)]
        own = cache.steps.clone() if cache.steps is not None else None
        parent.fill_(-1), draft.zero_(), target.zero_(), qkv.zero_()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                step()
        torch.cuda.synchronize()
        for t, was in zip((cache.pages.table, cache.pages.length, cache.pages.free_list, cache.pages.n_free, cache.codes), state):
            assert torch.equal(t, was)  # a capture runs nothing
        assert own is None or torch.equal(own, cache.steps)
    for k in range(4):
        trees = [ref.random_tree(rng, n, 4) for n in new]
        parent.copy_(i32([p for t in trees for p in t] + [0] * 3))
        draft.copy_(i32([rng.randrange(3) for _ in range(N)])), target.copy_(i32([rng.randrange(3) for _ in range(N)]))
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(k)).bfloat16())
        graph.replay() if captured else step()
        assert ctx.check_status() == 0
        path = [p for p, _ in (ref.accept(t, draft[a: a + len(t)].tolist(), target[a: a + len(t)].tolist()) for t, a in zip(trees, begins(new)))]
        assert n_kept.tolist() == [len(p) for p in path]
        # the accepted tokens one after another; the drafted step wrote the same vectors at the same positions
        for i in range(max(len(p) for p in path)):
            one = [1 if i < len(p) else 0 for p in path]
            qb, sl, po = ctx.page_plan(plain.pages, i32(one), n_rows=B, pos0=4)
            take = [begins(new)[b] + path[b][i] for b in range(B) if one[b]]
            x = torch.cat((qkv[take], qkv[:B - len(take)]))
            q1 = ctx.qk_norm_rope_kv4_paged_append(plain, x, None, None, 0.0, po, sl, theta)
            o1 = ctx.attn_kv4_paged(plain, q1, qb, 1, sm, ctx.attn_kv4_paged_workspace(plain, B, 1))
            assert torch.equal(q1[: len(take)], q[take])
            # two kernels, each within the tolerance of the definition: their distance is at most both
            where = qb.tolist()
            _, tol = paged_ref.attention(plain, q1, where, plain.pages.length.tolist(), sm)
            assert torch.all((o1[: len(take)].double() - out[take].double()).abs() <= 2 * tol[: len(take)])
        now = cache.pages.length.tolist()
        assert now == plain.pages.length.tolist()
        for b in range(B):
            at = lambda c: torch.tensor([int(c.pages.table[b, t // page]) * page + t % page for t in range(now[b])], device="cuda")
            assert torch.equal(ctx.kv4_paged_read(cache, at(cache)), ctx.kv4_paged_read(plain, at(plain)))
        taken = sum(paged_ref.up(n, page) for n in now)
        assert int(cache.pages.n_free) + taken == cache.pages.n_pages
    assert ctx.check_status() == 0


# ---- what the calls allow ------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_prefix", [0, 4])
@pytest.mark.parametrize("steps", ["head", "vector"])
def test_fewer_cached_keys_than_drafts(ctx, n_prefix, steps):
    """The first drafts have no place: nobody sees them, and a row that sees nothing else (and no prefix) is zero."""
    check(ctx, [3, 0, 40], see([5, 4, 40], 2), n_prefix=n_prefix, steps=steps)


def test_rows_strides_and_output_over_the_queries(ctx):
    lengths, new = [500, 300, 2000], [9, 40, 17]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, seed=9)
    begin, trees = begins(new), see(new, 3)
    wide = paged_ref.queries(begin[-1], 12, seed=9)
    q, mask = wide[:, :8], ref.words_of(trees, 2, begin[-1])
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    assert torch.all((call(ctx, cache, q, begin, 40, mask).double() - want).abs() <= tol)
    dense = q.contiguous()
    call(ctx, cache, dense, begin, 40, mask, out=dense)
    assert torch.all((dense.double() - want).abs() <= tol)
    assert ctx.check_status() == 0


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_a_cache_of_more_than_four_gigabytes(ctx, steps):
    """Pages whose codes lie beyond 2^32 bytes."""
    Hkv, page, n_pages = 8, 128, 36000
    lengths, new = [300, 140], [10, 3]
    codes = torch.zeros((n_pages, Hkv, 2, page, 64), dtype=torch.uint8, device="cuda")
    assert codes.numel() > 2**32
    ids = [n_pages - 1 - 7 * i for i in range(5)]
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in ids:
        codes[i] = torch.randint(0, 256, codes[i].shape, generator=g, device="cuda", dtype=torch.uint8)
    pages = binding.Pages(i32([ids[:3], ids[3:] + [-1]]), i32(lengths), torch.zeros(n_pages, dtype=torch.int32, device="cuda"), i32([0]), page)
    own = torch.rand((n_pages, Hkv, 2, page), generator=g, device="cuda") + 0.3 if steps == "vector" else None
    s = torch.full((Hkv,), 0.5, device="cuda")
    cache = binding.KV4PagedCache(pages, None, None, codes, 2 * Hkv, s_k=s, s_v=s, steps=own)
    begin, trees = begins(new), see(new, 2)
    q = paged_ref.queries(13, 2 * Hkv)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    assert torch.all((call(ctx, cache, q, begin, 10, ref.words_of(trees, 1, 13)).double() - want).abs() <= tol)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, 50, 3)
    ws = ctx.attn_kv4_paged_workspace(cache, 13, 10)
    out = ctx.attn_kv4_paged_window(cache, q, i32(begin), 10, 50, 128**-0.5, ws, n_sink=3)
    assert torch.all((out.double() - want).abs() <= tol)
    before = codes[ids[0], :, :, :3].clone()
    kept = i32([0, 9, 8] + [-1] * 7 + [0, -1, -1])
    pages.length.copy_(i32([293, 138]))  # 3 of 10, 1 of 3 stay
    ctx.kv4_paged_keep(cache, i32(begin), kept, i32([3, 1]))
    last = codes[ids[2], :, :, 34:44]  # places 290 .. 299
    assert ctx.check_status() == 0 and torch.equal(last[:, :, 1], last[:, :, 9]) and torch.equal(codes[ids[0], :, :, :3], before)


def test_two_contexts_on_two_streams(ctx):
    """Trees of few and of many columns and windowed prompts side by side, again and again: each gives what it gives alone."""
    other = binding.Context()
    try:
        jobs = []
        for c, seed in ((ctx, 1), (other, 2)):
            lengths, new = ([3000, 700, 90], [5, 8, 3]) if seed == 1 else ([2500, 900], [100, 64])
            cache = paged_ref.make_cache(lengths, 8, 2, 16, steps="vector", seed=seed)
            begin, q = begins(new), paged_ref.queries(sum(new), 8, seed=seed)
            mask, qb, ws = ref.words_of(see(new, 3), 4, sum(new)), i32(begin), c.attn_kv4_paged_tree_workspace(cache, sum(new), max(new))
            ws2, out, out2 = c.attn_kv4_paged_workspace(cache, sum(new), max(new)), torch.zeros_like(q), torch.zeros_like(q)

            def run(c=c, cache=cache, q=q, qb=qb, mask=mask, ws=ws, ws2=ws2, out=out, out2=out2, most=max(new)):
                c.attn_kv4_paged_tree(cache, q, qb, most, mask, 128**-0.5, ws, out=out)
                c.attn_kv4_paged_window(cache, q, qb, most, 300, 128**-0.5, ws2, out=out2)
                return out, out2

            jobs.append((run, [t.clone() for t in run()], torch.cuda.Stream(), c))
        torch.cuda.synchronize()
        for _ in range(20):
            for run, _, stream, _ in jobs:
                with torch.cuda.stream(stream):
                    run()
        torch.cuda.synchronize()
        for run, want, stream, c in jobs:
            with torch.cuda.stream(stream):
                assert all(torch.equal(a, b) for a, b in zip(run(), want)) and c.check_status() == 0
    finally:
        other.close()


def test_two_captured_graphs_share_a_workspace(ctx):
    lengths, new = [3000, 700], [9, 40]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, seed=3)
    begin, q = begins(new), paged_ref.queries(49, 8, seed=3)
    qb, mask = i32(begin), ref.words_of(see(new, 3), 2, 49)
    ws = ctx.attn_kv4_paged_tree_workspace(cache, 49, 40)
    outs, graphs = [torch.zeros_like(q) for _ in range(2)], []
    calls = [lambda: ctx.attn_kv4_paged_tree(cache, q, qb, 40, mask, 128**-0.5, ws, out=outs[0]),
             lambda: ctx.attn_kv4_paged_tree(cache, q, qb, 40, mask, 128**-0.5, ws, window=400, n_sink=5, out=outs[1])]
    want = [f().clone() for f in calls]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for f in calls:
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                f()
        for k in range(6):
            for o in outs:
                o.zero_()
            graphs[k & 1].replay()
            graphs[1 - (k & 1)].replay()
            s.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    torch.cuda.synchronize()
    assert ctx.check_status() == 0


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_every_number_of_columns(ctx, steps):
    """Rows of 32, 64 and 128 columns, by the size of the call; a token's heads on both sides of a warp's 32 columns."""
    for B, n, ctx_len, Hq, Hkv in ((40, 8, 300, 8, 2), (60, 13, 400, 10, 2), (80, 16, 500, 4, 1), (60, 18, 600, 14, 2), (40, 30, 700, 8, 2)):
        new = [n - b % 3 for b in range(B)]
        check(ctx, [ctx_len + 7 * b for b in range(B)], see(new, 4), Hq=Hq, Hkv=Hkv, steps=steps, hide=False)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 0.0])
@pytest.mark.parametrize("n", [7, 40, 120])
def test_a_draft_without_numbers_stays_in_its_branch(ctx, n, bad):
    """Own steps that are no number, of a draft: rows that do not see it keep their results."""
    lengths = [300, 64 + n]
    cache = paged_ref.make_cache(lengths, 8, 2, 16, steps="vector", seed=5)
    begin, trees = [0, n, 2 * n], see([n, n], 3, seed=5)
    q = paged_ref.queries(2 * n, 8, seed=5)
    want, tol = ref.attention(cache, q, begin, lengths, 128**-0.5, trees=trees)
    table = cache.pages.table.tolist()
    for b, u in ((0, 2), (1, n - 2)):
        c = lengths[b] - n + u
        cache.steps[table[b][c // 16], :, :, c % 16] = bad
    out = call(ctx, cache, q, begin, n, ref.words_of(trees, 4, 2 * n))
    apart = torch.tensor([not row[u] for b, u in ((0, 2), (1, n - 2)) for row in trees[b]], device="cuda")
    assert 0 < apart.sum() < 2 * n
    assert torch.all((out.double() - want).abs()[apart] <= tol[apart])
    if bad != bad:
        assert torch.all(out[~apart].isnan())
    assert ctx.check_status() == 0


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("window", [64, 130, 500])
def test_own_masks_through_a_window(ctx, window, steps):
    """Any mask, not only a tree's: the place of a row, and with it its window, follows from how many drafts it sees. No key before every row's window is read."""
    rng, new, lengths = random.Random(window), [64, 33, 1], [900, 40, 333]
    trees = [[[rng.random() < 0.5 for _ in range(n)] for _ in range(n)] for n in new]
    check(ctx, lengths, trees, steps=steps, window=window, n_sink=3, hide=False)
    for row in trees:
        row[0] = [True] + [False] * (len(row) - 1)  # a row that sees itself alone has the earliest window
    check(ctx, lengths, trees, steps=steps, window=window, n_sink=3)
