"""The paged KV4 operators on the GPU against their definitions in 64 bits (tests/paged_ref.py): pages and slots, norm + rotary position with the
write into the cache, ragged attention, and a run of them together."""
import math
import random

import pytest
import torch

from paper_2410_05265_b200 import binding

import paged_ref as ref

pytestmark = pytest.mark.gpu
D, DEV = 128, "cuda"


@pytest.fixture(scope="module")
def ctx():
    return binding.Context()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ================================================================================================ pages
def page_state(B, page, seed, longest=200, spare=7, width=None):
    r = random.Random(seed)
    length = [r.choice([0, r.randint(0, longest), page * r.randint(0, longest // page)]) for _ in range(B)]
    width = width or ref.up(longest, page) * 3 + 1
    need = [ref.up(l, page) for l in length]
    n_pages = sum(need) + spare
    ids = list(range(n_pages))
    r.shuffle(ids)
    table, at = [], 0
    for k in need:
        table.append(ids[at: at + k] + [-9] * (width - k))
        at += k
    free = ids[at:] + [-5] * at
    return table, length, free, n_pages - at, n_pages


def pages_of(table, length, free, n_free, page):
    t = i32(table).reshape(len(table), -1) if table else torch.zeros((0, 4), dtype=torch.int32, device=DEV)
    return binding.Pages(t, i32(length), i32(free), i32([n_free]), page)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("B", [1, 2, 37, 600, 1500])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_plan_is_the_definition(ctx, B, page, pad):
    table, length, free, n_free, n_pages = page_state(B, page, seed=B + page, spare=3 * B + 20)
    r = random.Random(B * page + pad)
    n_new = [r.choice([0, 1, 1, r.randint(0, 40)]) for _ in range(B)]
    want = ref.plan(table, length, free, n_free, n_new, page, 4, sum(n_new) + pad, n_pages)
    assert want is not None
    pg = pages_of(table, length, free, n_free, page)
    begin, slot, pos = ctx.page_plan(pg, i32(n_new), n_rows=sum(n_new) + pad, pos0=4)
    ctx.check()
    assert pg.table.tolist() == want[0] and pg.length.tolist() == want[1] and pg.n_free.tolist() == [want[2]]
    assert begin.tolist() == want[3] and slot.tolist() == want[4] and pos.tolist() == want[5]
    assert pg.free_list.tolist() == free


def test_plan_of_many_rows(ctx):
    """Rows by the ten thousand: the form with several CTAs, in place and out of place."""
    B, page = 33, 32
    table, length, free, n_free, n_pages = page_state(B, page, 5, longest=3000, spare=3000, width=400)
    n_new = [(b * 37) % 1400 for b in range(B)]
    rows = sum(n_new) + 3
    want = ref.plan(table, length, free, n_free, n_new, page, 0, rows, n_pages)
    for in_place in (False, True):
        pg = pages_of(table, length, free, n_free, page)
        out_len, out_free = (None, None) if in_place else (i32([0] * B), i32([0]))
        begin, slot, pos = ctx.page_plan(pg, i32(n_new), n_rows=rows, len_out=out_len, n_free_out=out_free)
        ctx.check()
        assert (pg.length if in_place else out_len).tolist() == want[1] and (pg.n_free if in_place else out_free).tolist() == [want[2]]
        assert in_place or (pg.length.tolist() == length and pg.n_free.tolist() == [n_free])
        assert pg.table.tolist() == want[0] and begin.tolist() == want[3] and slot.tolist() == want[4] and pos.tolist() == want[5]


def test_plan_at_the_largest_batch(ctx):
    B, page = 8192, 16
    length = [(7 * b) % 50 for b in range(B)]
    need = [ref.up(l, page) for l in length]
    n_pages = sum(need) + B
    table, at = [], 0
    for k in need:
        table.append(list(range(at, at + k)) + [-1] * (5 - k))
        at += k
    free = list(range(at, n_pages)) + [0] * at
    n_new = [1 if b % 3 else 0 for b in range(B)]
    want = ref.plan(table, length, free, n_pages - at, n_new, page, 1, sum(n_new), n_pages)
    pg = pages_of(table, length, free, n_pages - at, page)
    begin, slot, pos = ctx.page_plan(pg, i32(n_new), n_rows=sum(n_new), pos0=1)
    ctx.check()
    assert (pg.table.tolist(), pg.length.tolist(), pg.n_free.tolist()[0], begin.tolist(), slot.tolist(), pos.tolist()) == want


@pytest.mark.parametrize("case", ["pages", "rows", "width", "length", "count", "n_free"])
@pytest.mark.parametrize("rows", [40, 5000])
def test_a_step_that_cannot_be_served_changes_nothing(ctx, case, rows):
    page, width = 16, 6
    table, length, free, n_free = [[3, 1, -1, -1, -1, -1], [0, -1, -1, -1, -1, -1], [-1] * 6], [20, 16, 0], [2, 4, 5, 6, 7, 8, 9, 9, 9, 9], 7
    n_new = [1, 1, 3]
    if case == "pages":
        n_new = [70, 70, 70]
    if case == "rows":
        n_new, rows = [20, 15, 6], 40
    if case == "width":
        n_new = [1, 81, 0]
    if case == "length":
        length[2] = -3
    if case == "count":
        n_new[1] = -1
    if case == "n_free":
        n_free = 11
    pg = pages_of(table, length, free, n_free, page)
    begin, slot, pos = ctx.page_plan(pg, i32(n_new), n_rows=rows)
    assert ctx.check_status() == 2
    assert pg.table.tolist() == table and pg.length.tolist() == length and pg.n_free.tolist() == [n_free] and pg.free_list.tolist() == free
    assert begin.tolist() == [0] * 4 and slot.tolist() == [-1] * rows and pos.tolist() == [0] * rows


def test_plan_reports_ids_that_are_none(ctx):
    pg = pages_of([[0, -1, -1, -1]], [10], [1, 77, 5], 2, 16)  # the first page taken is id 77 of 3
    begin, slot, pos = ctx.page_plan(pg, i32([8]), n_rows=8)
    assert ctx.check_status() == 2
    assert slot.tolist() == list(range(10, 16)) + [-1, -1] and pos.tolist() == list(range(10, 18))
    assert pg.table.tolist() == [[0, -1, -1, -1]]


@pytest.mark.parametrize("B,page", [(1, 16), (9, 64), (700, 16), (1100, 32)])
def test_release_is_the_definition(ctx, B, page):
    table, length, free, n_free, n_pages = page_state(B, page, seed=B, spare=2)
    r = random.Random(B)
    done = [r.choice([0, 0, 1, -3]) for _ in range(B)]
    want_free, want_len = ref.release(table, length, free, n_free, done, page, n_pages)
    for in_place in (False, True):
        pg = pages_of(table, length, free, n_free, page)
        a, b = (None, None) if in_place else (i32([0] * B), i32([0]))
        ctx.page_release(pg, i32(done), len_out=a, n_free_out=b)
        ctx.check()
        assert (pg.length if in_place else a).tolist() == want_len and (pg.n_free if in_place else b).tolist() == [len(want_free)]
        assert pg.free_list.tolist()[: len(want_free)] == want_free and pg.free_list.tolist()[len(want_free):] == free[len(want_free):]
        assert pg.table.tolist() == table


def test_release_refuses_what_the_list_cannot_hold(ctx):
    for length, n_free in (([20, 16], 3), ([-1, 16], 1), ([1000, 16], 0)):
        pg = pages_of([[3, 1, -1], [0, -1, -1]], length, [2, 4, 9, 9, 9], n_free, 16)
        ctx.page_release(pg, i32([1, 1]))
        assert ctx.check_status() == 2
        assert pg.length.tolist() == length and pg.n_free.tolist() == [n_free] and pg.free_list.tolist() == [2, 4, 9, 9, 9]


def test_pages_go_round(ctx):
    """Requests come and go for many steps: every page is free or belongs to one sequence, and never to two."""
    B, page, n_pages, r = 12, 16, 60, random.Random(3)
    pg = binding.Pages(i32([[0] * 12 for _ in range(B)]), i32([0] * B), i32(list(range(n_pages))), i32([n_pages]), page)
    length = [0] * B
    for _ in range(60):
        done = [1 if l and r.random() < 0.2 else 0 for l in length]
        ctx.page_release(pg, i32(done))
        length = [0 if d else l for d, l in zip(done, length)]
        n_new = [r.choice([0, 1, 1, 1, 30]) if l + 30 <= 12 * page else 0 for l in length]
        while sum(ref.up(l + n, page) for l, n in zip(length, n_new)) > n_pages:
            n_new[max(range(B), key=lambda b: n_new[b])] = 0
        ctx.page_plan(pg, i32(n_new), n_rows=sum(n_new))
        length = [l + n for l, n in zip(length, n_new)]
        ctx.check()
        assert pg.length.tolist() == length
        table, n_free = pg.table.tolist(), pg.n_free.item()
        held = [i for b, l in enumerate(length) for i in table[b][: ref.up(l, page)]]
        assert sorted(held + pg.free_list.tolist()[:n_free]) == list(range(n_pages))


# ================================================================================================ norm + rotary position
SECTIONS = {1: (64,), 2: (16, 48), 3: (16, 24, 24)}


def heads(N, H, seed, scale=1.7, cols=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn((N, cols or H, D), generator=g, device=DEV)).bfloat16()


def gains(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(1 + 0.2 * torch.randn(D, generator=g, device=DEV)).bfloat16() for _ in range(2)]


def positions(axes, N, seed, top=140000):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, top, (axes, N), generator=g, device=DEV, dtype=torch.int32)


def assert_heads(got, want, what):
    """fp32 arithmetic: sums of 128 squares, a product or two for the rotation, angles off by 2^-22 of a radian and seven additions of the transform stay
    below 2^-15 of the head's largest magnitude (times sqrt(128) for what the transform may gather); the store rounds by 2^-8 of the value."""
    top = want.abs().amax(-1, keepdim=True)
    bad = (got.double() - want).abs() > want.abs() * 2.0**-8 + top * 2.0**-15 + 2.0**-126
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}"


@pytest.mark.parametrize("N,Hq,Hk", [(1, 32, 8), (1, 1, 0), (1, 0, 3), (3, 5, 1), (7, 7, 7), (33, 6, 2), (700, 8, 1), (5000, 3, 2)])
@pytest.mark.parametrize("axes", [1, 2, 3])
@pytest.mark.parametrize("norm,rotate", [(True, False), (False, True), (True, True), (False, False)])
def test_qk_norm_rope_is_the_definition(ctx, N, Hq, Hk, axes, norm, rotate):
    x, pos, sec = heads(N, Hq + Hk, N + axes), positions(axes, N, N), SECTIONS[axes]
    gq, gk = gains(N) if norm else (None, None)
    y = ctx.qk_norm_rope(x, Hq, gq, gk, 1e-5, pos if axes > 1 else pos[0], 500000.0, sections=sec if axes > 1 else None, rotate=rotate)
    ctx.check()
    want = torch.cat((ref.norm_rope(x[:, :Hq], gq, 1e-5, pos, 500000.0, sec, rotate), ref.norm_rope(x[:, Hq:], gk, 1e-5, pos, 500000.0, sec, rotate)), 1)
    assert_heads(y, want, "qk_norm_rope")


def test_qk_norm_rope_in_place_strided_and_far(ctx):
    """Columns of a wider projection, in place and into another stride; positions up to the largest int32 and below zero; zero heads; tiny and huge
    values."""
    N, Hq, Hk = 21, 6, 2
    wide = heads(N, 11, 4)
    wide[3, 2] = 0
    wide[4, 1] *= 1e-15
    wide[5, 0] *= 1e15
    gq, gk = gains(8)
    pos = positions(1, N, 3)
    pos[0, :3] = i32([2**31 - 1, -5, 0])
    want = torch.cat((ref.norm_rope(wide[:, :Hq], gq, 1e-6, pos, 10000.0, (64,), False), ref.norm_rope(wide[:, Hq: Hq + Hk], gk, 1e-6, pos, 10000.0, (64,), False)), 1)
    keep = wide.clone()
    out = torch.full((N, Hq + Hk + 1, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.qk_norm_rope(wide[:, : Hq + Hk], Hq, gq, gk, 1e-6, pos, 10000.0, out=out[:, : Hq + Hk])
    assert_heads(out[:, : Hq + Hk], want, "strided")
    assert torch.equal(wide, keep) and (out[:, Hq + Hk:] == 7.0).all()
    ctx.qk_norm_rope(wide[:, : Hq + Hk], Hq, gq, gk, 1e-6, pos, 10000.0, out=wide[:, : Hq + Hk])
    ctx.check()
    assert torch.equal(wide[:, : Hq + Hk], out[:, : Hq + Hk]) and torch.equal(wide[:, Hq + Hk:], keep[:, Hq + Hk:])


def test_qk_norm_rope_agrees_with_rope(ctx):
    """Without gains and with positions that count up it is pq_rope and pq_rope_rotate, up to the rounding of the store."""
    x = heads(40, 5, 2)
    pos = torch.arange(9, 49, dtype=torch.int32, device=DEV)
    for rotate in (False, True):
        a, b = ctx.qk_norm_rope(x, 3, None, None, 0.0, pos, 500000.0, rotate=rotate), ctx.rope(x, 9, 500000.0, rotate=rotate)
        top = b.double().abs().amax(-1, keepdim=True)
        assert ((a.double() - b.double()).abs() <= 2 * 2.0**-8 * b.double().abs() + top * 2.0**-14).all()


# ================================================================================================ append and read
@pytest.mark.parametrize("N,Hq,Hkv,page", [(1, 32, 8, 16), (1, 5, 1, 128), (19, 8, 8, 32), (130, 6, 2, 64), (900, 4, 1, 16), (2600, 2, 1, 128)])
@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("norm,rotate,axes", [(True, False, 1), (True, True, 3), (False, True, 2), (False, False, 1)])
def test_append_writes_codes_steps_and_queries(ctx, N, Hq, Hkv, page, steps, norm, rotate, axes):
    cache = ref.make_cache([N], Hq, Hkv, page, steps, seed=N, extra_pages=4)
    before, before_steps = cache.codes.clone(), None if cache.steps is None else cache.steps.clone()
    qkv = heads(N, Hq + 2 * Hkv, N + Hkv)
    if N > 5:
        qkv[2] = 0  # a vector of zeros takes the step 1
        qkv[4, Hq:] *= 1e-20
    pos, sec = positions(axes, N, N + 1), SECTIONS[axes]
    gq, gk = gains(N) if norm else (None, None)
    n_slots = cache.codes.shape[0] * page
    g = torch.Generator(device=DEV).manual_seed(N)
    slot = torch.randperm(n_slots, generator=g, device=DEV)[:N]
    skip = torch.rand(N, generator=g, device=DEV) < (0.2 if N > 5 else 0.0)
    slot[skip] = -1
    q_out = torch.full((N, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx.qk_norm_rope_kv4_paged_append(cache, qkv.view(N, -1), gq, gk, 1e-5, pos if axes > 1 else pos[0], slot, 500000.0, sections=sec if axes > 1 else None,
                                      rotate=rotate, q_out=q_out)
    ctx.check()
    live = ~skip
    assert_heads(q_out[live], ref.norm_rope(qkv[:, :Hq], gq, 1e-5, pos, 500000.0, sec, rotate)[live], "queries")
    assert (q_out[skip] == 3.0).all()
    k, v = ref.norm_rope(qkv[:, Hq: Hq + Hkv], gk, 1e-5, pos, 500000.0, sec, rotate), qkv[:, Hq + Hkv:].double()
    codes, st = [], []
    for y, s in ((k, cache.s_k), (v, cache.s_v)):
        s = ref.step_of(y) if steps == "vector" else s[None].expand(N, -1)
        codes.append(ref.codes_of(y, s[..., None]))
        st.append(s)
    codes, st = torch.stack(codes, 1), torch.stack(st, 1)  # [N, 2, Hkv, 128], [N, 2, Hkv]
    where = slot[live]
    got = ref.unpack(cache.codes).permute(0, 3, 2, 1, 4).reshape(n_slots, 2, Hkv, D)
    assert torch.equal(got[where].to(torch.int8), codes[live])
    others = torch.ones(n_slots, dtype=torch.bool, device=DEV)
    others[where] = False
    assert torch.equal(got[others], ref.unpack(before).permute(0, 3, 2, 1, 4).reshape(n_slots, 2, Hkv, D)[others])
    if steps == "vector":
        flat = lambda t: t.permute(0, 3, 2, 1).reshape(n_slots, 2, Hkv)
        assert torch.equal(flat(cache.steps)[others], flat(before_steps)[others])
        # the key's step comes from a maximum in 64 bits: off by its rounding to fp32 at most, where the reference's last bits differ
        assert ((flat(cache.steps)[where] - st[live]).abs() <= 2.0**-23 * st[live]).all()
    kv = torch.full((N, 2, Hkv, D), 5.0, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_paged_read(cache, slot, out=kv)
    ctx.check()
    used = flat(cache.steps)[where] if steps == "vector" else st[live]
    assert torch.equal(kv[live], (codes[live].float() * used[..., None]).bfloat16())
    assert (kv[skip] == 5.0).all()


def test_append_in_place_and_from_a_wider_matrix(ctx):
    N, Hq, Hkv = 50, 4, 2
    cols = (Hq + 2 * Hkv) * D
    wide = torch.zeros((N, cols + 64), dtype=torch.bfloat16, device=DEV)
    wide[:, :cols] = heads(N, Hq + 2 * Hkv, 6).view(N, cols)
    gq, gk = gains(1)
    pos, slot = positions(1, N, 5), torch.arange(N, device=DEV)
    a, b = (ref.make_cache([N], Hq, Hkv, 32, "vector", seed=1) for _ in range(2))
    q = ctx.qk_norm_rope_kv4_paged_append(a, wide[:, :cols].contiguous(), gq, gk, 1e-5, pos, slot, 500000.0, rotate=True)
    rest = wide[:, Hq * D:].clone()
    ctx.qk_norm_rope_kv4_paged_append(b, wide[:, :cols], gq, gk, 1e-5, pos, slot, 500000.0, rotate=True, q_out=wide[:, : Hq * D].unflatten(1, (Hq, D)))
    ctx.check()
    assert torch.equal(wide[:, : Hq * D].reshape(N, Hq, D), q) and torch.equal(wide[:, Hq * D:], rest)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.steps, b.steps)


def test_keys_do_not_depend_on_how_a_prompt_is_cut(ctx):
    """A prompt cached at once, in chunks and token by token leaves the same bytes."""
    N, Hq, Hkv = 300, 4, 2
    qkv, pos, (gq, gk) = heads(N, Hq + 2 * Hkv, 9).view(N, -1), positions(1, N, 2)[0], gains(3)
    caches = [ref.make_cache([N], Hq, Hkv, 16, "vector", seed=2) for _ in range(3)]
    slot = torch.arange(N, device=DEV)
    for c, size in zip(caches, (N, 77, 1)):
        for lo in range(0, N, size):
            hi = min(N, lo + size)
            ctx.qk_norm_rope_kv4_paged_append(c, qkv[lo:hi], gq, gk, 1e-5, pos[lo:hi], slot[lo:hi], 500000.0)
    ctx.check()
    assert all(torch.equal(caches[0].codes, c.codes) and torch.equal(caches[0].steps, c.steps) for c in caches[1:])


def test_slots_past_the_cache_are_skipped_and_reported(ctx):
    cache = ref.make_cache([20], 2, 1, 16, seed=4)
    before = cache.codes.clone()
    n_slots = cache.codes.shape[0] * 16
    slot = torch.tensor([n_slots, 2**40, -1, -(2**40)], device=DEV)
    q = torch.full((4, 2, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx.qk_norm_rope_kv4_paged_append(cache, heads(4, 4, 1).view(4, -1), None, None, 0.0, positions(1, 4, 1), slot, 1e4, q_out=q)
    assert ctx.check_status() == 2
    assert torch.equal(cache.codes, before) and (q == 3.0).all()
    out = torch.full((4, 2, 1, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_paged_read(cache, slot, out=out)
    assert ctx.check_status() == 2 and (out == 3.0).all()


# ================================================================================================ attention
def attend(ctx, cache, lengths, new, seed=1, scale=1.2, pad=0, max_new=None, max_len=0, sm_scale=1 / math.sqrt(D)):
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    N = begin[-1] + pad
    q = ref.queries(N, cache.Hq, seed, scale)
    out = torch.full((N, cache.Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
    mn = max(new + [1]) if max_new is None else max_new
    ws = ctx.attn_kv4_paged_workspace(cache, N, mn)
    ctx.attn_kv4_paged(cache, q, i32(begin), mn, sm_scale, ws, max_len=max_len, out=out)
    ctx.check()
    return q, begin, out


def check_attention(ctx, cache, lengths, new, **kw):
    q, begin, out = attend(ctx, cache, lengths, new, **kw)
    want, tol = ref.attention(cache, q, begin, lengths, kw.get("sm_scale", 1 / math.sqrt(D)))
    n = begin[-1]
    bad = ~((out[:n].double() - want[:n]).abs() <= tol[:n])
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}; worst {float(((out[:n].double() - want[:n]).abs() / tol[:n].clamp(min=1e-30)).max())} of the tolerance"
    assert (out[n:] == 9.0).all()
    return out


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 1), (4, 4), (6, 2), (5, 1), (14, 2)])
def test_decode_lengths_around_every_border(ctx, steps, page, Hq, Hkv):
    lengths = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 300, 511, 513]
    cache = ref.make_cache(lengths, Hq, Hkv, page, steps, seed=page + Hq)
    check_attention(ctx, cache, lengths, [1] * len(lengths))
    check_attention(ctx, cache, lengths, [1] * len(lengths), max_len=max(lengths), pad=3)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,Hq,Hkv", [([1021], 32, 8), ([5], 8, 8), ([40000], 8, 1), ([9000, 1, 130, 20000, 0, 64], 16, 2), ([4097] * 3, 64, 8),
                                            ([700 + 13 * i for i in range(90)], 8, 4), ([1 + (37 * i) % 600 for i in range(400)], 4, 2)])
@pytest.mark.parametrize("bound", [False, True])
def test_decode_batches(ctx, steps, lengths, Hq, Hkv, bound):
    """One sequence, long ones whose keys many workers share, batches that fill the chip many times over; with and without a bound on the lengths."""
    cache = ref.make_cache(lengths, Hq, Hkv, 16 if len(lengths) > 2 else 64, steps, seed=len(lengths), width=4096 if len(lengths) < 10 else 200)
    check_attention(ctx, cache, lengths, [1] * len(lengths), max_len=max(lengths) if bound else 0)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("n_prefix", [0, 1, 5, 64])
def test_decode_prefix_lengths_and_empty_sequences(ctx, steps, n_prefix):
    lengths = [0, 1, 200, 0, 40]
    cache = ref.make_cache(lengths, 8, 2, 32, steps, n_prefix=n_prefix, seed=n_prefix)
    out = check_attention(ctx, cache, lengths, [1] * 5)
    if n_prefix == 0:
        assert (out[0] == 0).all() and (out[3] == 0).all()
    check_attention(ctx, cache, lengths, [1, 0, 1, 0, 1], pad=2)  # sequences without a row
    check_attention(ctx, cache, lengths, [0] * 5, pad=1)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 1e25])
def test_decode_queries_of_any_magnitude(ctx, steps, scale):
    """A query is scaled into fp16 by a power of two per head: its own magnitude is not limited by fp16."""
    lengths = [3, 150, 900]
    cache = ref.make_cache(lengths, 8, 2, 16, steps, seed=3)
    check_attention(ctx, cache, lengths, [1] * 3, scale=scale, sm_scale=min(1 / math.sqrt(D), 20 / scale / D) if scale > 1 else 1 / math.sqrt(D) / scale)


@pytest.mark.parametrize("lo,hi", [(-50.0, -40.0), (40.0, 50.0), (-20.0, 20.0)])
def test_decode_own_steps_of_any_magnitude(ctx, lo, hi):
    """Steps far apart: a weight carries its value's step in the exponent, so that no step is lost against another."""
    lengths = [1, 70, 1000]
    cache = ref.make_cache(lengths, 4, 2, 16, "vector", n_prefix=0, seed=5, step_range=(lo, hi))
    cache.steps[:, :, 0] = 0.4  # keys of ordinary size: it is the values that differ
    check_attention(ctx, cache, lengths, [1] * 3)


def test_decode_scores_that_climb(ctx):
    """The largest score comes last and far above the others, where the reference exponent has to move in every block."""
    lengths = [2000]
    cache = ref.make_cache(lengths, 8, 1, 16, "vector", seed=6)
    order = cache.pages.table[0, :125].long()
    cache.steps[order, :, 0] = torch.linspace(0.01, 6.0, 2000, device=DEV).view(125, 1, 16)
    check_attention(ctx, cache, lengths, [1])


def test_decode_ids_that_are_none_do_not_fault(ctx):
    cache = ref.make_cache([100, 40], 4, 2, 16, seed=8)
    cache.pages.table[0, 3] = 10**6
    cache.pages.table[0, 5] = -1
    q, ws = ref.queries(2, 4), ctx.attn_kv4_paged_workspace(cache, 2, 1)
    out = ctx.attn_kv4_paged(cache, q, i32([0, 1, 2]), 1, 0.1, ws)
    assert ctx.check_status() == 2
    cache.pages.table[0] = 0  # (the reference does not look at it)
    want, tol = ref.attention(cache, q[1:], [0, 0, 1], [0, 40], 0.1)
    assert ((out[1:].double() - want).abs() <= tol).all()  # the other sequence is as it should be


def test_lengths_and_rows_out_of_range_are_reported(ctx):
    cache = ref.make_cache([100, 40], 4, 2, 16, seed=8, width=8)
    q = ref.queries(4, 4)
    ws = ctx.attn_kv4_paged_workspace(cache, 4, 1)
    for begin, length in (([0, 2, 3], None), ([0, 1, 2], [-4, 40]), ([0, 1, 2], [100, 129])):
        if length:
            cache.pages.length.copy_(i32(length))
        ctx.attn_kv4_paged(cache, q, i32(begin), 1, 0.1, ws)
        assert ctx.check_status() == 2
        cache.pages.length.copy_(i32([100, 40]))


def test_results_do_not_depend_on_timing(ctx):
    lengths = [30000, 2, 9000, 4500]
    for steps in ("head", "vector"):
        cache = ref.make_cache(lengths, 16, 2, 16, steps, seed=9)
        first = attend(ctx, cache, lengths, [1] * 4)[2]
        for _ in range(20):
            assert torch.equal(first, attend(ctx, cache, lengths, [1] * 4)[2])


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 1), (4, 4), (6, 2), (5, 1), (7, 1), (4, 2), (12, 4)])
@pytest.mark.parametrize("page,n_prefix", [(16, 4), (32, 0), (64, 64), (128, 1)])
def test_prompts_of_many_lengths(ctx, steps, Hq, Hkv, page, n_prefix):
    """Whole prompts, chunks behind cached keys and single tokens in one batch; row tiles and key tiles that are full, nearly empty and one more."""
    new = [2, 3, 17, 33, 64, 65, 1, 127, 128, 129, 0, 200, 1]
    lengths = [2, 3, 17, 40, 64, 65, 500, 256, 128, 400, 30, 201, 1]
    cache = ref.make_cache(lengths, Hq, Hkv, page, steps, seed=page + Hq, n_prefix=n_prefix)
    check_attention(ctx, cache, lengths, new, pad=2)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [
    ([700], [700], 8, 2), ([5000], [2], 8, 1), ([20000], [5], 16, 2), ([3000], [300], 4, 4), ([9000, 100, 4000], [40, 100, 2], 8, 1), ([2], [2], 1, 1),
    ([257 + 3 * i for i in range(40)], [2 + (11 * i) % 90 for i in range(40)], 4, 1), ([4 + i % 3 for i in range(300)], [2 + i % 3 for i in range(300)], 2, 2)])
def test_chunks_that_several_workers_share(ctx, steps, lengths, new, Hq, Hkv):
    cache = ref.make_cache(lengths, Hq, Hkv, 32, steps, seed=len(lengths))
    check_attention(ctx, cache, lengths, new)


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_rows_without_keys(ctx, steps):
    """More rows than cached keys: the first rows see the prefix alone, or nothing."""
    for n_prefix in (0, 3):
        lengths, new = [3, 0, 150], [9, 4, 200]
        cache = ref.make_cache(lengths, 8, 2, 16, steps, n_prefix=n_prefix, seed=2)
        out = check_attention(ctx, cache, lengths, new)
        if n_prefix == 0:
            assert (out[:6] == 0).all() and (out[9:13] == 0).all()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 1e25])
def test_prompt_queries_of_any_magnitude(ctx, steps, scale):
    lengths = [150, 90]
    cache = ref.make_cache(lengths, 8, 2, 16, steps, seed=3)
    check_attention(ctx, cache, lengths, [150, 20], scale=scale, sm_scale=min(1 / math.sqrt(D), 20 / scale / D) if scale > 1 else 1 / math.sqrt(D) / scale)


@pytest.mark.parametrize("lo,hi", [(-50.0, -40.0), (40.0, 50.0), (-20.0, 20.0)])
def test_prompt_own_steps_of_any_magnitude(ctx, lo, hi):
    lengths = [70, 600]
    cache = ref.make_cache(lengths, 4, 2, 16, "vector", n_prefix=0, seed=5, step_range=(lo, hi))
    cache.steps[:, :, 0] = 0.4
    check_attention(ctx, cache, lengths, [70, 40])


def test_prompt_scores_that_climb(ctx):
    lengths = [800]
    cache = ref.make_cache(lengths, 8, 1, 16, "vector", seed=6)
    order = cache.pages.table[0, :50].long()
    cache.steps[order, :, 0] = torch.linspace(0.01, 6.0, 800, device=DEV).view(50, 1, 16)
    check_attention(ctx, cache, lengths, [300])


def test_prompt_ids_that_are_none_do_not_fault(ctx):
    cache = ref.make_cache([300, 40], 4, 2, 16, seed=8)
    cache.pages.table[0, 3] = 10**6
    cache.pages.table[0, 18] = -1
    q, ws = ref.queries(14, 4), ctx.attn_kv4_paged_workspace(cache, 14, 10)
    out = ctx.attn_kv4_paged(cache, q, i32([0, 10, 14]), 10, 0.1, ws)
    assert ctx.check_status() == 2
    cache.pages.table[0] = 0
    want, tol = ref.attention(cache, q[10:], [0, 0, 4], [0, 40], 0.1)
    assert ((out[10:].double() - want).abs() <= tol).all()


def test_prompt_rows_out_of_range_are_reported(ctx):
    cache = ref.make_cache([100, 40], 4, 2, 16, seed=8, width=8)
    for begin, length, rows, max_new in (([0, 5, 9], None, 9, 4), ([0, 5, 9], [-4, 40], 9, 5), ([0, 5, 9], [100, 129], 9, 5), ([0, 5, 12], None, 9, 7), ([-3, 5, 9], None, 9, 8),
                                         ([4, 2, 9], None, 9, 9)):
        if length:
            cache.pages.length.copy_(i32(length))
        out = torch.full((rows, 4, D), 9.0, dtype=torch.bfloat16, device=DEV)
        ctx.attn_kv4_paged(cache, ref.queries(rows, 4), i32(begin), max_new, 0.1, ctx.attn_kv4_paged_workspace(cache, rows, max_new), out=out)
        assert ctx.check_status() == 2
        cache.pages.length.copy_(i32([100, 40]))
        if begin == [0, 5, 9] and max_new == 4:
            assert (out[:5] == 9.0).all() and (out[5:] != 9.0).any()  # the sequence that is too long is left out, the other is not


def test_prompt_results_do_not_depend_on_timing(ctx):
    lengths, new = [9000, 700, 300, 4500], [30, 700, 3, 150]
    for steps in ("head", "vector"):
        cache = ref.make_cache(lengths, 16, 2, 16, steps, seed=9)
        first = attend(ctx, cache, lengths, new)[2]
        for _ in range(20):
            assert torch.equal(first, attend(ctx, cache, lengths, new)[2])
