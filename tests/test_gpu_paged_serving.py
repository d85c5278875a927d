"""The paged KV4 operators as a server uses them: release -> plan -> append -> attention over many steps of a ragged batch, captured and replayed,
on other streams, with waits that run out, and far into large caches."""
import math
import random

import pytest
import torch

from paper_2410_05265_b200 import binding

import paged_ref as ref

pytestmark = pytest.mark.gpu
D, DEV = 128, "cuda"
SCALE = 1 / math.sqrt(D)
PQ_ERR_TIMEOUT = 6


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.check()
    c.close()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def empty_cache(B, n_pages, page, width, Hq, Hkv, steps, n_prefix, seed=0):
    """A cache without tokens whose pages are all free, in a mixed order."""
    c = ref.make_cache([0] * B, Hq, Hkv, page, steps, n_prefix, seed=seed, extra_pages=n_pages, width=width)
    c.codes.fill_(0x5A)
    return c


def projection(N, Hq, Hkv, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn((N, (Hq + 2 * Hkv) * D), generator=g, device=DEV).bfloat16()


def gains(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return tuple((1 + 0.2 * torch.randn(D, generator=g, device=DEV)).bfloat16() for _ in range(2))


def slots_of(cache, b, n):
    page = cache.pages.page
    c = torch.arange(n, device=DEV)
    return cache.pages.table[b].long()[c // page] * page + c % page


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("page,Hq,Hkv,n_prefix,rotate", [(16, 8, 2, 4, True), (64, 5, 1, 0, False), (128, 4, 4, 64, True), (32, 16, 2, 1, False)])
def test_steps_of_a_server(ctx, steps, page, Hq, Hkv, n_prefix, rotate):
    """Sequences come, are cached in chunks, go on token by token, wait, and leave; their pages are given to others. The bookkeeping is the one in plain
    Python, what a sequence has in the cache is what a cache of its own gets when it is appended at once, bit for bit, and each step's
    attention is the definition's over the cache as it is."""
    B, pad = 6, 3
    r = random.Random(page)
    width, n_pages = ref.up(420, page), ref.up(420, page) * B // 2
    cache = empty_cache(B, n_pages, page, width, Hq, Hkv, steps, n_prefix, seed=page)
    pg, (gq, gk) = cache.pages, gains(3)
    table, length, free, n_free = pg.table.tolist(), [0] * B, pg.free_list.tolist(), n_pages
    rows = {b: [] for b in range(B)}  # projections of the tokens that a sequence holds
    step, refused, released = 0, 0, 0
    while step < 24:
        done = [1 if l > 0 and (l > 300 or r.random() < 0.08) else 0 for l in length]
        back = ref.release(table, length, free, n_free, done, page, n_pages)
        ctx.page_release(pg, i32(done))
        free, length, n_free = back[0], back[1], len(back[0])
        released += sum(done)
        for b in range(B):
            if done[b]:
                rows[b] = []
        n_new = [r.choice([1, 1, 1, 0]) if length[b] else r.choice([0, 1, 2, 37, 128, 130]) for b in range(B)]
        if step % 5 == 2:  # a chunk behind what is cached
            n_new[r.randrange(B)] += r.choice([2, 33, 100])
        want = ref.plan(table, length, free, n_free, n_new, page, n_prefix, sum(n_new) + pad, n_pages)
        begin, slot, pos = ctx.page_plan(pg, i32(n_new), n_rows=sum(n_new) + pad, pos0=n_prefix)
        if want is None:  # too few pages: nothing has changed, the step is tried again with what the next releases leave
            assert ctx.check_status() == 2
            assert pg.length.tolist() == length and pg.n_free.tolist() == [n_free]
            refused += 1
            length_before = max(range(B), key=lambda b: length[b])
            back = ref.release(table, length, free, n_free, [int(b == length_before) for b in range(B)], page, n_pages)
            ctx.page_release(pg, i32([int(b == length_before) for b in range(B)]))
            free, length, n_free = back[0], back[1], len(back[0])
            rows[length_before] = []
            continue
        ctx.check()
        table, length, n_free = want[0], want[1], want[2]
        assert begin.tolist() == want[3] and slot.tolist() == want[4] and pos.tolist() == want[5]
        free = free[:n_free]
        N = sum(n_new) + pad
        qkv = projection(N, Hq, Hkv, 100 * page + step)
        q = torch.full((N, Hq, D), 2.0, dtype=torch.bfloat16, device=DEV)
        ctx.qk_norm_rope_kv4_paged_append(cache, qkv, gq, gk, 1e-5, pos, slot, 500000.0, rotate=rotate, q_out=q)
        out = torch.full((N, Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
        mn = max(n_new + [1])
        ctx.attn_kv4_paged(cache, q, begin, mn, SCALE, ctx.attn_kv4_paged_workspace(cache, N, mn), max_len=max(length) if step % 2 else 0, out=out)
        ctx.check()
        for b in range(B):
            rows[b] += [qkv[t] for t in range(want[3][b], want[3][b + 1])]
        exact, tol = ref.attention(cache, q, want[3], length, SCALE)
        n = want[3][-1]
        assert ((out[:n].double() - exact[:n]).abs() <= tol[:n]).all()
        assert (out[n:] == 9.0).all() and (q[n:] == 2.0).all()
        step += 1
    assert released > 0 and max(length) > 0
    for b in range(B):
        n = length[b]
        assert len(rows[b]) == n
        if n == 0:
            continue
        own = empty_cache(1, ref.up(n, page), page, ref.up(n, page), Hq, Hkv, steps, n_prefix, seed=page)
        own.pages.table.copy_(torch.arange(ref.up(n, page), dtype=torch.int32, device=DEV).expand(1, -1)[:, : own.pages.max_pages])
        if steps == "head":
            own.s_k.copy_(cache.s_k), own.s_v.copy_(cache.s_v)
        at = torch.arange(n, device=DEV)
        ctx.qk_norm_rope_kv4_paged_append(own, torch.stack(rows[b]), gq, gk, 1e-5, (at + n_prefix).int(), at, 500000.0, rotate=rotate)
        assert torch.equal(ctx.kv4_paged_read(cache, slots_of(cache, b, n)), ctx.kv4_paged_read(own, at))
    ctx.check()


def test_the_binding_refuses(ctx):
    """Shapes, types, strides and places that the calls do not take are refused before anything is launched."""
    cache = ref.make_cache([20, 5], 4, 2, 16, seed=4)
    pg, q, begin = cache.pages, ref.queries(3, 4), i32([0, 2, 3])
    ws = ctx.attn_kv4_paged_workspace(cache, 3, 2)
    qkv, slot, pos, (gq, gk) = projection(3, 4, 2, 1), torch.arange(3, device=DEV), i32([0, 1, 2]), gains(2)
    out = (i32([0] * 3), torch.zeros(3, dtype=torch.int64, device=DEV), i32([0] * 3))
    attn = lambda **k: ctx.attn_kv4_paged(**{**dict(cache=cache, q=q, q_begin=begin, max_new=2, sm_scale=SCALE, ws=ws), **k})
    rope = lambda **k: ctx.qk_norm_rope(**{**dict(x=q, Hq=4, gq=gq, gk=gk, eps=1e-5, pos=pos, theta=1e4), **k})
    append = lambda **k: ctx.qk_norm_rope_kv4_paged_append(**{**dict(cache=cache, qkv=qkv, gq=gq, gk=gk, eps=1e-5, pos=pos, slot=slot, theta=1e4), **k})
    plan = lambda **k: ctx.page_plan(**{**dict(pages=pg, n_new=i32([1, 2]), out=out), **k})
    state = [t.clone() for t in (cache.codes, pg.table, pg.length, pg.n_free, q)]
    for call in (lambda: attn(q=q.half()), lambda: attn(q=q.cpu()), lambda: attn(q_begin=begin.long()), lambda: attn(ws=ws.int()), lambda: attn(out=q.float()),
                 lambda: rope(x=q.float()), lambda: rope(pos=pos.long()), lambda: rope(gq=gq.float()), lambda: rope(out=q.cpu()), lambda: append(qkv=qkv.half()),
                 lambda: append(slot=pos), lambda: append(q_out=q.float()), lambda: plan(n_new=slot[:2]), lambda: plan(out=(out[0], pos, out[2])),
                 lambda: ctx.page_release(pg, slot[:2]), lambda: ctx.kv4_paged_read(cache, pos), lambda: plan(n_new=i32([1, 2]).cpu())):
        with pytest.raises(TypeError):
            call()
    wide = torch.zeros((3, 8, D), dtype=torch.bfloat16, device=DEV)
    for call in (lambda: attn(q=wide), lambda: attn(q=wide[:, ::2]), lambda: attn(q_begin=begin[:2]), lambda: attn(out=wide[:, :4]), lambda: attn(out=q[:2]),
                 lambda: rope(pos=pos[:2]), lambda: rope(gq=gq[:64]), lambda: rope(gk=None), lambda: rope(gq=None), lambda: rope(pos=i32([0] * 6)[::2]),
                 lambda: rope(pos=i32([[0] * 3] * 2), sections=[64]), lambda: rope(out=q[:2]), lambda: append(qkv=qkv[:, :-128]), lambda: append(slot=slot[:2]),
                 lambda: append(slot=torch.arange(6, device=DEV)[::2]), lambda: append(q_out=wide), lambda: plan(n_new=i32([1])), lambda: plan(n_rows=4),
                 lambda: plan(len_out=i32([0])), lambda: plan(n_free_out=i32([0, 0])), lambda: ctx.page_release(pg, i32([1])),
                 lambda: ctx.kv4_paged_read(cache, slot, out=wide)):
        with pytest.raises(AssertionError):
            call()
    ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (cache.codes, pg.table, pg.length, pg.n_free, q)))


class Loop:
    """One step of token-by-token serving on fixed buffers."""

    def __init__(self, ctx, steps, lengths, new, Hq=8, Hkv=2, page=16, spare=60, ws=None, seed=5):
        self.ctx = ctx
        self.cache = ref.make_cache(lengths, Hq, Hkv, page, steps, seed=seed, extra_pages=spare, width=max(ref.up(n, page) for n in lengths) + 60)
        self.new, self.N = i32(new), sum(new) + 2
        self.plan = (i32([0] * (len(new) + 1)), torch.zeros(self.N, dtype=torch.int64, device=DEV), i32([0] * self.N))
        self.qkv, (self.gq, self.gk) = projection(self.N, Hq, Hkv, seed), gains(seed)
        self.q = torch.zeros((self.N, Hq, D), dtype=torch.bfloat16, device=DEV)
        self.out, self.most = torch.zeros_like(self.q), max(new)
        self.ws = ctx.attn_kv4_paged_workspace(self.cache, self.N, self.most) if ws is None else ws

    def step(self):
        self.ctx.page_plan(self.cache.pages, self.new, out=self.plan)
        self.ctx.qk_norm_rope_kv4_paged_append(self.cache, self.qkv, self.gq, self.gk, 1e-5, self.plan[2], self.plan[1], 1e4, q_out=self.q)
        self.ctx.attn_kv4_paged(self.cache, self.q, self.plan[0], self.most, SCALE, self.ws, out=self.out)

    def state(self):
        c = self.cache
        return [c.codes, c.pages.table, c.pages.length, c.pages.free_list, c.pages.n_free, self.out] + ([c.steps] if c.steps is not None else [])

    def captured(self):
        """The step as a graph; the state is what it was before."""
        keep = [t.clone() for t in self.state()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()  # (loads the kernels)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        for t, k in zip(self.state(), keep):
            t.copy_(k)
        return graph


SERVED = [([700, 3, 64, 0], [1, 1, 1, 1]), ([9000, 50], [1, 1]), ([300, 0, 17, 4000], [40, 130, 1, 3])]


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,new", SERVED)
def test_replays_of_a_captured_step_are_the_eager_steps(ctx, steps, lengths, new):
    """The plan advances the state in place: every replay is the next step."""
    eager, graphed = (Loop(ctx, steps, lengths, new) for _ in range(2))
    graph = graphed.captured()
    for _ in range(5):
        eager.step()
        graph.replay()
        ctx.check()
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), graphed.state()))
    assert eager.cache.pages.length.tolist() == [l + 5 * n for l, n in zip(lengths, new)]


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_two_graphs_share_a_workspace(ctx, steps):
    """Captured against one workspace and replayed in turn on one stream without a wait between them."""
    need = max((Loop(ctx, steps, *s).ws for s in SERVED), key=lambda t: t.numel())
    ws = torch.full_like(need, 0xFF)  # what a workspace holds before a call does not matter: here NaN
    alone, shared = [Loop(ctx, steps, *s) for s in SERVED], [Loop(ctx, steps, *s, ws=ws) for s in SERVED]
    graphs = [s.captured() for s in shared]
    for _ in range(4):
        for a in alone:
            a.step()
        for g in graphs:
            g.replay()
    ctx.check()
    for a, s in zip(alone, shared):
        assert all(torch.equal(x, y) for x, y in zip(a.state(), s.state()))


@pytest.mark.parametrize("which", [(0, 1), (2, 2), (1, 2)])
def test_two_contexts_on_two_streams(ctx, which):
    other = binding.Context()
    served = [SERVED[w] for w in which]
    ref_loops, loops = [Loop(ctx, "vector", *s) for s in served], [Loop(c, "vector", *s) for c, s in zip((ctx, other), served)]
    for l in ref_loops:
        for _ in range(5):
            l.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in loops]
    for _ in range(5):
        for l, s in zip(loops, streams):
            with torch.cuda.stream(s):
                l.step()
    for l, s in zip(loops, streams):
        with torch.cuda.stream(s):
            l.ctx.check()
    for a, b in zip(ref_loops, loops):
        assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))
    other.close()


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_calls_in_a_row_are_in_order(ctx, steps):
    """Calls back to back give what they give with a wait after each: the kernels for single tokens and for several rows run beside one another, and neither
    may begin before the append ends or end after its successor begins."""
    runs = []
    for sync in (False, True):
        loop, outs = Loop(ctx, steps, [500, 0, 2000, 90], [1, 60, 1, 5]), []
        for i in range(8):
            loop.qkv.copy_(projection(loop.N, 8, 2, 40 + i))
            loop.step()
            if sync:
                torch.cuda.synchronize()
            outs.append(loop.out.clone())
            loop.out.zero_()
        ctx.check()
        runs.append(outs + loop.state())
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_a_wait_that_runs_out_is_reported_and_the_context_stays_usable():
    ctx = binding.Context()
    seen = []
    for steps in ("head", "vector"):
        for lengths, new in SERVED + [([3000], [700])]:
            loop = Loop(ctx, steps, lengths, new)
            loop.step()
            ctx.check()
            good = loop.out.clone()
            for limit in (16, 2000):
                ctx.set_wait_limit(limit)  # a few clocks: no copy from memory is that fast
                ctx.attn_kv4_paged(loop.cache, loop.q, loop.plan[0], loop.most, SCALE, loop.ws, out=loop.out)
                seen.append(ctx.check_status())
                assert ctx.check_status() == 0
                ctx.set_wait_limit(0)
                ctx.attn_kv4_paged(loop.cache, loop.q, loop.plan[0], loop.most, SCALE, loop.ws, out=loop.out)
                assert ctx.check_status() == 0 and torch.equal(loop.out, good)
    assert all(s in (0, PQ_ERR_TIMEOUT) for s in seen), seen
    ctx.close()


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_nothing_to_do(ctx, steps):
    cache = ref.make_cache([0, 0], 4, 2, 16, steps, n_prefix=0, extra_pages=2)
    pg = cache.pages
    begin, slot, pos = ctx.page_plan(pg, i32([0, 0]), n_rows=0)
    assert begin.tolist() == [0, 0, 0] and slot.numel() == pos.numel() == 0
    ctx.page_release(pg, i32([1, 1]))
    empty = torch.empty((0, 8 * D), dtype=torch.bfloat16, device=DEV)
    assert ctx.qk_norm_rope_kv4_paged_append(cache, empty, None, None, 0.0, pos, slot, 1e4).shape == (0, 4, D)
    assert ctx.qk_norm_rope(empty.view(0, 8, D), 4, None, None, 0.0, pos, 1e4).shape == (0, 8, D)
    assert ctx.kv4_paged_read(cache, slot).shape == (0, 2, 2, D)
    ws = ctx.attn_kv4_paged_workspace(cache, 0, 1)
    assert ctx.attn_kv4_paged(cache, torch.empty((0, 4, D), dtype=torch.bfloat16, device=DEV), begin, 1, SCALE, ws).shape == (0, 4, D)
    # rows of a step that no sequence has stay as they are
    out = torch.full((3, 4, D), 9.0, dtype=torch.bfloat16, device=DEV)
    for mn in (1, 3):
        ctx.attn_kv4_paged(cache, ref.queries(3, 4), begin, mn, SCALE, ctx.attn_kv4_paged_workspace(cache, 3, mn), out=out)
    ctx.check()
    assert (out == 9.0).all() and pg.n_free.tolist() == [2]
    # no sequences at all
    none = binding.KV4PagedCache(binding.Pages(torch.zeros((0, 4), dtype=torch.int32, device=DEV), i32([]), pg.free_list, pg.n_free, 16), None, None,
                                 cache.codes, 4, s_k=cache.s_k, s_v=cache.s_v, steps=cache.steps)
    begin, slot, pos = ctx.page_plan(none.pages, i32([]), n_rows=2)
    ctx.page_release(none.pages, i32([]))
    ctx.attn_kv4_paged(none, ref.queries(3, 4), begin, 2, SCALE, ctx.attn_kv4_paged_workspace(none, 3, 2), out=out)
    ctx.check()
    assert begin.tolist() == [0] and slot.tolist() == [-1, -1] and (out == 9.0).all()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,new,Hq,Hkv", [([700, 3, 9000, 40], [1, 1, 1, 1], 8, 2), ([40], [1], 8, 8), ([700, 300, 20, 9000], [700, 1, 20, 33], 16, 4),
                                                ([6000], [300], 6, 2)])
def test_the_output_may_be_the_queries(ctx, steps, lengths, new, Hq, Hkv):
    cache = ref.make_cache(lengths, Hq, Hkv, 16, steps, seed=3)
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    q = ref.queries(begin[-1], Hq)
    ws = ctx.attn_kv4_paged_workspace(cache, begin[-1], max(new))
    want = ctx.attn_kv4_paged(cache, q, i32(begin), max(new), SCALE, ws)
    assert torch.equal(ctx.attn_kv4_paged(cache, q, i32(begin), max(new), SCALE, ws, out=q), want)
    ctx.check()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("lengths,bound,Hq,Hkv,n_prefix", [([5000], 0, 8, 8, 4), ([12000], 12000, 32, 8, 1), ([3200, 5000], 0, 16, 4, 0), ([0], 6000, 8, 1, 64), ([1], 6000, 8, 1, 0),
                                                           ([130, 4097], 9000, 14, 2, 5), ([9, 700, 33], 4000, 3, 3, 2)])
def test_few_long_sequences(ctx, steps, lengths, bound, Hq, Hkv, n_prefix):
    """Wide clusters to a (sequence, KV head), most of whose CTAs may have nothing to do."""
    cache = ref.make_cache(lengths, Hq, Hkv, 16, steps, n_prefix, seed=11, width=max(ref.up(max(lengths + [bound]), 16), 1))
    B = len(lengths)
    q, begin = ref.queries(B, Hq), list(range(B + 1))
    out = ctx.attn_kv4_paged(cache, q, i32(begin), 1, SCALE, ctx.attn_kv4_paged_workspace(cache, B, 1), max_len=bound)
    again = ctx.attn_kv4_paged(cache, q, i32(begin), 1, SCALE, ctx.attn_kv4_paged_workspace(cache, B, 1), max_len=bound)
    ctx.check()
    want, tol = ref.attention(cache, q, begin, lengths, SCALE)
    assert ((out.double() - want).abs() <= tol).all() and torch.equal(out, again)


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("ragged", [False, True])
def test_the_largest_batch(ctx, steps, ragged):
    """8192 sequences of a few tokens, single rows or several; a sample of them against the definition."""
    r = random.Random(5)
    B = 8192
    new = [r.choice([0, 1, 2, 5]) if ragged else r.choice([0, 1, 1, 1]) for _ in range(B)]
    lengths = [n + r.choice([0, 0, 3, 17, 60]) for n in new]
    cache = ref.make_cache(lengths, 3, 1, 16, steps, n_prefix=1, seed=7)
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    q = ref.queries(begin[-1], 3)
    out = ctx.attn_kv4_paged(cache, q, i32(begin), 5 if ragged else 1, SCALE, ctx.attn_kv4_paged_workspace(cache, begin[-1], 5 if ragged else 1))
    ctx.check()
    for lo in (0, 1000, 4095, B - 40):
        some = range(lo, lo + 40)
        part = binding.KV4PagedCache(binding.Pages(cache.pages.table[lo: lo + 40].contiguous(), cache.pages.length[lo: lo + 40].contiguous(), cache.pages.free_list,
                                                   cache.pages.n_free, 16), cache.prefix_k, cache.prefix_v, cache.codes, 3, s_k=cache.s_k, s_v=cache.s_v,
                                     steps=cache.steps)
        r0, r1 = begin[lo], begin[lo + 40]
        want, tol = ref.attention(part, q[r0:r1], [begin[b] - r0 for b in some] + [r1 - r0], [lengths[b] for b in some], SCALE)
        assert ((out[r0:r1].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("steps", ["head", "vector"])
def test_offsets_past_32_bits(ctx, steps):
    """A cache of more than 2^32 bytes whose pages in use lie at its end, query rows that are 2^30 elements apart."""
    Hq, Hkv, page, n_pages = 8, 4, 128, 70000
    lengths, new, rows = [333, 40], [3, 1], 4
    codes = torch.zeros((n_pages, Hkv, 2, page, D // 2), dtype=torch.uint8, device=DEV)
    assert codes.numel() > 2**32
    small = ref.make_cache(lengths, Hq, Hkv, page, steps, seed=1, width=4)
    assert small.codes.shape[0] < 40
    far = n_pages - 40
    codes[far: far + small.codes.shape[0]] = small.codes
    st = None
    if steps == "vector":
        st = torch.ones((n_pages, Hkv, 2, page), device=DEV)
        st[far: far + small.codes.shape[0]] = small.steps
    table = torch.where(small.pages.table >= 0, small.pages.table + far, small.pages.table)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[0] = n_pages - 1
    big = binding.KV4PagedCache(binding.Pages(table, small.pages.length.clone(), free, i32([1]), page), small.prefix_k, small.prefix_v, codes, Hq,
                                s_k=small.s_k, s_v=small.s_v, steps=st)
    q = ref.queries(rows, Hq)
    wide = torch.empty((rows - 1) * 2**30 + Hq * D, dtype=torch.bfloat16, device=DEV).as_strided((rows, Hq, D), (2**30, D, 1))
    wide.copy_(q)
    begin = i32([0, 3, 4])
    ws = ctx.attn_kv4_paged_workspace(big, rows, 3)
    a, b = ctx.attn_kv4_paged(small, q, begin, 3, SCALE, ws), ctx.attn_kv4_paged(big, wide, begin, 3, SCALE, ws)
    ctx.check()
    assert torch.equal(a, b)
    # a new token on the very last page, written and read there
    begin, slot, pos = ctx.page_plan(big.pages, i32([52, 0]), n_rows=52)
    assert slot.tolist()[51] == (n_pages - 1) * page and big.pages.table[0, 3].item() == n_pages - 1
    qkv, (gq, gk) = projection(52, Hq, Hkv, 3), gains(1)
    ctx.qk_norm_rope_kv4_paged_append(big, qkv, gq, gk, 1e-5, pos, slot, 1e4)
    own = empty_cache(1, 1, 128, 1, Hq, Hkv, steps, 0)
    if steps == "head":
        own.s_k.copy_(big.s_k), own.s_v.copy_(big.s_v)
    at = torch.arange(52, device=DEV)
    ctx.qk_norm_rope_kv4_paged_append(own, qkv, gq, gk, 1e-5, pos, at, 1e4)
    assert torch.equal(ctx.kv4_paged_read(big, slot), ctx.kv4_paged_read(own, at))
    ctx.check()
