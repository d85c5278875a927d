"""Arguments that the paged KV4 entry points refuse, checked without a GPU: a refused call returns before it touches the device. The
context is a zeroed block of memory that only the checks look at."""
import ctypes

import pytest

from paper_2410_05265_b200 import binding, build

OK, INVALID, SHAPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4
AT = 1 << 20  # an aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.fixture
def ctx():
    block = (ctypes.c_char * 256)()
    yield ctypes.cast(block, ctypes.c_void_p)


def pages(**kw):
    a = dict(table=AT, len=AT, free_list=AT, n_free=AT, B=4, max_pages=8, page=16, n_pages=40)
    a.update(kw)
    return binding.PagesStruct(*(a[n] for n, _ in binding.PagesStruct._fields_))


def cache(pg=None, **kw):
    a = dict(pages=pg or pages(), prefix_k=AT, prefix_v=AT, codes=AT, steps=0, s_k=AT, s_v=AT, Hq=8, Hkv=2, D=128, n_prefix=4)
    a.update(kw)
    return binding.KV4PagedStruct(*(a[n] for n, _ in binding.KV4PagedStruct._fields_))


BAD_PAGES = [(dict(table=0), INVALID), (dict(len=0), INVALID), (dict(free_list=0), INVALID), (dict(n_free=0), INVALID), (dict(B=-1), INVALID),
             (dict(max_pages=-1), INVALID), (dict(n_pages=-1), INVALID), (dict(page=8), SHAPE), (dict(page=48), SHAPE), (dict(page=0), SHAPE),
             (dict(B=8193), SHAPE), (dict(max_pages=1 << 27), SHAPE)]
BAD_CACHE = [(dict(codes=0), INVALID), (dict(s_k=0), INVALID), (dict(s_v=0), INVALID), (dict(prefix_k=0), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
             (dict(n_prefix=-1), INVALID), (dict(D=64), SHAPE), (dict(Hq=9), SHAPE), (dict(Hq=18), SHAPE), (dict(n_prefix=65), SHAPE),
             (dict(codes=AT + 8), ALIGN), (dict(steps=AT + 4), ALIGN), (dict(prefix_v=AT + 2), ALIGN)]


def plan(lib, ctx, pg, **kw):
    a = dict(n_new=AT, pos0=0, n_rows=10, q_begin=AT, slot=AT, pos=AT, len_out=AT, n_free_out=AT)
    a.update(kw)
    return lib.pq_page_plan(ctx, ctypes.byref(pg), a["n_new"], a["pos0"], a["n_rows"], a["q_begin"], a["slot"], a["pos"], a["len_out"], a["n_free_out"], None)


@pytest.mark.parametrize("kw,want", BAD_PAGES)
def test_page_calls_refuse_bad_tables(lib, ctx, kw, want):
    pg = pages(**kw)
    assert plan(lib, ctx, pg) == want
    assert lib.pq_page_release(ctx, ctypes.byref(pg), AT, AT, AT, None) == want
    assert lib.pq_kv4_paged_read(ctx, ctypes.byref(cache(pg)), AT, 3, AT, None) == want
    assert attn(lib, ctx, cache(pg)) == want
    assert append(lib, ctx, cache(pg)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n_new=0), INVALID), (dict(q_begin=0), INVALID), (dict(slot=0), INVALID), (dict(pos=0), INVALID), (dict(len_out=0), INVALID),
    (dict(n_free_out=0), INVALID), (dict(n_rows=-1), INVALID), (dict(pos0=-1), INVALID), (dict(n_rows=1 << 31), SHAPE), (dict(pos0=2**31 - 100), SHAPE),
    (dict(slot=AT + 8), ALIGN), (dict(pos=AT + 4), ALIGN),
])
def test_page_plan_refuses(lib, ctx, kw, want):
    assert plan(lib, ctx, pages(), **kw) == want
    assert lib.pq_page_plan(None, ctypes.byref(pages()), AT, 0, 1, AT, AT, AT, AT, AT, None) == INVALID


def test_page_release_refuses(lib, ctx):
    pg = ctypes.byref(pages())
    for args in ((0, AT, AT), (AT, 0, AT), (AT, AT, 0)):
        assert lib.pq_page_release(ctx, pg, *args, None) == INVALID
    assert lib.pq_page_release(None, pg, AT, AT, AT, None) == INVALID


def rope(lib, ctx, **kw):
    a = dict(x=AT, N=5, Hq=4, Hk=2, D=128, ld=6 * 128, gq=AT, gk=AT, eps=1e-5, pos=AT, axes=1, ld_pos=5, sections=None, theta=1e4, rotate=0, y=2 * AT, ldy=6 * 128)
    a.update(kw)
    sec = (ctypes.c_int32 * len(a["sections"]))(*a["sections"]) if a["sections"] is not None else None
    return lib.pq_qk_norm_rope(ctx, a["x"], a["N"], a["Hq"], a["Hk"], a["D"], a["ld"], a["gq"], a["gk"], a["eps"], a["pos"], a["axes"], a["ld_pos"], sec,
                               a["theta"], a["rotate"], a["y"], a["ldy"], None)


BAD_ROPE = [(dict(x=0), INVALID), (dict(pos=0), INVALID), (dict(gq=0), INVALID), (dict(gk=0), INVALID), (dict(N=-1), INVALID), (dict(eps=-1.0), INVALID),
            (dict(eps=float("nan")), INVALID), (dict(theta=0.0), INVALID), (dict(theta=float("inf")), INVALID), (dict(axes=0), INVALID), (dict(axes=4), INVALID),
            (dict(axes=2), INVALID), (dict(axes=2, sections=[32, 32], ld_pos=4), INVALID), (dict(axes=2, sections=[70, -6]), INVALID),
            (dict(axes=3, sections=[16, 24, 23]), SHAPE), (dict(axes=1, sections=[63]), SHAPE), (dict(ld=5 * 128), INVALID), (dict(ld=6 * 128 + 4), ALIGN)]


@pytest.mark.parametrize("kw,want", BAD_ROPE + [(dict(y=0), INVALID), (dict(Hq=-1), INVALID), (dict(Hq=0, Hk=0), INVALID), (dict(D=64), SHAPE), (dict(ldy=128), INVALID),
                                                (dict(y=AT, ldy=8 * 128), INVALID), (dict(x=AT + 8), ALIGN), (dict(y=AT + 2), ALIGN), (dict(gq=AT + 8), ALIGN)])
def test_qk_norm_rope_refuses(lib, ctx, kw, want):
    assert rope(lib, ctx, **kw) == want


def append(lib, ctx, c, **kw):
    a = dict(x=AT, N=5, ld=12 * 128, gq=AT, gk=AT, eps=1e-5, pos=AT, axes=1, ld_pos=5, sections=None, theta=1e4, rotate=0, slot=AT, q_out=2 * AT, ldq=8 * 128)
    a.update(kw)
    sec = (ctypes.c_int32 * len(a["sections"]))(*a["sections"]) if a["sections"] is not None else None
    return lib.pq_qk_norm_rope_kv4_paged_append(ctx, ctypes.byref(c), a["x"], a["N"], a["ld"], a["gq"], a["gk"], a["eps"], a["pos"], a["axes"], a["ld_pos"], sec,
                                                a["theta"], a["rotate"], a["slot"], a["q_out"], a["ldq"], None)


@pytest.mark.parametrize("kw,want", [(k, w) for k, w in BAD_ROPE if "ld" not in k] + [
    (dict(slot=0), INVALID), (dict(q_out=0), INVALID), (dict(ld=11 * 128), INVALID), (dict(ldq=7 * 128), INVALID), (dict(q_out=AT), INVALID),
    (dict(ld=12 * 128 + 4), ALIGN), (dict(q_out=2 * AT + 4), ALIGN)])
def test_append_refuses(lib, ctx, kw, want):
    assert append(lib, ctx, cache(), **kw) == want


def attn(lib, ctx, c, **kw):
    a = dict(q=AT, ldq=8 * 128, q_begin=AT, n_rows=6, max_new=3, max_len=0, out=AT, scale=0.1, ws=AT, ws_bytes=1 << 40)
    a.update(kw)
    return lib.pq_attn_kv4_paged(ctx, ctypes.byref(c), a["q"], a["ldq"], a["q_begin"], a["n_rows"], a["max_new"], a["max_len"], a["out"], a["scale"], a["ws"],
                                 a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_cache_calls_refuse_bad_caches(lib, ctx, kw, want):
    c = cache(**kw)
    assert attn(lib, ctx, c, ldq=18 * 128) == want
    assert append(lib, ctx, c, ld=30 * 128, ldq=18 * 128) == want
    assert lib.pq_kv4_paged_read(ctx, ctypes.byref(c), AT, 3, AT, None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=0), INVALID), (dict(q_begin=0), INVALID), (dict(out=0), INVALID), (dict(n_rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(max_len=-1), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(ldq=7 * 128), INVALID),
    (dict(n_rows=1 << 31), SHAPE), (dict(q=AT + 8), ALIGN), (dict(out=AT + 8), ALIGN), (dict(ws=AT + 8), ALIGN), (dict(ldq=8 * 128 + 4), ALIGN), (dict(ws=0), WORKSPACE),
])
def test_attention_refuses(lib, ctx, kw, want):
    assert attn(lib, ctx, cache(), **kw) == want


def test_read_refuses(lib, ctx):
    c = ctypes.byref(cache())
    assert lib.pq_kv4_paged_read(ctx, c, AT, -1, AT, None) == INVALID
    assert lib.pq_kv4_paged_read(ctx, c, 0, 3, AT, None) == INVALID
    assert lib.pq_kv4_paged_read(ctx, c, AT, 3, 0, None) == INVALID
    assert lib.pq_kv4_paged_read(ctx, c, AT, 3, AT + 8, None) == ALIGN


def test_calls_without_rows_do_nothing(lib, ctx):
    """No launch (there may be no device): the status is that of a call that has nothing to do."""
    assert rope(lib, ctx, N=0, x=0, y=0, pos=0) == OK
    assert append(lib, ctx, cache(), N=0, x=0, q_out=0, slot=0) == OK
    assert lib.pq_kv4_paged_read(ctx, ctypes.byref(cache()), 0, 0, 0, None) == OK
    assert attn(lib, ctx, cache(), n_rows=0, q=0, out=0) == OK
    assert attn(lib, ctx, cache(pages(B=0))) == OK
    assert attn(lib, ctx, cache(), max_new=0) == OK


def test_workspace_of_nothing_is_nothing(lib, ctx):
    assert lib.pq_attn_kv4_paged_workspace_bytes(None, ctypes.byref(cache()), 4, 1) == 0
    assert lib.pq_attn_kv4_paged_workspace_bytes(ctx, ctypes.byref(cache(D=64)), 4, 1) == 0
    assert lib.pq_attn_kv4_paged_workspace_bytes(ctx, ctypes.byref(cache()), 0, 1) == 0


def test_in_place_with_another_stride_is_refused_of_several_rows_only(lib, ctx):
    """The distance of a single row says nothing: the next thing to refuse (here gains that are not aligned) is reached."""
    assert append(lib, ctx, cache(), N=2, q_out=AT, gq=AT + 8) == INVALID
    assert append(lib, ctx, cache(), N=1, q_out=AT, gq=AT + 8) == ALIGN
    assert rope(lib, ctx, N=2, y=AT, ldy=8 * 128, gq=AT + 8) == INVALID
    assert rope(lib, ctx, N=1, y=AT, ldy=8 * 128, gq=AT + 8) == ALIGN
