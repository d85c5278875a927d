"""What the entry points of windowed attention and of drafted trees refuse, checked without a GPU (a refused call returns before it touches the device), their order
under programmatic dependent launch, read from the sources, and tables and caches on another device."""
import ctypes
import re

import pytest
import torch

from test_launch_order import TRIGGER, kernel_body
from test_paged_devices import Fake, cache_on, ctx as fake_ctx, pages_on  # noqa: F401 (a fixture)
from test_paged_refusals import ALIGN, AT, BAD_CACHE, BAD_PAGES, INVALID, OK, SHAPE, WORKSPACE, cache, ctx, lib, pages  # noqa: F401 (fixtures)


def window(lib, ctx, c, **kw):
    a = dict(q=AT, ldq=8 * 128, q_begin=AT, n_rows=6, max_new=3, max_len=0, window=5, n_sink=0, out=AT, scale=0.1, ws=AT, ws_bytes=1 << 40)
    a.update(kw)
    return lib.pq_attn_kv4_paged_window(ctx, ctypes.byref(c), a["q"], a["ldq"], a["q_begin"], a["n_rows"], a["max_new"], a["max_len"], a["window"], a["n_sink"],
                                        a["out"], a["scale"], a["ws"], a["ws_bytes"], None)


def tree(lib, ctx, c, **kw):
    a = dict(q=AT, ldq=8 * 128, q_begin=AT, n_rows=6, max_new=3, max_len=0, mask=AT, words=1, window=0, n_sink=0, out=AT, scale=0.1, ws=AT, ws_bytes=1 << 40)
    a.update(kw)
    return lib.pq_attn_kv4_paged_tree(ctx, ctypes.byref(c), a["q"], a["ldq"], a["q_begin"], a["n_rows"], a["max_new"], a["max_len"], a["mask"], a["words"], a["window"],
                                      a["n_sink"], a["out"], a["scale"], a["ws"], a["ws_bytes"], None)


def plan(lib, ctx, pg, **kw):
    a = dict(parent=AT, q_begin=AT, n_rows=10, pos0=0, mask=AT, words=1, pos=AT)
    a.update(kw)
    return lib.pq_tree_plan(ctx, ctypes.byref(pg), a["parent"], a["q_begin"], a["n_rows"], a["pos0"], a["mask"], a["words"], a["pos"], None)


def accept(lib, ctx, **kw):
    a = dict(q_begin=AT, B=4, parent=AT, draft=AT, target=AT, n_rows=10, kept=AT, n_kept=AT, next=AT)
    a.update(kw)
    return lib.pq_tree_accept(ctx, a["q_begin"], a["B"], a["parent"], a["draft"], a["target"], a["n_rows"], a["kept"], a["n_kept"], a["next"], None)


def keep(lib, ctx, pg, q_begin=AT, n_kept=AT, len_out=AT, n_free_out=AT):
    return lib.pq_page_keep(ctx, ctypes.byref(pg), q_begin, n_kept, len_out, n_free_out, None)


def move(lib, ctx, c, q_begin=AT, kept=AT, n_kept=AT, n_rows=6):
    return lib.pq_kv4_paged_keep(ctx, ctypes.byref(c), q_begin, kept, n_kept, n_rows, None)


@pytest.mark.parametrize("kw,want", BAD_PAGES)
def test_bad_tables(lib, ctx, kw, want):
    pg = pages(**kw)
    assert plan(lib, ctx, pg) == want and keep(lib, ctx, pg) == want
    assert move(lib, ctx, cache(pg)) == want and window(lib, ctx, cache(pg)) == want and tree(lib, ctx, cache(pg)) == want


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_bad_caches(lib, ctx, kw, want):
    c = cache(**kw)
    assert move(lib, ctx, c) == want and window(lib, ctx, c, ldq=18 * 128) == want and tree(lib, ctx, c, ldq=18 * 128) == want


ATTENTION = [
    (dict(q=0), INVALID), (dict(q_begin=0), INVALID), (dict(out=0), INVALID), (dict(n_rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(max_len=-1), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(ldq=7 * 128), INVALID), (dict(n_rows=1 << 31), SHAPE),
    (dict(q=AT + 8), ALIGN), (dict(out=AT + 8), ALIGN), (dict(ws=AT + 8), ALIGN), (dict(ldq=8 * 128 + 4), ALIGN), (dict(ws=0), WORKSPACE), (dict(n_sink=-1), INVALID),
    (dict(window=-1), INVALID)]


@pytest.mark.parametrize("kw,want", ATTENTION + [(dict(window=0), INVALID)])
def test_window_refuses(lib, ctx, kw, want):
    assert window(lib, ctx, cache(), **kw) == want


@pytest.mark.parametrize("kw,want", ATTENTION + [(dict(mask=0), INVALID), (dict(words=-1), INVALID), (dict(words=0), SHAPE), (dict(max_new=33), SHAPE),
                                                 (dict(max_new=129, words=5), SHAPE), (dict(window=2), SHAPE)])
def test_tree_attention_refuses(lib, ctx, kw, want):
    assert tree(lib, ctx, cache(), **kw) == want


@pytest.mark.parametrize("kw,want", [(dict(parent=0), INVALID), (dict(q_begin=0), INVALID), (dict(mask=0), INVALID), (dict(pos=0), INVALID), (dict(n_rows=-1), INVALID),
                                     (dict(pos0=-1), INVALID), (dict(words=0), INVALID), (dict(words=5), SHAPE), (dict(n_rows=1 << 31), SHAPE), (dict(pos0=2**31 - 100), SHAPE)])
def test_tree_plan_refuses(lib, ctx, kw, want):
    assert plan(lib, ctx, pages(), **kw) == want
    assert plan(lib, None, pages()) == INVALID


@pytest.mark.parametrize("kw,want", [(dict(q_begin=0), INVALID), (dict(B=-1), INVALID), (dict(parent=0), INVALID), (dict(draft=0), INVALID), (dict(target=0), INVALID),
                                     (dict(kept=0), INVALID), (dict(n_kept=0), INVALID), (dict(next=0), INVALID), (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 31), SHAPE),
                                     (dict(B=8193), SHAPE)])
def test_tree_accept_refuses(lib, ctx, kw, want):
    assert accept(lib, ctx, **kw) == want
    assert accept(lib, None) == INVALID


def test_keeping_refuses(lib, ctx):
    for kw in (dict(q_begin=0), dict(n_kept=0), dict(len_out=0), dict(n_free_out=0)):
        assert keep(lib, ctx, pages(), **kw) == INVALID
    for kw in (dict(q_begin=0), dict(kept=0), dict(n_kept=0), dict(n_rows=-1)):
        assert move(lib, ctx, cache(), **kw) == INVALID
    assert keep(lib, None, pages()) == INVALID and move(lib, None, cache()) == INVALID and move(lib, ctx, cache(), n_rows=1 << 31) == SHAPE


def test_calls_without_rows_do_nothing(lib, ctx):
    for kw in (dict(n_rows=0, q=0, out=0), dict(max_new=0)):
        assert window(lib, ctx, cache(), **kw) == OK and tree(lib, ctx, cache(), **kw) == OK
    assert tree(lib, ctx, cache(pages(B=0))) == OK and window(lib, ctx, cache(pages(B=0))) == OK
    assert plan(lib, ctx, pages(), n_rows=0, parent=0, mask=0, pos=0) == OK
    assert accept(lib, ctx, B=0, n_rows=0, q_begin=0, parent=0, draft=0, target=0, kept=0, n_kept=0, next=0) == OK
    assert move(lib, ctx, cache(), n_rows=0, kept=0) == OK and move(lib, ctx, cache(pages(B=0))) == OK


def test_workspace_of_nothing_is_nothing(lib, ctx):
    assert lib.pq_attn_kv4_paged_tree_workspace_bytes(None, ctypes.byref(cache()), 4, 1) == 0
    assert lib.pq_attn_kv4_paged_tree_workspace_bytes(ctx, ctypes.byref(cache(D=64)), 4, 1) == 0
    assert lib.pq_attn_kv4_paged_tree_workspace_bytes(ctx, ctypes.byref(cache()), 0, 1) == 0


@pytest.mark.parametrize("source,name", [("pq_pages.cu", "page_keep_kernel"), ("pq_tree.cu", "kv4_paged_keep_kernel")])
def test_writers_of_lengths_and_caches_never_trigger(source, name):
    assert not TRIGGER.search(kernel_body(source, name))


@pytest.mark.parametrize("source,name", [("pq_pages.cu", "page_keep_kernel"), ("pq_tree.cu", "kv4_paged_keep_kernel"), ("pq_tree.cu", "tree_plan_kernel"),
                                         ("pq_tree.cu", "tree_accept_kernel"), ("pq_paged_tree.cu", "paged_tree_kernel")])
def test_the_wait_comes_before_every_read_and_before_the_trigger(source, name):
    body = kernel_body(source, name)
    wait = body.index("pdl_wait")
    assert wait < re.search(r"ld_dep|__ldcg|tma_load|cp_async|tree_rows|padding_rows|report\(", body).start()
    trigger = TRIGGER.search(body)
    assert trigger is None or wait < trigger.start()
    assert "__ldg(" not in body and "ld.global.nc" not in body


def test_a_cache_of_another_device_is_refused(fake_ctx):  # noqa: F811
    c = fake_ctx
    t = lambda dtype, *shape: Fake(dtype, shape, 0)
    i32, bf16, u8 = torch.int32, torch.bfloat16, torch.uint8
    q, out, ws, begin, mask = t(bf16, 5, 4, 128), t(bf16, 5, 4, 128), t(u8, 100), t(i32, 3), t(i32, 5, 1)
    calls = {
        "pq_attn_kv4_paged_window": lambda at: c.attn_kv4_paged_window(cache_on(at), q, begin, 3, 9, 0.1, ws, out=out),
        "pq_attn_kv4_paged_tree": lambda at: c.attn_kv4_paged_tree(cache_on(at), q, begin, 3, mask, 0.1, ws, out=out),
        "pq_tree_plan": lambda at: c.tree_plan(pages_on(at), t(i32, 5), begin, out=(mask, t(i32, 5))),
        "pq_page_keep": lambda at: c.page_keep(pages_on(at), begin, t(i32, 2)),
        "pq_kv4_paged_keep": lambda at: c.kv4_paged_keep(cache_on(at), begin, t(i32, 5), t(i32, 2)),
        "pq_tree_accept": lambda at: c.tree_accept(begin, t(i32, 5), t(i32, 5), t(i32, 5), out=(Fake(i32, (5,), at), t(i32, 2), t(i32, 2))),
    }
    for name, call in calls.items():
        c.called.clear()
        call(0)
        assert c.called == [name]
        with pytest.raises(ValueError):
            call(1)
        assert c.called == [name]
