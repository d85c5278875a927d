"""The operators of paged KV4 serving on representative calls: block tables and slot maps built on the GPU, norm and rotary position of the
query and key heads in one pass (with the write into the paged 4-bit cache), attention over that cache.

Head counts are those of the Llama-3-8B and Llama-3-70B layers of `inputs.py` (32 and 64 query heads on 8 KV heads) and, in drawn cases,
a few other ratios; four prefixed tokens stay in fp16, as everywhere in this repository.

    listed()  the fixed cases          draw(rng)  one more case of the same ranges
    prepare   inputs, caches, output buffers
    run       one pass: the plain form with elementary torch operations, or (own) the calls of the framework
    exact     the same results in 64 bits, written from the definitions row by row
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

D = 128
DEV = "cuda"
THETA = 500000.0
EPS = 1e-5
N_PREFIX = 4  # prefixed tokens, fp16, seen by every sequence
SECTIONS = (16, 24, 24)  # rotary frequencies that follow the time, the height and the width of a token with three positions
SM_SCALE = 1.0 / math.sqrt(D)


def listed():
    return [
        # scheduler step of a decode batch: every sequence gets one more token, few of them a new page
        dict(name="pages_decode_64", kind="pages", B=64, page=16, ctx=4096, new=1, fresh=0.0, ended=0.05, pad=0),
        # scheduler step of a large server: some requests end, others start with their whole prompts, the rest decode
        dict(name="pages_mixed_512", kind="pages", B=512, page=32, ctx=8192, new=2048, fresh=0.1, ended=0.1, pad=77),
        # one token of one sequence: latency
        dict(name="norm_rope_1", kind="norm_rope", N=1, Hq=32, Hkv=8, axes=1, norm=True, rotate=False),
        # a prompt with images, three positions to a token, keys rotated for 4-bit storage
        dict(name="norm_rope_axes_4099", kind="norm_rope", N=4099, Hq=64, Hkv=8, axes=3, norm=True, rotate=True),
        # a decode step's new tokens into the cache, padded to the batch of a captured graph
        dict(name="append_48", kind="append", N=48, pad=15, Hq=32, Hkv=8, page=16, axes=1, norm=True, rotate=False, steps="head", prompt=False),
        # prompts of a prefill, every cached vector with its own step
        dict(name="append_axes_6001", kind="append", N=6001, pad=143, Hq=64, Hkv=8, page=64, axes=3, norm=True, rotate=True, steps="vector", prompt=True),
        # one sequence, one token: interactive decoding
        dict(name="decode_1x1021", kind="attn", B=1, ctx=1021, ragged=False, new=1, share=0.0, pad=0, Hq=32, Hkv=8, page=16, steps="head"),
        # a batch of ragged sequences whose cached vectors carry their own steps
        dict(name="decode_48x6000", kind="attn", B=48, ctx=6000, ragged=True, new=1, share=0.0, pad=0, Hq=32, Hkv=8, page=16, steps="vector"),
        # few sequences with long caches on the large layer
        dict(name="decode_5x50000", kind="attn", B=5, ctx=50000, ragged=True, new=1, share=0.0, pad=0, Hq=64, Hkv=8, page=64, steps="head"),
        # short prompts and single tokens in one ragged batch, padded behind
        dict(name="mixed_16x515", kind="attn", B=16, ctx=515, ragged=True, new=515, share=0.5, pad=9, Hq=32, Hkv=8, page=16, steps="head"),
        # prompts of several lengths, vectors with their own steps
        dict(name="prefill_4x2000", kind="attn", B=4, ctx=2000, ragged=True, new=2000, share=1.0, pad=0, Hq=32, Hkv=8, page=32, steps="vector"),
        # one chunk of a long prompt on the large layer
        dict(name="chunk_2048_of_24000", kind="attn", B=1, ctx=24000, ragged=False, new=2048, share=1.0, pad=0, Hq=64, Hkv=8, page=64, steps="head"),
    ]


def draw(rng):
    log = lambda lo, hi: min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))
    kind = rng.choice(["pages", "norm_rope", "append", "attn", "attn", "attn"])
    Hq, Hkv = rng.choice([(32, 8), (64, 8), (32, 8), (64, 8), (8, 8), (6, 2), (5, 1), (7, 1)])
    page, steps = rng.choice([16, 32, 64, 128]), rng.choice(["head", "vector"])
    axes, norm, rotate, pad = rng.choice([1, 1, 2, 3]), rng.random() < 0.75, rng.random() < 0.5, rng.choice([0, 0, log(1, 200)])
    if kind == "pages":
        B = log(1, 512)
        return dict(kind=kind, B=B, page=page, ctx=log(16, 16384), new=rng.choice([1, log(2, 2048)]), fresh=rng.choice([0.0, 0.1, 0.5]),
                    ended=rng.choice([0.0, 0.1, 0.5]), pad=pad)
    if kind == "norm_rope":
        return dict(kind=kind, N=log(1, 4099), Hq=Hq, Hkv=Hkv, axes=axes, norm=norm, rotate=rotate)
    if kind == "append":
        return dict(kind=kind, N=log(1, 6001), pad=pad, Hq=Hq, Hkv=Hkv, page=page, axes=axes, norm=norm, rotate=rotate, steps=steps,
                    prompt=rng.random() < 0.5)
    form = rng.choice(["decode", "decode", "mixed", "prompts", "chunk"])
    ragged = rng.random() < 0.7
    if form == "decode":
        B = log(1, 128)
        return dict(kind=kind, B=B, ctx=log(1, min(60000, 250000 // B)), ragged=ragged, new=1, share=0.0, pad=pad, Hq=Hq, Hkv=Hkv, page=page, steps=steps)
    if form == "mixed":
        return dict(kind=kind, B=log(2, 32), ctx=log(17, 1500), ragged=True, new=log(2, 1500), share=0.5, pad=pad, Hq=Hq, Hkv=Hkv, page=page, steps=steps)
    if form == "prompts":
        B = log(1, 8)
        n = log(2, 4096 // B)
        return dict(kind=kind, B=B, ctx=n, ragged=ragged, new=n, share=1.0, pad=pad, Hq=Hq, Hkv=Hkv, page=page, steps=steps)
    new = log(2, 2048)
    return dict(kind=kind, B=1, ctx=log(new, 24000), ragged=False, new=new, share=1.0, pad=pad, Hq=Hq, Hkv=Hkv, page=page, steps=steps)


# ---- inputs -----------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=1)
def _ctx():
    from paper_2410_05265_b200 import binding

    return binding.Context()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 29)


def _randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _up(a, b):
    return -(-a // b)


def _plan_lengths(case):
    """(cached, new, ended) of every sequence: a fixed mixture of running, fresh, ended and idle requests."""
    r = random.Random(case["B"] * 7919 + case["ctx"])
    cached, new, ended = [], [], []
    for _ in range(case["B"]):
        u = r.random()
        n = r.randint(1, case["ctx"])
        if u < case["fresh"]:
            cached.append(0), new.append(r.randint(1, case["new"])), ended.append(0)
        elif u < case["fresh"] + case["ended"]:
            cached.append(n), new.append(0), ended.append(1)
        elif u > 0.97:  # a sequence that waits
            cached.append(n), new.append(0), ended.append(0)
        else:
            cached.append(n), new.append(1), ended.append(0)
    return cached, new, ended


def _attn_lengths(case):
    """(cached with the new ones, new) of every sequence."""
    r = random.Random(case["B"] * 104729 + case["ctx"] * 31 + case["new"])
    total, new = [], []
    for b in range(case["B"]):
        n = r.randint(max(1, case["new"] // 2), case["new"]) if case["ragged"] else case["new"]
        if r.random() >= case["share"]:
            n = 1
        t = r.randint(max(1, case["ctx"] // 4), case["ctx"]) if case["ragged"] and b else case["ctx"]
        total.append(max(t, n)), new.append(n)
    return total, new


def _tables(g, lengths, page, width, n_pages):
    """Block table [B, width] of pages scattered over the pool (-1 behind a sequence's own) and the ids that are left, in any order."""
    ids = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    need = [_up(n, page) for n in lengths]
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at: at + k]
        at += k
    return table, ids[at:]


def prepare(case, seed):
    return {"pages": _prepare_pages, "norm_rope": _prepare_norm_rope, "append": _prepare_append, "attn": _prepare_attn}[case["kind"]](case, seed)


def _prepare_pages(case, seed):
    g, P = _gen(seed), case["page"]
    cached, new, ended = _plan_lengths(case)
    after = [c + n for c, n in zip(cached, new)]
    width = _up(max(after) + 1, P) + 3
    n_pages = sum(_up(a, P) for a in after) + 5
    table, left = _tables(g, cached, P, width, n_pages)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[: left.numel()] = left
    n_rows = sum(new) + case["pad"]
    z = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt, device=DEV)
    return dict(kind="pages", page=P, n_rows=n_rows, width=width, table=table, free=free, n_free=_ints([left.numel()]), len=_ints(cached), n_new=_ints(new),
                done=_ints(ended), len1=z(case["B"]), n_free1=z(1), len2=z(case["B"]), n_free2=z(1), q_begin=z(case["B"] + 1),
                slot=z(n_rows, torch.int64), pos=z(n_rows))


def _positions(g, case, N):
    """Text positions count up from a random start; with several axes most tokens belong to images, whose rows and columns are small steps."""
    start = int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
    if case.get("prompt", True):
        t = start + torch.arange(N, device=DEV)
    else:
        t = torch.randint(0, 131072, (N,), generator=g, device=DEV)
    pos = t[None].repeat(case["axes"], 1)
    for a in range(1, case["axes"]):
        pos[a] = t // 64 + torch.randint(0, 64, (N,), generator=g, device=DEV)
    return pos.to(torch.int32).contiguous()


def _sections(axes):
    return (64,) if axes == 1 else (SECTIONS[0], 64 - SECTIONS[0]) if axes == 2 else SECTIONS


def _gains(g, case):
    if not case["norm"]:
        return None, None
    return tuple((1.0 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))


def _prepare_norm_rope(case, seed):
    g, N, H = _gen(seed), case["N"], case["Hq"] + case["Hkv"]
    gq, gk = _gains(g, case)
    x = _randn(g, N, H + case["Hkv"], D, scale=1.7)[:, :H]  # the q and k heads of a q|k|v projection
    return dict(kind="norm_rope", x=x, Hq=case["Hq"], Hk=case["Hkv"], gq=gq, gk=gk, pos=_positions(g, case, N), sections=_sections(case["axes"]),
                rotate=case["rotate"], out=torch.zeros((N, H, D), dtype=torch.bfloat16, device=DEV))


def _steps(g, case, n_pages):
    """(s_k, s_v, steps): one step for a KV head, or one for each cached vector."""
    Hkv = case["Hkv"]
    if case["steps"] == "head":
        s_k, s_v = ((0.45 + 0.2 * torch.rand(Hkv, generator=g, device=DEV)) for _ in range(2))
        return s_k, s_v, None
    return None, None, torch.exp2(0.5 * torch.randn((n_pages, Hkv, 2, case["page"]), generator=g, device=DEV) - 1.2)


def _prefix(g, Hkv):
    """Keys and values of the prefixed tokens: keys that draw attention, small values."""
    return _randn(g, Hkv, N_PREFIX, D, scale=1.5, dtype=torch.float16), _randn(g, Hkv, N_PREFIX, D, scale=0.3, dtype=torch.float16)


def _prepare_append(case, seed):
    g, N, pad, Hq, Hkv, P = _gen(seed), case["N"], case["pad"], case["Hq"], case["Hkv"], case["page"]
    gq, gk = _gains(g, case)
    rows = N + pad
    n_pages = (_up(N, P) if case["prompt"] else N) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int64)
    r = torch.arange(N, device=DEV)
    slot = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
    slot[:N] = perm[r // P] * P + r % P if case["prompt"] else perm[r] * P + torch.randint(0, P, (N,), generator=g, device=DEV)
    s_k, s_v, steps = _steps(g, case, n_pages)
    pk, pv = _prefix(g, Hkv)
    z = lambda *sh: torch.zeros(sh, dtype=torch.bfloat16, device=DEV)
    return dict(kind="append", qkv=_randn(g, rows, (Hq + 2 * Hkv) * D, scale=1.7 if case["norm"] else 1.0), Hq=Hq, Hkv=Hkv, page=P, gq=gq, gk=gk,
                pos=_positions(g, case, rows), sections=_sections(case["axes"]), rotate=case["rotate"], slot=slot,
                codes=torch.zeros((n_pages, Hkv, 2, P, D // 2), dtype=torch.uint8, device=DEV), s_k=s_k, s_v=s_v, steps=steps, pk=pk, pv=pv,
                table=torch.full((1, n_pages), -1, dtype=torch.int32, device=DEV), len=_ints([0]), free=z(n_pages).to(torch.int32), n_free=_ints([0]),
                q_out=z(rows, Hq, D), kv_out=z(rows, 2, Hkv, D))


def _prepare_attn(case, seed):
    g, B, Hq, Hkv, P = _gen(seed), case["B"], case["Hq"], case["Hkv"], case["page"]
    total, new = _attn_lengths(case)
    n_pages = sum(_up(t, P) for t in total) + 5
    width = _up(max(total), P) + 2
    table, left = _tables(g, total, P, width, n_pages)
    codes = torch.empty((n_pages, Hkv, 2, P, D // 2), dtype=torch.uint8, device=DEV)
    flat = codes.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):  # codes as values of spread 2.6 steps leave them
        part = flat[lo: lo + (1 << 26)]
        c = torch.clamp(torch.round(2.6 * torch.randn((2, part.numel()), generator=g, device=DEV)), -8, 7).to(torch.int16)
        part.copy_(((c[0] & 15) | ((c[1] & 15) << 4)).to(torch.uint8))
    s_k, s_v, steps = _steps(g, case, n_pages)
    pk, pv = _prefix(g, Hkv)
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    N = begin[-1] + case["pad"]
    b_of = [b for b, n in enumerate(new) for _ in range(n)]
    t_of = [t for n in new for t in range(n)]
    return dict(kind="attn", page=P, Hq=Hq, Hkv=Hkv, codes=codes, table=table, len=_ints(total), free=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
                n_free=_ints([0]), s_k=s_k, s_v=s_v, steps=steps, pk=pk, pv=pv, q=_randn(g, N, Hq, D, scale=1.2), q_begin=_ints(begin), n_new=_ints(new),
                max_new=max(new), max_len=max(total), row_b=_ints(b_of, torch.int64), row_t=_ints(t_of, torch.int64),
                out=torch.zeros((N, Hq, D), dtype=torch.bfloat16, device=DEV))


# ---- the plain forms --------------------------------------------------------------------------------------
def run(state):
    return {"pages": _run_pages, "norm_rope": _run_norm_rope, "append": _run_append, "attn": _run_attn}[state["kind"]](state)


def _run_pages(s):
    """A scheduler step: the pages of ended requests go back, the new tokens get pages, slots and positions."""
    if own:
        from paper_2410_05265_b200 import binding

        if "pages" not in s:
            s["pages"] = binding.Pages(s["table"], s["len"], s["free"], s["n_free"], s["page"])
            s["after"] = binding.Pages(s["table"], s["len1"], s["free"], s["n_free1"], s["page"])
        _ctx().page_release(s["pages"], s["done"], len_out=s["len1"], n_free_out=s["n_free1"])
        _ctx().page_plan(s["after"], s["n_new"], pos0=N_PREFIX, out=(s["q_begin"], s["slot"], s["pos"]), len_out=s["len2"], n_free_out=s["n_free2"])
        return s["table"], s["free"], s["n_free2"], s["len2"], s["q_begin"], s["slot"], s["pos"]
    P, n_pages, B = s["page"], s["free"].numel(), s["len"].numel()
    # release: entry j of an ended sequence goes to free[n_free + what the ended ones before it give back + j]
    done = s["done"] != 0
    back = torch.where(done, (s["len"] + P - 1) // P, 0).to(torch.int64)
    at = s["n_free"].to(torch.int64) + torch.cumsum(back, 0) - back
    j = torch.arange(s["width"], device=DEV)[None]
    free = torch.cat((s["free"], s["free"][:1]))  # the last place takes what belongs nowhere
    free.scatter_(0, torch.where(j < back[:, None], at[:, None] + j, n_pages).reshape(-1), s["table"].reshape(-1))
    free = free[:n_pages]
    n_free1 = s["n_free"].to(torch.int64) + back.sum()
    len1 = torch.where(done, 0, s["len"]).to(torch.int64)
    # plan: page k of all that are taken is free[n_free - 1 - k]
    n_new = s["n_new"].to(torch.int64)
    old, now = (len1 + P - 1) // P, (len1 + n_new + P - 1) // P
    k0 = torch.cumsum(now - old, 0) - (now - old)
    take = (n_free1 - 1 - k0[:, None] - (j - old[:, None])).clamp(0, n_pages - 1)
    table = torch.where((j >= old[:, None]) & (j < now[:, None]), free[take], s["table"])
    end = torch.cumsum(n_new, 0)
    r = torch.arange(s["n_rows"], device=DEV)
    b = (end[None] <= r[:, None]).sum(1).clamp(max=B - 1)
    live = r < end[-1]
    p = len1[b] + r - (end - n_new)[b]
    slot = torch.where(live, table[b, torch.where(live, p // P, 0)].to(torch.int64) * P + p % P, -1)
    pos = torch.where(live, p + N_PREFIX, 0).to(torch.int32)
    q_begin = torch.cat((end[:1] * 0, end)).to(torch.int32)
    return table, free, (n_free1 - (now - old).sum()).reshape(1).to(torch.int32), (len1 + n_new).to(torch.int32), q_begin, slot, pos


def _angles(pos, sections):
    """cos and sin [N, 1, 64] in 64 bits."""
    axis = torch.cat([torch.full((n,), a, dtype=torch.int64, device=DEV) for a, n in enumerate(sections)])
    i = torch.arange(D // 2, device=DEV, dtype=torch.float64)
    ang = pos.to(torch.float64)[axis].T * THETA ** (-2.0 * i / D)
    return torch.cos(ang)[:, None], torch.sin(ang)[:, None]


def _hadamard(dtype):
    i = torch.arange(D, device=DEV)
    m = i[:, None] & i[None]
    bits = sum((m >> k) & 1 for k in range(7))
    return (1 - 2 * (bits % 2)).to(dtype) / math.sqrt(D)


def _norm_rope(x, gain, c, s, rotate, dtype):
    """x [N, H, 128] -> normed, rotated by position (and by the Hadamard matrix) in `dtype`."""
    v = x.to(dtype)
    if gain is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * gain.to(dtype)
    a, b, c, s = v[..., : D // 2], v[..., D // 2:], c.to(dtype), s.to(dtype)
    y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return y @ _hadamard(dtype) if rotate else y


def _run_norm_rope(s):
    if own:
        return _ctx().qk_norm_rope(s["x"], s["Hq"], s["gq"], s["gk"], EPS, s["pos"], THETA, sections=s["sections"], rotate=s["rotate"], out=s["out"])
    c, si = _angles(s["pos"], s["sections"])
    q = _norm_rope(s["x"][:, : s["Hq"]], s["gq"], c, si, s["rotate"], torch.float32)
    k = _norm_rope(s["x"][:, s["Hq"]:], s["gk"], c, si, s["rotate"], torch.float32)
    return torch.cat((q, k), 1).to(torch.bfloat16)


def _nibbles(c):
    """Packed codes [..., 64] -> values [..., 128] in fp32."""
    lo = ((c & 15) ^ 8).to(torch.int8) - 8
    hi = ((c >> 4) ^ 8).to(torch.int8) - 8
    return torch.stack((lo, hi), -1).flatten(-2).to(torch.float32)


def _paged_cache(s):
    if "cache" not in s:
        from paper_2410_05265_b200 import binding

        pages = binding.Pages(s["table"], s["len"], s["free"], s["n_free"], s["page"])
        s["cache"] = binding.KV4PagedCache(pages, s["pk"], s["pv"], s["codes"], s["Hq"], s_k=s["s_k"], s_v=s["s_v"], steps=s["steps"])
    return s["cache"]


def _run_append(s):
    """New tokens into the cache, and their values as a reader of the cache finds them. Rows with slot -1 are left alone."""
    if own:
        cache = _paged_cache(s)
        _ctx().qk_norm_rope_kv4_paged_append(cache, s["qkv"], s["gq"], s["gk"], EPS, s["pos"], s["slot"], THETA, sections=s["sections"],
                                             rotate=s["rotate"], q_out=s["q_out"])
        _ctx().kv4_paged_read(cache, s["slot"], out=s["kv_out"])
        return s["q_out"], s["kv_out"]
    Hq, Hkv, P = s["Hq"], s["Hkv"], s["page"]
    x = s["qkv"].view(-1, Hq + 2 * Hkv, D)
    c, si = _angles(s["pos"], s["sections"])
    live = (s["slot"] >= 0)[:, None, None]
    q = torch.where(live, _norm_rope(x[:, :Hq], s["gq"], c, si, s["rotate"], torch.float32).to(torch.bfloat16), s["q_out"])
    # the keys in 64 bits: a code next to a border is decided by the last bits
    k = _norm_rope(x[:, Hq: Hq + Hkv], s["gk"], c, si, s["rotate"], torch.float64)
    v = x[:, Hq + Hkv:].to(torch.float32)
    if s["steps"] is None:
        sk, sv = s["s_k"][None, :, None].expand(k.shape[0], -1, 1), s["s_v"][None, :, None].expand(k.shape[0], -1, 1)
    else:
        seven = torch.full((), 7.0, device=DEV)
        sk = (k.abs().amax(-1, keepdim=True) / 7.0).to(torch.float32)
        sv = v.abs().amax(-1, keepdim=True) / seven
    codes = torch.stack((torch.round((k / sk.to(torch.float64)).to(torch.float32)), torch.round(v / sv)), 1).clamp(-8, 7).to(torch.int16) & 15
    packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8)  # [N, 2, Hkv, 64]
    n_slots = s["codes"].shape[0] * P
    to = torch.where(s["slot"] >= 0, s["slot"], n_slots)
    rows = torch.zeros((n_slots + 1, 2, Hkv, D // 2), dtype=torch.uint8, device=DEV)  # token-major here; the last row takes what belongs nowhere
    rows[:n_slots] = s["codes"].permute(0, 3, 2, 1, 4).reshape(n_slots, 2, Hkv, D // 2)
    rows[to] = packed
    s["codes"].copy_(rows[:n_slots].view(-1, P, 2, Hkv, D // 2).permute(0, 3, 2, 1, 4))
    values = _nibbles(rows[to]) * torch.stack((sk, sv), 1)
    return q, torch.where(live[..., None], values.to(torch.bfloat16), s["kv_out"])


def _run_attn(s):
    if own:
        cache = _paged_cache(s)
        if "ws" not in s:
            s["ws"] = _ctx().attn_kv4_paged_workspace(cache, s["q"].shape[0], s["max_new"])
        return _ctx().attn_kv4_paged(cache, s["q"], s["q_begin"], s["max_new"], SM_SCALE, s["ws"], max_len=s["max_len"], out=s["out"])
    P, Hq, Hkv, B, L, n = s["page"], s["Hq"], s["Hkv"], s["len"].numel(), s["max_len"], s["max_new"]
    G, width = Hq // Hkv, _up(s["max_len"], s["page"])
    page = s["table"][:, :width].clamp(min=0).to(torch.int64)
    kv = _nibbles(s["codes"][page])  # [B, width, Hkv, 2, P, 128]
    if s["steps"] is None:
        kv *= torch.stack((s["s_k"], s["s_v"]), 1)[:, :, None, None]
    else:
        kv *= s["steps"][page][..., None]
    kv = kv.permute(3, 0, 2, 1, 4, 5).reshape(2, B, Hkv, width * P, D)[:, :, :, :L]
    k, v = (torch.cat((pre.to(torch.float32)[None].expand(B, -1, -1, -1), t), 2) for pre, t in ((s["pk"], kv[0]), (s["pv"], kv[1])))
    q = torch.zeros((B, n, Hq, D), device=DEV)
    q[s["row_b"], s["row_t"]] = s["q"][: s["row_b"].numel()].to(torch.float32)
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    x = q @ k.transpose(-1, -2)
    x *= SM_SCALE
    last = s["len"][:, None] - s["n_new"][:, None] + torch.arange(n, device=DEV)[None]  # the last cached key of row t
    hidden = torch.arange(N_PREFIX + L, device=DEV)[None, None] > N_PREFIX + last[..., None]
    x.view(B, Hkv, n, G, -1).masked_fill_(hidden[:, None, :, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    o = (x @ v) / x.sum(-1, keepdim=True)
    o = o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)[s["row_b"], s["row_t"]].to(torch.bfloat16)
    return torch.cat((o, s["out"][o.shape[0]:]))


# ---- work -------------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "pages":
        cached, new, ended = _plan_lengths(case)
        P = case["page"]
        taken = sum(_up(c + n, P) - _up(c, P) for c, n in zip(cached, new))
        back = sum(_up(c, P) for c, e in zip(cached, ended) if e)
        # lengths, new tokens and flags read, lengths and offsets written; a taken page is read and written, so is one that goes back
        return dict(bytes=case["B"] * 20 + 8 * (taken + back) + 12 * (sum(new) + case["pad"]), flops=0)
    H = case["Hq"] + case["Hkv"]
    if case["kind"] == "norm_rope":
        return dict(bytes=case["N"] * (H * 512 + 4 * case["axes"]), flops=case["N"] * H * D * (22 if case["rotate"] else 8))
    if case["kind"] == "append":
        a_step = 8 * case["Hkv"] if case["steps"] == "vector" else 0
        write = (H + case["Hkv"]) * 256 + case["Hq"] * 256 + case["Hkv"] * 128 + a_step + 8 + 4 * case["axes"]
        read = case["Hkv"] * (128 + 512) + a_step + 8
        return dict(bytes=case["N"] * (write + read) + 16 * case["pad"], flops=case["N"] * (H * D * (22 if case["rotate"] else 8) + 4 * case["Hkv"] * D))
    total, new = _attn_lengths(case)
    pairs = sum(n * (N_PREFIX + t - n) + n * (n + 1) // 2 for t, n in zip(total, new))
    a_key = 128 + (8 if case["steps"] == "vector" else 0)
    return dict(bytes=case["Hkv"] * (a_key * sum(total) + N_PREFIX * 512) + sum(new) * case["Hq"] * 512, flops=4 * D * case["Hq"] * pairs)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "pages":
        return None
    s = prepare(case, seed)
    return {"norm_rope": _exact_norm_rope, "append": _exact_append, "attn": _exact_attn}[case["kind"]](s)


def _exact_heads(x, gain, pos, sections, rotate):
    """Row by definition: y_i + j y_{i+64} = (v_i + j v_{i+64}) e^{j angle}; then the Walsh-Hadamard transform by butterflies."""
    v = x.to(torch.float64)
    if gain is not None:
        v = v * torch.rsqrt(v.square().sum(-1, keepdim=True) / D + EPS) * gain.to(torch.float64)
    parts, lo = [], 0
    for axis, n in enumerate(sections):
        freq = torch.exp(torch.arange(lo, lo + n, device=DEV, dtype=torch.float64) * (-math.log(THETA) / 64))
        turn = pos[axis].to(torch.float64)[:, None] * freq[None]
        parts.append(torch.polar(torch.ones_like(turn), turn))
        lo += n
    z = torch.complex(v[..., :64].contiguous(), v[..., 64:].contiguous()) * torch.cat(parts, 1)[:, None]
    y = torch.cat((z.real, z.imag), -1)
    if rotate:
        h = 1
        while h < D:
            y = y.view(*y.shape[:2], D // (2 * h), 2, h)
            y = torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).flatten(-3)
            h *= 2
        y = y / math.sqrt(D)
    return y


def _exact_norm_rope(s):
    q = _exact_heads(s["x"][:, : s["Hq"]], s["gq"], s["pos"], s["sections"], s["rotate"])
    return torch.cat((q, _exact_heads(s["x"][:, s["Hq"]:], s["gk"], s["pos"], s["sections"], s["rotate"])), 1)


def _exact_append(s):
    Hq, Hkv = s["Hq"], s["Hkv"]
    x = s["qkv"].view(-1, Hq + 2 * Hkv, D)
    q = _exact_heads(x[:, :Hq], s["gq"], s["pos"], s["sections"], s["rotate"])
    kv = [_exact_heads(x[:, Hq: Hq + Hkv], s["gk"], s["pos"], s["sections"], s["rotate"]), x[:, Hq + Hkv:].to(torch.float64)]
    if s["steps"] is None:
        step = [t.to(torch.float64)[None, :, None] for t in (s["s_k"], s["s_v"])]
    else:
        step = [(t.abs().amax(-1, keepdim=True) / 7).to(torch.float32).to(torch.float64) for t in kv]
    # by the interface's rule a code rounds the quotient in 32 bits (half of a vector's maximum is 3.5 steps, wherever the step was rounded to)
    values = torch.stack([torch.clamp(torch.round((t / st).to(torch.float32)), -8, 7) * st for t, st in zip(kv, step)], 1)
    live = s["slot"] >= 0
    return torch.where(live[:, None, None], q, 0.0), torch.where(live[:, None, None, None], values, 0.0)


def _exact_attn(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    P, G = s["page"], s["Hq"] // s["Hkv"]
    begin, lengths = s["q_begin"].tolist(), s["len"].tolist()
    for b, n_keys in enumerate(lengths):
        r0, n = begin[b], begin[b + 1] - begin[b]
        page = s["table"][b, : _up(n_keys, P)].to(torch.int64)
        for h in range(s["Hkv"]):
            keys = []
            for which, pre, head in ((0, s["pk"], s["s_k"]), (1, s["pv"], s["s_v"])):
                c = s["codes"][page, h, which].reshape(-1, D // 2)[:n_keys].to(torch.int16)
                val = torch.stack((c % 16, c // 16), -1).flatten(1).to(torch.float64)
                val = torch.where(val > 7, val - 16, val)
                step = head[h].to(torch.float64) if s["steps"] is None else s["steps"][page, h, which].reshape(-1)[:n_keys, None].to(torch.float64)
                keys.append(torch.cat((pre[h].to(torch.float64), val * step)))
            for lo in range(0, n, 256):  # bounded score matrices
                hi = min(n, lo + 256)
                q = s["q"][r0 + lo: r0 + hi, h * G: (h + 1) * G].to(torch.float64)
                x = (q.reshape(-1, D) @ keys[0].T).view(hi - lo, G, -1) * SM_SCALE
                seen = N_PREFIX + n_keys - n + 1 + torch.arange(lo, hi, device=DEV)
                x = x.masked_fill(torch.arange(x.shape[-1], device=DEV)[None, None] >= seen[:, None, None], -math.inf)
                w = torch.softmax(x, -1).view(-1, x.shape[-1])
                out[r0 + lo: r0 + hi, h * G: (h + 1) * G] = (w @ keys[1]).view(hi - lo, G, D)
    return out
