"""Speculative decoding and windowed layers over the paged 4-bit cache, on representative calls: attention with a sliding window and first tokens that
stay visible, attention of a tree of drafted tokens, the plan of such trees (ancestors, positions) and what follows a verification (the accepted path,
the pages that go back, the moves inside the cache).

Head counts are those of the Llama-3-8B and Llama-3-70B layers of `inputs.py` (32 and 64 query heads on 8 KV heads) and, in drawn cases, a few other
ratios; four prefixed tokens stay in fp16, as everywhere in this repository, and are visible to every token, whatever the window.

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
N_PREFIX = 4  # prefixed tokens, fp16, seen by every token
SM_SCALE = 1.0 / math.sqrt(D)
VOCAB = 128256
MOST_DRAFTS = 128


def listed():
    window = dict(kind="window", ragged=True, pad=0, Hq=32, Hkv=8, page=16, steps="head", sinks=0)
    tree = dict(kind="tree", ragged=True, pad=0, Hq=32, Hkv=8, page=16, steps="head", window=0, sinks=0)
    return [
        # one sequence, one token, far behind its first ones: interactive decoding on a windowed layer
        dict(window, name="window_1x30000", B=1, ctx=30000, new=1, share=0.0, window=1024),
        # a decode batch; cached vectors with their own steps
        dict(window, name="window_64x16000", B=64, ctx=16000, new=1, share=0.0, window=4096, steps="vector", pad=3),
        # prompts of several lengths, the first four tokens of each stay visible
        dict(window, name="window_prompts_4x2900", B=4, ctx=2900, new=2900, share=1.0, window=1000, sinks=4, page=32, steps="vector"),
        # one chunk of a long prompt on the large layer
        dict(window, name="window_chunk_2048_of_32000", B=1, ctx=32000, new=2048, share=1.0, window=4096, Hq=64, page=64, ragged=False),
        # one sequence verifies a small tree: interactive decoding with drafts
        dict(tree, name="tree_1x26_at_1021", B=1, ctx=1021, new=26, width=6),
        # a batch of short chains of drafts, cached vectors with their own steps, padded to the batch of a captured graph
        dict(tree, name="tree_48x5_at_6000", B=48, ctx=6000, new=5, width=1, steps="vector", pad=15),
        # trees of 64 on the large layer behind long contexts
        dict(tree, name="tree_12x64_at_16000", B=12, ctx=16000, new=64, width=9, Hq=64, page=64),
        # trees on a windowed layer
        dict(tree, name="tree_window_16x33_at_9000", B=16, ctx=9000, new=33, width=5, window=2048, sinks=4, page=32),
        # ancestors and positions of one tree: latency
        dict(kind="plan", name="plan_1x26", B=1, ctx=4000, new=26, width=6, ragged=False, pad=0),
        # a large server's trees
        dict(kind="plan", name="plan_512x64", B=512, ctx=8000, new=64, width=9, ragged=True, pad=77),
        # what follows a verification of one tree
        dict(kind="accept", name="accept_1x26", B=1, ctx=1021, new=26, width=6, ragged=False, pad=0, Hq=32, Hkv=8, page=16, steps="head"),
        # the same for a batch, cached vectors with their own steps
        dict(kind="accept", name="accept_128x60", B=128, ctx=2000, new=60, width=8, ragged=True, pad=9, Hq=32, Hkv=8, page=16, steps="vector"),
    ]


def draw(rng):
    log = lambda lo, hi: min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))
    kind = rng.choice(["window", "window", "window", "tree", "tree", "tree", "plan", "accept"])
    Hq, Hkv = rng.choice([(32, 8), (64, 8), (32, 8), (64, 8), (8, 8), (6, 2), (5, 1), (7, 1)])
    page, steps, pad = rng.choice([16, 32, 64, 128]), rng.choice(["head", "vector"]), rng.choice([0, 0, log(1, 100)])
    ragged, sinks = rng.random() < 0.7, rng.choice([0, 0, 4, log(1, 300)])
    both = dict(kind=kind, ragged=ragged, pad=pad)
    cache = dict(both, Hq=Hq, Hkv=Hkv, page=page, steps=steps)
    if kind == "plan":
        return dict(both, B=log(1, 512), ctx=log(1, 8000), new=log(1, 64), width=log(1, 12))
    if kind == "accept":
        return dict(cache, B=log(1, 128), ctx=log(1, 2000), new=log(1, 60), width=log(1, 12))
    if kind == "tree":
        B, new = log(1, 48), log(2, 64)
        ctx = log(new, min(30000, 190000 // B))
        return dict(cache, B=B, ctx=ctx, new=new, width=log(1, 12), window=rng.choice([0, 0, log(64, 8192)]), sinks=sinks)
    form = rng.choice(["decode", "decode", "mixed", "prompts", "chunk"])
    cache.update(window=log(16, 8192 if form == "decode" else 4096), sinks=sinks)
    if form == "decode":
        B = log(1, 128)
        return dict(cache, B=B, ctx=log(1, min(60000, 500000 // B)), new=1, share=0.0)
    if form == "mixed":
        return dict(cache, B=log(2, 32), ctx=log(17, 1500), ragged=True, new=log(2, 1500), share=0.5)
    if form == "prompts":
        B = log(1, 8)
        n = log(2, 4096 // B)
        return dict(cache, B=B, ctx=n, new=n, share=1.0)
    new = log(2, 2048)
    return dict(cache, B=1, ctx=log(new, 30000), ragged=False, new=new, share=1.0)


# ---- inputs -----------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=1)
def _ctx():
    from paper_2410_05265_b200 import binding

    return binding.Context()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 31)


def _randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _up(a, b):
    return -(-a // b)


def _lengths(case):
    """(cached tokens with the new ones, new ones) of every sequence."""
    r = random.Random(case["B"] * 104729 + case["ctx"] * 31 + case["new"])
    total, new = [], []
    for b in range(case["B"]):
        n = r.randint(max(1, case["new"] // 2), case["new"]) if case["ragged"] else case["new"]
        if r.random() >= case.get("share", 1.0):
            n = 1
        t = r.randint(max(1, case["ctx"] // 4), case["ctx"]) if case["ragged"] and b else case["ctx"]
        total.append(max(t, n)), new.append(n)
    return total, new


def _trees(case):
    """Parents of every sequence's drafts (row 0 is the root): a draft hangs on one of the `width` rows before it."""
    r = random.Random(case["B"] * 7919 + case["ctx"] * 13 + case["new"] + case["width"])
    return [[-1] + [r.randint(max(0, t - case["width"]), t - 1) for t in range(1, n)] for n in _lengths(case)[1]]


def _ancestors(parent):
    """For every row the rows it sees, itself among them, as bits of one integer."""
    seen = []
    for t, p in enumerate(parent):
        seen.append((1 << t) | (seen[p] if p >= 0 else 0))
    return seen


def _mask_words(parents, words, rows):
    out = []
    for parent in parents:
        for bits in _ancestors(parent):
            w = [(bits >> (32 * i)) & 0xFFFFFFFF for i in range(words)]
            out.append([x - (1 << 32) if x >= 1 << 31 else x for x in w])
    return _ints(out + [[0] * words] * (rows - len(out)))


def _paged(g, case, total):
    """Codes as values of spread 2.6 steps leave them, on pages scattered over the pool, with steps, prefix and block table (-1 behind a sequence's pages)."""
    Hkv, P = case["Hkv"], case["page"]
    need = [_up(t, P) for t in total]
    n_pages = sum(need) + 5
    ids = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    table = torch.full((len(total), max(need) + 2), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at: at + k]
        at += k
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[: n_pages - at] = ids[at:]
    codes = torch.empty((n_pages, Hkv, 2, P, D // 2), dtype=torch.uint8, device=DEV)
    flat = codes.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        part = flat[lo: lo + (1 << 26)]
        c = torch.clamp(torch.round(2.6 * torch.randn((2, part.numel()), generator=g, device=DEV)), -8, 7).to(torch.int16)
        part.copy_(((c[0] & 15) | ((c[1] & 15) << 4)).to(torch.uint8))
    s_k = s_v = steps = None
    if case["steps"] == "head":
        s_k, s_v = ((0.45 + 0.2 * torch.rand(Hkv, generator=g, device=DEV)) for _ in range(2))
    else:
        steps = torch.exp2(0.5 * torch.randn((n_pages, Hkv, 2, P), generator=g, device=DEV) - 1.2)
    pk, pv = _randn(g, Hkv, N_PREFIX, D, scale=1.5, dtype=torch.float16), _randn(g, Hkv, N_PREFIX, D, scale=0.3, dtype=torch.float16)
    return dict(page=P, Hq=case["Hq"], Hkv=Hkv, codes=codes, table=table, len=_ints(total), free=free, n_free=_ints([n_pages - at]), s_k=s_k, s_v=s_v,
                steps=steps, pk=pk, pv=pv)


def _rows(new):
    """(q_begin, sequence of every row, its place among the sequence's rows)."""
    begin = [0]
    for n in new:
        begin.append(begin[-1] + n)
    return dict(q_begin=_ints(begin), row_b=_ints([b for b, n in enumerate(new) for _ in range(n)], torch.int64),
                row_t=_ints([t for n in new for t in range(n)], torch.int64), n_new=_ints(new), max_new=max(new), live=begin[-1])


def prepare(case, seed):
    return {"window": _prepare_attn, "tree": _prepare_attn, "plan": _prepare_plan, "accept": _prepare_accept}[case["kind"]](case, seed)


def _prepare_attn(case, seed):
    g = _gen(seed)
    total, new = _lengths(case)
    s = dict(_paged(g, case, total), kind=case["kind"], window=case["window"], sinks=case["sinks"], max_len=max(total), **_rows(new))
    N = s["live"] + case["pad"]
    s["mask"] = _mask_words(_trees(case), _up(s["max_new"], 32), N) if case["kind"] == "tree" else None
    s["q"], s["out"] = _randn(g, N, case["Hq"], D, scale=1.2), torch.zeros((N, case["Hq"], D), dtype=torch.bfloat16, device=DEV)
    return s


def _prepare_plan(case, seed):
    total, new = _lengths(case)
    total = [t + int(seed) % 97 for t in total]
    s = dict(_rows(new), kind="plan", B=case["B"], len=_ints(total))
    N = s["live"] + case["pad"]
    trees = _trees(case)
    if seed % 2:  # other trees of the same sizes: the draft in the middle hangs on the root
        trees = [[0 if 0 < t == len(p) // 2 else q for t, q in enumerate(p)] for p in trees]
    s["parent"] = _ints([q for p in trees for q in p] + [0] * case["pad"])
    s["mask"], s["pos"] = torch.zeros((N, _up(s["max_new"], 32)), dtype=torch.int32, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)
    return s


def _tokens(trees, seed):
    """Drafted tokens and the model's choice after each: a path of every tree is accepted, whose rows move from behind the accepted ones (so that a pass can
    be repeated on the same cache)."""
    r = random.Random(int(seed) * 31 + len(trees))
    draft, target = [], []
    for parent in trees:
        n = len(parent)
        tok, choice = [r.randrange(VOCAB) for _ in range(n)], [r.randrange(VOCAB) for _ in range(n)]
        path = [0]
        while r.random() < 0.8:
            children = [c for c in range(path[-1] + 1, n) if parent[c] == path[-1]]
            if not children:
                break
            path.append(r.choice(children))
        while any(p != i and p < len(path) for i, p in enumerate(path)):
            path.pop()
        for i, p in enumerate(path):
            if i + 1 < len(path):
                for c in range(p + 1, n):  # no sibling before it has the same token
                    if parent[c] == p and c != path[i + 1] and tok[c] == tok[path[i + 1]]:
                        tok[c] = (tok[c] + 1) % VOCAB
                choice[p] = tok[path[i + 1]]
            else:
                while any(parent[c] == p and tok[c] == choice[p] for c in range(p + 1, n)):
                    choice[p] = (choice[p] + 1) % VOCAB
        draft.extend(tok), target.extend(choice)
    return draft, target


def _prepare_accept(case, seed):
    g = _gen(seed)
    total, new = _lengths(case)
    trees = _trees(case)
    draft, target = _tokens(trees, seed)
    pad = case["pad"]
    s = dict(_paged(g, case, total), kind="accept", **_rows(new))
    N, B = s["live"] + pad, case["B"]
    s["parent"] = _ints([q for p in trees for q in p] + [0] * pad)
    s["draft"], s["target"] = _ints(draft + [0] * pad), _ints(target + [0] * pad)
    place = s["len"].to(torch.int64)[s["row_b"]] - s["n_new"].to(torch.int64)[s["row_b"]] + s["row_t"]
    s["slot"] = torch.full((N,), -1, dtype=torch.int64, device=DEV)
    s["slot"][: s["live"]] = s["table"][s["row_b"], place // s["page"]].to(torch.int64) * s["page"] + place % s["page"]
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    s.update(kept=z(N), n_kept=z(B), next=z(B), len1=z(B), n_free1=z(1), kv_out=torch.zeros((N, 2, case["Hkv"], D), dtype=torch.bfloat16, device=DEV))
    return s


# ---- the plain forms --------------------------------------------------------------------------------------
def run(state):
    return {"window": _run_attn, "tree": _run_attn, "plan": _run_plan, "accept": _run_accept}[state["kind"]](state)


def _nibbles(c):
    """Packed codes [..., 64] -> values [..., 128] in fp32."""
    lo = ((c & 15) ^ 8).to(torch.int8) - 8
    hi = ((c >> 4) ^ 8).to(torch.int8) - 8
    return torch.stack((lo, hi), -1).flatten(-2).to(torch.float32)


def _cache(s, length):
    from paper_2410_05265_b200 import binding

    pages = binding.Pages(s["table"], length, s["free"], s["n_free"], s["page"])
    return binding.KV4PagedCache(pages, s["pk"], s["pv"], s["codes"], s["Hq"], s_k=s["s_k"], s_v=s["s_v"], steps=s["steps"])


def _bits(mask, n):
    """Mask words int32 [N, words] -> truth values [N, n]."""
    j = torch.arange(n, device=DEV)
    return ((mask.to(torch.int64)[:, j // 32] >> (j % 32)) & 1) != 0


def _run_attn(s):
    if own:
        if "cache" not in s:
            s["cache"] = _cache(s, s["len"])
            s["ws"] = (_ctx().attn_kv4_paged_workspace if s["mask"] is None else _ctx().attn_kv4_paged_tree_workspace)(s["cache"], s["q"].shape[0], s["max_new"])
        if s["mask"] is None:
            return _ctx().attn_kv4_paged_window(s["cache"], s["q"], s["q_begin"], s["max_new"], s["window"], SM_SCALE, s["ws"], n_sink=s["sinks"],
                                                max_len=s["max_len"], out=s["out"])
        return _ctx().attn_kv4_paged_tree(s["cache"], s["q"], s["q_begin"], s["max_new"], s["mask"], SM_SCALE, s["ws"], window=s["window"], n_sink=s["sinks"],
                                          max_len=s["max_len"], out=s["out"])
    P, Hq, Hkv, B, L, n = s["page"], s["Hq"], s["Hkv"], s["len"].numel(), s["max_len"], s["max_new"]
    G, width, rows = Hq // Hkv, _up(s["max_len"], s["page"]), s["live"]
    page = s["table"][:, :width].clamp(min=0).to(torch.int64)
    kv = _nibbles(s["codes"][page])  # [B, width, Hkv, 2, P, 128]
    if s["steps"] is None:
        kv *= torch.stack((s["s_k"], s["s_v"]), 1)[:, :, None, None]
    else:
        kv *= s["steps"][page][..., None]
    kv = kv.permute(3, 0, 2, 1, 4, 5).reshape(2, B, Hkv, width * P, D)[:, :, :, :L]
    k, v = (torch.cat((pre.to(torch.float32)[None].expand(B, -1, -1, -1), t), 2) for pre, t in ((s["pk"], kv[0]), (s["pv"], kv[1])))
    q = torch.zeros((B, n, Hq, D), device=DEV)
    q[s["row_b"], s["row_t"]] = s["q"][:rows].to(torch.float32)
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    x = q @ k.transpose(-1, -2)
    x *= SM_SCALE
    j = torch.arange(L, device=DEV)
    before = (s["len"] - s["n_new"]).to(torch.int64)  # cached tokens before the new rows
    if s["mask"] is None:
        place = before[:, None] + torch.arange(n, device=DEV)[None]
        seen = j <= place[..., None]
    else:
        sees = torch.zeros((B, n, n), dtype=torch.bool, device=DEV)
        sees[s["row_b"], s["row_t"]] = _bits(s["mask"][:rows], n)
        place = before[:, None] + sees.sum(-1) - 1
        rel = j[None] - before[:, None]
        new = torch.gather(sees, 2, rel.clamp(0, n - 1)[:, None].expand(B, n, L))
        seen = (rel < 0)[:, None] | (new & (rel < n)[:, None])
    if s["window"]:
        seen &= (j > place[..., None] - s["window"]) | (j < s["sinks"])
    seen = torch.cat((torch.ones((B, n, N_PREFIX), dtype=torch.bool, device=DEV), seen), 2)
    x.view(B, Hkv, n, G, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    o = (x @ v) / x.sum(-1, keepdim=True)
    o = o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)[s["row_b"], s["row_t"]].to(torch.bfloat16)
    return torch.cat((o, s["out"][rows:]))


def _run_plan(s):
    """Ancestors and positions of every draft. A row without a parent follows the cached tokens."""
    if own:
        if "pages" not in s:  # a table without pages: the plan reads the lengths only
            from paper_2410_05265_b200 import binding

            B = s["B"]
            s["pages"] = binding.Pages(torch.zeros((B, 1024), dtype=torch.int32, device=DEV), s["len"], _ints([0]), _ints([0]), 16)
        _ctx().tree_plan(s["pages"], s["parent"], s["q_begin"], pos0=N_PREFIX, out=(s["mask"], s["pos"]))
        return s["mask"], s["pos"]
    N, words, rows = s["parent"].numel(), s["mask"].shape[1], s["live"]
    t = torch.zeros(N + 1, dtype=torch.int64, device=DEV)
    t[:rows] = s["row_t"]
    up = torch.full((N + 1,), N, dtype=torch.int64, device=DEV)  # the parent's row; N: none
    p = s["parent"][:rows].to(torch.int64)
    up[:rows] = torch.where(p >= 0, s["q_begin"].to(torch.int64)[s["row_b"]] + p, N)
    bits = torch.zeros((N + 1, words), dtype=torch.int64, device=DEV)
    bits[:rows] = torch.where(torch.arange(words, device=DEV)[None] == (t // 32)[:rows, None], 1 << (t % 32)[:rows, None], 0)
    depth = (up < N).to(torch.int64)
    for _ in range(MOST_DRAFTS.bit_length() - 1):  # twice as many generations each time
        bits |= bits[up]
        depth += depth[up]
        up = up[up]
    base = (s["len"] - s["n_new"]).to(torch.int64)[s["row_b"]]
    pos = torch.zeros(N, dtype=torch.int64, device=DEV)
    pos[:rows] = N_PREFIX + base + depth[:rows]
    return torch.where(bits >= 1 << 31, bits - (1 << 32), bits)[:N].to(torch.int32), pos.to(torch.int32)


def _run_accept(s):
    """The accepted path of every tree, the pages that hold no token any more, the moves inside the cache, and the drafts' slots as a reader finds them."""
    if own:
        if "cache" not in s:
            s["cache"], s["after"] = _cache(s, s["len"]), _cache(s, s["len1"])
        _ctx().tree_accept(s["q_begin"], s["parent"], s["draft"], s["target"], out=(s["kept"], s["n_kept"], s["next"]))
        _ctx().page_keep(s["cache"].pages, s["q_begin"], s["n_kept"], len_out=s["len1"], n_free_out=s["n_free1"])
        _ctx().kv4_paged_keep(s["after"], s["q_begin"], s["kept"], s["n_kept"])
        _ctx().kv4_paged_read(s["after"], s["slot"], out=s["kv_out"])
        return s["kept"], s["n_kept"], s["next"], s["len1"], s["free"], s["n_free1"], s["kv_out"]
    B, n, P, rows, N = s["len"].numel(), s["max_new"], s["page"], s["live"], s["parent"].numel()
    dense = lambda t, fill: torch.full((B, n), fill, dtype=torch.int64, device=DEV).index_put((s["row_b"], s["row_t"]), t[:rows].to(torch.int64))
    parent, draft, target = dense(s["parent"], -2), dense(s["draft"], -1), dense(s["target"], -3)
    j = torch.arange(n, device=DEV)[None]
    at, count = torch.zeros(B, dtype=torch.int64, device=DEV), torch.ones(B, dtype=torch.int64, device=DEV)
    path = torch.full((B, n), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    alive = torch.ones(B, dtype=torch.bool, device=DEV)
    for i in range(1, n):
        fits = (parent == at[:, None]) & (draft == target.gather(1, at[:, None]))
        child = torch.where(fits, j, n).amin(1)
        alive = alive & (child < n)
        at = torch.where(alive, child, at)
        path[:, i] = torch.where(alive, child, -1)
        count += alive
    nxt = target.gather(1, at[:, None])[:, 0]
    kept = torch.full((N,), -1, dtype=torch.int64, device=DEV)
    kept[:rows] = path[s["row_b"], s["row_t"]]
    # pages behind the new end go back, sequence by sequence
    base = (s["len"] - s["n_new"]).to(torch.int64)
    len1 = base + count
    first, back = _up(len1, P), _up(s["len"].to(torch.int64), P) - _up(len1, P)
    n_free = s["n_free"].to(torch.int64)
    start = n_free + torch.cumsum(back, 0) - back
    width, n_pages = s["table"].shape[1], s["free"].numel()
    w = torch.arange(width, device=DEV)[None]
    goes = (w >= first[:, None]) & (w < (first + back)[:, None])
    free = torch.cat((s["free"], s["free"][:1]))  # the last place takes what belongs nowhere
    free.scatter_(0, torch.where(goes, start[:, None] + w - first[:, None], n_pages).reshape(-1), s["table"].reshape(-1))
    # the moves: a token-major copy of the cache, its last row takes what belongs nowhere
    src = torch.where(path >= 0, base[:, None] + path, 0)
    dst = torch.where(path >= 0, base[:, None] + j, 0)
    slot_of = lambda place: torch.gather(s["table"].to(torch.int64), 1, place // P) * P + place % P
    ok, n_slots = path >= 0, s["codes"].shape[0] * P
    src, dst = slot_of(src)[ok], slot_of(dst)[ok]
    flat = s["codes"].permute(0, 3, 2, 1, 4).reshape(n_slots, 2, s["Hkv"], D // 2)
    flat[dst] = flat[src]
    s["codes"].copy_(flat.view(-1, P, 2, s["Hkv"], D // 2).permute(0, 3, 2, 1, 4))
    if s["steps"] is not None:
        st = s["steps"].permute(0, 3, 2, 1).reshape(n_slots, 2, s["Hkv"])
        st[dst] = st[src]
        s["steps"].copy_(st.view(-1, P, 2, s["Hkv"]).permute(0, 3, 2, 1))
    slot = s["slot"].clamp(min=0)
    step = torch.stack((s["s_k"], s["s_v"]))[None] if s["steps"] is None else st[slot]
    values = (_nibbles(flat[slot]) * step[..., None]).to(torch.bfloat16)
    kv = torch.where((s["slot"] >= 0)[:, None, None, None], values, s["kv_out"])
    i32 = lambda t: t.to(torch.int32)
    return i32(kept), i32(count), i32(nxt), i32(len1), free[:n_pages], i32((n_free + back.sum()).reshape(1)), kv


# ---- work -------------------------------------------------------------------------------------------------
def work(case):
    total, new = _lengths(case)
    rows = sum(new)
    if case["kind"] == "plan":  # a parent read, a mask and a position written; offsets and lengths
        return dict(bytes=rows * (8 + 4 * _up(max(new), 32)) + 8 * case["B"], flops=0)
    if case["kind"] == "accept":
        # parents, drafts and choices read, paths written; offsets, lengths and counts; every draft's vectors read once (most of the moved rows among them) and
        # handed out
        vector = 64 + (4 if case["steps"] == "vector" else 0)
        return dict(bytes=rows * 16 + 20 * case["B"] + rows * case["Hkv"] * 2 * (vector + 256), flops=rows * case["Hkv"] * 2 * D)
    window, sinks = case["window"] or 1 << 40, case["sinks"]
    pairs = keys = 0
    trees = _trees(case) if case["kind"] == "tree" else [None] * case["B"]
    for t, n, parent in zip(total, new, trees):
        base, first = t - n, t
        for i, bits in enumerate(_ancestors(parent) if parent else range(n)):
            place = base + (bits.bit_count() - 1 if parent else i)
            lo = max(0, place - window + 1)
            pairs += N_PREFIX + place + 1 - lo + min(lo, sinks)
            first = min(first, lo)
        keys += t - first + min(first, sinks)
    a_key = 128 + (8 if case["steps"] == "vector" else 0)
    return dict(bytes=case["Hkv"] * (a_key * keys + N_PREFIX * 512) + rows * case["Hq"] * 512, flops=4 * D * case["Hq"] * pairs)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "plan":
        return None
    if case["kind"] == "accept":
        return _exact_accept(case, seed)
    return _exact_attn(case, seed)


def _exact_attn(case, seed):
    s = prepare(case, seed)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    P, G, window, sinks = s["page"], s["Hq"] // s["Hkv"], case["window"] or 1 << 40, case["sinks"]
    total, new = _lengths(case)
    trees = _trees(case) if case["kind"] == "tree" else None
    r0 = 0
    for b, (n_keys, n) in enumerate(zip(total, new)):
        page = s["table"][b, : _up(n_keys, P)].to(torch.int64)
        base = n_keys - n
        for lo in range(0, n, 256):  # bounded score matrices
            hi = min(n, lo + 256)
            rows = range(lo, hi)
            if trees is None:
                place = [base + t for t in rows]
                seen_new = None
            else:
                bits = _ancestors(trees[b])
                place = [base + bits[t].bit_count() - 1 for t in rows]
                seen_new = torch.tensor([[bool(bits[t] >> u & 1) for u in range(n)] for t in rows], device=DEV)
            first = max(0, min(place) - window + 1)
            pick = [i for i in range(min(first, sinks))] if first else []
            keys = torch.cat((torch.tensor(pick, dtype=torch.int64, device=DEV), torch.arange(first, n_keys, device=DEV)))  # those that some row sees
            at = torch.tensor(place, device=DEV)[:, None]
            see = (keys[None] > at - window) | (keys[None] < sinks)
            if seen_new is None:
                see &= keys[None] <= at
            else:
                is_new = keys >= base
                see &= ~is_new[None] | seen_new[:, (keys - base).clamp(min=0)]
            see = torch.cat((torch.ones((hi - lo, N_PREFIX), dtype=torch.bool, device=DEV), see), 1)
            for h in range(s["Hkv"]):
                kv = []
                for which, pre, head in ((0, s["pk"], s["s_k"]), (1, s["pv"], s["s_v"])):
                    c = s["codes"][page[keys // P], h, which, keys % P].to(torch.int16)
                    val = torch.stack((c % 16, c // 16), -1).flatten(1).to(torch.float64)
                    val = torch.where(val > 7, val - 16, val)
                    step = head[h].to(torch.float64) if s["steps"] is None else s["steps"][page[keys // P], h, which, keys % P][:, None].to(torch.float64)
                    kv.append(torch.cat((pre[h].to(torch.float64), val * step)))
                q = s["q"][r0 + lo: r0 + hi, h * G: (h + 1) * G].to(torch.float64)
                x = (q.reshape(-1, D) @ kv[0].T).view(hi - lo, G, -1) * SM_SCALE
                w = torch.softmax(x.masked_fill(~see[:, None], -math.inf), -1).view(-1, x.shape[-1])
                out[r0 + lo: r0 + hi, h * G: (h + 1) * G] = (w @ kv[1]).view(hi - lo, G, D)
        r0 += n
    return out


def _exact_accept(case, seed):
    s = prepare(case, seed)
    total, new = _lengths(case)
    trees, (draft, target) = _trees(case), _tokens(_trees(case), seed)
    P, r0 = s["page"], 0
    table = s["table"].tolist()
    come_from = [0] * (sum(new) + case["pad"])  # the slot whose vectors a row's slot holds in the end
    for b, (t, n) in enumerate(zip(total, new)):
        slot = [table[b][c // P] * P + c % P for c in range(t - n, t)]
        come_from[r0: r0 + n] = slot
        row, i = 0, 0
        while True:
            nxt = [c for c in range(n) if trees[b][c] == row and draft[r0 + c] == target[r0 + row]]
            if not nxt:
                break
            row, i = nxt[0], i + 1
            come_from[r0 + i] = slot[row]
        r0 += n
    at = _ints(come_from, torch.int64)
    c = s["codes"][at // P, :, :, at % P].to(torch.int16)  # [N, Hkv, 2, 64]
    val = torch.stack((c % 16, c // 16), -1).flatten(3).to(torch.float64)
    val = torch.where(val > 7, val - 16, val)
    step = torch.stack((s["s_k"], s["s_v"]), 1)[None] if s["steps"] is None else s["steps"][at // P, :, :, at % P]
    val = (val * step.to(torch.float64)[..., None]).permute(0, 2, 1, 3)
    return None, None, None, None, None, None, torch.where((s["slot"] >= 0)[:, None, None, None], val, 0.0)
