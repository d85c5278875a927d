"""The paged KV4 operators in 64 bits, written from their definitions with plain Python and torch, and builders of small caches."""
import math
import random

import torch

from paper_2410_05265_b200 import binding

D = 128


def up(a, b):
    return -(-a // b)


# ---- pages -------------------------------------------------------------------------------------------------
def plan(table, length, free, n_free, n_new, page, pos0, n_rows, n_pages):
    """(table, len, n_free, q_begin, slot, pos) of a step, or None where it cannot be served; lists of ints."""
    width = len(table[0]) if table else 0
    if any(l < 0 or n < 0 or l + n > width * page for l, n in zip(length, n_new)) or sum(n_new) > n_rows:
        return None
    need = [up(l + n, page) - up(l, page) for l, n in zip(length, n_new)]
    if sum(need) > n_free:
        return None
    table, stack, begin, slot, pos = [list(r) for r in table], list(free[:n_free]), [0], [], []
    for b, (l, n) in enumerate(zip(length, n_new)):
        for j in range(need[b]):
            table[b][up(l, page) + j] = stack.pop()
        for c in range(l, l + n):
            slot.append(table[b][c // page] * page + c % page)
            pos.append(pos0 + c)
        begin.append(begin[-1] + n)
    pad = n_rows - len(slot)
    return table, [l + n for l, n in zip(length, n_new)], len(stack), begin, slot + [-1] * pad, pos + [0] * pad


def release(table, length, free, n_free, done, page, n_pages):
    back = [i for b, d in enumerate(done) if d for i in table[b][: up(length[b], page)]]
    if n_free + len(back) > n_pages:
        return None
    return list(free[:n_free]) + back, [0 if d else l for l, d in zip(length, done)]


# ---- heads -------------------------------------------------------------------------------------------------
def hadamard(dev):
    i = torch.arange(D, device=dev)
    m = i[:, None] & i[None]
    return (1 - 2 * (sum((m >> k) & 1 for k in range(7)) % 2)).double() / math.sqrt(D)


def norm_rope(x, gain, eps, pos, theta, sections, rotate):
    """x bf16 [N, H, 128], pos int32 [axes, N] -> float64 [N, H, 128]."""
    v = x.double()
    if gain is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * gain.double()
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device=x.device)
    i = torch.arange(64, device=x.device, dtype=torch.float64)
    ang = pos.double()[axis].T * theta ** (-2.0 * i / 128)
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    a, b = v[..., :64], v[..., 64:]
    y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return y @ hadamard(x.device) if rotate else y


def step_of(y):
    mx = y.abs().amax(-1)
    return torch.where(mx < 2.0**-57, 1.0, (mx / 7).float().double()).float()


def codes_of(y, s):
    return torch.clamp(torch.round((y / s.double()).float()), -8, 7).to(torch.int8)


def unpack(c):
    c = c.to(torch.int16)
    lo, hi = ((c & 15) ^ 8) - 8, ((c >> 4) ^ 8) - 8
    return torch.stack((lo, hi), -1).flatten(-2)


# ---- attention ---------------------------------------------------------------------------------------------
def attention(cache, q, begin, lengths, sm_scale):
    """(float64 outputs, tolerance) of every row.

    A row is sum w v / sum w. A weight is off by its rounding to fp16 (2^-11) and by its exponent's error: the score is a sum of 128 products
    in fp32, off by at most 2^-23 (a truncating accumulation) x 128 x sum |q||k|, times ln 2 in log2 units; the hardware's 2^x and log2 add 2^-20. A relative
    error e of the weights moves the quotient by at most 2 e max|v|. The result is rounded to bf16: 2^-8 of the value, and twice the
    smallest normal number for results that vanish."""
    pages = cache.pages
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    table = pages.table.tolist()
    G = cache.Hq // cache.Hkv
    for b, n_keys in enumerate(lengths):
        r0, n = begin[b], begin[b + 1] - begin[b]
        if n == 0:
            continue
        ids = torch.tensor(table[b][: up(n_keys, pages.page)], dtype=torch.int64, device=q.device)
        kv = unpack(cache.codes[ids]).double()  # [pages, Hkv, 2, page, 128]
        if cache.steps is not None:
            kv = kv * cache.steps[ids].double()[..., None]
        else:
            kv = kv * torch.stack((cache.s_k, cache.s_v), 1).double()[None, :, :, None, None]
        kv = kv.permute(1, 2, 0, 3, 4).reshape(cache.Hkv, 2, -1, D)[:, :, :n_keys]
        k, v = kv[:, 0], kv[:, 1]
        if cache.n_prefix:
            k, v = torch.cat((cache.prefix_k.double(), k), 1), torch.cat((cache.prefix_v.double(), v), 1)
        for t in range(n):
            seen = cache.n_prefix + max(0, n_keys - n + t + 1)
            if seen == 0:
                continue
            qr = q[r0 + t].double().view(cache.Hkv, G, D)
            x = qr @ k[:, :seen].transpose(1, 2) * sm_scale
            w = torch.softmax(x, -1)
            o = w @ v[:, :seen]
            off = (qr.abs() @ k[:, :seen].abs().transpose(1, 2)).amax(-1, keepdim=True) * sm_scale * 2.0**-16
            e = 2.0**-11 + 2.0**-20 + off
            out[r0 + t] = o.reshape(cache.Hq, D)
            tol[r0 + t] = (o.abs() * 2.0**-8 + 2 * e * v[:, :seen].abs().amax((1, 2))[:, None, None] + 2.0**-125).reshape(cache.Hq, D)
    return out, tol


def make_cache(lengths, Hq, Hkv, page, steps="head", n_prefix=4, seed=0, spread=2.6, extra_pages=3, width=None, step_range=(-1.5, 0.5), device="cuda"):
    """A cache of random codes whose pages lie scattered over the pool; entries behind a sequence's pages hold ids that are none."""
    g = torch.Generator(device=device).manual_seed(seed)
    rng = random.Random(seed)
    need = [up(n, page) for n in lengths]
    n_pages = sum(need) + extra_pages
    ids = list(range(n_pages))
    rng.shuffle(ids)
    width = width or max(need + [1]) + 2
    table, at = [], 0
    for k in need:
        table.append(ids[at: at + k] + [-7] * (width - k))
        at += k
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)
    free = ids[at:] + [0] * at
    pages = binding.Pages(i32(table), i32(lengths), i32(free), i32([n_pages - at]), page)
    c = torch.clamp(torch.round(spread * torch.randn((n_pages, Hkv, 2, page, D), generator=g, device=device)), -8, 7).to(torch.int16) & 15
    codes = (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)
    lo, hi = step_range
    rand = lambda *sh: torch.exp2(lo + (hi - lo) * torch.rand(sh, generator=g, device=device))
    s_k, s_v, st = (None, None, rand(n_pages, Hkv, 2, page)) if steps == "vector" else (rand(Hkv), rand(Hkv), None)
    pk = pv = None
    if n_prefix:
        pk, pv = (torch.randn((Hkv, n_prefix, D), generator=g, device=device).mul_(s).half() for s in (1.5, 0.5))
    return binding.KV4PagedCache(pages, pk, pv, codes.contiguous(), Hq, s_k=s_k, s_v=s_v, steps=st)


def queries(n, Hq, seed=1, scale=1.2, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed + 1000)
    return (scale * torch.randn((n, Hq, D), generator=g, device=device)).bfloat16()
