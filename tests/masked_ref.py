"""Windowed attention, attention of drafted trees and what follows a verification, from their definitions: 64 bits, plain Python and torch."""
import random

import torch

from paged_ref import D, unpack, up


def visible(n_keys, n, t, window=0, n_sink=0, sees=None):
    """Truth values of the cached keys of a sequence for its row t of n; sees [n][n]: what the rows see of one another (None: those before them)."""
    j = torch.arange(n_keys)
    base = n_keys - n
    if sees is None:
        place, see = base + t, j <= base + t
    else:
        row = torch.tensor(sees[t])
        row[t] = True
        place = base + int(row.sum()) - 1
        see = j < base
        see[max(base, 0):] |= row[max(base, 0) - base:]
    return see & ((j > place - window) | (j < n_sink)) if window else see


def attention(cache, q, begin, lengths, sm_scale, window=0, n_sink=0, trees=None):
    """(float64 outputs, tolerance) of every row; trees: for every sequence what its rows see of one another.

    The tolerance is counted as in paged_ref.attention: a weight is off by its rounding to fp16 (2^-11), by the hardware's 2^x and log2 (2^-20) and by its score's
    error (a sum of 128 products in fp32: 2^-23 x 128 x sum |q||k|, in log2 units times ln 2); a relative error e of the weights moves the quotient by 2 e max|v| at
    most over the visible keys; the result is rounded to bf16 (2^-8), twice the smallest normal number where it vanishes."""
    pages = cache.pages
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    table = pages.table.tolist()
    G = cache.Hq // cache.Hkv
    for b, n_keys in enumerate(lengths):
        r0, n = begin[b], begin[b + 1] - begin[b]
        for t in range(n):
            keys = torch.nonzero(visible(n_keys, n, t, window, n_sink, trees[b] if trees else None))[:, 0].tolist()
            at = torch.tensor([table[b][c // pages.page] * pages.page + c % pages.page for c in keys], dtype=torch.int64, device=q.device)
            page, inside = at // pages.page, at % pages.page
            kv = unpack(cache.codes[page, :, :, inside]).double()  # [keys, Hkv, 2, 128]
            if cache.steps is not None:
                kv = kv * cache.steps[page, :, :, inside].double()[..., None]
            else:
                kv = kv * torch.stack((cache.s_k, cache.s_v), 1).double()[None, ..., None]
            k, v = kv[:, :, 0].transpose(0, 1), kv[:, :, 1].transpose(0, 1)
            if cache.n_prefix:
                k, v = torch.cat((cache.prefix_k.double(), k), 1), torch.cat((cache.prefix_v.double(), v), 1)
            if k.shape[1] == 0:
                continue
            qr = q[r0 + t].double().view(cache.Hkv, G, D)
            w = torch.softmax(qr @ k.transpose(1, 2) * sm_scale, -1)
            o = w @ v
            off = (qr.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True) * sm_scale * 2.0**-16
            e = 2.0**-11 + 2.0**-20 + off
            out[r0 + t] = o.reshape(cache.Hq, D)
            tol[r0 + t] = (o.abs() * 2.0**-8 + 2 * e * v.abs().amax((1, 2))[:, None, None] + 2.0**-125).reshape(cache.Hq, D)
    return out, tol


def hide_unseen_pages(cache, begin, lengths, window, n_sink, trees=None):
    """Ids that are none where no row of the sequence sees a key of the page; with own steps no number in the steps of the keys that no row sees."""
    pages, used = cache.pages, set()
    table = pages.table.tolist()
    for b, n_keys in enumerate(lengths):
        n = begin[b + 1] - begin[b]
        if n == 0:
            continue
        see = torch.stack([visible(n_keys, n, t, window, n_sink, trees[b] if trees else None) for t in range(n)]).any(0).tolist()
        for c in range(n_keys):
            if see[c]:
                used.add(table[b][c // pages.page] * pages.page + c % pages.page)
        for w in range(up(n_keys, pages.page)):
            if not any(see[w * pages.page: (w + 1) * pages.page]):
                pages.table[b, w] = -9 - b
    if cache.steps is not None:
        keep = torch.zeros(cache.codes.shape[0] * pages.page, dtype=torch.bool)
        keep[sorted(used)] = True
        keep = keep.view(-1, 1, 1, pages.page).to(cache.steps.device)
        cache.steps.copy_(torch.where(keep, cache.steps, torch.full_like(cache.steps, float("nan"))))


def random_tree(rng, n, width, roots=1):
    return [-1 if t < roots else rng.randint(max(0, t - width), t - 1) for t in range(n)]


def ancestors(parent):
    """[n][n] truth values: what every row sees of its tree."""
    n, out = len(parent), []
    for t, p in enumerate(parent):
        row = [False] * n
        if p >= 0:
            row = list(out[p])
        row[t] = True
        out.append(row)
    return out


def words_of(trees, words, n_rows, device="cuda"):
    rows = []
    for sees in trees:
        for row in sees:
            bits = sum(1 << u for u, s in enumerate(row) if s)
            w = [(bits >> (32 * i)) & 0xFFFFFFFF for i in range(words)]
            rows.append([x - (1 << 32) if x >> 31 else x for x in w])
    return torch.tensor(rows + [[0] * words] * (n_rows - len(rows)), dtype=torch.int32, device=device).reshape(n_rows, words)


def accept(parent, draft, target):
    """(path, choice after its last row) of one tree."""
    if not parent:
        return [], -1
    path = [0]
    while True:
        r = path[-1]
        nxt = [c for c in range(1, len(parent)) if parent[c] == r and draft[c] == target[r]]
        if not nxt:
            return path, target[r]
        path.append(nxt[0])
