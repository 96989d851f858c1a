"""The paged cache and drafted decoding in 64 bits on the CPU, as include/wnw.h defines them, for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch


def clamp(x, hi):
    return min(max(int(x), 0), hi)


def place(table, b, row, page, pages):
    """(page, row in it) of a sequence's row, or None where there is no page."""
    if row >= table.shape[1] * page:
        return None
    p = int(table[b, row // page])
    return (p, row % page) if 0 <= p < pages else None


def rotate(x, position, freq, dim, pairs, amplitude):
    """x [..., d] double at a position -> (rotated, |x0| + |x1| of each element's pair, which elements are rotated)."""
    y, size = x.clone(), torch.zeros_like(x)
    h = dim // 2
    if h:
        a = (torch.arange(0, dim, 2), torch.arange(1, dim, 2)) if pairs else (torch.arange(h), torch.arange(h) + h)
        angle = torch.from_numpy(np.asarray(freq, dtype=np.float64)) * float(position)
        c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
        x0, x1 = x[..., a[0]], x[..., a[1]]
        y[..., a[0]], y[..., a[1]] = x0 * c - x1 * s, x1 * c + x0 * s
        for i in a:
            size[..., i] = (x0.abs() + x1.abs()) * abs(amplitude)
    return y, size


def ancestors(parent):
    """[n][n] bool: token i sees token j."""
    n = len(parent)
    see = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parent):
        if 0 <= p < i:
            see[i] = see[p]
        see[i, i] = True
    return see


def words(see):
    """[n][n] bool -> int64 [n][(n + 63) / 64]."""
    n = see.shape[0]
    w = (n + 63) // 64
    out = np.zeros((n, w), dtype=np.uint64)
    for i, j in zip(*np.nonzero(see)):
        out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return torch.from_numpy(out.view(np.int64))


def gather(pool, table, b, layers, rows, page):
    """(rows 0 .. rows - 1 of sequence b [layers][H][rows][d] double, zeros without a page; which have one)."""
    P, L, H, _, D = pool.shape
    out = torch.zeros((len(layers), H, rows, D), dtype=torch.float64)
    there = torch.zeros(rows, dtype=torch.bool)
    for j in range(-(-rows // page)):
        p, r1 = int(table[b, j]), min(rows, (j + 1) * page)
        if 0 <= p < P:
            out[:, :, j * page: r1] = pool[p, layers, :, : r1 - j * page].double()
            there[j * page: r1] = True
    return out, there


def attend(q, k, v, table, page, lens, counts, see=None, layer0=0):
    """q [B][nl][Hq][n][d] (any float type), pools k, v -> out, lse, and for error bounds sum p |v|, the largest logit's
    sum |q k| / sqrt(d), and rows seen; tokens past a count are NaN.  see: [B] of [n][n] bool, or None (causal)."""
    B, nl, Hq, n, D = q.shape
    H, cap = k.shape[2], table.shape[1] * page
    G, layers = Hq // H, list(range(layer0, layer0 + nl))
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:-1], math.nan, dtype=torch.float64)
    absv, absq, seen = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    for b in range(B):
        T = clamp(lens[b], cap)
        c = min(clamp(counts[b], n), T)
        kk, there = gather(k, table, b, layers, T, page)
        vv, _ = gather(v, table, b, layers, T, page)
        for i in range(c):
            sees = there.clone()
            if see is None:
                sees[T - c + i + 1:] = False
            else:
                sees[T - c:] &= torch.from_numpy(see[b][i, :c])
            for hq in range(Hq):
                k_, v_, q_ = kk[:, hq // G, sees], vv[:, hq // G, sees], q[b, :, hq, i].double()
                x = (k_ @ q_.unsqueeze(-1)).squeeze(-1) / math.sqrt(D)
                lse[b, :, hq, i] = torch.logsumexp(x, dim=-1) if sees.any() else -math.inf
                p = torch.softmax(x, dim=-1)
                out[b, :, hq, i] = (p.unsqueeze(1) @ v_).squeeze(1)
                absv[b, :, hq, i] = (p.unsqueeze(1) @ v_.abs()).squeeze(1)
                if sees.any():
                    absq[b, :, hq, i] = (k_.abs() @ q_.abs().unsqueeze(-1)).squeeze(-1).amax(dim=-1) / math.sqrt(D)
                seen[b, :, hq, i] = int(sees.sum())
    return out, lse, absv, absq, seen


def verify(token, parent, count, target, draft, uniform):
    """One sequence: (path, next).  parent: list or None; target, draft [n + 1][V] arrays; uniform [n + 1]."""
    n, V = len(token), target.shape[1]
    parent = [i - 1 for i in range(n)] if parent is None else [p if 0 <= p < i else -1 for i, p in enumerate(parent)]
    node, path = -1, []
    while True:
        p, s, moved = target[node + 1].astype(np.float64), 1.0, False
        for i in range(clamp(count, n)):
            if parent[i] != node or i <= node:
                continue
            x = token[i]
            if not 0 <= x < V:
                if draft is not None:
                    p = np.maximum(p - draft[node + 1], 0)
                    p = p / p.sum() if p.sum() > 0 else p
                continue
            q = draft[node + 1].astype(np.float64) if draft is not None else None
            if float(uniform[i]) * (q[x] if q is not None else s) < p[x]:
                node, moved = i, True
                path.append(i)
                break
            if q is not None:
                p = np.maximum(p - q, 0)
                p = p / p.sum() if p.sum() > 0 else p
            else:
                s -= p[x]
                p[x] = 0
        if not moved:
            break
    if not p.sum() > 0:
        p = np.maximum(target[node + 1].astype(np.float64), 0)
    total = p.cumsum()
    if not 0 < total[-1] < math.inf:
        return path, -1
    over = np.nonzero((total > float(uniform[n]) * total[-1]) & (p > 0))[0]
    return path, int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])
