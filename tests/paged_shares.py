"""How wnw_paged_attend shares a call out, found again on the host, so that a test can say which way it goes; and its
outputs in 64 bits on the GPU, for calls that are too large for paged_reference."""
from __future__ import annotations

import math

import numpy as np
import torch

BLOCK_COST, MIN_PIECE = 8, 4


def clamp(x, hi):
    return min(max(int(x), 0), hi)


def block_rows(rows):
    """Query rows of a block, for so many of a KV-head."""
    return next((r for r in (16, 32, 64, 128) if rows <= r), 256)


def at_least(x, inv):
    return int(np.float32(np.float32(x) * inv) * np.float32(1.000001)) + 1


def piece_len(tiles, most):
    n = -(-tiles // most)
    return -(-tiles // n)


def share(W, cfg, n_layers, q_heads, n, lens, counts=None, max_len=0):
    """(query rows of a block, "whole" / "pieces" / "line", work-groups)."""
    G, heads = q_heads // cfg.kv_heads, n_layers * cfg.kv_heads
    RB = block_rows(G * n)
    need = W.wnw_paged_attend_workspace(cfg, n_layers, q_heads, n, max_len)
    if need == 0:
        return RB, "whole", cfg.batch * heads * -(-G * n // RB)
    groups, rest = divmod(need, 2 * RB * (cfg.head_dim * 4 + 8))
    assert rest == 0
    tile, cap = 64 if cfg.head_dim == 64 or RB > 32 else 32, cfg.table_width * cfg.page
    units = [-(-clamp(n if counts is None else counts[b], n) * G // RB) * heads for b in range(cfg.batch)]
    tiles = [max(1, -(-clamp(x, cap) // tile)) for x in lens]
    total = sum((t + BLOCK_COST) * u for t, u in zip(tiles, units))
    per = max(at_least(total, np.float32(1) / np.float32(groups)), MIN_PIECE)
    if sum(units) < groups:
        longest = max([t for t, u in zip(tiles, units) if u], default=0)
        p = min(max(at_least(total - sum(units) * BLOCK_COST, np.float32(1) / np.float32(groups - sum(units))), MIN_PIECE), longest)
        if p and piece_len(longest, p) <= per:
            return RB, "pieces", groups
    return RB, "line", groups


def exact(q, k, v, table, page, lens, counts, see=None):
    """What paged_reference.attend gives, computed and left where q is: q [B][L][Hq][n][d], pools and table there too, every
    entry of which that a sequence uses has a page; see: [B] of [n][n] bool, or None."""
    B, L, Hq, n, D = q.shape
    H = k.shape[2]
    G = Hq // H
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:-1], math.nan, dtype=torch.float64, device=q.device)
    absv, absq, seen = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    for b in range(B):
        T = clamp(lens[b], table.shape[1] * page)
        c = min(clamp(counts[b], n), T)
        if not c:
            continue
        used = table[b, : -(-T // page)].long()
        kk, vv = (x[used].permute(1, 2, 0, 3, 4).reshape(L, H, -1, D)[:, :, :T].double() for x in (k, v))
        sees = torch.ones((c, T), dtype=torch.bool)
        own = np.tril(np.ones((n, n), dtype=bool)) if see is None else see[b]
        sees[:, T - c:] = torch.from_numpy(own[:c, :c].copy())
        unseen = ~sees.to(q.device)
        for l in range(L):
            rows = q[b, l, :, :c].double().reshape(H, G * c, D)
            keys = kk[l].transpose(-1, -2).contiguous()
            x = (torch.matmul(rows, keys) / math.sqrt(D)).reshape(H, G, c, T).masked_fill(unseen, -math.inf)
            size = (torch.matmul(rows.abs(), keys.abs()) / math.sqrt(D)).reshape(H, G, c, T).masked_fill(unseen, 0.0)
            p = torch.softmax(x, dim=-1).reshape(H, G * c, T)
            lse[b, l, :, :c] = torch.logsumexp(x, dim=-1).reshape(Hq, c)
            absq[b, l, :, :c] = size.amax(dim=-1).reshape(Hq, c)
            out[b, l, :, :c] = torch.matmul(p, vv[l]).reshape(Hq, c, D)
            absv[b, l, :, :c] = torch.matmul(p, vv[l].abs()).reshape(Hq, c, D)
        seen[b, :, :, :c] = sees.sum(dim=-1).double().to(q.device)
    return out, lse, absv, absq, seen


# Softmax weights one by one.  Logits are k / sqrt(d) for one element k of a row of K, a multiple of 1 / 16 in -8 .. 8, and the largest, 8, is in
# every tile; a dimension of the output is one row's weight over their sum.  Then nothing but the weights is rounded: in units of 2^-24,
#   the scale (log2 e rounded, sqrt(d) rounded, their quotient) is off by 3, so that a weight is by 3 |x - 8| ln 2 <= 3 * 16 / sqrt(d) <= 6;
#   k times the scale and less the maximum are two steps, of at most 1.45 and 2.89: ln 2 * 4.34 <= 3.01; the exponential 2^-22: 4; the
#   product with 1 / sum: 1.  The sum itself is common to all of a query row's outputs.
WEIGHT_SPREAD = (6 + 2 * (3.01 + 4 + 1)) * 2.0 ** -24


def weight_keys(g, *shape):
    """Rows of K [..., rows][d]."""
    k = torch.randint(-128, 128, shape, generator=g, device=g.device).float() / 16
    k[..., ::8, :] = 8.0
    return k


def weight_rows(g, rows, d):
    """Which row every dimension of the output is the weight of, -1: none."""
    at = torch.randperm(rows, generator=g, device=g.device)[:d]
    return torch.cat([at, at.new_full((d - len(at),), -1)])


def weight_spread(out, want):
    """How far apart the ratios of weights and exact ones are, over every query row's outputs [..., d] that are not zero."""
    some = want > 0
    r = torch.where(some, out / torch.where(some, want, torch.ones_like(want)), torch.ones_like(want) * math.nan)
    top, low = torch.where(some, r, -math.inf).amax(dim=-1), torch.where(some, r, math.inf).amin(dim=-1)
    return top / low - 1
