"""The 8-bit cache in 64 bits on the CPU: the arithmetic that include/wnw.h defines, row by row and block by
block, for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch

INT8, E4M3 = 0, 1
TINY = 2.0 ** -126


def e4m3_grid():
    """The non-negative finite e4m3 numbers by code 0 .. 126."""
    return np.array([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127])


def numbers(fmt):
    """What the 256 bytes stand for, before the scale."""
    if fmt == INT8:
        return np.arange(256) - 128.0
    g = np.concatenate([e4m3_grid(), [np.nan]])
    return np.concatenate([g, -g])


def scale_of(amax, fmt):
    if not np.isfinite(amax):
        return math.nan
    if fmt == INT8:
        return max(float(np.float32(np.float64(amax) / 127)), TINY)
    s = TINY
    while amax > 448 * s:
        s *= 2
    return s


def round_to(x, s, fmt):
    """Codes' numbers of x under scale s: nearest, ties to even (double; exact for the tests' inputs)."""
    y = np.asarray(x, dtype=np.float64) / s
    if fmt == INT8:
        return np.rint(y)
    g = e4m3_grid()
    a = np.abs(y)
    hi = np.clip(np.searchsorted(g, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = g[hi] - a, a - g[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(g[pick], y)


class Cache:
    """Numbers [B][L][H][capacity][d] and scales of K or V."""

    def __init__(self, B, L, H, cap, D, block, fmt):
        self.num = np.zeros((B, L, H, cap, D))
        self.scale = np.full((B, L, H, cap // block), np.nan)
        self.block, self.fmt, self.cap = block, fmt, cap

    def write(self, x, pos, count, layer0=0):
        """x [B][nl][H][n][d] double."""
        for b in range(x.shape[0]):
            p = min(max(int(pos[b]), 0), self.cap)
            e = min(p + min(max(int(count[b]), 0), x.shape[3]), self.cap)
            if e == p:
                continue
            for j in range(p // self.block, (e - 1) // self.block + 1):
                r0, r1 = max(p, j * self.block), min(e, (j + 1) * self.block)
                for l in range(x.shape[1]):
                    for h in range(x.shape[2]):
                        rows = x[b, l, h, r0 - p: r1 - p]
                        s = scale_of(np.abs(rows).max(), self.fmt)
                        n = self.num[b, layer0 + l, h]
                        if p > j * self.block:
                            was = self.scale[b, layer0 + l, h, j]
                            s = math.nan if math.isnan(was) or math.isnan(s) else max(was, s)
                            if s > was:
                                n[j * self.block: p] = round_to(n[j * self.block: p] * was, s, self.fmt)
                        self.scale[b, layer0 + l, h, j] = s
                        n[r0:r1] = 0.0 if math.isnan(s) else round_to(rows, s, self.fmt)

    def values(self):
        return self.num * np.repeat(self.scale, self.block, axis=3)[..., None]


def v_place(r):
    return r % 16 // 4 * 16 + r // 16 * 4 + r % 4


def decode_k(t, fmt):
    return numbers(fmt)[t.cpu().numpy()]


def decode_v(t, fmt):
    x = numbers(fmt)[t.cpu().numpy()][..., [v_place(r) for r in range(64)]]
    x = np.swapaxes(x, -1, -2)
    return x.reshape(*x.shape[:3], -1, x.shape[-1])


def encode(num, fmt):
    """Bytes of numbers [B][L][H][capacity][d] as torch uint8 in K's layout."""
    if fmt == INT8:
        return torch.from_numpy((num + 128).astype(np.uint8))
    code = np.searchsorted(e4m3_grid(), np.abs(num)) + 128 * np.signbit(num)
    return torch.from_numpy(code.astype(np.uint8))


def k_to_v(k):
    """K's byte layout -> V's."""
    order = np.argsort([v_place(r) for r in range(64)])
    return k.unflatten(3, (-1, 64))[..., order, :].transpose(-1, -2).contiguous()


def attend(q, k, v, lens, counts, block):
    """float64 tensors q [B][L][Hq][n][d], k, v [B][L][H][cap][d] -> out, lse, mass, and for error bounds
    sum_t p |v|, for each output row the largest sum_d |q k| / sqrt(d), and rows seen times the largest |v|.  Tokens past a count are NaN."""
    B, L, Hq, n, D = q.shape
    H, cap = k.shape[2], k.shape[3]
    G = Hq // H
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:-1], math.nan, dtype=torch.float64)
    mass = torch.full((B, L, Hq, n, cap // block), math.nan, dtype=torch.float64)
    absv, absq, sumv = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    for b in range(B):
        T, c = min(max(int(lens[b]), 0), cap), min(max(int(counts[b]), 0), n)
        for i in range(c):
            see = max(0, min(T, T - c + i + 1))
            for hq in range(Hq):
                kk, vv = k[b, :, hq // G, :see], v[b, :, hq // G, :see]
                qq = q[b, :, hq, i]
                x = (kk @ qq.unsqueeze(-1)).squeeze(-1) / math.sqrt(D)     # [L][see]
                lse[b, :, hq, i] = torch.logsumexp(x, dim=-1) if see else -math.inf
                p = torch.softmax(x, dim=-1)
                out[b, :, hq, i] = (p.unsqueeze(1) @ vv).squeeze(1)
                w = torch.zeros((L, cap), dtype=torch.float64)
                w[:, :see] = p
                mass[b, :, hq, i] = w.unflatten(-1, (-1, block)).sum(dim=-1)
                absv[b, :, hq, i] = (p.unsqueeze(1) @ vv.abs()).squeeze(1)
                if see:
                    absq[b, :, hq, i] = (kk.abs() @ qq.abs().unsqueeze(-1)).squeeze(-1).amax(dim=-1) / math.sqrt(D)
                    sumv[b, :, hq, i] = see * vv.abs().amax(dim=(1, 2))
    return out, lse, mass, absv, absq, sumv


def attend_fast(q, k, v, lens, counts, block):
    """attend() with a product per sequence, on the tensors' device."""
    B, L, Hq, n, D = q.shape
    H, cap = k.shape[2], k.shape[3]
    G = Hq // H
    outs = [[] for _ in range(6)]
    key = torch.arange(cap, device=q.device)
    for b in range(B):
        T, c = min(max(int(lens[b]), 0), cap), min(max(int(counts[b]), 0), n)
        limit = (T - c + torch.arange(n, device=q.device) + 1).clamp(0, T)          # rows that token i sees
        sees = key < limit[:, None]
        qq = q[b].reshape(L, H, G * n, D)
        dead = (key >= T)[:, None]
        kk, vv = k[b].masked_fill(dead, 0.0), v[b].masked_fill(dead, 0.0)
        x = (qq @ kk.transpose(-1, -2) / math.sqrt(D)).reshape(L, H, G, n, cap).masked_fill(~sees, -math.inf)
        lse = torch.logsumexp(x, dim=-1)
        p = torch.where(sees, torch.exp(x - lse.unsqueeze(-1)), 0.0)
        absq = (qq.abs() @ kk.abs().transpose(-1, -2) / math.sqrt(D)).reshape(L, H, G, n, cap).masked_fill(~sees, 0.0).amax(dim=-1)
        pr = p.reshape(L, H, G * n, cap)
        got = ((pr @ vv), lse, p.unflatten(-1, (-1, block)).sum(dim=-1), (pr @ vv.abs()), absq,
               (limit * vv.abs().amax(dim=(2, 3))[:, :, None, None]).expand(L, H, G, n))
        token = torch.arange(n, device=q.device) < c
        for o, t, width in zip(outs, got, (D, None, cap // block, D, None, None)):
            t = t.reshape(L, Hq, n, *([width] if width else []))
            gone = (~token).reshape(1, 1, n, *([1] if width else []))
            o.append(t.masked_fill(gone, math.nan) if o is not outs[3] and o is not outs[4] and o is not outs[5] else t)
    return tuple(torch.stack(o) for o in outs)
