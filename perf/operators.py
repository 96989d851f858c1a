"""The operators of the 8-bit cache and their plain forms: quantising a KV cache as it is written, reading it
back, and attention over it.

A case is a dict of plain values.  `kind` says which call a pass makes:

* "store"    new K and V rows are quantised into the cache behind the rows that are there, and the last rows
             of every sequence are read back (wnw_quant_write, wnw_quant_read);
* "read"     rows of the cache as they stand for (wnw_quant_read);
* "attend"   attention of a sequence's last n tokens over its cache: output, log-sum-exp of every query row
             and, for single tokens, the softmax mass of every block of rows (wnw_quant_attend).

The cache of a batch: K as bytes [B][L][H_kv][capacity][d]; V as bytes [B][L][H_kv][capacity / 64][d][64], the
rows of a tile of 64 in the order that _place() gives; a scale for every `block` rows of a head,
fp32 [B][L][H_kv][capacity / block].  A byte is code + 128 (int8, code in -127 .. 127) or an e4m3 number.

Shapes are those of the backbones in synth/configs.py (30 layers, 32 query / 8 KV heads; 36 layers, 16 / 2;
one layer, 24 / 8), with ten minutes to an hour of audio, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

TILE = 64
VOXTRAL = dict(layers=30, q_heads=32, kv_heads=8)
QWEN = dict(layers=36, q_heads=16, kv_heads=2)
ONE = dict(layers=1, q_heads=24, kv_heads=8)


def _store(name, shape, rows, n, fmt, block, **kw):
    c = dict(kind="store", batch=1, rows=rows, n=n, back=n, fmt=fmt, block=block, head_dim=128, ragged=False, bf16=True)
    c.update(shape, **kw)
    return dict(c, name=name) if name else c


def _read(name, shape, rows, fmt, block, **kw):
    c = dict(kind="read", batch=1, rows=rows, fmt=fmt, block=block, head_dim=128, ragged=False, bf16=False)
    c.update(shape, **kw)
    return dict(c, name=name) if name else c


def _attend(name, shape, rows, n, fmt, block, **kw):
    c = dict(kind="attend", batch=1, rows=rows, n=n, fmt=fmt, block=block, head_dim=128, ragged=False, bf16=False,
             mass=n == 1)
    c.update(shape, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token joins one layer's cache of 40 s of audio; its last two chunks are read back
        _store("append_tiny", ONE, 1063, 1, "int8", 32, back=64),
        # a batch of three at ragged positions takes a few tokens at once (a draft that was accepted)
        _store("append_b3", VOXTRAL, 9377, 7, "e4m3", 64, batch=3, back=64, ragged=True),
        # the prompt of ten minutes of audio on the 2-KV-head backbone, as prefill leaves it
        _store("fill_qwen", QWEN, 0, 7756, "int8", 32),
        # the same on the 8-KV-head backbone
        _store("fill_voxtral", VOXTRAL, 0, 15512, "e4m3", 64),
        # a batch's caches read back in 32 bits, for calibration
        _read("read_b4", QWEN, 7756, "int8", 16, batch=4, ragged=True),
        # a generated token attends: the smallest cache, one layer
        _attend("token_tiny", ONE, 1064, 1, "int8", 32),
        # all layers, ten minutes at 12.5 tokens/s
        _attend("token_qwen", QWEN, 7756, 1, "e4m3", 32),
        # all layers, ten minutes at 25 tokens/s, bf16 output
        _attend("token_voxtral", VOXTRAL, 15512, 1, "int8", 64, bf16=True),
        # an hour of audio
        _attend("token_hour", VOXTRAL, 91024, 1, "e4m3", 64),
        # a serving batch of sixteen ragged sequences (one empty, one of a single row), one layer, smaller heads
        _attend("token_b16", dict(layers=1, q_heads=32, kv_heads=8), 20011, 1, "int8", 16, batch=16, ragged=True,
                head_dim=64, bf16=True),
        # a draft of five tokens is checked, a batch of three
        _attend("draft_b3", VOXTRAL, 9381, 5, "int8", 64, batch=3, ragged=True),
        # a layer's instruction tokens over ten minutes of audio
        _attend("text_voxtral", dict(VOXTRAL, layers=2), 15512, 512, "e4m3", 64, bf16=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges (lengths on a logarithmic scale, odd ones among them)."""
    kind = rng.choice(["store", "store", "read", "attend", "attend", "attend", "attend", "attend"])
    kv = rng.choice([1, 2, 3, 8])
    shape = dict(rng.choice([VOXTRAL, QWEN, dict(layers=rng.randint(1, 8), q_heads=24, kv_heads=8),
                             dict(layers=rng.randint(1, 4), q_heads=kv * rng.choice([1, 2, 5, 8, 16]), kv_heads=kv)]))
    batch = rng.choice([1, 1, 2, 3, 5, 16])
    heads = batch * shape["layers"] * shape["kv_heads"]
    kw = dict(batch=batch, ragged=batch > 1 and rng.random() < 0.7, head_dim=rng.choice([128, 128, 64]),
              bf16=rng.random() < 0.5)
    fmt, block = rng.choice(["int8", "e4m3"]), rng.choice([16, 32, 64])
    if kind == "attend":
        n = rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 512)])
        top = min(91024, 240 * 91024 // heads)
        if n > 1:
            top = min(top, 2 * 32 * 512 * 15512 // (batch * shape["layers"] * shape["q_heads"] * n))
        rows = max(n, _log_int(rng, 1, max(2, top)))
        return _attend("", shape, rows, n, fmt, block, **kw)
    top = min(15512, 240 * 15512 // heads)
    if kind == "read":
        return _read("", shape, _log_int(rng, 1, top), fmt, block, **kw)
    if rng.random() < 0.5:
        return _store("", shape, 0, _log_int(rng, 20, max(21, top)), fmt, block, **kw)
    return _store("", shape, _log_int(rng, 1, top), rng.randint(1, 9), fmt, block, back=64, **kw)


# ---- sizes and layout ------------------------------------------------------------------------


def _lengths(c, most):
    """Rows of every sequence; ragged: the first has the most, one has a single row, one none."""
    B = c["batch"]
    if not c["ragged"]:
        return [most] * B
    r = [max(1, int(most * math.exp(-3 * ((b * 0.618) % 1.0)))) if most else 0 for b in range(B)]
    if B >= 4 and most:
        r[1], r[2] = 1, 0
    return r


def _counts(c, n):
    """Tokens of every sequence in a call: up to n."""
    return [max(1, n - b) if c["ragged"] else n for b in range(c["batch"])]


def _capacity(c):
    most = c["rows"] + (c["n"] if c["kind"] == "store" else 0)
    return (most + TILE - 1) // TILE * TILE + TILE


def _place(r):
    """Where row r (0 .. 63) of a tile stands in the V tile: rows 16 b + 4 h + i at 16 h + 4 b + i."""
    return r % 16 // 4 * 16 + r // 16 * 4 + r % 4


def _k_rows(k):
    """[B][capacity][L][H_kv][d], a view of K's bytes."""
    return k.permute(0, 3, 1, 2, 4)


def _v_rows(v):
    """[B][tile][16-row part][4-row part][row][L][H_kv][d], a view of V's bytes: the places of _place()."""
    return v.unflatten(-1, (4, 4, 4)).permute(0, 3, 6, 5, 7, 1, 2, 4)


def _at(idx):
    """Indexes of rows idx in _v_rows()."""
    return idx // TILE, idx % TILE // 16, idx % 16 // 4, idx % 4


# ---- inputs ----------------------------------------------------------------------------------


def _rng(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 64 + tag) % (1 << 62))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, H, T, D):
    """Keys of a layer: normal, a direction shared by 64 neighbours, and two channels with a large constant."""
    k = _normal(g, H, T, D) + _normal(g, H, -(-T // 64), D).repeat_interleave(64, dim=1)[:, :T]
    k *= math.sqrt(0.5)
    k[:, :, ::D // 2] += 4.0
    return k


class State:
    """What a program holds between calls."""

    def __init__(self, **kw):
        self.__dict__.update(kw)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    B, L, H, D, cap = c["batch"], c["layers"], c["kv_heads"], c["head_dim"], _capacity(c)
    g = _rng(seed, 1)
    s = State(kind=c["kind"], fmt=c["fmt"], block=c["block"], scale=1.0 / math.sqrt(D), top=max(c["rows"], 1), mass=None)
    s.k = torch.empty((B, L, H, cap, D), dtype=torch.uint8, device="cuda")
    s.v = torch.empty((B, L, H, cap // TILE, D, TILE), dtype=torch.uint8, device="cuda")
    s.ks, s.vs = (torch.empty((B, L, H, cap // c["block"]), device="cuda") for _ in range(2))
    out = torch.bfloat16 if c["bf16"] else torch.float32
    if c["kind"] == "attend":
        n, Hq = c["n"], c["q_heads"]
        lens, counts = _lengths(c, c["rows"]), _counts(c, n)
        counts = [min(a, b) for a, b in zip(counts, lens)]
        s.len, s.count = _ints(lens), _ints(counts)
        s.q = torch.empty((B, L, Hq, n, D), dtype=torch.bfloat16, device="cuda")
        s.out = torch.zeros((B, L, Hq, n, D), dtype=out, device="cuda")
        s.lse = torch.zeros((B, L, Hq, n), device="cuda")
        if c["mass"]:
            s.mass = torch.zeros((B, L, Hq, cap // c["block"]), device="cuda")
    # the cache as earlier calls left it (rows behind a sequence's last one are from an earlier use)
    for b in range(B):
        for l in range(L):
            k, v = _keys(g, H, cap, D), _normal(g, H, cap, D)
            if c["kind"] == "attend":    # a query leans towards one of its sequence's keys
                at = torch.randint(0, max(lens[b], 1), (H, Hq // H * n, 1), generator=g, device="cuda")
                lean = k.gather(1, at.expand(-1, -1, D)).reshape(Hq, n, D)
                s.q[b, l] = _normal(g, Hq, n, D) + 0.7 * lean
            for x, scales in ((k, s.ks), (v, s.vs)):
                scales[b, l] = _scale(x.bfloat16().float().abs().unflatten(1, (-1, c["block"])).amax(dim=(2, 3)), c["fmt"])
            k, v = (_code(x.bfloat16().float(), t[b, l].repeat_interleave(c["block"], dim=1).unsqueeze(-1), c["fmt"])
                    for x, t in ((k, s.ks), (v, s.vs)))
            s.k[b, l] = k
            _v_rows(s.v)[b, ..., l, :, :] = v.transpose(0, 1).unflatten(0, (-1, 4, 4, 4))
    if c["kind"] == "store":
        n, back = c["n"], c["back"]
        pos, counts = _lengths(c, c["rows"]), _counts(c, n)
        ends = [a + b for a, b in zip(pos, counts)]
        s.pos, s.count = _ints(pos), _ints(counts)
        s.rpos, s.rcount = _ints([max(0, e - back) for e in ends]), _ints([min(back, e) for e in ends])
        s.xk, s.xv = (torch.empty((B, L, H, n, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for b in range(B):
            for l in range(L):
                # a generated token's rows are of any size
                s.xk[b, l] = _keys(g, H, n, D) * (torch.exp(0.5 * _normal(g, H, n, 1)) if c["rows"] else 1.0)
                s.xv[b, l] = _normal(g, H, n, D) * (torch.exp(0.5 * _normal(g, H, n, 1)) if c["rows"] else 1.0)
    elif c["kind"] == "read":
        back = c["rows"]
        s.rpos, s.rcount = _ints([0] * B), _ints(_lengths(c, c["rows"]))
    if c["kind"] != "attend":
        s.ko, s.vo = (torch.zeros((B, L, H, back, D), dtype=out, device="cuda") for _ in range(2))
    if own:
        from paper_2608_22704_amd import wnw as W
        s.W = W
        s.cfg = W.make_quant_config(B, L, H, cap, c["block"], W.WNW_QUANT_INT8 if c["fmt"] == "int8" else W.WNW_QUANT_E4M3,
                                    head_dim=D, flags=W.WNW_F_OUT_BF16 if c["bf16"] else 0)
        s.cache = W.QuantCache(s.k, s.v, s.ks, s.vs)
        if c["kind"] == "attend":
            need = W.wnw_quant_attend_workspace(s.cfg, L, c["q_heads"], c["n"], max_len=c["rows"])
            s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ---- the plain form --------------------------------------------------------------------------


def _scale(amax, fmt):
    """The scale of blocks whose largest magnitude is amax (fp32)."""
    if fmt == "int8":
        return (amax.double() / 127).float().clamp_min(2.0 ** -126)
    m, e = torch.frexp(amax)                                    # amax = m 2^e, m in [1/2, 1)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-126, 127)  # amax <= 448 * 2^e
    return ((e + 127) << 23).int().view(torch.float32)


def _code(x, s, fmt):
    """Bytes of values x (fp32) under scales s: nearest, ties to even."""
    if fmt == "int8":
        return ((x.double() / s.double()).round().clamp(-127, 127) + 128).to(torch.uint8)
    return (x / s).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)   # exact quotients: s is a power of two


def _number(codes, fmt):
    """What bytes stand for, before the scale (fp32)."""
    return codes.float() - 128 if fmt == "int8" else codes.view(torch.float8_e4m3fn).float()


def _write(s, x, codes, at, scales, idx, blk, new, old):
    """Rows idx [B][W] of one of K and V: whole blocks blk [B][W / block], new rows from x, old rows kept."""
    b = torch.arange(len(idx), device=idx.device)[:, None]
    nb = blk.shape[1]
    rows = x.permute(0, 3, 1, 2, 4)[b, (idx - s.pos[:, None]).clamp(0, x.shape[3] - 1)].float()   # [B][W][L][H_kv][d]
    amax = torch.where(new[..., None, None], rows.abs().amax(dim=-1), 0.0).unflatten(1, (nb, -1)).amax(dim=2)
    was = scales.permute(0, 3, 1, 2)[b, blk]
    there = old.unflatten(1, (nb, -1)).any(dim=2)[..., None, None]
    now = torch.where(there, torch.maximum(was, _scale(amax, s.fmt)), _scale(amax, s.fmt))
    touched = new.unflatten(1, (nb, -1)).any(dim=2)[..., None, None]
    now = torch.where(touched, now, was)
    wide = [t.repeat_interleave(s.block, dim=1).unsqueeze(-1) for t in (was, now)]
    had = codes[(b, *at)]
    kept = _code(_number(had, s.fmt).double() * wide[0], wide[1], s.fmt)
    put = torch.where(new[..., None, None, None], _code(rows, wide[1], s.fmt),
                      torch.where(old[..., None, None, None], kept, had))
    codes[(b, *at)] = put
    scales.permute(0, 3, 1, 2)[b, blk] = now


def _read_back(s, codes, at, scales, idx, live, out):
    b = torch.arange(len(idx), device=idx.device)[:, None]
    x = _number(codes[(b, *at)], s.fmt) * scales.permute(0, 3, 1, 2)[b, idx // s.block].unsqueeze(-1)
    return torch.where(live[..., None, None, None], x, 0.0).permute(0, 2, 3, 1, 4).to(out.dtype).contiguous()


def _plain_store(s):
    n = s.xk.shape[3]
    first = s.pos.long() // s.block
    blk = first[:, None] + torch.arange((n + s.block - 2) // s.block + 1, device=first.device)
    idx = (blk[..., None] * s.block + torch.arange(s.block, device=first.device)).flatten(1)
    end = (s.pos + s.count).long()[:, None]
    new, old = (idx >= s.pos[:, None]) & (idx < end), idx < s.pos[:, None]
    _write(s, s.xk, _k_rows(s.k), (idx,), s.ks, idx, blk, new, old)
    _write(s, s.xv, _v_rows(s.v), _at(idx), s.vs, idx, blk, new, old)
    return _plain_read(s)


def _plain_read(s):
    back = s.ko.shape[3]
    j = torch.arange(back, device=s.rpos.device)
    idx = s.rpos.long()[:, None] + j
    live = j < s.rcount[:, None]
    return (_read_back(s, _k_rows(s.k), (idx,), s.ks, idx, live, s.ko),
            _read_back(s, _v_rows(s.v), _at(idx), s.vs, idx, live, s.vo))


def _plain_attend(s):
    B, L, Hq, n, D = s.q.shape
    H = s.k.shape[2]
    top = (s.top + TILE - 1) // TILE * TILE
    key = torch.arange(top, device=s.q.device)
    live = (key < s.len[:, None])[:, None, None, :, None]
    scale = lambda t: t[..., :top // s.block].repeat_interleave(s.block, dim=3).unsqueeze(-1)   # noqa: E731
    k = torch.where(live, _number(s.k[:, :, :, :top], s.fmt) * scale(s.ks), 0.0)
    v = s.v[:, :, :, :top // TILE].unflatten(-1, (4, 4, 4)).permute(0, 1, 2, 3, 6, 5, 7, 4).reshape(B, L, H, top, D)
    v = torch.where(live, _number(v, s.fmt) * scale(s.vs), 0.0)
    q = s.q.float().reshape(B, L, H, Hq // H * n, D)
    x = (torch.matmul(q, k.transpose(-1, -2)) * s.scale).reshape(B, L, Hq, n, top)
    sees = key <= (s.len - s.count)[:, None, None] + torch.arange(n, device=key.device)[:, None]   # [B][n][top]
    token = (torch.arange(n, device=key.device) < s.count[:, None])[:, None, None]                 # [B][1][1][n]
    x = x.masked_fill(~(sees & (key < s.len[:, None, None]))[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(dim=-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = torch.matmul(p.reshape(B, L, H, Hq // H * n, top), v).reshape(B, L, Hq, n, D)
    got = [torch.where(token.unsqueeze(-1), out, 0.0).to(s.out.dtype),
           torch.where(token, (m + torch.log(total)).squeeze(-1), 0.0)]
    if s.mass is not None:
        w = torch.where(token.unsqueeze(-1), p, 0.0).reshape(B, L, Hq, top // s.block, s.block).sum(dim=-1)
        got.append(torch.nn.functional.pad(w, (0, s.mass.shape[-1] - w.shape[-1])))
    return got


# ---- one pass --------------------------------------------------------------------------------


def run(s):
    if not own:
        return {"store": _plain_store, "read": _plain_read, "attend": _plain_attend}[s.kind](s)
    if s.kind == "attend":
        s.W.wnw_quant_attend(s.cfg, s.cache, s.q, s.out, s.len, s.count, s.lse, s.mass, s.workspace, max_len=s.top)
        return [s.out, s.lse] + ([] if s.mass is None else [s.mass])
    if s.kind == "store":
        s.W.wnw_quant_write(s.cfg, s.cache, s.xk, s.xv, s.pos, s.count)
    s.W.wnw_quant_read(s.cfg, s.cache, s.ko, s.vo, s.rpos, s.rcount)
    return s.ko, s.vo


# ---- what a pass cannot do without -----------------------------------------------------------


def work(c):
    L, H, D, block = c["layers"], c["kv_heads"], c["head_dim"], c["block"]
    out = 2 if c["bf16"] else 4
    kept = 2 * L * H * (D + 4 / block)     # bytes of a cache row, K and V
    if c["kind"] == "attend":
        lens = _lengths(c, c["rows"])
        counts = [min(a, b) for a, b in zip(_counts(c, c["n"]), lens)]
        tokens, Hq = sum(counts), c["q_heads"]
        io = L * Hq * tokens * (D * (2 + out) + 4)
        if c["mass"]:
            io += L * Hq * sum(lens) / block * 4
        pairs = sum(n * (t - n) + n * (n + 1) / 2 for t, n in zip(lens, counts))
        return {"bytes": sum(lens) * kept + io, "flops": L * Hq * pairs * 4 * D}
    if c["kind"] == "read":
        rows = sum(_lengths(c, c["rows"]))
        return {"bytes": rows * (kept + 2 * L * H * D * out), "flops": rows * 2 * L * H * D}
    pos, counts = _lengths(c, c["rows"]), _counts(c, c["n"])
    rows, back = sum(counts), sum(min(c["back"], a + b) for a, b in zip(pos, counts))
    return {"bytes": rows * (2 * L * H * D * 2 + kept) + back * 2 * L * H * D * out + max(0, back - rows) * kept,
            "flops": (3 * rows + back) * 2 * L * H * D}


# ---- the same in 64 bits ---------------------------------------------------------------------


def _grid():
    """The non-negative e4m3 numbers in order, by code 0 .. 126."""
    return torch.tensor([(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device="cuda")


def _exact_scale(top, fmt):
    if fmt == "int8":
        s = (top / 127).float().double()
    else:
        s = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300) / 448)))
        s = torch.where(s * 448 < top, s * 2, torch.where(s * 224 >= top, s / 2, s))
    return s.clamp_min(2.0 ** -126)


def _exact_round(x, s, fmt):
    """The nearest multiple of s (int8) or of s times an e4m3 number, ties to the even code."""
    a = x.abs()
    if fmt == "int8":
        n = torch.floor(a / s)
        n = n + torch.sign(a - n * s).clamp_max(0)               # the quotient may have been rounded up
        rest = 2 * (a - n * s)
        n = n + ((rest > s) | ((rest == s) & (n % 2 == 1)))
        return torch.sign(x) * n.clamp_max(127) * s
    grid = _grid()
    a = a / s
    hi = torch.searchsorted(grid, a).clamp_max(126)
    lo = (hi - 1).clamp_min(0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.sign(x) * grid[pick] * s


def _exact_values(codes, scales, block, fmt, v):
    """Values [H_kv][rows][d] of a layer's bytes, double."""
    if v:
        place = torch.tensor([_place(r) for r in range(TILE)], device=codes.device)
        codes = codes[..., place].transpose(-1, -2).flatten(1, 2)
    grid = _grid()
    nan = torch.full((1,), math.nan, dtype=torch.float64, device="cuda")
    table = torch.arange(256, device="cuda", dtype=torch.float64) - 128 if fmt == "int8" else torch.cat([grid, nan, -grid, nan])
    return table[codes.int()] * scales.double().repeat_interleave(block, dim=1).unsqueeze(-1)


def _exact_store(c, s):
    block, fmt, back = c["block"], c["fmt"], c["back"]
    got = []
    for codes, scales, x, is_v in ((s.k, s.ks, s.xk, False), (s.v, s.vs, s.xv, True)):
        out = torch.zeros((c["batch"], c["layers"], c["kv_heads"], back, c["head_dim"]), dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            pos, n, first, cnt = (int(t[b]) for t in (s.pos, s.count, s.rpos, s.rcount))
            for l in range(c["layers"]):
                if pos:
                    full = _exact_values(codes[b, l], scales[b, l], block, fmt, is_v)
                else:
                    full = torch.zeros((c["kv_heads"], _capacity(c), c["head_dim"]), dtype=torch.float64, device="cuda")
                old_top = scales[b, l].double()
                full[:, pos: pos + n] = x[b, l, :, :n].double()
                j0, j1 = pos // block, -(-(pos + n) // block)
                part = full[:, j0 * block: j1 * block].unflatten(1, (-1, block))
                row = torch.arange(j0 * block, j1 * block, device="cuda").reshape(-1, block)
                new, old = (row >= pos) & (row < pos + n), row < pos
                sc = _exact_scale((part.abs().amax(dim=-1) * new).amax(dim=-1), fmt)
                sc = torch.where(old.any(dim=1), torch.maximum(sc, old_top[:, j0: j1]), sc)[..., None, None]
                full[:, j0 * block: j1 * block] = _exact_round(part, sc, fmt).flatten(1, 2)
                out[b, l, :, :cnt] = full[:, first: first + cnt]
        got.append(out)
    return got


def _exact_attend(c, s):
    B, L, Hq, n, D = s.q.shape
    G, block = Hq // c["kv_heads"], c["block"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, L, Hq, n), dtype=torch.float64, device="cuda")
    mass = torch.zeros((B, L, Hq, _capacity(c) // block), dtype=torch.float64, device="cuda")
    for b in range(B):
        T, cnt = int(s.len[b]), int(s.count[b])
        if not cnt:
            continue
        tiles = -(-T // TILE)
        later = torch.ones((cnt, T), dtype=torch.bool, device="cuda").triu(T - cnt + 1)
        for l in range(L):
            k, v = (_exact_values(x, sc[b, l, :, : tiles * TILE // block], block, c["fmt"], is_v)[:, :T] for x, sc, is_v in
                    ((s.k[b, l, :, : tiles * TILE], s.ks, False), (s.v[b, l, :, :tiles], s.vs, True)))
            for h in range(c["kv_heads"]):
                x = s.q[b, l, h * G: (h + 1) * G, :cnt].double().flatten(0, 1) @ k[h].T.contiguous() / math.sqrt(D)
                x = x.unflatten(0, (G, cnt)).masked_fill(later, -math.inf)
                lse[b, l, h * G: (h + 1) * G, :cnt] = torch.logsumexp(x, dim=-1)
                p = torch.softmax(x, dim=-1)
                out[b, l, h * G: (h + 1) * G, :cnt] = (p.flatten(0, 1) @ v[h]).unflatten(0, (G, cnt))
                if c["mass"]:
                    w = torch.nn.functional.pad(p[:, 0], (0, -T % block)).unflatten(-1, (-1, block)).sum(dim=-1)
                    mass[b, l, h * G: (h + 1) * G, : w.shape[-1]] = w
    return [out, lse] + ([mass] if c["mass"] else [])


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "attend":
        return _exact_attend(c, s)
    if c["kind"] == "store":
        return _exact_store(c, s)
    got = []
    for codes, scales, is_v in ((s.k, s.ks, False), (s.v, s.vs, True)):
        out = torch.zeros(s.ko.shape, dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            n = int(s.rcount[b])
            for l in range(c["layers"]):
                out[b, l, :, :n] = _exact_values(codes[b, l], scales[b, l], c["block"], c["fmt"], is_v)[:, :n]
        got.append(out)
    return got
