"""The operators of drafted decoding over a paged cache and their plain forms: a draft's tree, appending rows to
the pages with their positions' rotation, attention over the pages, verification, and keeping the accepted rows.

A case is a dict of plain values.  `kind` says which call a pass makes:

* "tree"     parents of the drafted tokens -> the bits of their ancestors and their positions (wnw_draft_tree);
* "append"   new K and V rows join the pages behind the rows that are there, K and the queries rotated by their
             positions (wnw_paged_append);
* "attend"   attention of a sequence's last n tokens over its pages, which see each other causally or as their
             tree says: output and log-sum-exp of every query row (wnw_paged_attend);
* "verify"   which drafted tokens stand, given the target's and the draft's probabilities and uniform numbers,
             and the token after them (wnw_draft_verify);
* "keep"     the rows of the tokens that stand move to the end of their sequence (wnw_paged_keep).

The cache of a batch: K and V as bf16 [pages][L][H_kv][page][d]; table int32 [B][width], the page of a sequence's
rows page j .. page (j + 1) - 1.  Pages are handed out in no order.

Shapes are those of the backbones in synth/configs.py (30 layers, 32 query / 8 KV heads; 36 layers, 16 / 2;
one layer, 24 / 8), with up to ten minutes of audio, and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

VOXTRAL = dict(layers=30, q_heads=32, kv_heads=8)
QWEN = dict(layers=36, q_heads=16, kv_heads=2)
ONE = dict(layers=1, q_heads=24, kv_heads=8)


def _tree(name, batch, n, shape, ragged):
    c = dict(kind="tree", batch=batch, n=n, tree=shape, ragged=ragged)
    return dict(c, name=name) if name else c


def _cache(name, kind, shape, rows, n, page, **kw):
    c = dict(kind=kind, batch=1, rows=rows, n=n, page=page, head_dim=128, ragged=False)
    c.update(shape, **kw)
    return dict(c, name=name) if name else c


def _append(name, shape, rows, n, page, **kw):
    return _cache(name, "append", shape, rows, n, page, **dict(dict(rotated=128, halves=True, queries=True, far=0, scaled=1.0), **kw))


def _attend(name, shape, rows, n, page, **kw):
    return _cache(name, "attend", shape, rows, n, page, **dict(dict(tree="", bf16=True), **kw))


def _verify(name, batch, n, vocab, **kw):
    c = dict(kind="verify", batch=batch, n=n, vocab=vocab, tree="", draft=True, ragged=False, near=1.0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the plan of a draft of sixteen tokens, one sequence: the smallest call there is
        _tree("tree_16", 1, 16, "wide", False),
        # a serving batch of sixteen drafts of up to 512 tokens
        _tree("tree_512_b16", 16, 512, "deep", True),
        # a generated token of all layers joins ten minutes of audio, its queries rotated beside its keys
        _append("append_token", VOXTRAL, 15512, 1, 16),
        # the prompt of ten minutes of audio, all layers, half of every head rotated, a context scaled by four
        _append("append_prompt", QWEN, 0, 7756, 64, rotated=64, halves=False, scaled=4.0),
        # a generated token attends: the smallest cache, one layer, fp32 outputs
        _attend("token_tiny", ONE, 1064, 1, 16, bf16=False),
        # all layers, ten minutes at 25 tokens/s
        _attend("token_voxtral", VOXTRAL, 15512, 1, 16),
        # four ragged sequences check a tree of 64 drafted tokens each, eight layers
        _attend("tree_b4", dict(VOXTRAL, layers=8), 15512, 64, 32, batch=4, ragged=True, tree="wide"),
        # two layers' instruction tokens over ten minutes of audio (a causal block)
        _attend("text_voxtral", dict(VOXTRAL, layers=2), 15512, 512, 128),
        # five tokens drafted one after the other, a single sequence
        _verify("verify_chain", 1, 5, 32000),
        # eight trees of 64 drafted tokens, a large vocabulary
        _verify("verify_tree", 8, 64, 131072, tree="wide", ragged=True),
        # three of a small draft's tokens stand, one layer
        _cache("keep_tiny", "keep", ONE, 1000, 16, 16, stand=3),
        # a batch of eight, all layers, up to eight tokens stand
        _cache("keep_b8", "keep", VOXTRAL, 1900, 64, 32, batch=8, ragged=True, stand=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges (lengths on a logarithmic scale, odd ones among them)."""
    kind = rng.choice(["tree", "append", "append", "attend", "attend", "attend", "attend", "attend", "verify", "verify", "keep"])
    batch = rng.choice([1, 1, 2, 3, 5, 16])
    ragged = batch > 1 and rng.random() < 0.7
    if kind == "tree":
        return _tree("", batch, _log_int(rng, 2, 512), rng.choice(["wide", "deep"]), ragged)
    if kind == "verify":
        n, vocab = _log_int(rng, 1, 64), _log_int(rng, 500, 131072)
        while batch * (n + 1) * vocab > 8 * 65 * 131072:
            n = n // 2
        return _verify("", batch, n, vocab, tree=rng.choice(["", "wide", "deep"]), draft=rng.random() < 0.6, ragged=ragged,
                       near=rng.choice([0.3, 1.0, 2.0]))
    kv = rng.choice([1, 2, 3, 8])
    shape = dict(rng.choice([VOXTRAL, QWEN, dict(layers=rng.randint(1, 8), q_heads=24, kv_heads=8),
                             dict(layers=rng.randint(1, 4), q_heads=kv * rng.choice([1, 2, 5, 8, 16]), kv_heads=kv)]))
    heads = batch * shape["layers"] * shape["kv_heads"]
    page, kw = rng.choice([16, 32, 64, 128]), dict(batch=batch, ragged=ragged, head_dim=rng.choice([128, 128, 64]))
    if kind == "keep":
        return _cache("", "keep", shape, _log_int(rng, 1, min(4000, 8 * 240 * 1900 // heads)), rng.randint(4, 64), page,
                      stand=rng.randint(1, 8), **kw)
    if kind == "append":
        rotated = kw["head_dim"] if rng.random() < 0.5 else 2 * rng.randint(0, kw["head_dim"] // 2)
        total = batch * shape["layers"] * (2 * shape["kv_heads"] + shape["q_heads"])
        n = rng.choice([1, rng.randint(2, 64), _log_int(rng, 16, max(17, min(15512, 36 * 20 * 7756 // total)))])
        rows = 0 if n > 64 else _log_int(rng, 1, max(2, min(15512, 240 * 15512 // heads)))
        return _append("", shape, rows, n, page, rotated=rotated, halves=rng.random() < 0.6, queries=rng.random() < 0.7,
                       far=rng.choice([0, 0, 1000003, 9999991]), scaled=rng.choice([1.0, 1.0, 4.0, 8.0]), **kw)
    n = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 64), _log_int(rng, 10, 512)])
    top = min(15512, 240 * 15512 // heads)
    if n > 1:
        top = max(n, min(top, 2 * 32 * 512 * 15512 // (batch * shape["layers"] * shape["q_heads"] * n)))
    rows = max(n, _log_int(rng, 1, max(2, top)))
    return _attend("", shape, rows, n, page, tree=rng.choice(["", "wide", "deep"]) if 1 < n <= 512 else "",
                   bf16=rng.random() < 0.6, **kw)


# ---- sizes -----------------------------------------------------------------------------------


def _lengths(c, most):
    """Rows of every sequence; ragged: the first has the most, one has a single row, one none."""
    B = c["batch"]
    if not c["ragged"]:
        return [most] * B
    r = [max(1, int(most * math.exp(-3 * ((b * 0.618) % 1.0)))) if most else 0 for b in range(B)]
    if B >= 4 and most:
        r[1], r[2] = 1, 0
    return r


def _counts(c):
    """Tokens of every sequence in a call: up to n."""
    return [max(1, c["n"] - b) if c["ragged"] else c["n"] for b in range(c["batch"])]


def _attend_sizes(c):
    lens = _lengths(c, c["rows"])
    return lens, [min(a, b) for a, b in zip(_counts(c), lens)]


def _width(c):
    """Pages of a sequence: room for its rows and a draft behind them."""
    return (c["rows"] + c["n"]) // c["page"] + 2


def _parents(c, seed):
    """[B][n]: -1 or an earlier token.  wide: a few tokens deep, several after each; deep: mostly one after the other."""
    rng = random.Random(seed)
    got = []
    for _ in range(c["batch"]):
        if not c["tree"]:
            got.append([i - 1 for i in range(c["n"])])
        elif c["tree"] == "deep":
            got.append([i - 1 if i == 0 or rng.random() < 0.8 else rng.randint(-1, i - 1) for i in range(c["n"])])
        else:
            first = min(c["n"], rng.randint(2, 5))
            got.append([-1 if i < first else min(i - 1, max(0, int((i - first) / rng.uniform(1.5, 4.0)))) for i in range(c["n"])])
    return got


# ---- inputs ----------------------------------------------------------------------------------


def _rng(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 64 + tag) % (1 << 62))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gumbel(g, *shape):
    u = torch.rand(shape, generator=g, device="cuda").clamp(1e-30, 1 - 2 ** -24)
    return -torch.log(-torch.log(u))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class State:
    """What a program holds between calls."""

    def __init__(self, **kw):
        self.__dict__.update(kw)


def _keys(g, P, H, page, D):
    """Keys of pages: normal, a direction shared by a page, and two channels with a large constant."""
    k = math.sqrt(0.5) * (_normal(g, P, H, page, D) + _normal(g, P, H, 1, D))
    k[..., ::D // 2] += 4.0
    return k


def _prepare_cache(c, seed, g):
    B, L, H, D, page, width = c["batch"], c["layers"], c["kv_heads"], c["head_dim"], c["page"], _width(c)
    pages = B * width + 3
    s = State(kind=c["kind"], page=page, top=max(c["rows"], 1))
    order = torch.randperm(pages, generator=g, device="cuda")[:B * width]
    s.table = order.int().reshape(B, width)
    s.k, s.v = (torch.empty((pages, L, H, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for l in range(L):
        s.k[:, l] = _keys(g, pages, H, page, D)
        s.v[:, l] = _normal(g, pages, H, page, D)
    if own:
        from paper_2608_22704_amd import wnw as W
        s.W = W
        s.cfg = W.make_paged_config(B, L, H, page, pages, width, head_dim=D,
                                    flags=W.WNW_F_OUT_BF16 if c.get("bf16") else 0)
        s.cache = W.PagedCache(s.k, s.v, s.table)
    return s


def _frequencies(dim, scaled):
    """fp32 radians per position of the pairs of `dim` rotated elements: 10^6 to the power -2 i / dim; a longer context by
    `scaled`: what turns less than once over 8192 positions slows down by it, what turns over 4 times stays."""
    f = 1e6 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / max(dim, 1))
    keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
    return (f * keep + f / scaled * (1 - keep)).float().cuda()


def _prepare_append(c, seed, g):
    s = _prepare_cache(c, seed, g)
    B, L, H, D, n = c["batch"], c["layers"], c["kv_heads"], c["head_dim"], c["n"]
    s.at, s.count = _ints(_lengths(c, c["rows"])), _ints(_counts(c))
    s.xk, s.xv = (torch.empty((B, L, H, n, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s.q = torch.empty((B, L, c["q_heads"], n, D), dtype=torch.bfloat16, device="cuda") if c["queries"] else None
    for l in range(L):
        s.xk[:, l] = _keys(g, B, H, n, D)
        s.xv[:, l] = _normal(g, B, H, n, D)
        if s.q is not None:
            s.q[:, l] = _normal(g, B, c["q_heads"], n, D)
    s.q_out = torch.zeros_like(s.q) if s.q is not None else None
    s.freq = _frequencies(c["rotated"], c["scaled"])
    s.dim, s.halves = c["rotated"], c["halves"]
    s.amplitude = 0.1 * math.log(c["scaled"]) + 1.0
    # a sequence whose earlier part is no longer in the cache has positions far ahead of its rows
    s.position = s.at[:, None] + torch.arange(n, dtype=torch.int32, device="cuda") + c["far"] if c["far"] else None
    if own:
        s.rotary = s.W.make_rotary(s.freq, s.dim, s.W.WNW_ROTARY_HALVES if s.halves else s.W.WNW_ROTARY_PAIRS, s.amplitude)
    return s


def _ancestors(parent):
    """[n][n]: token j is token i or before it on its path."""
    n = len(parent)
    see = [[False] * n for _ in range(n)]
    for i, p in enumerate(parent):
        if p >= 0:
            see[i] = list(see[p])
        see[i][i] = True
    return see


def _prepare_attend(c, seed, g):
    s = _prepare_cache(c, seed, g)
    B, L, Hq, D, n, page = c["batch"], c["layers"], c["q_heads"], c["head_dim"], c["n"], c["page"]
    lens, counts = _attend_sizes(c)
    s.len, s.count = _ints(lens), _ints(counts)
    s.q = torch.empty((B, L, Hq, n, D), dtype=torch.bfloat16, device="cuda")
    for b in range(B):      # a query leans towards one of its sequence's keys
        at = torch.randint(0, max(lens[b], 1), (n,), generator=g, device="cuda")
        lean = s.k[s.table[b, at // page].long(), :, :, at % page].float()                     # [n][L][H_kv][d]
        lean = lean.permute(1, 2, 0, 3).repeat_interleave(Hq // c["kv_heads"], dim=1)
        s.q[b] = _normal(g, L, Hq, n, D) + 0.7 * lean
    s.mask = None
    if c["tree"]:
        see = torch.tensor([_ancestors(p) for p in _parents(c, seed)], device="cuda")          # [B][n][n]
        see = torch.nn.functional.pad(see, (0, -n % 64)).unflatten(-1, (-1, 64)).long()
        s.mask = (see << torch.arange(64, device="cuda")).sum(dim=-1)
    s.out = torch.zeros((B, L, Hq, n, D), dtype=torch.bfloat16 if c["bf16"] else torch.float32, device="cuda")
    s.lse = torch.zeros((B, L, Hq, n), device="cuda")
    s.scale = 1.0 / math.sqrt(D)
    if own:
        need = s.W.wnw_paged_attend_workspace(s.cfg, L, Hq, n, max_len=s.top)
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def _prepare_keep(c, seed, g):
    s = _prepare_cache(c, seed, g)
    rng, paths, counts = random.Random(seed), [], []
    for b in range(c["batch"]):
        stand = min(c["n"], c["stand"] if not c["ragged"] else max(0, c["stand"] - b))
        p = sorted(rng.sample(range(c["n"]), stand))
        paths.append(p + [-1] * (c["n"] - stand))
        counts.append(stand)
    s.base, s.path, s.count = _ints(_lengths(c, c["rows"])), _ints(paths), _ints(counts)
    return s


def _prepare_tree(c, seed):
    B, n = c["batch"], c["n"]
    s = State(kind="tree", parent=_ints(_parents(c, seed)), count=_ints(_counts(c)))
    s.base = _ints([random.Random(seed + b).randint(0, 100000) for b in range(B)])
    s.mask = torch.zeros((B, n, (n + 63) // 64), dtype=torch.int64, device="cuda")
    s.position = torch.zeros((B, n), dtype=torch.int32, device="cuda")
    if own:
        from paper_2608_22704_amd import wnw as W
        s.W = W
    return s


def _prepare_verify(c, seed, g):
    B, n, V = c["batch"], c["n"], c["vocab"]
    s = State(kind="verify", vocab=V, chain=not c["tree"], count=_ints(_counts(c) if n else [0] * B))
    s.parent = _ints(_parents(c, seed)).reshape(B, n)
    s.target = torch.empty((B, n + 1, V), device="cuda")
    s.draft = torch.empty((B, n + 1, V), device="cuda") if c["draft"] else None
    s.token = torch.empty((B, n), dtype=torch.int32, device="cuda")
    for b in range(B):
        # what comes after each token: a few likely tokens and many rare ones (the k-th likeliest has about k^-1.4 of the
        # first one's share); the draft model is `near` the target
        x = 1.4 * _gumbel(g, n + 1, V)
        y = x + c["near"] * _normal(g, n + 1, V)
        s.target[b] = torch.softmax(x, dim=-1)
        if s.draft is not None:
            s.draft[b] = torch.softmax(y, dim=-1)
        if n:
            rows = s.parent[b].long() + 1
            # drawn from the draft's row, or its likeliest tokens in turn
            if s.draft is not None:
                s.token[b] = (y[rows] + _gumbel(g, n, V)).argmax(dim=-1)
            else:
                best = y.topk(min(V, n + 1), dim=-1).indices
                turn, seen = [], {}
                for p in s.parent[b].tolist():
                    turn.append(seen.get(p, 0))
                    seen[p] = turn[-1] + 1
                s.token[b] = best[rows, torch.tensor(turn, device="cuda")]
    s.uniform = torch.rand((B, n + 1), generator=g, device="cuda")
    s.path = torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    s.accepted, s.next = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    if own:
        from paper_2608_22704_amd import wnw as W
        s.W = W
        need = W.wnw_draft_verify_workspace(B, n, V)
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


def prepare(c, seed):
    if c["kind"] == "tree":
        return _prepare_tree(c, seed)
    g = _rng(seed, 1)
    return {"append": _prepare_append, "attend": _prepare_attend, "keep": _prepare_keep, "verify": _prepare_verify}[c["kind"]](c, seed, g)


# ---- the plain forms -------------------------------------------------------------------------


def _plain_tree(s):
    B, n = s.parent.shape
    i = torch.arange(n, device=s.parent.device)
    see = ((i == s.parent[..., None]) | (i == i[:, None])).float()
    reach = 1
    while reach < n:
        see = (torch.matmul(see, see) > 0).float()
        reach *= 2
    live = i < s.count[:, None]
    bits = torch.nn.functional.pad(see, (0, -n % 64)).unflatten(-1, (-1, 64)).long()
    mask = (bits << torch.arange(64, device=i.device)).sum(dim=-1)
    position = s.base[:, None] + see.sum(dim=-1).int() - 1
    return torch.where(live[..., None], mask, s.mask), torch.where(live, position, s.position)


def _rows(s, at, n):
    """Where rows at .. at + n - 1 of every sequence are: pages and rows of them, [B][n]."""
    r = at.long()[:, None] + torch.arange(n, device=at.device)
    return torch.gather(s.table.long(), 1, r // s.page), r % s.page


def _plain_rotate(s, x, position):
    """x [B][L][H][n][d] rotated by positions [B][n]."""
    if not s.dim:
        return x
    angle = position.double()[..., None] * s.freq.double()
    c, sn = ((f(angle) * s.amplitude).float()[:, None, None] for f in (torch.cos, torch.sin))
    r = x[..., :s.dim].float()
    if s.halves:
        a, b = r[..., :s.dim // 2], r[..., s.dim // 2:]
        y = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
    else:
        a, b = r[..., ::2], r[..., 1::2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
    return torch.cat([y.bfloat16(), x[..., s.dim:]], dim=-1)


def _plain_append(s):
    n = s.xk.shape[3]
    position = s.position if s.position is not None else s.at[:, None] + torch.arange(n, dtype=torch.int32, device=s.at.device)
    live = torch.arange(n, device=s.at.device) < s.count[:, None]
    page, row = _rows(s, s.at, n)
    for pool, x in ((s.k, _plain_rotate(s, s.xk, position)), (s.v, s.xv)):
        pool[page, :, :, row] = torch.where(live[..., None, None, None], x.permute(0, 3, 1, 2, 4), pool[page, :, :, row])
    if s.q is None:
        return s.k, s.v
    s.q_out.copy_(torch.where(live[:, None, None, :, None], _plain_rotate(s, s.q, position), s.q_out))
    return s.k, s.v, s.q_out


def _plain_attend(s):
    B, L, Hq, n, D = s.q.shape
    H = s.k.shape[2]
    most = (s.top + s.page - 1) // s.page
    top = most * s.page
    key = torch.arange(top, device=s.q.device)
    live = (key < s.len[:, None])[:, None, None, :, None]
    table = s.table[:, :most].long()
    k, v = (torch.where(live, x[table].permute(0, 2, 3, 1, 4, 5).reshape(B, L, H, top, D).float(), 0.0) for x in (s.k, s.v))
    q = s.q.float().reshape(B, L, H, Hq // H * n, D)
    x = (torch.matmul(q, k.transpose(-1, -2)) * s.scale).reshape(B, L, Hq, n, top)
    base = (s.len - s.count)[:, None, None]
    j = key - base                                                                             # [B][1][top]
    if s.mask is None:
        sees = j <= torch.arange(n, device=key.device)[:, None]
    else:
        at = j.clamp(0, n - 1).expand(B, n, top)
        sees = (j < 0) | ((torch.gather(s.mask, 2, at // 64) >> (at % 64)) & 1 == 1)
    sees = sees & (key < s.len[:, None, None])
    token = (torch.arange(n, device=key.device) < s.count[:, None])[:, None, None]             # [B][1][1][n]
    x = x.masked_fill(~sees[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(dim=-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = torch.matmul(p.reshape(B, L, H, Hq // H * n, top), v).reshape(B, L, Hq, n, D)
    return (torch.where(token.unsqueeze(-1), out, 0.0).to(s.out.dtype),
            torch.where(token, (m + torch.log(total)).squeeze(-1), 0.0))


def _plain_verify(s):
    B, n = s.token.shape
    V = s.vocab
    b = torch.arange(B, device=s.token.device)
    at = torch.full((B,), -1, dtype=torch.int32, device=b.device)       # the token that stands last
    rest = s.target[:, 0].double()                                      # what is left of the row behind it, and of its sum
    left = torch.ones(B, dtype=torch.float64, device=b.device)
    path, accepted = torch.full_like(s.path, -1), torch.zeros_like(s.accepted)
    place = torch.arange(n, device=b.device)
    for i in range(n):
        x = s.token[:, i].long()
        turn = (s.parent[:, i] == at) & (i < s.count)
        p = rest[b, x]
        if s.draft is not None:
            q = s.draft[b, at.long() + 1].double()
            stands = turn & (s.uniform[:, i].double() * q[b, x] * left < p)
            less = (rest - q).clamp_min(0)
            total = less.sum(dim=-1, keepdim=True)
            less = torch.where(total > 0, less / total, 0.0)
        else:
            stands = turn & (s.uniform[:, i].double() * left < p)
            less = rest.scatter(1, x[:, None], 0.0)
            left = torch.where(turn & ~stands, left - p, left)
        path = torch.where(stands[:, None] & (place == accepted[:, None]), i, path)
        accepted = accepted + stands.int()
        at = torch.where(stands, i, at)
        left = torch.where(stands, 1.0, left)
        rest = torch.where(stands[:, None], s.target[:, i + 1].double(), torch.where((turn & ~stands)[:, None], less, rest))
    row = s.target[b, at.long() + 1].double()
    rest = torch.where(rest.sum(dim=-1, keepdim=True) > 0, rest, row)
    run_sum = rest.cumsum(dim=-1)
    over = run_sum > s.uniform[:, n:].double() * run_sum[:, -1:]
    first = torch.where(over & (rest > 0), torch.arange(V, device=b.device), V).amin(dim=-1)
    last = torch.where(rest > 0, torch.arange(V, device=b.device), -1).amax(dim=-1)
    return path, accepted, torch.where(first < V, first, last).int()


def _plain_keep(s):
    n = s.path.shape[1]
    live = torch.arange(n, device=s.path.device) < s.count[:, None]
    page, row = _rows(s, s.base, n)
    p = s.path.clamp_min(0).long()
    from_page, from_row = torch.gather(page, 1, p), torch.gather(row, 1, p)
    for pool in (s.k, s.v):
        pool[page, :, :, row] = torch.where(live[..., None, None, None], pool[from_page, :, :, from_row], pool[page, :, :, row])
    return s.k, s.v


# ---- one pass --------------------------------------------------------------------------------


def run(s):
    if not own:
        return {"tree": _plain_tree, "append": _plain_append, "attend": _plain_attend, "verify": _plain_verify,
                "keep": _plain_keep}[s.kind](s)
    if s.kind == "tree":
        s.W.wnw_draft_tree(s.parent, s.base, s.mask, s.position, s.count)
        return s.mask, s.position
    if s.kind == "append":
        s.W.wnw_paged_append(s.cfg, s.cache, s.xk, s.xv, s.at, s.count, q_dev=s.q, q_out=s.q_out, rotary=s.rotary,
                             position_dev=s.position)
        return (s.k, s.v) if s.q is None else (s.k, s.v, s.q_out)
    if s.kind == "attend":
        s.W.wnw_paged_attend(s.cfg, s.cache, s.q, s.out, s.len, s.count, mask_dev=s.mask, lse_dev=s.lse,
                             workspace=s.workspace, max_len=s.top)
        return s.out, s.lse
    if s.kind == "verify":
        s.W.wnw_draft_verify(s.token, s.target, s.uniform, s.path, s.accepted, s.next, draft_dev=s.draft,
                             parent_dev=None if s.chain else s.parent, count_dev=s.count, workspace=s.workspace)
        return s.path, s.accepted, s.next
    s.W.wnw_paged_keep(s.cfg, s.cache, s.base, s.path, s.count)
    return s.k, s.v


# ---- what a pass cannot do without -----------------------------------------------------------


def work(c):
    if c["kind"] == "tree":
        tokens = sum(_counts(c))
        return {"bytes": tokens * (4 + 4 + 8 * ((c["n"] + 63) // 64)), "flops": tokens * c["n"]}
    if c["kind"] == "verify":
        rows = 2 if c["draft"] else 1       # the row that the next token is drawn from, at least
        return {"bytes": c["batch"] * (4 * rows * c["vocab"] + 20 * c["n"] + 8), "flops": 4 * c["batch"] * c["vocab"]}
    L, H, D = c["layers"], c["kv_heads"], c["head_dim"]
    if c["kind"] == "keep":
        stand = sum(min(c["n"], max(0, c["stand"] - (b if c["ragged"] else 0))) for b in range(c["batch"]))
        return {"bytes": 2 * stand * L * H * 2 * D * 2, "flops": 0}
    if c["kind"] == "append":
        vectors = sum(_counts(c)) * L * (2 * H + (c["q_heads"] if c["queries"] else 0))
        return {"bytes": vectors * D * 2 * 2, "flops": 3 * vectors * c["rotated"]}
    lens, counts = _attend_sizes(c)
    tokens, Hq = sum(counts), c["q_heads"]
    pairs = sum(n * (t - n) + n * (n + 1) / 2 for t, n in zip(lens, counts))
    io = L * Hq * tokens * (D * (2 + (2 if c["bf16"] else 4)) + 4)
    return {"bytes": sum(lens) * L * H * D * 4 + io, "flops": L * Hq * pairs * 4 * D}


# ---- the same in 64 bits ---------------------------------------------------------------------


def _exact_pages(s, pool, b, T):
    """Rows 0 .. T - 1 of sequence b, [L][H_kv][T][d] double."""
    used = s.table[b, : -(-T // s.page)].long()
    return torch.cat([pool[p] for p in used], dim=2)[:, :, :T].double()


def _exact_append(c, s):
    B, L, _, n, D = s.xk.shape
    h = s.dim // 2
    i = torch.arange(D, device="cuda")
    turned = i < s.dim
    if s.halves:
        pair, other, sign = i % max(h, 1), torch.where(i < h, i + h, i - h), torch.where(i < h, -1.0, 1.0)
    else:
        pair, other, sign = i // 2, i ^ 1, torch.where(i % 2 == 0, -1.0, 1.0)
    pair, other = pair.clamp(0, max(h - 1, 0)), torch.where(turned, other, i)
    freq = s.freq.double() if h else torch.zeros(1, dtype=torch.float64, device="cuda")
    outs = [s.k.double(), s.v.double()] + ([] if s.q is None else [torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")])
    for b in range(B):
        at, cnt = int(s.at[b]), int(s.count[b])
        row = torch.arange(at, at + cnt, device="cuda")
        # angles without their positions' whole turns, so that far positions lose nothing
        a = torch.remainder((row + c["far"]).double()[:, None] * freq, 2 * math.pi)[:, pair]               # [cnt][d]
        cs = torch.where(turned, torch.cos(a) * s.amplitude, 1.0)
        sn = torch.where(turned, torch.sin(a) * sign * s.amplitude, 0.0)
        p, r = s.table[b, row // s.page].long(), row % s.page
        x = s.xk[b, :, :, :cnt].double()
        outs[0][p, :, :, r] = (x * cs + x[..., other] * sn).permute(2, 0, 1, 3)
        outs[1][p, :, :, r] = s.xv[b, :, :, :cnt].double().permute(2, 0, 1, 3)
        if s.q is not None:
            x = s.q[b, :, :, :cnt].double()
            outs[2][b, :, :, :cnt] = x * cs + x[..., other] * sn
    return outs


def _exact_attend(c, s):
    B, L, Hq, n, D = s.q.shape
    G = Hq // c["kv_heads"]
    parents = [[i - 1 for i in range(n)]] * B if s.mask is None else s.parents
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, L, Hq, n), dtype=torch.float64, device="cuda")
    for b in range(B):
        T, cnt = int(s.len[b]), int(s.count[b])
        if not cnt:
            continue
        unseen = torch.zeros((cnt, T), dtype=torch.bool, device="cuda")
        unseen[:, T - cnt:] = ~torch.tensor(_ancestors(parents[b]), device="cuda")[:cnt, :cnt]
        ks, vs = _exact_pages(s, s.k, b, T), _exact_pages(s, s.v, b, T)
        for l in range(L):
            for h in range(c["kv_heads"]):
                x = s.q[b, l, h * G: (h + 1) * G, :cnt].double().flatten(0, 1) @ ks[l, h].T.contiguous() / math.sqrt(D)
                x = x.unflatten(0, (G, cnt)).masked_fill(unseen, -math.inf)
                lse[b, l, h * G: (h + 1) * G, :cnt] = torch.logsumexp(x, dim=-1)
                out[b, l, h * G: (h + 1) * G, :cnt] = (torch.softmax(x, dim=-1).flatten(0, 1) @ vs[l, h]).unflatten(0, (G, cnt))
    return out, lse


def _exact_verify(c, s):
    B, n = s.token.shape
    path, accepted, after = torch.full_like(s.path, -1), torch.zeros_like(s.accepted), torch.zeros_like(s.next)
    for b in range(B):
        parent, token, u = s.parent[b].tolist(), s.token[b].tolist(), s.uniform[b].double().tolist()
        node, got = -1, []
        while True:
            p, left, moved = s.target[b, node + 1].double(), 1.0, False
            for i in range(int(s.count[b])):
                if parent[i] != node:
                    continue
                t = token[i]
                q = s.draft[b, node + 1].double() if s.draft is not None else None
                if u[i] * (float(q[t]) if q is not None else left) < float(p[t]):
                    node, moved = i, True
                    got.append(i)
                    break
                if q is not None:
                    p = (p - q).clamp_min(0)
                    p = p / p.sum() if float(p.sum()) > 0 else p
                else:
                    left -= float(p[t])
                    p = p.index_fill(0, torch.tensor([t], device="cuda"), 0.0)
            if not moved:
                break
        if not float(p.sum()) > 0:
            p = s.target[b, node + 1].double()
        sums = p.cumsum(dim=0)
        hit = torch.searchsorted(sums, u[n] * sums[-1], right=True).reshape(1)
        accepted[b], after[b] = len(got), hit.clamp_max(int(p.nonzero().max()))[0]
        path[b, : len(got)] = _ints(got)
    return path, accepted, after


def _exact_tree(c, seed, s):
    mask, position = torch.zeros_like(s.mask), torch.zeros_like(s.position)
    bits, depths = [], []
    for see in map(_ancestors, _parents(c, seed)):
        rows = [sum(1 << j for j, v in enumerate(r) if v) for r in see]
        words = [[(r >> (64 * w)) & (2 ** 64 - 1) for w in range(mask.shape[2])] for r in rows]
        bits.append([[x - 2 ** 64 if x >> 63 else x for x in w] for w in words])
        depths.append([bin(r).count("1") - 1 for r in rows])
    for b, cnt in enumerate(_counts(c)):
        mask[b, :cnt] = torch.tensor(bits[b][:cnt], device="cuda").reshape(cnt, -1)
        position[b, :cnt] = _ints(depths[b][:cnt]) + s.base[b]
    return mask, position


def _exact_keep(c, s):
    outs = []
    for pool in (s.k, s.v):
        y = pool.double()
        for b in range(c["batch"]):
            base = int(s.base[b])
            place = lambda r: (int(s.table[b, r // s.page]), r % s.page)   # noqa: E731
            for i in range(int(s.count[b])):
                (p, r), (fp, fr) = place(base + i), place(base + int(s.path[b, i]))
                y[p, :, :, r] = pool[fp, :, :, fr].double()
        outs.append(y)
    return outs


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "tree":
        return _exact_tree(c, seed, s)
    if c["kind"] == "attend" and c["tree"]:
        s.parents = _parents(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep}[c["kind"]](c, s)
