"""GPU tests of the paged cache (wnw_paged_append, wnw_paged_attend, wnw_paged_keep) and of drafts (wnw_draft_tree,
wnw_draft_verify) against the same arithmetic in 64 bits on the CPU (paged_reference.py).  Copied rows and whole numbers have
to be equal.

A rotated element y = amplitude (x0 cos - x1 sin): the angle's turns are exact but for 2^-53 of them and rounded to 2^-24 of at most half
a turn, so the angle is off by pi 2^-24, cosine and sine by as much and their own two steps (2^-23), the amplitude's product and the two of
the sum by 2^-24 each: together below 2^-21 (|x0| + |x1|) amplitude; and half a step of bf16, 2^-8 |y|, at the end.

Attention: products of bf16 are exact in fp32 and d of them are summed, so a base-2 logit is off by at most (d + 3) 2^-24
sum|q k| / sqrt(d) log2(e) with its scaling and the subtraction of the maximum (at most twice that magnitude); a weight by ln 2 times
that, its exponential by 2^-22, and the denominator alike.  T products are summed in fp32 (T 2^-24 at worst, taken with the joins).
bf16 outputs add half a step, 2^-8 |y|; with more than 32 query rows of a KV-head the weights that multiply V are rounded to bf16
as well, 2^-8 of sum p |v|.
"""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests.wnw_harness import log

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def W():
    from paper_2608_22704_amd import wnw
    return wnw


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(g, *shape):
    """bf16 rows whose sizes vary by row."""
    return (torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn((*shape[:-1], 1), generator=g))).bfloat16()


def new_cache(W, g, B, L, H, D, page, width, spare=2, bf16=False, holes=()):
    """A cache whose pages hold earlier rows, handed out in no order; holes: (sequence, entry) without a page."""
    pages = B * width + spare
    cfg = W.make_paged_config(B, L, H, page, pages, width, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    c = W.make_paged_cache(cfg)
    table = torch.randperm(pages, generator=g)[:B * width].reshape(B, width).int()
    for i, (b, j) in enumerate(holes):
        table[b, j] = (-1, pages, -2147483648, 2147483647)[i % 4]
    c.table.copy_(table)
    for x in (c.k, c.v):
        x.copy_(rows(g, *x.shape))
    return cfg, c


# ---- appending -------------------------------------------------------------------------------

ROTATIONS = [(0, False), (128, False), (128, True), (64, False), (64, True), (80, False), (16, False), (2, False), (2, True), (6, False),
             (34, False), (46, True), (126, False), (100, False)]


def check_append(W, dim, pairs, D, page, n, at, count, first=0, nl=2, position=None, amplitude=1.0, holes=(), queries=5, keys=True, freq=None):
    g = torch.Generator().manual_seed(dim * 1000 + n * 10 + D)
    B, L, H, width = len(at), 3, 3, max(2, -(-(max(x for x in at if x < 10000) + n) // page))
    log(f"[case] append dim={dim} pairs={pairs} d={D} page={page} n={n} at={at} count={count} layers={first}+{nl} queries={queries} keys={keys}")
    cfg, c = new_cache(W, g, B, L, H, D, page, width, holes=holes)
    k0, v0, table = c.k.cpu().clone(), c.v.cpu().clone(), c.table.cpu()
    xk, xv = rows(g, B, nl, H, n, D), rows(g, B, nl, H, n, D)
    xq = rows(g, B, nl, queries, n, D) if queries else None
    if freq is None:
        freq = W.wnw_rotary_frequencies(dim, 1e4, 2.0, 1.0, 4.0, 4096)
    rotary = W.make_rotary(torch.from_numpy(freq).cuda(), dim, W.WNW_ROTARY_PAIRS if pairs else W.WNW_ROTARY_HALVES, amplitude)
    q = xq.cuda() if queries else None
    out = torch.full_like(q, 7.0) if queries else None
    W.wnw_paged_append(cfg, c, xk.cuda() if keys else None, xv.cuda() if keys else None, i32(at), None if count is None else i32(count), q_dev=q,
                       q_out=out, rotary=rotary, position_dev=None if position is None else i32(position), first_layer=first)
    torch.cuda.synchronize()
    if queries:
        assert torch.equal(q.cpu(), xq)
    k1, v1 = c.k.cpu(), c.v.cpu()
    counts = [n] * B if count is None else [R.clamp(x, n) for x in count]
    rotated = torch.zeros(D, dtype=torch.bool)
    rotated[:dim] = True

    def check(got, x, p):
        want, size = R.rotate(x.double(), p, freq, dim, pairs, amplitude)
        assert torch.equal(got[..., ~rotated], x[..., ~rotated])
        err = (got.double() - want).abs()
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -21 * size
        assert (err <= bound)[..., rotated].all(), float((err - bound).max())

    for b in range(B):
        a = R.clamp(at[b], width * page)
        for i in range(counts[b]):
            p = position[b][i] if position is not None else a + i
            if queries:
                check(out[b, :, :, i].cpu(), xq[b, :, :, i], p)
            to = R.place(table, b, a + i, page, cfg.pages)
            if to is None or not keys:
                continue
            check(k1[to[0], first: first + nl, :, to[1]], xk[b, :, :, i], p)
            assert torch.equal(v1[to[0], first: first + nl, :, to[1]], xv[b, :, :, i])
            for new, old in ((k1, k0), (v1, v0)):
                new[to[0], first: first + nl, :, to[1]] = old[to[0], first: first + nl, :, to[1]]
        if queries:
            assert (out[b, :, :, counts[b]:] == 7.0).all()
    assert torch.equal(k1, k0) and torch.equal(v1, v0)      # nothing else changed


@pytest.mark.parametrize("dim,pairs", ROTATIONS)
@pytest.mark.parametrize("D", [64, 128])
def test_append_rotations(W, dim, pairs, D):
    check_append(W, min(dim, D), pairs, D, 16, 5, [3, 30], [5, 2], amplitude=1.25)


@pytest.mark.parametrize("n", [1, 2, 3, 8, 15, 16, 17, 33, 100])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 64), (128, 256), (64, 32), (128, 128)])
def test_append_sizes(W, n, D, page):
    check_append(W, 64, False, D, page, n, [0, page - 1, 37], [n, 1, 0], first=1, nl=2)
    check_append(W, D, True, D, page, n, [page, 2 * page + 5], None, first=0, nl=1, queries=0)


def test_append_positions(W):
    far = [[0, 1, 2147483647], [-1, -2147483648, 16777217]]
    for dim, pairs in ((128, False), (128, True), (64, False)):
        check_append(W, dim, pairs, 128, 32, 3, [5, 40], None, position=far)
    # frequencies at which 32 bits would not know the angle at all, and none
    check_append(W, 8, False, 128, 32, 3, [5, 40], None, position=far, freq=np.array([1.0, 3.1415927, 1e-8, 0.0], dtype=np.float32))


def test_append_outside(W):
    """Lengths and counts outside their ranges, rows past the capacity, entries without a page."""
    check_append(W, 64, False, 128, 16, 20, [20, -5, 50], [25, -1, 20], holes=[(0, 2), (2, 4)])
    check_append(W, 64, False, 128, 16, 20, [64, 1 << 30, 60], [20, 3, 7], holes=[(0, 0), (1, 0), (2, 3), (0, 3)])


def test_append_queries_alone(W):
    check_append(W, 64, True, 128, 16, 4, [20, 7], [4, 1], keys=False)


def test_append_in_place_and_without_rotation(W):
    log("[case] append in place; without rotation")
    g = torch.Generator().manual_seed(4)
    cfg, c = new_cache(W, g, 1, 1, 2, 128, 32, 4)
    x, q = rows(g, 1, 1, 2, 40, 128).cuda(), rows(g, 1, 1, 6, 40, 128).cuda()
    rot = W.make_rotary(torch.from_numpy(W.wnw_rotary_frequencies(128, 1e4)).cuda(), 128)
    out = torch.empty_like(q)
    W.wnw_paged_append(cfg, c, x, x, i32([3]), q_dev=q, q_out=out, rotary=rot)
    k = c.k.clone()
    same = q.clone()
    W.wnw_paged_append(cfg, c, x, x, i32([3]), q_dev=same, q_out=same, rotary=rot)
    assert torch.equal(same, out) and torch.equal(c.k, k)
    W.wnw_paged_append(cfg, c, x, x, i32([3]), q_dev=q, q_out=out)
    assert torch.equal(out, q)
    for i in range(40):
        p, r = R.place(c.table.cpu(), 0, 3 + i, 32, cfg.pages)
        assert torch.equal(c.k[p, 0, :, r], x[0, 0, :, i]) and torch.equal(c.v[p, 0, :, r], x[0, 0, :, i])


def test_append_numbers_that_are_not_finite(W):
    """They stay where they are, and reach their pair and nothing else."""
    log("[case] append inf, NaN")
    g = torch.Generator().manual_seed(5)
    cfg, c = new_cache(W, g, 1, 1, 1, 64, 16, 2)
    x = rows(g, 1, 1, 1, 3, 64)
    x[..., 0, 3], x[..., 1, 40], x[..., 2, 63] = math.inf, math.nan, -math.inf
    rot = W.make_rotary(torch.from_numpy(W.wnw_rotary_frequencies(48, 1e4)).cuda(), 48)
    W.wnw_paged_append(cfg, c, x.cuda(), x.cuda(), i32([1]), rotary=rot)
    got = torch.stack([c.k[R.place(c.table.cpu(), 0, 1 + i, 16, cfg.pages)[0], 0, 0, 1 + i] for i in range(3)]).cpu()
    bad = ~torch.isfinite(got)
    assert bad.nonzero().tolist() == [[0, 3], [0, 27], [1, 16], [1, 40], [2, 63]]
    assert got[2, 63] == -math.inf


# ---- attention -------------------------------------------------------------------------------


def logit_bound(D, absq, T):
    lerr = (D + 3) * EPS * absq * math.log2(math.e) * 4
    return lerr, 2 * (math.log(2) * 2 * lerr + 2.0 ** -22)


def check_outputs(out, lse, ref, D, bf16, rounded_weights):
    """out, lse (CPU) against paged_reference.attend's; tokens past a count hold 7."""
    want, wlse, absv, absq, seen = ref
    gone = torch.isnan(wlse)
    assert (out[gone] == 7.0).all() and (lse[gone] == 7.0).all()
    live = ~gone
    lerr, werr = logit_bound(D, absq, seen)
    empty = live & (wlse == -math.inf)
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
    some = live & ~empty
    bound = (werr + seen * EPS + 4 * EPS).unsqueeze(-1) * absv
    if rounded_weights:
        bound = bound + 2.0 ** -8 * absv
    if bf16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    err = (out.double() - want).abs()
    assert torch.isfinite(out[some]).all()
    worst = (err - bound)[some]
    assert (worst <= 0).all(), (float(worst.max()), float(err[some].max()))
    lbound = (math.log(2) * 2 * lerr + 2.0 ** -22 + seen * EPS + 4 * EPS * (1 + wlse.abs()))[some]
    assert ((lse.double() - wlse)[some].abs() <= lbound).all(), float(((lse.double() - wlse)[some].abs() - lbound).max())


def some_tree(g, n):
    return [-1 if i == 0 or g.random() < 0.1 else (i - 1 if g.random() < 0.5 else int(g.integers(-1, i))) for i in range(n)]


def run_attend(W, cfg, c, q, lens, counts, mask=None, max_len=0, first=0, workspace_fill=0xFF, stream=None):
    n = q.shape[3]
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16 if cfg.flags else torch.float32, device="cuda")
    lse = torch.full(q.shape[:-1], 7.0, device="cuda")
    ws = torch.full((max(16, W.wnw_paged_attend_workspace(cfg, q.shape[1], q.shape[2], n, max_len)),), workspace_fill, dtype=torch.uint8, device="cuda")
    W.wnw_paged_attend(cfg, c, q, out, i32(lens), None if counts is None else i32(counts), mask_dev=mask, lse_dev=lse, workspace=ws, max_len=max_len,
                       first_layer=first, stream=stream)
    return out, lse


def check_attend(W, H, G, D, page, n, lens, counts, tree, bf16=False, L=2, first=0, nl=None, max_len=0, holes=(), see=None, seed=0):
    B = len(lens)
    nl = nl or L - first
    width = max(1, -(-max(1, n, *[x for x in lens if x < 100000]) // page))
    log(f"[case] attend H={H} G={G} d={D} page={page} n={n} lens={lens} counts={counts} tree={tree} bf16={bf16} layers={first}+{nl} holes={holes}")
    g = torch.Generator().manual_seed(seed + n * 100 + D)
    rng = np.random.default_rng(seed + n)
    cfg, c = new_cache(W, g, B, L, H, D, page, width, bf16=bf16, holes=holes)
    # rows that no sequence has hold what must not matter
    k, v, table = c.k.cpu(), c.v.cpu(), c.table.cpu()
    for pool, junk in ((k, math.nan), (v, math.inf)):
        keep = torch.zeros(pool.shape[0], page, dtype=torch.bool)
        for b in range(B):
            for r in range(R.clamp(lens[b], width * page)):
                to = R.place(table, b, r, page, cfg.pages)
                if to:
                    keep[to] = True
        pool.permute(0, 3, 1, 2, 4)[~keep] = junk
    c.k.copy_(k)
    c.v.copy_(v)
    q = rows(g, B, nl, H * G, n, D)
    if tree and see is None:
        see = [R.ancestors(some_tree(rng, n)) for _ in range(B)]
    mask = torch.stack([R.words(s) for s in see]).cuda() if see is not None else None
    out, lse = run_attend(W, cfg, c, q.cuda(), lens, counts, mask, max_len, first)
    torch.cuda.synchronize()
    ref = R.attend(q, k, v, table, page, lens, counts or [n] * B, see, first)
    check_outputs(out.cpu(), lse.cpu(), ref, D, bf16, bf16 and G * n > 32)


LENGTHS = [[1], [0, 1, 2], [31, 32, 33], [63, 64, 65, 16], [127, 128, 129], [300, 5, 0, 177]]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("D,page,G,bf16", [(128, 16, 4, False), (64, 16, 1, True), (128, 32, 3, True), (64, 128, 16, False), (128, 64, 20, False),
                                           (64, 32, 40, True)])
def test_single_tokens(W, lens, D, page, G, bf16):
    check_attend(W, 2, G, D, page, 1, lens, None, False, bf16)


@pytest.mark.parametrize("n", [2, 5, 8, 9, 16, 17, 33, 64, 65, 70, 130])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("D,page,G", [(128, 16, 1), (64, 64, 4), (128, 32, 2), (64, 16, 3)])
def test_drafts(W, n, tree, D, page, G):
    top = n + 61
    check_attend(W, 2, G, D, page, n, [top, n, max(1, n // 2), 200 + n], [n, n, n, max(1, n - 3)], tree, bf16=(n + G) % 2 == 0, seed=n)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_a_prompt(W, D, bf16):
    check_attend(W, 1, 2, D, 64, 200, [200, 333], [200, 190], False, bf16, L=1)
    check_attend(W, 1, 5, D, 16, 100, [413], None, False, bf16, L=1)


@pytest.mark.parametrize("B,H,L,nl", [(1, 1, 1, 1), (1, 3, 1, 1), (2, 5, 1, 1), (1, 8, 1, 1), (3, 3, 2, 1), (2, 3, 3, 2), (2, 8, 1, 1)])
def test_prompts_of_any_number_of_heads(W, B, H, L, nl):
    """Several blocks of rows a head, which are dealt out to the dies."""
    check_attend(W, H, 1, 64, 16, 600, [600, 37, 555][:B], [600, 37, 520][:B], False, L=L, first=L - nl, nl=nl)
    check_attend(W, H, 3, 128, 32, 200, [300, 200, 170][:B], [200, 150, 0][:B], True, bf16=True, L=L, first=L - nl, nl=nl)


@pytest.mark.parametrize("D", [64, 128])
def test_long_sequences_that_are_shared(W, D):
    """Parts of a cache for many work-groups, the join, ragged batches."""
    check_attend(W, 1, 4, D, 32, 1, [5000, 1, 0, 777, 3001], None, False, L=1)
    check_attend(W, 2, 4, D, 16, 6, [2100, 6, 1500], [6, 6, 2], True, L=1)
    check_attend(W, 1, 8, D, 16, 12, [2500, 900], [12, 12], True, bf16=True, L=1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,bf16", [(1, False), (6, True), (16, True), (16, False), (32, True), (32, False), (64, True), (50, False)])
def test_room_for_many_rows(W, n, bf16, D):
    """A capacity that no cache of the device holds: tiles are loaded past the caches."""
    log(f"[case] attend, large capacity, n={n} bf16={bf16} d={D}")
    g = torch.Generator().manual_seed(n)
    H, G, page, T = 8, 4, 16, 500
    cfg = W.make_paged_config(1, 1, H, page, 40, 16384, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    c = W.make_paged_cache(cfg)
    c.table[0, :32] = torch.randperm(40, generator=g)[:32].int().cuda()
    for x in (c.k, c.v):
        x.copy_(rows(g, *x.shape))
    q = rows(g, 1, 1, H * G, n, D)
    out, lse = run_attend(W, cfg, c, q.cuda(), [T], None)
    ref = R.attend(q, c.k.cpu(), c.v.cpu(), c.table.cpu(), page, [T], [n], None, 0)
    check_outputs(out.cpu(), lse.cpu(), ref, D, bf16, bf16 and G * n > 32)


def test_many_sequences(W):
    """More sequences than a wavefront has lanes."""
    g = np.random.default_rng(7)
    lens = [int(x) for x in g.integers(0, 90, 70)]
    check_attend(W, 1, 2, 64, 16, 1, lens, None, False, L=1)
    check_attend(W, 1, 2, 128, 16, 3, lens, [int(x) for x in g.integers(0, 4, 70)], True, L=1)


@pytest.mark.parametrize("G", [1, 8])
def test_masks_of_any_kind(W, G):
    """Rows that see nothing of the draft, or nothing at all, everything, or later tokens."""
    n = 70
    rng = np.random.default_rng(3)
    see = [np.zeros((n, n), dtype=bool), np.ones((n, n), dtype=bool), rng.random((n, n)) < 0.3, np.eye(n, dtype=bool)]
    see[2][5] = False
    check_attend(W, 1, G, 128, 16, n, [n, n + 30, n, n + 5], None, True, see=see)
    check_attend(W, 1, G, 64, 32, n, [n, n, n + 100, 40], [n, 3, n, n], True, bf16=True, see=see)


def test_pages_that_are_not_there(W):
    check_attend(W, 2, 2, 128, 16, 4, [100, 40, 200], None, True, holes=[(0, 0), (0, 3), (1, 2), (2, 12), (2, 5)])
    check_attend(W, 2, 2, 64, 16, 1, [100, 40, 30], None, False, holes=[(0, 6), (1, 0), (1, 1), (1, 2), (2, 0)])
    check_attend(W, 1, 20, 128, 32, 5, [100, 64], None, False, bf16=True, holes=[(0, 1), (1, 1), (1, 0)])
    check_attend(W, 1, 12, 64, 16, 4, [150, 64], None, True, holes=[(0, 0), (0, 5), (1, 1)])
    check_attend(W, 2, 16, 128, 16, 20, [400, 64, 90], None, True, bf16=True, holes=[(0, 2), (0, 24), (1, 1), (2, 0)])
    check_attend(W, 1, 16, 64, 64, 20, [700, 64, 90], None, False, holes=[(0, 4), (1, 0), (2, 1)])


def test_layers_lengths_and_counts(W):
    check_attend(W, 2, 3, 128, 16, 2, [50, 20], None, False, L=4, first=1, nl=2)
    check_attend(W, 2, 3, 128, 16, 5, [64, -3, 1 << 30, 50], [9, 5, -1, 2], False, max_len=7)
    check_attend(W, 2, 3, 64, 16, 5, [64, 64, 3, 50], [5, 5, 5, 2], True, max_len=64)


def test_bf16_outputs_are_the_fp32_ones_rounded(W):
    """Up to 32 query rows of a KV-head."""
    for n, G, lens in ((1, 4, [700, 33]), (5, 4, [300, 20]), (8, 4, [1000, 9]), (1, 32, [64, 65])):
        log(f"[case] bf16 outputs n={n} G={G}")
        g = torch.Generator().manual_seed(n)
        cfg, c = new_cache(W, g, 2, 1, 2, 128, 16, 64)
        q = rows(g, 2, 1, 2 * G, n, 128).cuda()
        full, _ = run_attend(W, cfg, c, q, lens, None)
        half = W.make_paged_config(2, 1, 2, 16, cfg.pages, 64, flags=W.WNW_F_OUT_BF16)
        short, _ = run_attend(W, half, c, q, lens, None)
        assert torch.equal(full.bfloat16(), short)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8, 12, 24])
def test_numbers_that_are_not_finite(W, D, G):
    """In rows that a token does not see they do nothing; in those that it sees they reach the outputs that they belong to."""
    log(f"[case] attend inf, NaN d={D} G={G}")
    g = torch.Generator().manual_seed(11)
    n, T, page = 6, 100, 16
    cfg, c = new_cache(W, g, 1, 1, 1, D, page, 8)
    table = c.table.cpu()
    see = R.ancestors([-1, 0, 0, 1, 2, -1])
    mask = R.words(see)[None].cuda()
    q = rows(g, 1, 1, G, n, D)
    clean, clean_lse = (x.cpu() for x in run_attend(W, cfg, c, q.cuda(), [T], None, mask))
    at = lambda r: R.place(table, 0, r, page, cfg.pages)   # noqa: E731
    # V of token 1 (seen by 1 and 3) and of the prefix; K of token 2 (seen by 2 and 4)
    v, k = c.v.cpu().clone(), c.k.cpu().clone()
    v2, k2 = v.clone(), k.clone()
    v2[at(T - n + 1)[0], 0, 0, at(T - n + 1)[1], 5] = math.inf
    v2[at(T - n + 1)[0], 0, 0, at(T - n + 1)[1], D - 1] = math.nan
    k2[at(T - n + 2)[0], 0, 0, at(T - n + 2)[1], 7] = math.nan
    c.v.copy_(v2)
    c.k.copy_(k2)
    out, lse = (x.cpu() for x in run_attend(W, cfg, c, q.cuda(), [T], None, mask))
    bad = ~torch.isfinite(out[0, 0])
    want = torch.zeros_like(bad)
    want[:, [1, 3], 5] = want[:, [1, 3], D - 1] = True
    want[:, [2, 4]] = True
    assert torch.equal(bad, want)
    assert torch.equal(out[0, 0][~want], clean[0, 0][~want])
    assert torch.isnan(lse[0, 0][:, [2, 4]]).all() and torch.equal(lse[0, 0][:, [0, 1, 3, 5]], clean_lse[0, 0][:, [0, 1, 3, 5]])
    # in the prefix everyone sees it
    v2 = v.clone()
    v2[at(3)[0], 0, 0, at(3)[1], 9] = -math.inf
    c.v.copy_(v2)
    c.k.copy_(k)
    out, _ = (x.cpu() for x in run_attend(W, cfg, c, q.cuda(), [T], None, mask))
    bad = ~torch.isfinite(out[0, 0])
    assert bad[:, :, 9].all() and bad.sum() == G * n
    # a query row
    c.v.copy_(v)
    for x in (math.inf, -math.inf, math.nan):
        q2 = q.clone()
        q2[0, 0, G - 1, 3, 2] = x
        out, lse = (t.cpu() for t in run_attend(W, cfg, c, q2.cuda(), [T], None, mask))
        want = torch.zeros((G, n), dtype=torch.bool)
        want[G - 1, 3] = True
        assert torch.equal(torch.isnan(out[0, 0]).all(dim=-1), want) and torch.equal(torch.isnan(lse[0, 0]), want)
        assert torch.equal(out[0, 0][~want], clean[0, 0][~want])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 20, 40, 80, 200])
def test_a_token_that_does_not_see_itself(W, D, G):
    """A single token whose mask leaves out its own row, in which there is no number."""
    log(f"[case] attend, own row unseen, d={D} G={G}")
    g = torch.Generator().manual_seed(5)
    T, page = 70, 16
    cfg, c = new_cache(W, g, 1, 1, 1, D, page, 5)
    to = R.place(c.table.cpu(), 0, T - 1, page, cfg.pages)
    c.k[to[0], 0, 0, to[1]] = math.nan
    c.v[to[0], 0, 0, to[1]] = math.inf
    q = rows(g, 1, 1, G, 1, D)
    see = [np.zeros((1, 1), dtype=bool)]
    out, lse = run_attend(W, cfg, c, q.cuda(), [T], None, R.words(see[0])[None].cuda())
    k, v = c.k.cpu(), c.v.cpu()
    check_outputs(out.cpu(), lse.cpu(), R.attend(q, k, v, c.table.cpu(), page, [T], [1], see, 0), D, False, False)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("G", [12, 24])
def test_rows_do_not_depend_on_the_rows_beside_them(W, G):
    """Bit for bit: a token's logits that grow along the cache move its own maximum alone."""
    log(f"[case] attend, rows beside each other, G={G}")
    g = torch.Generator().manual_seed(6)
    n, T, D, page = 6, 400, 128, 16
    cfg, c = new_cache(W, g, 1, 1, 1, D, page, 25, bf16=True)
    q = rows(g, 1, 1, G, n, D)
    clean, clean_lse = (x.cpu() for x in run_attend(W, cfg, c, q.cuda(), [T], None))
    q2 = q.clone()
    q2[0, 0, :, 4] *= 64
    out, lse = (x.cpu() for x in run_attend(W, cfg, c, q2.cuda(), [T], None))
    others = [0, 1, 2, 3, 5]
    assert torch.equal(out[0, 0][:, others], clean[0, 0][:, others]) and torch.equal(lse[0, 0][:, others], clean_lse[0, 0][:, others])
    assert not torch.equal(lse[0, 0][:, 4], clean_lse[0, 0][:, 4])


def test_offsets_past_32_bits(W):
    """Pages beyond 4 GiB of the buffers."""
    log("[case] paged, buffers above 4 GiB")
    B, L, H, D, page = 1, 2, 8, 128, 256
    pages = (5 << 30) // (L * H * page * D * 2)
    cfg = W.make_paged_config(B, L, H, page, pages, 3)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.zeros((pages, L, H, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 0, pages // 2 + 3]], dtype=torch.int32)
    c = W.PagedCache(k, v, table.cuda())
    x, y = rows(g, B, L, H, 600, D), rows(g, B, L, H, 600, D)
    W.wnw_paged_append(cfg, c, x.cuda(), y.cuda(), i32([0]))
    W.wnw_paged_keep(cfg, c, i32([500]), i32([[40, 90]]))
    x[:, :, :, [500, 501]], y[:, :, :, [500, 501]] = x[:, :, :, [540, 590]], y[:, :, :, [540, 590]]
    q = rows(g, B, L, 2 * H, 1, D)
    out, lse = run_attend(W, cfg, c, q.cuda(), [555], None)
    small = torch.zeros((3, L, H, page, D), dtype=torch.bfloat16)
    small_v = torch.zeros_like(small)
    for p in range(3):
        m = min(600, (p + 1) * page) - p * page
        small[p, :, :, :m], small_v[p, :, :, :m] = x[0, :, :, p * page: p * page + m], y[0, :, :, p * page: p * page + m]
    ref = R.attend(q, small, small_v, torch.tensor([[0, 1, 2]]), page, [555], [1])
    check_outputs(out.cpu(), lse.cpu(), ref, D, False, False)
    del k, v, c
    torch.cuda.empty_cache()


def test_graphs_and_streams(W):
    """Two captured graphs of attention on two streams, a workspace each, replayed at once, with lengths that change between the replays;
    the same call twice gives the same bits."""
    log("[case] paged attention captured")
    g = torch.Generator().manual_seed(2)
    B, H, G, D, page, n = 2, 2, 4, 128, 16, 5
    cfg, c = new_cache(W, g, B, 1, H, D, page, 130)
    rng = np.random.default_rng(5)
    q = rows(g, B, 1, H * G, n, D).cuda()
    lens = i32([2000, 300])
    mask = torch.stack([R.words(R.ancestors(some_tree(rng, n))) for _ in range(B)]).cuda()
    need = W.wnw_paged_attend_workspace(cfg, 1, H * G, n)
    sets = []
    for s in range(2):
        sets.append(dict(out=torch.zeros(q.shape, device="cuda"), lse=torch.zeros(q.shape[:-1], device="cuda"),
                         ws=torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda"), stream=torch.cuda.Stream(), graph=torch.cuda.CUDAGraph()))
    torch.cuda.synchronize()
    for s in sets:
        with torch.cuda.graph(s["graph"], stream=s["stream"]):
            W.wnw_paged_attend(cfg, c, q, s["out"], lens, mask_dev=mask, lse_dev=s["lse"], workspace=s["ws"])
    for step in range(4):
        lens.copy_(i32([2000 - 500 * step, 300 + 7 * step]))
        want, wlse = run_attend(W, cfg, c, q, lens.tolist(), None, mask)
        again, _ = run_attend(W, cfg, c, q, lens.tolist(), None, mask, workspace_fill=0)
        assert torch.equal(want, again)
        torch.cuda.synchronize()
        for s in sets:
            s["out"].zero_()
        torch.cuda.synchronize()
        for s in sets:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s in sets:
            assert torch.equal(s["out"], want) and torch.equal(s["lse"], wlse), step


# ---- keeping ---------------------------------------------------------------------------------


@pytest.mark.parametrize("D,page", [(128, 16), (64, 32), (128, 256)])
@pytest.mark.parametrize("base,paths,counts", [
    ([0, 5, 37], [[0, 1, 2], [1, 4, 9], [2, 3, 4]], None),
    ([15, 16, 30], [[3, 2, 9], [0, 5, 5], [-1, 3, 4]], [3, 3, 3]),
    ([20, 0, 3], [[7, 8, 30], [1, 2, 3], [4, 9, 11]], [5, -1, 2]),
    ([40, 60, 0], [[20, 23, 30], [3, 40, 2000000000], [2, 60, 62]], None),
])
def test_keep(W, D, page, base, paths, counts):
    log(f"[case] keep d={D} page={page} base={base} paths={paths} counts={counts}")
    check_keep(W, D, page, base, paths, counts, first=1, nl=1)


def check_keep(W, D, page, base, paths, counts, first=0, nl=None, L=2, holes=()):
    g = torch.Generator().manual_seed(3)
    B, n = len(base), len(paths[0])
    width = max(2, -(-64 // page))
    cfg, c = new_cache(W, g, B, L, 3, D, page, width, holes=holes)
    nl = nl or L - first
    want, table = [x.cpu().clone() for x in (c.k, c.v)], c.table.cpu()
    W.wnw_paged_keep(cfg, c, i32(base), i32(paths), None if counts is None else i32(counts), first_layer=first, n_layers=nl)
    torch.cuda.synchronize()
    cap = width * page
    for b in range(B):
        at = R.clamp(base[b], cap)
        for i in range(n if counts is None else R.clamp(counts[b], n)):
            p = paths[b][i]
            if p < 0 or at + p >= cap or (i and p <= paths[b][i - 1]):
                break
            src, dst = R.place(table, b, at + p, page, cfg.pages), R.place(table, b, at + i, page, cfg.pages)
            if src and dst:
                for x in want:
                    x[dst[0], first: first + nl, :, dst[1]] = x[src[0], first: first + nl, :, src[1]].clone()
    assert torch.equal(c.k.cpu(), want[0]) and torch.equal(c.v.cpu(), want[1])


def test_keep_long_paths(W):
    """Every entry of the step's registers, several steps, and sources that are later destinations."""
    log("[case] keep, long paths")
    rng = np.random.default_rng(1)
    for n in (16, 17, 31, 33, 70, 200):
        paths = [sorted(rng.choice(250, n, replace=False).tolist()), list(range(1, n + 1)), list(range(n))]
        g = torch.Generator().manual_seed(n)
        cfg, c = new_cache(W, g, 3, 1, 2, 128, 16, 20)
        want, table = [x.cpu().clone() for x in (c.k, c.v)], c.table.cpu()
        W.wnw_paged_keep(cfg, c, i32([30, 3, 11]), i32(paths))
        for b, base in enumerate([30, 3, 11]):
            for x in want:
                old = x.clone()
                for i in range(n):
                    src, dst = R.place(table, b, base + paths[b][i], 16, cfg.pages), R.place(table, b, base + i, 16, cfg.pages)
                    x[dst[0], :, :, dst[1]] = old[src[0], :, :, src[1]]
        assert torch.equal(c.k.cpu(), want[0]) and torch.equal(c.v.cpu(), want[1])


def test_keep_without_pages(W):
    log("[case] keep, entries without a page")
    check_keep(W, 128, 16, [14, 30], [[1, 3, 20, 33], [2, 9, 10, 19]], None, holes=[(0, 1), (1, 3)])


# ---- drafts ----------------------------------------------------------------------------------


@pytest.mark.parametrize("n", [1, 2, 7, 63, 64, 65, 128, 200, 511, 1024])
@pytest.mark.parametrize("kind", ["chain", "star", "random", "odd"])
def test_trees(W, n, kind):
    log(f"[case] tree n={n} {kind}")
    rng = np.random.default_rng(n)
    B = 3
    parents = [{"chain": [i - 1 for i in range(n)], "star": [-1] * n, "random": some_tree(rng, n),
                "odd": [int(rng.integers(-5, n + 5)) for _ in range(n)]}[kind] for _ in range(B)]
    counts = [n, n // 2, 0]
    base = [0, 1000000, 17]
    words = (n + 63) // 64
    mask, pos = torch.full((B, n, words), 5, dtype=torch.int64, device="cuda"), torch.full((B, n), -9, dtype=torch.int32, device="cuda")
    W.wnw_draft_tree(i32(parents), i32(base), mask, pos, i32(counts))
    only = torch.empty_like(pos)
    W.wnw_draft_tree(i32(parents), i32(base), None, only)
    for b in range(B):
        see = R.ancestors(parents[b])
        want, c = R.words(see), counts[b]
        assert torch.equal(mask[b, :c].cpu(), want[:c]) and (mask[b, c:] == 5).all()
        depth = see.sum(axis=1) - 1 + base[b]
        assert pos[b, :c].tolist() == depth[:c].tolist() and (pos[b, c:] == -9).all()
        assert only[b].tolist() == depth.tolist()


def run_verify(W, token, parent, count, target, draft, uniform):
    B, n = token.shape
    V = target.shape[2]
    path = torch.full((B, n), 99, dtype=torch.int32, device="cuda")
    acc, nxt = (torch.full((B,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.full((W.wnw_draft_verify_workspace(B, n, V),), 0xFF, dtype=torch.uint8, device="cuda")
    dev = lambda x, t: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()   # noqa: E731
    W.wnw_draft_verify(dev(token, torch.int32), dev(target, torch.float32), dev(uniform, torch.float32), path, acc, nxt,
                       draft_dev=dev(draft, torch.float32), parent_dev=dev(parent, torch.int32), count_dev=dev(count, torch.int32), workspace=ws)
    torch.cuda.synchronize()
    return path.cpu().tolist(), acc.tolist(), nxt.tolist()


def check_verify(W, token, parent, count, target, draft, uniform):
    got = run_verify(W, token, parent, count, target, draft, uniform)
    B, n = token.shape
    for b in range(B):
        path, nxt = R.verify(token[b].tolist(), None if parent is None else parent[b].tolist(), n if count is None else count[b],
                             target[b], None if draft is None else draft[b], uniform[b])
        assert got[0][b] == path + [-1] * (n - len(path)), (b, got[0][b], path)
        assert got[1][b] == len(path) and got[2][b] == nxt, (b, got[2][b], nxt)
    return got


def probabilities(rng, *shape, sharp=1.3):
    x = np.exp(sharp * rng.gumbel(size=shape))
    return (x / x.sum(axis=-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("V", [1, 2, 7, 100, 1023, 1024, 1025, 5000, 65536, 70001])
@pytest.mark.parametrize("n", [0, 1, 5, 40])
@pytest.mark.parametrize("with_draft", [False, True])
def test_verification(W, V, n, with_draft):
    log(f"[case] verify V={V} n={n} draft={with_draft}")
    rng = np.random.default_rng(V * 100 + n)
    B = 4
    target = probabilities(rng, B, n + 1, V)
    draft = probabilities(rng, B, n + 1, V, sharp=0.7) * 0.5 + target * 0.5 if with_draft else None
    draft = draft.astype(np.float32) if with_draft else None
    trees = [some_tree(rng, n) for _ in range(B - 1)] + [[-1] * n]
    for parent in (None, np.array(trees, dtype=np.int32).reshape(B, n)):
        p = [list(range(-1, n - 1))] * B if parent is None else trees
        src = draft if with_draft else target
        token = np.array([[int(rng.choice(V, p=src[b, p[b][i] + 1].astype(np.float64) / src[b, p[b][i] + 1].astype(np.float64).sum()))
                           for i in range(n)] for b in range(B)], dtype=np.int32).reshape(B, n)
        uniform = rng.random((B, n + 1)).astype(np.float32)
        check_verify(W, token, parent, None, target, draft, uniform)
        check_verify(W, token, parent, np.array([n, n // 2, 0, n], dtype=np.int32), target, draft, uniform * 0.2)


def test_verification_on_borders(W):
    """Every sibling refused, tokens outside the vocabulary, the same token twice, rows that are one token, nothing left, u = 0."""
    log("[case] verify, borders")
    V, n, B = 300, 12, 8
    rng = np.random.default_rng(9)
    target = probabilities(rng, B, n + 1, V)
    draft = probabilities(rng, B, n + 1, V)
    parent = np.full((B, n), -1, dtype=np.int32)
    token = np.array([rng.choice(V, n) for _ in range(B)], dtype=np.int32)
    uniform = np.full((B, n + 1), 0.999999, dtype=np.float32)
    uniform[:, n] = [0, 0.25, 0.5, 0.75, 0.999999, 0.1, 0.9, 0.3]
    token[1] = [-1, V, 2147483647, -2147483648] * 3
    token[2] = 5
    target[3] = 0
    target[3, :, 17] = 1          # greedy
    token[3, 4] = 17
    draft[4] = target[4]          # the draft is the target: the first token stands, and nothing is left where it does not
    uniform[4, :n] = 1.5
    target[5] = 0                 # no row at all
    uniform[6, :n] = 0
    target[7, :, ::2] = 0
    target[7] /= target[7].sum(axis=-1, keepdims=True)
    got = check_verify(W, token, parent, None, target, draft, uniform)
    assert got[1][3] >= 1 and got[0][3][0] == 4 and got[2][5] == -1 and got[2][3] == 17
    got = check_verify(W, token, parent, None, target, None, uniform)
    assert got[2][5] == -1


def test_verification_of_numbers_that_are_no_probabilities(W):
    log("[case] verify, inf and NaN")
    V, B = 2000, 3
    rng = np.random.default_rng(2)
    target = probabilities(rng, B, 2, V)
    target[0, 0, 1500] = math.inf
    target[1, 0, 3] = math.nan          # counts as 0
    target[2, 0] = -target[2, 0]
    _, acc, nxt = run_verify(W, np.full((B, 1), 3, dtype=np.int32), None, None, target, None, np.full((B, 2), 0.5, dtype=np.float32))
    assert acc == [0, 0, 0] or acc == [int(0.5 < target[0, 0, 3]), 0, 0]
    assert nxt[0] == -1 and nxt[2] == -1
    p = np.nan_to_num(target[1, 0].astype(np.float64))
    assert nxt[1] == int(np.nonzero(p.cumsum() > 0.5 * p.sum())[0][0])


# ---- together --------------------------------------------------------------------------------


@pytest.mark.parametrize("graphed", [False, True])
def test_drafted_decoding_is_decoding(W, graphed):
    """Steps of tree, append, attention, verification and keeping, and the same tokens one at a time: the caches agree bit for bit, and
    the outputs of the tokens that stood within the sum of both sides' bounds.  What a token's vectors are is a table."""
    log(f"[case] drafted decoding, graphed={graphed}")
    B, L, H, G, D, page, n, V = 2, 2, 2, 2, 128, 16, 9, 50
    g = torch.Generator().manual_seed(8)
    rng = np.random.default_rng(8)
    emb = [rows(g, V, L, h, D).cuda() for h in (H, H, H * G)]
    rot = W.make_rotary(torch.from_numpy(W.wnw_rotary_frequencies(D, 1e4)).cuda(), D)
    cfg, c = new_cache(W, g, B, L, H, D, page, 8)
    _, one = new_cache(W, g, B, L, H, D, page, 8)
    one.table.copy_(c.table)
    text = [[3, 1, 4, 1, 5], [9, 2, 6]]
    vectors = lambda toks: [e[toks].permute(0, 2, 3, 1, 4).contiguous() for e in emb]     # [B][n] -> [B][L][heads][n][D]  # noqa: E731
    first = torch.tensor([t + [0] * (5 - len(t)) for t in text], device="cuda")
    for cache in (c, one):
        k, v, _ = vectors(first)
        W.wnw_paged_append(cfg, cache, k, v, i32([0, 0]), i32([5, 3]), rotary=rot)
    base = i32([5, 3])
    token, parent = torch.zeros((B, n), dtype=torch.int64, device="cuda"), torch.zeros((B, n), dtype=torch.int32, device="cuda")
    mask, position = torch.zeros((B, n, 1), dtype=torch.int64, device="cuda"), torch.zeros((B, n), dtype=torch.int32, device="cuda")
    k, v, q = vectors(token)
    out, q_out, total = torch.zeros((B, L, H * G, n, D), device="cuda"), torch.zeros_like(q), torch.zeros_like(base)
    ws = torch.zeros(max(16, W.wnw_paged_attend_workspace(cfg, L, H * G, n)), dtype=torch.uint8, device="cuda")
    target, uniform = torch.zeros((B, n + 1, V), device="cuda"), torch.zeros((B, n + 1), device="cuda")
    path, acc, nxt = torch.zeros_like(parent), torch.zeros_like(base), torch.zeros_like(base)
    ws2 = torch.zeros(W.wnw_draft_verify_workspace(B, n, V), dtype=torch.uint8, device="cuda")
    short = torch.zeros((B, n), dtype=torch.int32, device="cuda")

    def step():
        W.wnw_draft_tree(parent, base, mask, position)
        W.wnw_paged_append(cfg, c, k, v, base, q_dev=q, q_out=q_out, rotary=rot, position_dev=position)
        total.copy_(base + n)
        W.wnw_paged_attend(cfg, c, q_out, out, total, mask_dev=mask, workspace=ws)
        short.copy_(token)
        W.wnw_draft_verify(short, target, uniform, path, acc, nxt, parent_dev=parent, workspace=ws2)
        W.wnw_paged_keep(cfg, c, base, path, acc)
        base.add_(acc)

    graph = None
    if graphed:
        saved = [x.clone() for x in (c.k, c.v, base)]
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for x, y in zip((c.k, c.v, base), saved):
            x.copy_(y)
        with torch.cuda.graph(graph):
            step()
        torch.cuda.synchronize()
    stood = 0
    for turn in range(6):
        trees = [some_tree(rng, n) for _ in range(B)]
        toks = rng.integers(0, V, (B, n))
        parent.copy_(i32(trees))
        token.copy_(torch.from_numpy(toks))
        for x, y in zip((k, v, q), vectors(token)):
            x.copy_(y)
        t = probabilities(rng, B, n + 1, V, sharp=0.1)
        for b in range(B):                       # the target likes a child of every node that has one
            for i, p in enumerate(trees[b]):
                t[b, p + 1] *= 0.5
                t[b, p + 1, toks[b, i]] += 0.5
        t /= t.sum(axis=-1, keepdims=True)
        target.copy_(torch.from_numpy(t))
        u = rng.random((B, n + 1)).astype(np.float32)
        uniform.copy_(torch.from_numpy(u))
        before = base.tolist()
        graph.replay() if graphed else step()
        torch.cuda.synchronize()
        for b in range(B):
            want, after = R.verify(toks[b].tolist(), trees[b], n, t[b].astype(np.float32), None, u[b])
            m = acc.tolist()[b]
            assert path[b, :m].tolist() == want and m == len(want) and nxt.tolist()[b] == after and base.tolist()[b] == before[b] + m
            stood += m
            for j, node in enumerate(want):      # one at a time
                at = [before[0], before[1]]
                at[b] += j
                k1, v1, q1 = vectors(torch.from_numpy(toks[:, [node]]).cuda())
                only = [0, 0]
                only[b] = 1
                turned = torch.zeros_like(q1)
                W.wnw_paged_append(cfg, one, k1, v1, i32(at), i32(only), q_dev=q1, q_out=turned, rotary=rot)
                lens = [at[0], at[1]]
                lens[b] += 1
                single, _ = run_attend(W, cfg, one, turned, lens, only)
                ref = R.attend(turned.cpu(), one.k.cpu(), one.v.cpu(), one.table.cpu(), page, lens, only)
                _, werr = logit_bound(D, ref[3][b, :, :, 0], 0)
                bound = 2 * (werr + ref[4][b, :, :, 0] * EPS + 4 * EPS).unsqueeze(-1) * ref[2][b, :, :, 0]
                assert ((single[b, :, :, 0] - out[b, :, :, node]).abs().cpu() <= bound).all(), (turn, b, j)
    assert stood >= 6
    table = c.table.cpu()
    for b, rows_there in enumerate(base.tolist()):
        for r in range(rows_there):
            p, o = R.place(table, b, r, page, cfg.pages)
            assert torch.equal(c.k[p, :, :, o], one.k[p, :, :, o]) and torch.equal(c.v[p, :, :, o], one.v[p, :, :, o]), (b, r)
