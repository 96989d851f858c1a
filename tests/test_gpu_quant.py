"""GPU tests of the 8-bit cache (wnw_quant_write, wnw_quant_read, wnw_quant_attend) against the same
arithmetic in 64 bits on the CPU (quant_reference.py).  Bytes and scales have to be equal.

Attention's tolerances, from the arithmetic: products of bytes and bf16 queries are exact in fp32 and d of them are
summed, so a base-2 logit is off by at most (d + 3) 2^-24 sum|q k| / sqrt(d) log2(e) with its two scalings and the
subtraction of the maximum (both at most twice that magnitude); a weight by ln 2 times that, its exponential by 2^-22, and the
denominator alike.  The weight is rounded to 2^-22 of itself (two fp16) or 2^-11 (one, half a step: 2^-12),
and T products are summed in fp32 (T 2^-24 at worst, taken with the joins).  bf16 outputs add half a step, 2^-8.
fp16 ends at 2^-24, where a weight of 1 in the block of the largest V scale seen, below 2^e, stands at up to 2^15: each weight
is off by up to 2^-25 there, which is 2^-40 2^e times its number in the output, where 2^e times a number is at most twice the
largest |v|: 2^-39 |v|max for each row seen.  With more than 32 query rows on a KV-head the maximum that weights are relative to lags
by up to 2^8, so that a weight of 1 stands at 2^7 or more: 2^-31 |v|max.
"""
import math

import numpy as np
import pytest
import torch

from tests import quant_reference as R
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


def rows(seed, *shape, spread=1.0):
    """bf16 rows whose sizes vary by row."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn((*shape[:-1], 1), generator=g))
    return x.bfloat16()


def new_cache(W, cfg, fill=0xA5):
    c = W.make_quant_cache(cfg)
    c.k.fill_(fill)
    c.v.fill_(fill)
    c.k_scale.fill_(-7.0)
    c.v_scale.fill_(-7.0)
    return c


def check_cache(c, refs, written, fmt):
    """Bytes of written rows and scales of their blocks equal the reference's; the others are as they were."""
    for got, scale, ref in ((R.decode_k(c.k, fmt), c.k_scale, refs[0]), (R.decode_v(c.v, fmt), c.v_scale, refs[1])):
        untouched = R.numbers(fmt)[0xA5]
        s = scale.cpu().numpy()
        blocks = written.reshape(*written.shape[:-1], -1, ref.block).any(axis=-1)
        assert np.array_equal(s[blocks], ref.scale[blocks].astype(np.float32), equal_nan=True)
        assert (s[~blocks] == -7.0).all()
        live = written & ~np.isnan(np.repeat(ref.scale, ref.block, axis=-1))
        assert np.array_equal(got[live], ref.num[live])
        assert (got[~written] == untouched).all()


# (rows of the sequences, tokens written next), one entry per call
WRITES = [
    [([0, 0], [1, 64])],
    [([0, 0], [63, 65]), ([63, 65], [1, 63]), ([64, 128], [64, 1])],
    [([0, 0], [130, 7]), ([130, 7], [0, 20]), ([130, 27], [5, 5]), ([100, 3], [3, 0])],
    [([0, 0], [190, 192]), ([190, -5], [10, 4]), ([191, 189], [9, 9]), ([-5, 300], [4, 4])],
]


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("block,D", [(16, 128), (32, 64), (64, 128), (32, 128), (64, 64)])
@pytest.mark.parametrize("which", range(len(WRITES)))
def test_writes(W, fmt, block, D, which):
    log(f"[case] quant write fmt={fmt} block={block} d={D} calls={WRITES[which]}")
    B, L, H, cap = 2, 2, 3, 192
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    written = np.zeros((B, L, H, cap), dtype=bool)
    for call, (pos, count) in enumerate(WRITES[which]):
        n = max(count)
        x = [rows(1000 * which + 10 * call + j, B, L, H, n, D) for j in range(2)]
        W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32(pos), i32(count))
        for ref, t in zip(refs, x):
            ref.write(t.double().numpy(), pos, count)
        for b in range(B):
            p = min(max(pos[b], 0), cap)
            if count[b] and p < cap:
                written[b, ..., p: min(p + count[b], cap)] = True
    torch.cuda.synchronize()
    check_cache(c, refs, written, fmt)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("block,D", [(16, 64), (32, 128), (64, 128)])
@pytest.mark.parametrize("n", [2, 5, 13, 16, 17])
def test_a_few_rows_at_a_time(W, fmt, block, D, n):
    """Up to n rows per call and sequence, across every boundary, until the cache is full; sizes that make scales grow."""
    log(f"[case] quant write, {n} rows at a time, fmt={fmt} block={block} d={D}")
    B, L, H, cap = 3, 1, 3, 192
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    g = np.random.default_rng(n)
    pos = [0, 0, 0]
    written = np.zeros((B, L, H, cap), dtype=bool)
    call = 0
    while min(pos) < cap:
        count = [int(k) for k in g.integers(0, n + 1, B)]
        x = [rows(100 * call + j, B, L, H, n, D, spread=2.0) for j in range(2)]
        W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32(pos), i32(count))
        for ref, t in zip(refs, x):
            ref.write(t.double().numpy(), pos, count)
        for b in range(B):
            written[b, ..., pos[b]: pos[b] + count[b]] = True
            pos[b] += count[b]
        call += 1
    torch.cuda.synchronize()
    check_cache(c, refs, written, fmt)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 3, 20])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_writes_that_are_not_finite(W, fmt, n, bad):
    """A block with such a row has the scale NaN, keeps it as rows join, and loses it when it is begun anew."""
    log(f"[case] quant write, not finite, fmt={fmt} n={n} {bad}")
    B, L, H, cap, D, block = 1, 1, 2, 128, 64, 32
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    written = np.zeros((B, L, H, cap), dtype=bool)
    # the bad value in head 1's K of the second call and V of the third; the last call begins the first block anew
    for call, pos in enumerate((0, n, 2 * n, 3 * n, 0)):
        x = [rows(10 * call + j, B, L, H, n, D) for j in range(2)]
        if call in (1, 2):
            x[call - 1][0, 0, 1, n - 1, 5] = bad
        W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32([pos]))
        for ref, t in zip(refs, x):
            ref.write(t.double().numpy(), [pos], [n])
        written[..., pos: pos + n] = True
        torch.cuda.synchronize()
        check_cache(c, refs, written, fmt)
    assert not np.isnan(refs[0].scale[..., 0]).any()


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("block", [16, 64])
def test_rows_one_by_one(W, fmt, block):
    """A row per call, of growing and shrinking sizes: a block's rows are rounded again as its scale grows."""
    log(f"[case] quant write, row by row, fmt={fmt} block={block}")
    B, L, H, cap, D, n = 1, 1, 2, 128, 128, 70
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    x = [rows(7 + j, B, L, H, n, D, spread=2.0) for j in range(2)]
    for i in range(n):
        W.wnw_quant_write(cfg, c, *(t[..., i: i + 1, :].contiguous().cuda() for t in x), i32([i]))
        for ref, t in zip(refs, x):
            ref.write(t[..., i: i + 1, :].double().numpy(), [i], [1])
    written = np.zeros((B, L, H, cap), dtype=bool)
    written[..., :n] = True
    torch.cuda.synchronize()
    check_cache(c, refs, written, fmt)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
def test_values_at_the_edges(W, fmt):
    """Ties, zeros, subnormals, the largest numbers, infinities and NaN."""
    log(f"[case] quant write, edges, fmt={fmt}")
    B, L, H, cap, D, block = 1, 1, 1, 64 * 6, 64, 64
    x = torch.zeros((B, L, H, cap, D))
    x[0, 0, 0, 0] = torch.arange(64) - 31.5                              # ties under the next row's scale
    x[0, 0, 0, 1, 0] = 127.0 if fmt == R.INT8 else 448.0
    x[0, 0, 0, 2] = (torch.arange(64) + 0.5) * (1.0 if fmt == R.INT8 else 2.0 ** -9)
    x[0, 0, 0, 3] = (torch.arange(64) + 64.0) * (1.0 if fmt == R.INT8 else 3.5)
    x[0, 0, 0, 64] = torch.linspace(-1, 1, 64) * 2.0 ** -120             # under the smallest scale
    x[0, 0, 0, 65, :2] = torch.tensor([2.0 ** -133, -0.0])
    x[0, 0, 0, 128] = torch.linspace(-1, 1, 64) * 3.3895e38               # near the largest bf16
    x[0, 0, 0, 192 + 5, 3] = math.inf
    x[0, 0, 0, 192 + 6] = 1.0
    x[0, 0, 0, 256 + 5, 3] = math.nan
    x[0, 0, 0, 256 + 60, 3] = 5.0
    x = x.bfloat16()
    y = -x
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    W.wnw_quant_write(cfg, c, x.cuda(), y.cuda(), i32([0]))
    # a NaN stays in its block when more rows come, and goes when the block is begun anew
    z = torch.ones((B, L, H, 3, D)).bfloat16()
    W.wnw_quant_write(cfg, c, z.cuda(), z.cuda(), i32([192 + 61]))
    W.wnw_quant_write(cfg, c, z.cuda(), z.cuda(), i32([256]))
    for ref, t in zip(refs, (x, y)):
        ref.write(t.double().numpy(), [0], [cap])
        ref.write(z.double().numpy(), [192 + 61], [3])
        ref.write(z.double().numpy(), [256], [3])
    torch.cuda.synchronize()
    check_cache(c, refs, np.ones((B, L, H, cap), dtype=bool), fmt)
    ko = torch.empty((B, L, H, cap, D), device="cuda")
    W.wnw_quant_read(cfg, c, ko, None, i32([0]))
    with np.errstate(invalid="ignore", over="ignore"):
        want = refs[0].values().astype(np.float32)
    got = ko.cpu().numpy()
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[0, 0, 0, 192:256]).all() and np.isfinite(got[0, 0, 0, 256:]).all()


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_read(W, fmt, bf16, D):
    log(f"[case] quant read fmt={fmt} bf16={bf16} d={D}")
    B, L, H, cap, block, n = 3, 2, 2, 256, 32, 150
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    c = new_cache(W, cfg)
    x = [rows(30 + j, B, L, H, cap, D) for j in range(2)]
    W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32([0] * B))
    refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
    for ref, t in zip(refs, x):
        ref.write(t.double().numpy(), [0] * B, [cap] * B)
    kind = torch.bfloat16 if bf16 else torch.float32
    pos, count = [0, 37, 200], [150, 0, 140]
    for layer, nl in ((0, 2), (1, 1)):
        for parts in ((True, True), (True, False), (False, True)):
            outs = [torch.full((B, nl, H, n, D), 3.0, dtype=kind, device="cuda") if p else None for p in parts]
            W.wnw_quant_read(cfg, c, *outs, i32(pos), i32(count), first_layer=layer)
            for o, ref in zip(outs, refs):
                if o is None:
                    continue
                want = torch.full((B, nl, H, n, D), 3.0, dtype=kind)
                vals = torch.from_numpy(ref.values())[:, layer: layer + nl]
                for b in range(B):
                    m = min(count[b], cap - pos[b])
                    want[b, :, :, :m] = vals[b, :, :, pos[b]: pos[b] + m].float().to(kind)
                assert torch.equal(o.cpu(), want)


def filled(W, cfg, lens, fmt, seed, garbage=True, scale_spread=0.5):
    """A cache of random rows: numbers in 64 bits, and device buffers in which everything behind the
    sequences' last rows is garbage (NaN scales, 0xFF bytes)."""
    B, L, H, cap, D, block = cfg.batch, cfg.layers, cfg.kv_heads, cfg.capacity, cfg.head_dim, cfg.block
    c = W.make_quant_cache(cfg)
    vals = []
    for j, (to, scale) in enumerate(((c.k, c.k_scale), (c.v, c.v_scale))):
        x = rows(seed + j, B, L, H, cap, D, spread=scale_spread).double().numpy()
        amax = np.abs(x).reshape(B, L, H, -1, block, D).max(axis=(4, 5))
        s = np.vectorize(lambda a: R.scale_of(a, fmt))(amax)
        num = R.round_to(x, np.repeat(s, block, axis=3)[..., None], fmt)
        vals.append(torch.from_numpy(num * np.repeat(s, block, axis=3)[..., None]))
        code, s = R.encode(num, fmt), torch.from_numpy(s.astype(np.float32))
        if garbage:
            for b in range(B):
                code[b, :, :, lens[b]:] = 0xFF
                s[b, :, :, -(-lens[b] // block):] = math.nan
        (to.copy_(code) if j == 0 else to.copy_(R.k_to_v(code)))
        scale.copy_(s)
    return c, vals


def bound(D, lens, absv, absq, sumv, bf16, H):
    """See the module's head: the bound of an output element, and of a logarithm and a mass (relative)."""
    logit = 4 * (D + 3) * EPS * absq + 8 * EPS
    T = max(lens) + 64
    rel = 2 * logit + 2.0 ** -21 + T * EPS
    floor = 2.0 ** (-31 if absq.shape[2] // H * absq.shape[3] > 32 else -39)
    out = absv * (rel + (2.0 ** -11 if bf16 else 2.0 ** -22)).unsqueeze(-1) + floor * sumv.unsqueeze(-1)
    return out, logit + 2.0 ** -21 + T * EPS, rel


def run_attend(W, cfg, c, q, lens, counts, mass=True, max_len=0, first_layer=0, count_dev=True):
    B, nl, Hq, n, D = q.shape
    kind = torch.bfloat16 if cfg.flags & W.WNW_F_OUT_BF16 else torch.float32
    out = torch.full(q.shape, 9.0, dtype=kind, device="cuda")
    lse = torch.full(q.shape[:-1], 9.0, device="cuda")
    m = torch.full((B, nl, Hq, cfg.capacity // cfg.block), 9.0, device="cuda") if mass and n == 1 else None
    ws = torch.full((W.wnw_quant_attend_workspace(cfg, nl, Hq, n, max_len=max_len),), 0xFF, dtype=torch.uint8, device="cuda")
    W.wnw_quant_attend(cfg, c, q.cuda(), out, i32(lens), i32(counts) if count_dev else None, lse, m, ws, max_len=max_len,
                       first_layer=first_layer)
    torch.cuda.synchronize()
    return out, lse, m


def check_attend(got, want, lens, counts, D, bf16, H):
    out, lse, mass = got
    w_out, w_lse, w_mass, absv, absq, sumv = want
    b_out, b_lse, b_mass = bound(D, lens, absv, absq, sumv, bf16, H)
    for b in range(out.shape[0]):
        c = min(max(counts[b], 0), out.shape[3])
        o, l = out[b, :, :, :c].double().cpu(), lse[b, :, :, :c].double().cpu()
        wo, wl = w_out[b, :, :, :c], w_lse[b, :, :, :c]
        tol = b_out[b, :, :, :c] + (2.0 ** -8 * wo.abs() if bf16 else 0.0)
        assert torch.equal(torch.isnan(o), torch.isnan(wo)), b
        assert bool(((o - wo).abs() <= tol)[~torch.isnan(wo)].all()), (b, float(((o - wo).abs() - tol).max()))
        fine = torch.isfinite(wl)
        assert torch.equal(l[~fine], wl[~fine]) or torch.isnan(wl[~fine]).any(), b
        assert bool(((l - wl).abs() <= b_lse[b, :, :, :c] + 4 * EPS * wl.abs())[fine].all()), b
        assert bool((out[b, :, :, c:] == 9.0).all()) and bool((lse[b, :, :, c:] == 9.0).all())
        if mass is None:
            continue
        if c == 0:
            assert bool((mass[b] == 9.0).all())
            continue
        m, wm = mass[b].double().cpu(), w_mass[b, :, :, 0]
        assert torch.equal(torch.isnan(m), torch.isnan(wm))
        # a NaN query has no bound: its blocks without rows, the only ones that are not NaN, have to be 0
        assert bool(((m - wm).abs() <= wm * b_mass[b, :, :, :1].nan_to_num(0.0) + 1e-37)[~torch.isnan(wm)].all()), b


# lens, tokens a call, counts, KV heads, group, block, d
SHAPES = [
    ([1, 2, 63, 64], 1, [1, 1, 1, 1], 2, 4, 32, 128),
    ([0, 65, 128, 1], 1, [1, 1, 0, 1], 2, 1, 16, 128),
    ([1000, 127, 129, 500], 1, [1, 1, 1, 1], 1, 3, 64, 64),
    ([2500], 1, [1], 1, 16, 16, 128),
    ([700], 1, [1], 1, 20, 32, 64),
    ([700, 3], 1, [1, 1], 2, 5, 64, 128),
    ([333, 70, 0], 1, [1, 1, 1], 1, 40, 32, 64),
    ([500], 1, [1], 2, 71, 16, 128),
    ([300, 2, 64, 0], 4, [4, 2, 3, 4], 2, 2, 32, 128),
    ([515, 80], 5, [5, 3], 1, 8, 64, 128),
    ([200, 17], 17, [17, 17], 2, 3, 16, 64),
    ([333, 64], 64, [64, 50], 1, 2, 32, 128),
    ([300, 130], 130, [129, 130], 1, 4, 64, 128),
    ([130, 90], 130, [130, 130], 1, 2, 16, 128),
    ([1500, 3], 40, [40, 2], 1, 7, 32, 64),
    ([70, 32, 33], 11, [11, 11, 3], 2, 3, 16, 128),
]


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"len{s[0][0]}_n{s[1]}_g{s[4]}_blk{s[5]}_d{s[6]}")
def test_attend(W, fmt, bf16, shape):
    lens, n, counts, H, G, block, D = shape
    log(f"[case] quant attend fmt={fmt} bf16={bf16} {shape}")
    B, L = len(lens), 2
    cap = (max(lens) + 63) // 64 * 64 + 64
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    c, (k, v) = filled(W, cfg, lens, fmt, 50)
    q = rows(70, B, L, H * G, n, D, spread=0.3)
    want = R.attend(q.double(), k, v, lens, counts, block)
    check_attend(run_attend(W, cfg, c, q, lens, counts), want, lens, counts, D, bf16, H)
    if n == 1:     # without masses, and with a bound of the lengths that does not hold
        check_attend(run_attend(W, cfg, c, q, lens, counts, mass=False), want, lens, counts, D, bf16, H)
        check_attend(run_attend(W, cfg, c, q, lens, counts, max_len=1), want, lens, counts, D, bf16, H)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 33])
def test_attend_split_cache(W, fmt, n):
    """One sequence and few heads over a long cache: the parts are joined."""
    log(f"[case] quant attend, split, fmt={fmt} n={n}")
    lens, H, G, block, D = [9001], 1, 2, 64, 128
    cfg = W.make_quant_config(1, 1, H, 9088, block, fmt, head_dim=D)
    c, (k, v) = filled(W, cfg, lens, fmt, 90)
    q = rows(91, 1, 1, H * G, n, D)
    want = R.attend(q.double(), k, v, lens, [n], block)
    check_attend(run_attend(W, cfg, c, q, lens, [n], count_dev=False), want, lens, [n], D, False, H)


@pytest.mark.parametrize("n", [1, 4, 70])
def test_lengths_and_counts_outside(W, n):
    """Lengths and counts outside their ranges count as the nearer end."""
    log(f"[case] quant attend, lengths outside, n={n}")
    H, G, block, D, cap = 2, 2, 32, 64, 192
    cfg = W.make_quant_config(4, 1, H, cap, block, R.INT8, head_dim=D)
    c, _ = filled(W, cfg, [cap] * 4, R.INT8, 21, garbage=False)
    q = rows(22, 4, 1, H * G, n, D)
    got = run_attend(W, cfg, c, q, [-7, cap + 1, 2**31 - 1, 50], [n, n, n + 9, -2])
    want = run_attend(W, cfg, c, q, [0, cap, cap, 50], [n, n, n, 0])
    for a, b in zip(got, want):
        assert a is b is None or torch.equal(a, b)


# How a call is shared out depends on its blocks of query rows and their tiles: a work-group per block, even pieces that
# are joined, or equal parts of all tiles in a line.  (lens, n, counts, layers, KV heads, group, block, d)
SHARED = {
    "token, a block each": ([900, 0, 64, 333], 1, None, 6, 8, 4, 32, 128),
    "token, a block each, d = 64": ([960, 577, 0], 1, None, 4, 8, 4, 32, 64),
    "token, a block each, streamed": ([9000], 1, None, 30, 8, 4, 16, 64),
    "token, many blocks": ([500, 30, 0, 449, 512], 1, None, 8, 8, 3, 16, 128),
    "token, pieces": ([5000, 63, 4097], 1, None, 2, 3, 2, 16, 128),
    "token, pieces, many sequences": ([3000 - 23 * b if b % 7 else b for b in range(130)], 1, None, 1, 1, 2, 64, 128),
    "token, pieces, 37 q-heads": ([5000, 63], 1, None, 1, 1, 37, 64, 128),
    "token, a line": ([10240, 10000], 1, None, 5, 17, 3, 64, 128),
    "token, a line, d = 64": ([36000, 35999], 1, None, 7, 10, 1, 32, 64),
    "32 rows, pieces": ([4000, 700], 6, [6, 5], 2, 3, 4, 64, 128),
    "32 rows, a block each": ([400, 70, 3], 6, [6, 5, 3], 10, 8, 5, 16, 64),
    "32 rows, a block each, many tiles": ([700, 130, 65], 6, [6, 5, 3], 10, 8, 5, 16, 64),
    "32 rows, a block each, d = 128": ([640, 129], 5, [5, 2], 8, 8, 4, 64, 128),
    "32 rows, a block each, streamed": ([4500], 5, [5], 30, 8, 4, 64, 128),
    "many rows, pieces": ([2000, 900], 50, [50, 33], 2, 2, 3, 16, 128),
    "64 rows, pieces": ([3000, 700], 12, [12, 7], 2, 2, 4, 64, 128),
    "64 rows, a line": ([700], 41, [41], 20, 30, 1, 32, 64),
    "64 rows, a block each": ([200, 130, 33, 0], 16, [16, 9, 16, 4], 4, 8, 4, 32, 128),
    "many rows, a line": ([700], 90, [90], 20, 30, 1, 32, 64),
    "many rows, a block each": ([200, 130], 140, [140, 100], 2, 2, 5, 32, 128),
}


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("name", SHARED)
def test_attend_shared_out(W, fmt, bf16, name):
    lens, n, counts, L, H, G, block, D = SHARED[name]
    log(f"[case] quant attend, {name}, fmt={fmt} bf16={bf16}")
    B = len(lens)
    counts = counts or [1] * B
    cap = (max(lens) + 63) // 64 * 64 + 64
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    g = torch.Generator(device="cuda").manual_seed(17)
    c = W.make_quant_cache(cfg)
    number = torch.from_numpy(np.nan_to_num(R.numbers(fmt))).cuda()
    vals = []
    for to, scale, is_v in ((c.k, c.k_scale, False), (c.v, c.v_scale, True)):
        code = torch.randint(1, 256, (B, L, H, cap, D), generator=g, device="cuda", dtype=torch.uint8)
        if fmt == R.E4M3:
            code = torch.where((code & 127) == 127, 0, code)
        mean = float(number[code.int()[0, 0, 0]].abs().mean())
        s = torch.exp(0.5 * torch.randn(scale.shape, generator=g, device="cuda")) / mean
        if not is_v:
            s *= 0.5
        vals.append(number[code.int()] * s.double().repeat_interleave(block, dim=3).unsqueeze(-1))
        for b in range(B):
            code[b, :, :, lens[b]:] = 0xFF
            s[b, :, :, -(-lens[b] // block):] = math.nan
        to.copy_(R.k_to_v(code) if is_v else code)
        scale.copy_(s)
        del code
    q = rows(18, B, L, H * G, n, D, spread=0.3).cuda()
    want = tuple(t.cpu() for t in R.attend_fast(q.double(), *vals, lens, counts, block))
    del vals
    check_attend(run_attend(W, cfg, c, q, lens, counts), want, lens, counts, D, bf16, H)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 9, 70])
def test_attend_poisoned_block(W, fmt, n):
    """A block whose scale is NaN: tokens that see one of its rows get NaN, the others nothing of it."""
    log(f"[case] quant attend, NaN block, fmt={fmt} n={n}")
    H, G, block, D, T = 1, 3, 16, 64, 170
    for bad in (T - n, 40, T - 1):
        for which in (0, 1):
            cfg = W.make_quant_config(1, 1, H, 192, block, fmt, head_dim=D)
            c, vals = filled(W, cfg, [T], fmt, 11)
            j = bad // block
            (c.k_scale, c.v_scale)[which][..., j] = math.nan
            vals[which][..., j * block: (j + 1) * block, :] = math.nan
            q = rows(12, 1, 1, H * G, n, D)
            got = run_attend(W, cfg, c, q, [T], [n])
            want = R.attend(q.double(), *vals, [T], [n], block)
            out, w = got[0].cpu(), want[0]
            assert torch.equal(torch.isnan(out), torch.isnan(w)), (bad, which)
            tol = bound(D, [T], *want[3:], False, H)[0]
            assert bool(((out - w).abs() <= tol)[~torch.isnan(w)].all()), (bad, which)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 40])
def test_attend_scales_and_queries_of_any_size(W, fmt, n):
    """V scales from 2^-40 to 2^40 in either order, queries from subnormal to huge, zero and NaN queries."""
    log(f"[case] quant attend, magnitudes, fmt={fmt} n={n}")
    H, G, block, D, T = 1, 4, 32, 128, 330
    cfg = W.make_quant_config(2, 1, H, 384, block, fmt, head_dim=D)
    c, (k, v) = filled(W, cfg, [T, T], fmt, 21)
    f = torch.pow(2.0, torch.linspace(-40, 40, 384 // block).round())
    f = torch.stack([f, f.flip(0)])[:, None, None]
    c.v_scale *= f.cuda()
    v *= f.repeat_interleave(block, dim=-1).unsqueeze(-1).double()
    q = rows(22, 2, 1, H * G, n, D)
    q[0, 0, 0] = 0.0
    q[0, 0, 1] *= 2.0 ** -130
    q[0, 0, 2] *= 8.0
    q[1, 0, 3, n - 1, 5] = math.nan
    want = R.attend(q.double(), k, v, [T, T], [n, n], block)
    check_attend(run_attend(W, cfg, c, q, [T, T], [n, n]), want, [T, T], [n, n], D, False, H)


def test_layers_one_by_one(W):
    """A model's way through the layers gives the bits of one call over all of them."""
    log("[case] quant, layer by layer")
    B, L, H, G, cap, D, n = 2, 3, 2, 2, 128, 128, 70
    cfg = W.make_quant_config(B, L, H, cap, 32, W.WNW_QUANT_INT8, head_dim=D)
    x = [rows(5 + j, B, L, H, n, D).cuda() for j in range(2)]
    q = rows(9, B, L, H * G, 1, D).cuda()
    a, b = new_cache(W, cfg), new_cache(W, cfg)
    W.wnw_quant_write(cfg, a, *x, i32([0, 20]))
    whole = run_attend(W, cfg, a, q, [70, 90], [1, 1])
    for l in range(L):
        W.wnw_quant_write(cfg, b, *(t[:, l: l + 1].contiguous() for t in x), i32([0, 20]), first_layer=l)
    torch.cuda.synchronize()
    for s, t in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        assert torch.equal(s, t)
    for l in range(L):
        one = run_attend(W, cfg, b, q[:, l: l + 1].contiguous(), [70, 90], [1, 1], first_layer=l)
        want = [t[:, l: l + 1] for t in whole]
        for s, t in zip(one, want):
            assert float((s - t)[~torch.isnan(t)].abs().max()) <= 1e-5      # parts may be cut elsewhere


def test_generation(W):
    """A prompt is written, then tokens one by one, each attending to everything so far, eagerly and as a
    captured step whose lengths move on the device; a draft of three tokens is taken back."""
    log("[case] quant, a prompt and generated tokens")
    B, L, H, G, cap, D, block = 2, 2, 2, 3, 320, 128, 32
    for fmt in (W.WNW_QUANT_INT8, W.WNW_QUANT_E4M3):
        cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
        prompt = [200, 61]
        x = [rows(40 + j, B, L, H, 200, D) for j in range(2)]
        steps = 24
        new = [rows(60 + j, steps, B, L, H, 1, D) for j in range(2)]
        q = rows(80, steps, B, L, H * G, 1, D)

        def fresh():
            c = new_cache(W, cfg)
            W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32([0, 0]), i32(prompt))
            return c
        eager, graphed = fresh(), fresh()
        length = i32(prompt)
        ws = torch.empty(W.wnw_quant_attend_workspace(cfg, L, H * G, 1), dtype=torch.uint8, device="cuda")
        bufs = [torch.empty_like(t[0], device="cuda") for t in (*new, q)]
        outs = [[torch.zeros((B, L, H * G, 1, D), device="cuda"), torch.zeros((B, L, H * G, 1), device="cuda"),
                 torch.zeros((B, L, H * G, cap // block), device="cuda")] for _ in range(2)]

        def step(c, out, length):
            W.wnw_quant_write(cfg, c, bufs[0], bufs[1], length)
            length += 1
            W.wnw_quant_attend(cfg, c, bufs[2], out[0], length, None, out[1], out[2], ws)
        # warm-up on a cache of its own, then the capture
        step(fresh(), outs[0], i32(prompt))
        glen = i32(prompt)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(graphed, outs[1], glen)
        refs = [R.Cache(B, L, H, cap, D, block, fmt) for _ in range(2)]
        for ref, t in zip(refs, x):
            ref.write(t.double().numpy(), [0, 0], prompt)
        for s in range(steps):
            for buf, t in zip(bufs, (*new, q)):
                buf.copy_(t[s])
            step(eager, outs[0], length)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(*outs):
                assert torch.equal(a, b), s
            lens = [p + s for p in prompt]
            for ref, t in zip(refs, new):
                ref.write(t[s].double().numpy(), lens, [1, 1])
            lens = [p + 1 for p in lens]
            want = R.attend(q[s].double(), *(torch.from_numpy(np.nan_to_num(r.values())) for r in refs), lens, [1, 1], block)
            check_attend(outs[0], want, lens, [1, 1], D, False, H)
        # three tokens are written as a draft, one of them stays, another follows
        at = [p + steps for p in prompt]
        draft = [rows(95 + j, B, L, H, 3, D) for j in range(2)]
        W.wnw_quant_write(cfg, eager, draft[0].cuda(), draft[1].cuda(), i32(at))
        W.wnw_quant_write(cfg, eager, new[0][0].cuda(), new[1][0].cuda(), i32([a + 1 for a in at]))
        for ref, d, t in zip(refs, draft, new):
            ref.write(d.double().numpy(), at, [3, 3])
            ref.write(t[0].double().numpy(), [a + 1 for a in at], [1, 1])
        lens = [a + 2 for a in at]
        got = run_attend(W, cfg, eager, q[0], lens, [1, 1])
        want = R.attend(q[0].double(), *(torch.from_numpy(np.nan_to_num(r.values())) for r in refs), lens, [1, 1], block)
        check_attend(got, want, lens, [1, 1], D, False, H)


def test_streams(W):
    """Calls in flight on two streams, a workspace each."""
    log("[case] quant attend on two streams")
    cfg = W.make_quant_config(1, 1, 1, 8192, 64, W.WNW_QUANT_INT8)
    c, (k, v) = filled(W, cfg, [8100], R.INT8, 33)
    q = [rows(34 + j, 1, 1, 2, 1, 128) for j in range(2)]
    dev = [t.cuda() for t in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    need = W.wnw_quant_attend_workspace(cfg, 1, 2, 1)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    lens = [8100, 4000]
    ld = [i32([t]) for t in lens]
    outs = [[torch.zeros((1, 1, 2, 1, 128), device="cuda") for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(10):
        for j in range(2):
            W.wnw_quant_attend(cfg, c, dev[j], outs[j][i], ld[j], workspace=ws[j], stream=streams[j])
    torch.cuda.synchronize()
    for j in range(2):
        want = R.attend(q[j].double(), k, v, [lens[j]], [1], 64)
        tol = bound(128, lens, *want[3:], False, 1)[0]
        for o in outs[j]:
            assert torch.equal(o, outs[j][0])
        assert bool(((outs[j][0].cpu() - want[0]).abs() <= tol).all())


def test_cache_over_4_gib(W):
    """Heads behind the first 4 GiB of K, and rows at the end of a long one."""
    log("[case] quant, more than 4 GiB of K")
    H, cap, D, block = 9, 1 << 22, 128, 64
    cfg = W.make_quant_config(1, 1, H, cap, block, W.WNW_QUANT_INT8)
    c = W.make_quant_cache(cfg)
    n = 200
    x = [rows(3 + j, 1, 1, H, n, D) for j in range(2)]
    refs = [R.Cache(1, 1, H, 256, D, block, R.INT8) for _ in range(2)]
    for ref, t in zip(refs, x):
        ref.write(t.double().numpy(), [0], [n])
    vals = [torch.from_numpy(r.values()) for r in refs]
    for at in (0, cap - 256):
        W.wnw_quant_write(cfg, c, x[0].cuda(), x[1].cuda(), i32([at]))
        outs = [torch.zeros((1, 1, H, n, D), device="cuda") for _ in range(2)]
        W.wnw_quant_read(cfg, c, *outs, i32([at]))
        for o, w in zip(outs, vals):
            assert torch.equal(o.cpu(), w[..., :n, :].float())
    q = rows(8, 1, 1, H, 1, D)
    want = R.attend(q.double(), vals[0][..., :256, :], vals[1][..., :256, :], [n], [1], block)
    got = run_attend(W, cfg, c, q, [n], [1], mass=False)
    tol = bound(D, [n], *want[3:], False, H)[0]
    assert bool(((got[0].cpu() - want[0]).abs() <= tol).all())
    # every row of the cache, keys and values the same: the output is that value whatever the lengths
    c.k.fill_(140)
    c.v.fill_(133)
    c.k_scale.fill_(0.5)
    c.v_scale.fill_(0.25)
    out, lse, _ = run_attend(W, cfg, c, q, [cap - 7], [1], mass=False)
    assert float((out - 1.25).abs().max()) <= 1.25 * (cap * EPS + 2.0 ** -20)
    logit = 6.0 * q.double().sum(dim=-1) / math.sqrt(D)
    assert float((lse.cpu() - (logit + math.log(cap - 7))).abs().max()) <= 1e-3


def test_refusals_with_device_tensors(W):
    log("[case] quant, refusals of the binding")
    cfg = W.make_quant_config(1, 1, 1, 64, 32, W.WNW_QUANT_INT8)
    c = W.make_quant_cache(cfg)
    x = torch.zeros((1, 1, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):     # on the host
        W.wnw_quant_write(cfg, c, x.cpu(), x.cpu(), i32([0]))
    with pytest.raises(ValueError):
        W.wnw_quant_write(cfg, c, x, x, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        W.wnw_quant_write(cfg, c, x, x, i32([0]).long())
    with pytest.raises(ValueError):     # not contiguous
        W.wnw_quant_write(cfg, c, x.transpose(3, 4).contiguous().transpose(3, 4), x, i32([0]))
    with pytest.raises(ValueError):     # another head dimension
        W.wnw_quant_write(cfg, c, x[..., :64].contiguous(), x[..., :64].contiguous(), i32([0]))
    out = torch.zeros((1, 1, 2, 1, 128), device="cuda")
    q = torch.zeros((1, 1, 2, 1, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(W.WnwError) as e:     # no workspace
        W.wnw_quant_attend(cfg, c, q, out, i32([5]))
    assert e.value.status == W.WNW_ERR_INVALID and "workspace" in str(e.value)
    with pytest.raises(TypeError):           # fp32 output into bf16
        W.wnw_quant_attend(cfg, c, q, out.bfloat16(), i32([5]))
    short = W.QuantCache(c.k[..., :32, :].contiguous(), c.v, c.k_scale, c.v_scale)
    with pytest.raises(ValueError):
        W.wnw_quant_attend(cfg, short, q, out, i32([5]))
