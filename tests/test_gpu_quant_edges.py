"""GPU tests of the 8-bit cache at the ends of what its header allows.  Tolerances of attention are those
of test_gpu_quant.py, whose head derives them."""
import math

import pytest
import torch

from tests import quant_reference as R
from tests.test_gpu_quant import SHAPES, SHARED, bound, check_attend, filled, i32, new_cache, rows, run_attend
from tests.wnw_harness import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def W():
    from paper_2608_22704_amd import wnw
    return wnw


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 16, 17, 130])
def test_a_sequence_that_writes_nothing(W, fmt, n):
    """Its bytes and scales stay as they are wherever pos is, inside a block too: another call may be writing that block."""
    log(f"[case] quant write, nothing of some sequences, fmt={fmt} n={n}")
    pos, count = [5, 37, 64, 191, 3, 21], [0, -4, 0, 0, n, 0]
    B, L, H, cap, D, block = len(pos), 1, 2, 192, 64, 32
    cfg = W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D)
    c = new_cache(W, cfg)
    x = [rows(60 + j, B, L, H, n, D).cuda() for j in range(2)]
    W.wnw_quant_write(cfg, c, *x, i32(pos), i32(count))
    torch.cuda.synchronize()
    for b in range(B):
        if count[b] > 0:
            assert bool((c.k[b] != 0xA5).any())
            continue
        for t in (c.k, c.v):
            assert bool((t[b] == 0xA5).all()), b
        for t in (c.k_scale, c.v_scale):
            assert bool((t[b] == -7.0).all()), b


# tokens a call of four query heads: 16, 32, 64 and 128 query rows to a block
TOKENS = [1, 6, 12, 40]


def scaled(c, vals, f, block):
    """Multiplies V by 2^f[j] in block j."""
    f = torch.pow(2.0, torch.as_tensor(f, dtype=torch.float64))
    c.v_scale *= f.float().cuda()
    vals[1].mul_(f.repeat_interleave(block).unsqueeze(-1))


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
def test_smallest_v_scales(W, fmt, D, n):
    """V scales from the smallest that a cache holds, 2^-126, on."""
    log(f"[case] quant attend, smallest V scales, fmt={fmt} n={n} d={D}")
    H, G, block, T, cap = 1, 4, 32, 330, 384
    cfg = W.make_quant_config(1, 1, H, cap, block, fmt, head_dim=D)
    c, vals = filled(W, cfg, [T], fmt, 41, garbage=False)
    low = torch.floor(torch.log2(c.v_scale.double())).cpu().reshape(-1)
    scaled(c, vals, -126 - low, block)
    assert bool((c.v_scale >= 2.0 ** -126).all()) and bool((c.v_scale < 2.0 ** -125).all())
    q = rows(42, 1, 1, H * G, n, D, spread=0.3)
    want = R.attend(q.double(), *vals, [T], [n], block)
    check_attend(run_attend(W, cfg, c, q, [T], [n]), want, [T], [n], D, False, H)


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2, 6, 12, 40, 64])
@pytest.mark.parametrize("before", [0, 1000])
def test_v_scales_of_rows_not_seen(W, fmt, D, n, before):
    """V scales that grow by 2^30 from block to block: a token's output knows nothing of the rows behind it, whose scales are
    2^30 and more above those that it sees."""
    log(f"[case] quant attend, V scales of later rows, fmt={fmt} n={n} d={D} rows in front {before}")
    H, G, block = 1, 4, 16
    T, first = before + n, before // block
    cap = (T + 63) // 64 * 64
    cfg = W.make_quant_config(1, 1, H, cap, block, fmt, head_dim=D)
    c, vals = filled(W, cfg, [T], fmt, 43)
    # (a token's own block and those behind it; all rows in front are alike)
    scaled(c, vals, [30.0 * min(max(j - first, 0), 4) - 60 for j in range(cap // block)], block)
    q = rows(44, 1, 1, H * G, n, D, spread=0.3)
    want = R.attend(q.double(), *vals, [T], [n], block)
    check_attend(run_attend(W, cfg, c, q, [T], [n]), want, [T], [n], D, False, H)


def check_not_finite(got, want, D, T, H):
    """Every output has NaN and infinities exactly where the reference has, and is within its bound elsewhere."""
    b_out, b_lse, b_mass = bound(D, [T], *want[3:], False, H)
    checks = [("out", got[0], want[0], b_out), ("lse", got[1], want[1], b_lse + 2.0 ** -22 * want[1].abs())]
    if got[2] is not None:       # single tokens
        checks.append(("mass", got[2], want[2][..., 0, :], want[2][..., 0, :] * b_mass + 1e-37))
    for name, g, w, tol in checks:
        g = g.double().cpu()
        assert torch.equal(torch.isnan(g), torch.isnan(w)), name
        assert torch.equal(torch.isinf(g), torch.isinf(w)) and torch.equal(g[torch.isinf(w)], w[torch.isinf(w)]), name
        fine = torch.isfinite(w)
        assert bool(((g - w).abs()[fine] <= tol.expand_as(w)[fine]).all()), name


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("n", [1, 9, 20, 70])
@pytest.mark.parametrize("which", ["K", "V"])
def test_a_nan_block_in_every_output(W, fmt, n, which):
    """K's: the log-sum-exp and all masses of a token that sees it are NaN; V's: the output alone."""
    log(f"[case] quant attend, NaN block of {which}, every output, fmt={fmt} n={n}")
    H, G, block, D, T = 1, 3, 16, 64, 170
    for bad in (T - n, 40, T - 1):
        cfg = W.make_quant_config(1, 1, H, 192, block, fmt, head_dim=D)
        c, vals = filled(W, cfg, [T], fmt, 11)
        j = bad // block
        (c.k_scale if which == "K" else c.v_scale)[..., j] = math.nan
        vals[which == "V"][..., j * block: (j + 1) * block, :] = math.nan
        q = rows(12, 1, 1, H * G, n, D)
        want = list(R.attend(q.double(), *vals, [T], [n], block))
        for e, t in zip((3, 4, 5), want[3:]):     # sizes for the bounds: without the block
            clean = [v.nan_to_num(0.0) for v in vals]
            want[e] = R.attend(q.double(), *clean, [T], [n], block)[e]
        if which == "V":
            assert torch.isfinite(want[1]).all() and torch.isnan(want[0]).any()
        check_not_finite(run_attend(W, cfg, c, q, [T], [n]), want, D, T, H)


@pytest.mark.parametrize("n", [1, 9, 20, 70])
def test_queries_that_are_not_finite(W, n):
    """A NaN or an infinity in a query: NaN in the outputs of its row alone, and -inf for a token that sees no row."""
    log(f"[case] quant attend, queries that are not finite, n={n}")
    H, G, block, D = 1, 3, 16, 64
    T = 170 if n == 1 else n - 1        # the first token sees no row where there are several
    cfg = W.make_quant_config(1, 1, H, 192, block, R.INT8, head_dim=D)
    c, vals = filled(W, cfg, [T], R.INT8, 13)
    q = rows(14, 1, 1, H * G, n, D)
    want = list(R.attend(q.double(), *vals, [T], [n], block))
    for hq, value in ((0, math.nan), (1, math.inf)):
        q[0, 0, hq, n - 1, 5] = value
        want[0][0, 0, hq, n - 1] = want[1][0, 0, hq, n - 1] = math.nan
        want[2][0, 0, hq, n - 1, : -(-T // block)] = math.nan
    got = run_attend(W, cfg, c, q, [T], [n])
    if n > 1:
        assert bool((want[1][..., 0] == -math.inf).all())
    check_not_finite(got, want, D, max(T, 1), H)


# every way of sharing work out, and every kernel: (lens, n, counts, layers, KV heads, group, block, d)
CALLS = [(lens, n, counts, 2, H, G, block, D) for lens, n, counts, H, G, block, D in SHAPES] + list(SHARED.values())


@pytest.mark.parametrize("fmt", [R.INT8, R.E4M3])
@pytest.mark.parametrize("call", CALLS, ids=lambda c: f"b{len(c[0])}_len{c[0][0]}_n{c[1]}_l{c[3]}_g{c[5]}_blk{c[6]}_d{c[7]}")
def test_bf16_outputs_are_the_fp32_ones_rounded(W, fmt, call):
    """The flag changes how a result is stored and nothing else: the same bits, rounded; the same statistics and masses."""
    lens, n, counts, L, H, G, block, D = call
    log(f"[case] quant attend, bf16 against fp32, fmt={fmt} n={n} {L} layers group {G} block {block} d={D}")
    B = len(lens)
    counts = counts or [1] * B
    cap = (max(lens) + 63) // 64 * 64 + 64
    cfg = [W.make_quant_config(B, L, H, cap, block, fmt, head_dim=D, flags=f) for f in (0, W.WNW_F_OUT_BF16)]
    g = torch.Generator(device="cuda").manual_seed(19)
    c = W.make_quant_cache(cfg[0])
    for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        t.random_(1, 127, generator=g)
        s.copy_(torch.exp(0.5 * torch.randn(s.shape, generator=g, device="cuda")) * 0.02)
    q = rows(20, B, L, H * G, n, D, spread=0.3)
    want, got = (run_attend(W, f, c, q, lens, counts) for f in cfg)
    assert torch.equal(got[0], want[0].bfloat16())
    for a, b in zip(got[1:], want[1:]):
        assert a is b is None or torch.equal(a, b)
