"""GPU tests of the paged cache and of drafted decoding at the ends of what the header allows: every kernel of attention with
every way of sharing a call out, numbers that are not finite, large vocabularies and batches, and the loop of a program that drafts."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import paged_shares as S
from tests.test_gpu_paged import check_outputs, i32, run_attend, some_tree
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


# tokens, q-heads per KV-head: 16, 32, 64, 128 and (two blocks of) 256 query rows to a block
BLOCKS = {16: (1, 4), 32: (5, 5), 64: (12, 4), 128: (9, 10), 256: (50, 6)}
# batch, layers, KV-heads, lengths: a work-group for every block, blocks in pieces, and all tiles in a line
WAYS = {"whole": (2, 1, 2, [200, 90]), "pieces": (2, 1, 2, [3000, 700]), "line": (3, 10, 20, [2000, 0, 700])}


def filled(W, seed, B, L, H, D, page, top, bf16):
    """A cache whose pages are handed out in no order, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-top // page)
    cfg = W.make_paged_config(B, L, H, page, B * width, width, head_dim=D, flags=W.WNW_F_OUT_BF16 if bf16 else 0)
    c = W.make_paged_cache(cfg)
    c.table.copy_(torch.randperm(B * width, generator=g, device="cuda").int().reshape(B, width))
    c.k.normal_(generator=g)
    c.v.normal_(generator=g)
    return cfg, c, g


def call(W, rb, way, D, tree, bf16):
    """(cfg, cache, queries, lengths, counts, what token sees what, its bits): checked to go the way it is named for."""
    n, G = BLOCKS[rb]
    B, L, H, lens = WAYS[way]
    cfg, c, g = filled(W, rb + D, B, L, H, D, 32, max(lens), bf16)
    q = torch.randn((B, L, H * G, n, D), generator=g, device="cuda").bfloat16()
    counts = [n, n, max(1, n - 3)][:B]
    assert S.share(W, cfg, L, H * G, n, lens, counts)[:2] == (rb, way)
    rng = np.random.default_rng(rb)
    see = [R.ancestors(some_tree(rng, n)) for _ in range(B)] if tree else None
    return cfg, c, q, lens, counts, see, torch.stack([R.words(s) for s in see]).cuda() if tree else None


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("rb", list(BLOCKS))
@pytest.mark.parametrize("D", [64, 128])
def test_bf16_outputs_are_the_fp32_ones_rounded(W, D, rb, way, tree):
    """The flag changes how a result is stored and nothing else: the same bits, rounded; the same log-sum-exp."""
    log(f"[case] attend, bf16 against fp32, {rb} rows a block, {way}, d={D} tree={tree}")
    cfg, c, q, lens, counts, _, mask = call(W, rb, way, D, tree, False)
    half = W.make_paged_config(cfg.batch, cfg.layers, cfg.kv_heads, cfg.page, cfg.pages, cfg.table_width, head_dim=D, flags=W.WNW_F_OUT_BF16)
    assert S.share(W, half, cfg.layers, q.shape[2], q.shape[3], lens, counts)[:2] == (rb, way)
    full, lse = run_attend(W, cfg, c, q, lens, counts, mask)
    short, short_lse = run_attend(W, half, c, q, lens, counts, mask)
    assert torch.equal(full.bfloat16(), short) and torch.equal(lse, short_lse)


@pytest.mark.parametrize("T,way", [(70, "whole"), (5000, "pieces")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 20, 40, 80, 200])
def test_logits_that_are_all_minus_infinity(W, D, G, T, way):
    """A token that gives no row any weight gets zeros and the log-sum-exp -inf, whatever is in the rows' V; one that gives some of them
    weight gets what is in all that it sees."""
    log(f"[case] attend, logits of -inf, d={D} G={G} T={T}")
    for n in (1, 2):
        cfg, c, g = filled(W, G, 1, 1, 1, D, 16, T, False)
        assert S.share(W, cfg, 1, G * n, n, [T])[1] == way
        q = torch.randn((1, 1, G, n, D), generator=g, device="cuda").bfloat16()
        q[..., 0] = 1.0
        c.k[..., 0] = -math.inf
        c.v[..., 5] = math.nan
        c.v[..., D - 1] = math.inf
        out, lse = run_attend(W, cfg, c, q, [T], None)
        assert bool((lse == -math.inf).all()) and bool((out == 0).all())
        # the last row but one has a finite key, and every token sees it
        page, row = R.place(c.table.cpu(), 0, T - 2, 16, cfg.pages)
        c.k[page, 0, 0, row, 0] = 0.25
        out, lse = run_attend(W, cfg, c, q, [T], None)
        bad = torch.zeros(D, dtype=torch.bool, device="cuda")
        bad[[5, D - 1]] = True
        assert bool(torch.isfinite(lse).all()) and bool((torch.isfinite(out) == ~bad).all())
        want = c.v[page, 0, 0, row].float()
        assert bool(((out - want).abs() <= 2.0 ** -22 * want.abs())[..., ~bad].all())      # a weight of one over a sum of one
