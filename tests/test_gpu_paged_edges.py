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
