"""The bound by which the GPU tests tell softmax weights of 24 bits from shorter ones holds for fp32 arithmetic and for no shorter weights."""
import math

import numpy as np
import pytest
import torch

from tests import paged_shares as S


def shortened(w, terms):
    """fp32 weights as so many bf16 terms: each the upper half of what is left (so that three are exact), or, negative, rounded."""
    out, rest = np.zeros_like(w, dtype=np.float64), w.copy()
    for _ in range(abs(terms)):
        if terms < 0:
            t = torch.from_numpy(rest).bfloat16().float().numpy()
        else:
            t = (rest.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        out += t
        rest = (rest - t).astype(np.float32)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [40, 100, 700, 3000])
def test_the_bound_of_the_weights(rows, d):
    g = torch.Generator().manual_seed(rows + d)
    k, at = S.weight_keys(g, rows, d), S.weight_rows(g, rows, d).numpy()
    there, k = at >= 0, k.double()
    scale = np.float32(1.4426950408889634) / np.sqrt(np.float32(d))
    worst = {}
    for e in range(0, d, 7):
        want = torch.softmax(k[:, e] / math.sqrt(d), dim=0)[at] * torch.from_numpy(there)
        x = (k[:, e].numpy().astype(np.float32) * scale).astype(np.float32)
        w = np.exp2((x - x.max()).astype(np.float64)).astype(np.float32)
        inv = np.float32(1) / w.sum(dtype=np.float32)
        for terms in (3, 2, 1, -2, -1):
            out = (shortened(w, terms)[at].astype(np.float32) * inv).astype(np.float64) * there
            spread = float(S.weight_spread(torch.from_numpy(out), want))
            worst.setdefault(terms, []).append(spread)
    assert max(worst[3]) <= S.WEIGHT_SPREAD
    for terms in (2, 1, -2, -1):
        assert min(worst[terms]) > S.WEIGHT_SPREAD, terms
