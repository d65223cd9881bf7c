"""A bias by distance over trees of drafts: an ancestor's distance is the one in the tree, and nothing of the one in
the cache, which may be 60 times as long, is left in the result."""
import math

import pytest
import torch

from test_gpu_decoder import _batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


@pytest.mark.parametrize("n,H", [(7, 2), (60, 2), (64, 4), (64, 8)])
@pytest.mark.parametrize("L", [0, 3, 150])
@pytest.mark.parametrize("shape", ["star", "chain", "comb"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_only_the_bias_counts(sp, n, H, L, shape, cap):
    """Queries of zero: the log of the sum is that of exp(-slope distance).  Its terms are off by 2^-22 of what they
    weigh (slope and log2(e), their product, 2^x) and by 2^-23 of the slope times a distance that counts, which is
    below 30; the log and its product by 2^-22: 2^-18 covers them."""
    ctx = sp.Context(0)
    cache, batch, *_ = _batch(sp, [n], [L + n], 32, 1, 64, 3)
    parents = {"star": [-1] + [0] * (n - 1), "chain": list(range(-1, n - 1)), "comb": [-1] + [max(0, i - 2) for i in range(1, n)]}[shape]
    bits, chains = [], []
    for i, p in enumerate(parents):
        bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        chains.append(bin(bits[i]).count("1"))
    tree = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device="cuda")
    slopes = torch.tensor([4.0, 3.3, 0.77, 0.01, 1e-3, 2.1, 1.7, 0.3][:H])
    q = torch.zeros(n, H, 64, dtype=torch.bfloat16, device="cuda")
    y, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
    sp.sparoa_ruled_attention(ctx, q, y, cache, batch, sp.ScoreRules(cap=cap, slopes=slopes.cuda(), tree=tree), lse=lse)
    ctx.sync()
    for i in range(n):
        # ancestors at 0, 1, ... and the cached tokens behind them
        far = torch.arange(L + chains[i], dtype=torch.float64)
        want = torch.logsumexp(-slopes.double()[:, None] * far, 1)
        err = (lse[i].double().cpu() - want).abs()
        assert (err <= 2.0 ** -18).all(), f"token {i}: {err.max() / 2 ** -18:.2f} of what is allowed"
    ctx.close()
