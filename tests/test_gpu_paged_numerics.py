"""Attention over a paged cache where its arithmetic can go wrong: scores far from zero, weights below the
normal range, weights that have to keep more bits than bf16 has.  Both kernels (max_q chooses), items of one
and of two tiles of 128 rows, items that several CTAs share."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


@pytest.fixture(scope="module")
def ctx(sp):
    c = sp.Context(0)
    yield c
    c.sync()
    c.close()


def _g(seed):
    return torch.Generator().manual_seed(seed)


def _run(sp, ctx, q, k, v, scale, max_q, causal=False):
    """q [n, H, D], k and v [L, KH, D] (fp32, exact in bf16): y and log-sum-exp of one sequence, in 64 bits."""
    n, H, D = q.shape
    L, KH = k.shape[:2]
    page = 32
    pages = -(-L // page)
    pools = []
    order = torch.randperm(pages, generator=_g(L))
    for t in (k, v):
        flat = torch.full((pages * page, KH, D), float("nan"))
        flat[:L] = t
        pool = torch.empty(pages, KH, page, D)
        pool[order] = flat.view(pages, page, KH, D).transpose(1, 2)
        pools.append(pool.to(torch.bfloat16).cuda())
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    batch = sp.PagedBatch(ints([0, n]), ints([L]), order.to(torch.int32).view(1, pages).cuda(), max_q=max_q)
    y = torch.full((n, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, H), float("nan"), device="cuda")
    sp.sparoa_paged_attention(ctx, q.to(torch.bfloat16).cuda(), y, sp.KVCache(*pools), batch, scale=scale, causal=causal, lse=lse)
    ctx.sync()
    return y.double().cpu(), lse.double().cpu()


def _plain(q, k, v, scale):
    """y, log-sum-exp and sum p |v| in 64 bits, no mask."""
    G = q.shape[1] // k.shape[1]
    kd, vd = (t.double().repeat_interleave(G, 1) for t in (k, v))
    s = torch.einsum("nhd,lhd->nhl", q.double(), kd) * scale
    p = torch.softmax(s, -1)
    mix = lambda w: torch.einsum("nhl,lhd->nhd", p, w)  # noqa: E731
    return mix(vd), torch.logsumexp(s, -1), mix(vd.abs())


# (new tokens, heads over one key head, max_q): few rows, a tile, two tiles
FORMS = [(4, 4, 4), (4, 8, 4), (25, 4, 25), (100, 4, 100), (70, 2, 1)]


@pytest.mark.parametrize("n,H,max_q", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [500, 2000, 9000])
def test_scores_far_from_zero(sp, ctx, n, H, max_q, D, L):
    """Scores of 2^24 plus a few even units, exact in fp32, of which the weights depend on the differences
    alone.  A maximum scaled by log2(e) / 8 is rounded to a quarter there: weights of keys that are taken
    with different maxima have to go by the same rounded number, or they are off by up to a fifth.  Rounding
    of the weights 2^-8 at most, of the result 2^-8; the log-sum-exp is within two roundings of itself."""
    g = _g(L + D)
    q, k = torch.zeros(n, H, D), torch.zeros(L, 1, D)
    q[..., 0] = 4096.0
    k[..., 0] = 4096.0
    q[..., 1] = torch.randint(1, 3, (n, H), generator=g).float()
    t = torch.arange(L)
    k[:, 0, 1] = (2 * ((5 * (t // 128)) % 11) + 2 * ((7 * t) % 5)).float()
    v = ((0.25 * torch.randn(L, 1, D, generator=g)) + ((t // 128) % 2).float()[:, None, None]).to(torch.bfloat16).float()
    want, wl, size = _plain(q, k, v, 0.125)
    y, lse = _run(sp, ctx, q, k, v, 0.125, max_q)
    worst = ((y - want).abs() / (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * size)).max()
    assert worst <= 1, f"{worst:.2f} of the tolerance"
    assert ((lse - wl).abs() <= 2.0 ** -22 * wl.abs()).all()


@pytest.mark.parametrize("n,H,max_q", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("unit", [1, 2, 3])
def test_scores_far_from_zero_that_grow(sp, ctx, n, H, max_q, D, unit):
    """As above, with maxima that outgrow those of the units before by 2^9, and values that make up for it."""
    g = _g(unit + D)
    L = 512
    q, k = torch.zeros(n, H, D), torch.zeros(L, 1, D)
    q[..., 0] = 4096.0
    k[..., 0] = 4096.0
    q[..., 1] = 1.0
    t = torch.arange(L)
    k[:, 0, 1] = (2 * ((7 * t) % 5)).float()
    k[unit * 128:, 0, 1] += 50
    v = torch.randn(L, 1, D, generator=g)
    v[:unit * 128] += 2.0
    v[:unit * 128] *= 512.0
    v = v.to(torch.bfloat16).float()
    want, wl, size = _plain(q, k, v, 0.125)
    y, lse = _run(sp, ctx, q, k, v, 0.125, max_q)
    worst = ((y - want).abs() / (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * size)).max()
    assert worst <= 1, f"{worst:.2f} of the tolerance"
    assert ((lse - wl).abs() <= 2.0 ** -22 * wl.abs()).all()


@pytest.mark.parametrize("n,H,max_q", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("small,large", [(0, 1), (1, 0), (0, 40), (100, 3), (0, 200), (200, 0), (0, 300), (300, 0), (5, 4000), (4000, 5)])
def test_weights_below_the_normal_range(sp, ctx, n, H, max_q, D, small, large):
    """Key `small` has a value of 2^125 and a weight of 2^-128.4 (key `large` scores 712 / 8 higher: in its
    block of keys, another one, another unit or another CTA's): fp32 and bf16 hold such weights as subnormals,
    and the output is 2^-3.4.  A weight that is rounded to bf16 there is a multiple of 2^-133: within
    2^-134 / 2^-128.4 = 2.1 %; the result's own rounding is 2^-9."""
    L = max(600, max(small, large) + 90)
    q, k, v = torch.zeros(n, H, D), torch.zeros(L, 1, D), torch.zeros(L, 1, D)
    q[..., 0] = 8.0
    k[..., 0] = -1024.0
    k[small, 0, 0], k[large, 0, 0] = 0.0, 89.0
    v[small, 0, 0] = 2.0 ** 125
    want, wl, _ = _plain(q, k, v, 0.125)
    y, lse = _run(sp, ctx, q, k, v, 0.125, max_q)
    assert want[0, 0, 0] > 0.09
    assert (y[..., 0] / want[..., 0] - 1).abs().max() <= 0.021 + 2.0 ** -9
    assert not y[..., 1:].any() and torch.allclose(lse, wl, rtol=1e-6)


@pytest.mark.parametrize("n,H,max_q", [(1, 1, 1), (4, 4, 4), (2, 8, 2), (17, 1, 17), (4, 8, 4), (32, 4, 32), (40, 2, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("a,b,L", [(0, 1, 2), (3, 90, 100), (0, 130, 300), (5, 280, 300), (1, 4000, 5000)])
def test_weights_of_few_rows_keep_16_bits(sp, ctx, n, H, max_q, D, a, b, L):
    """Up to 128 rows per key head go into the product with their weights in two bf16 parts.  Two keys of
    nearly one weight and opposite values: the result is the difference of the weights, small beside them,
    so that its own rounding hides nothing.  Two parts leave 2^-16 of a weight, fp32 scores below 4 at most
    128 2^-24 4 = 2^-15: 2^-14 of sum p |v| together with the result's 2^-8.  Weights of one part exceed that by far."""
    g = _g(D + L + n)
    q, k, v = torch.zeros(n, H, D), torch.zeros(L, 1, D), torch.zeros(L, 1, D)
    q[..., 0] = 1 + 0.5 * torch.rand(n, H, generator=g)
    q[..., 1] = 64.0
    q = q.to(torch.bfloat16).float()
    k[..., 1] = -64.0                       # keys without weight
    k[a, 0, :2] = torch.tensor([2.0, 0.0])
    k[b, 0, :2] = torch.tensor([1.75, 0.0])
    v[a, 0], v[b, 0] = 1.0, -1.0
    v[a, 0, 1], v[b, 0, 1] = 0.75, -0.625
    scale = 0.125
    want, wl, size = _plain(q, k, v, scale)
    y, lse = _run(sp, ctx, q, k, v, scale, max_q)
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -14 * size
    worst = ((y - want).abs() / tol).max()
    assert worst <= 1, f"{worst:.2f} of the tolerance"
    assert ((lse - wl).abs() <= 1e-5).all()


