"""Batches over a paged cache by their lists: wrong ones, long ones, heads of another size."""
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


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


@pytest.mark.parametrize("start,kv,T,bad", [
    ([0, 2, 5], [40, 60], 4, [1]),          # rows past the tensor
    ([0, 3, 2], [40, 60], 4, [1]),          # decreasing
    ([0, 2, 4], [40, -1], 4, [1]),          # a negative length
    ([0, 2, 4], [40, 97], 4, [1]),          # a length past the table's row
    ([-1, 2, 4], [40, 60], 4, [0]),         # rows before the tensor
    ([0, 2, 1, 4], [40, 60, 50], 4, [1])])
def test_rope_reports_bad_lists(sp, ctx, start, kv, T, bad):
    """Lists on the device that say something impossible are reported, and the cache of the sequences that
    they speak of is as it was: a count of rows that is too large would move every key to an earlier place."""
    H, KH, D, page = 4, 2, 64, 16
    B, width = len(kv), 6
    k = torch.full((B * width, KH, page, D), 3.0, dtype=torch.bfloat16, device="cuda")
    cache = sp.KVCache(k, k.clone())
    table = torch.arange(B * width, dtype=torch.int32).view(B, width)
    batch = sp.PagedBatch(_ints(start), _ints(kv), table.cuda(), max_q=4)
    x = torch.randn(T, (H + 2 * KH) * D, generator=_g(1)).to(torch.bfloat16).cuda()
    q = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_rope_append(ctx, x, q, cache, batch, sp.Rope(64))
    with pytest.raises(sp.SparoaError) as e:
        ctx.sync()
    assert e.value.status == sp.ERR_INVALID_ARG
    for pool in (cache.k, cache.v):
        same = (pool == 3).flatten(1).all(1).cpu().view(B, width).all(1)
        assert same[bad].all(), same
    # rows that belong to no sequence are no error
    good = sp.PagedBatch(_ints([0, 2, 3]), _ints([40, 60]), table[:2].contiguous().cuda(), max_q=2)
    sp.sparoa_rope_append(ctx, x, q, cache, good, sp.Rope(64))
    ctx.sync()


def test_heads_of_another_size(sp, ctx):
    """Rows given as heads have heads of the cache's size; flat rows are cut into them."""
    cache = sp.KVCache(*(torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    batch = sp.PagedBatch(_ints([0, 2]), _ints([20]), _ints([[0, 1]]), max_q=2)
    new = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    rope = sp.Rope(64)
    for q, y in ((new(2, 2, 128), new(2, 2, 128)), (new(2, 8, 32), new(2, 8, 32))):
        with pytest.raises(sp.SparoaError):
            sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    for qkv, q in ((new(2, 8, 64), new(2, 2, 128)), (new(2, 4, 128), new(2, 4, 64)), (new(2, 512), new(2, 8, 32))):
        with pytest.raises(sp.SparoaError):
            sp.sparoa_rope_append(ctx, qkv, q, cache, batch, rope)
    for q in (new(2, 4, 64), new(2, 256)):
        sp.sparoa_rope_append(ctx, new(2, 8, 64), q, cache, batch, rope)
        sp.sparoa_rope_append(ctx, new(2, 512), q, cache, batch, rope)
        sp.sparoa_paged_attention(ctx, q, new(2, 4, 64), cache, batch)
        sp.sparoa_paged_attention(ctx, q, new(2, 256), cache, batch)
    ctx.sync()


@pytest.mark.parametrize("B", [33, 40, 129, 300, 1024])
@pytest.mark.parametrize("form", ["single", "ragged", "chunks"])
def test_many_sequences(sp, ctx, B, form):
    """Batches longer than a warp, than the CTAs' 128, 256 and 384 threads: every sequence's tokens are
    rotated and cached at their places, and see their own cached tokens."""
    H, KH, D, page = 4, 2, 64, 16
    g = _g(B)
    new = [1] * B if form == "single" else torch.randint(0, 4, (B,), generator=g).tolist()
    if form == "chunks":
        new[B // 2], new[-1] = 70, 33
    kv = [n + int(t) for n, t in zip(new, torch.randint(0, 90, (B,), generator=g))]
    kv[3] = 1500
    T, width = sum(new), -(-max(kv) // page)
    need = [-(-n // page) for n in kv]
    order = torch.randperm(sum(need), generator=g)
    table = torch.full((B, width), -1, dtype=torch.int32)
    keys = [torch.randn(2, KH, n, D, generator=g).to(torch.bfloat16) for n in kv]
    k, v = (torch.full((sum(need), KH, page, D), float("nan"), dtype=torch.bfloat16) for _ in range(2))
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m].to(torch.int32)
        for i in range(m):
            e = min(page, kv[b] - i * page)
            for pool, src in ((k, keys[b][0]), (v, keys[b][1])):
                pool[order[at + i], :, :e] = src[:, i * page:i * page + e]
        at += m
    start = torch.tensor([0] + new).cumsum(0)
    batch = sp.PagedBatch(start.to(torch.int32).cuda(), _ints(kv), table.cuda(), max_q=max(new))
    # (no rotation: what is appended is the keys themselves, which are cached already, with other values)
    cache = sp.KVCache(k.cuda(), v.cuda())
    qkv = torch.empty(T, H + 2 * KH, D, dtype=torch.bfloat16)
    qkv[:, :H] = torch.randn(T, H, D, generator=g).to(torch.bfloat16)
    for b, n in enumerate(new):
        rows = slice(int(start[b]), int(start[b]) + n)
        keys[b][1, :, kv[b] - n:] = torch.randn(KH, n, D, generator=g).to(torch.bfloat16)
        qkv[rows, H:H + KH] = keys[b][0, :, kv[b] - n:].transpose(0, 1)
        qkv[rows, H + KH:] = keys[b][1, :, kv[b] - n:].transpose(0, 1)
    q = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
    y = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sp.sparoa_rope_append(ctx, qkv.view(T, -1).cuda(), q, cache, batch, sp.Rope(0))
    sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    ctx.sync()
    assert torch.equal(q.cpu(), qkv[:, :H])
    y = y.double().cpu()
    for b, n in enumerate(new):
        for h in range(H):
            rows = slice(int(start[b]), int(start[b]) + n)
            s = qkv[rows, h].double() @ keys[b][0, h // 2].double().t() / D ** 0.5
            keep = torch.arange(kv[b])[None] <= torch.arange(kv[b] - n, kv[b])[:, None]
            p = torch.softmax(s.masked_fill(~keep, float("-inf")), -1)
            val = keys[b][1, h // 2].double()
            tol = 2.0 ** -8 * (p @ val).abs() + (2.0 ** -8 + 2.0 ** -12) * (p @ val.abs())
            assert ((y[rows, h] - p @ val).abs() <= tol).all(), (b, n, kv[b], h)
