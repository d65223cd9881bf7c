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
