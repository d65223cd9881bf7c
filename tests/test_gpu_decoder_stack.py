"""The decoder stack on the GPU: logits of ragged prompts in chunks and of single tokens against a plain
64-bit model that rounds to bf16 where the stack hands bf16 from one operator to the next."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


def _b(t):
    return t.to(torch.bfloat16).double()


def _plain(model, tokens):
    """Logits [n, vocab] of one sequence, all tokens at once."""
    def norm(v, n):
        return _b(v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * n.weight.cpu().double())

    H, KH, D = model.heads, model.kv_heads, model.head_dim
    n = len(tokens)
    x = model.embed.cpu()[tokens].double()
    f = 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    ang = torch.arange(n, dtype=torch.float64)[:, None] * f
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    mask = torch.ones(n, n, dtype=torch.bool).tril()
    w = [{k: v.cpu().double() for k, v in layer.items() if isinstance(v, torch.Tensor)} for layer in model.layers]
    for i, m in enumerate(w):
        y = norm(x, model.layers[i]["n1"])
        qkv = _b(y @ m["qkv"].t()).view(n, H + 2 * KH, D)
        lo, hi = qkv[:, :H + KH, :D // 2], qkv[:, :H + KH, D // 2:]
        qk = _b(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))
        q, k = qk[:, :H].transpose(0, 1), qk[:, H:].repeat_interleave(H // KH, 1).transpose(0, 1)
        v = qkv[:, H + KH:].repeat_interleave(H // KH, 1).transpose(0, 1)
        p = torch.softmax((q @ k.transpose(1, 2) / D ** 0.5).masked_fill(~mask, float("-inf")), -1)
        a = _b((p @ v).transpose(0, 1).reshape(n, H * D))
        x = x + m["g1"] * _b(a @ m["o"].t())
        h = _b((norm(x, model.layers[i]["n2"]) @ m["w1"].t()).relu())
        x = x + m["g2"] * _b(h @ m["w2"].t())
    return norm(x, model.last) @ model.embed.cpu().double().t()


def _close(got, want, what):
    """A chain of about 20 operators whose bf16 results may round the other way: each moves the
    logits by about 2^-9 of their size, 20 of them by sqrt(20) 2^-9 = 1e-2; twice that is allowed."""
    err = torch.linalg.norm(got.double().cpu() - want) / torch.linalg.norm(want)
    assert torch.isfinite(got).all() and err <= 2e-2, f"{what}: {err:.2e}"


@pytest.mark.parametrize("heads,kv_heads,head_dim,page", [(8, 2, 64, 16), (4, 4, 64, 64), (6, 1, 128, 32)])
def test_logits(sp, heads, kv_heads, head_dim, page):
    from paper_2511_19457_gb300.decoder import Decoder
    ctx = sp.Context(0)
    model = Decoder(ctx, layers=2, dim=256, heads=heads, kv_heads=kv_heads, head_dim=head_dim, hidden=512, vocab=504,
                    pages=64, page_size=page)
    g = torch.Generator().manual_seed(3)
    tokens = [torch.randint(0, 504, (n,), generator=g).tolist() for n in (150, 3, 70)]
    want = [_plain(model, t) for t in tokens]
    # chunks of different lengths, then single tokens, all sequences of a step together
    steps = [(100, 1, 40), (40, 1, 20), (9, 1, 9), (1, 0, 1)]
    at = [0, 0, 0]
    for new in steps:
        live = [i for i in range(3) if new[i]]
        flat = [t for i in live for t in tokens[i][at[i]:at[i] + new[i]]]
        got = model.forward(torch.tensor(flat).cuda(), live, [new[i] for i in live])
        ctx.sync()
        row = 0
        for i in live:
            _close(got[row:row + new[i]], want[i][at[i]:at[i] + new[i]], f"sequence {i} at {at[i]}")
            row += new[i]
            at[i] += new[i]
    assert at == [150, 3, 70]
    ctx.close()


def test_generate_and_pages(sp):
    """Greedy tokens are the same again; pages come back, after a failure too; a full cache says so."""
    from paper_2511_19457_gb300.decoder import Decoder
    ctx = sp.Context(0)
    model = Decoder(ctx, layers=1, dim=128, heads=2, kv_heads=1, head_dim=64, hidden=256, vocab=64, pages=20, page_size=16)
    prompts = [[1, 2, 3] * 20, [5], [7] * 33]
    a = model.generate(prompts, 5, chunk=64)
    assert len(model.pages.free) == 20 and not model.pages.held
    assert [len(t) for t in a] == [5, 5, 5] and all(0 <= t < 64 for s in a for t in s)
    assert a == model.generate(prompts, 5, chunk=64)
    with pytest.raises(RuntimeError):
        model.generate([[2] * 10, [1] * 400], 1, chunk=400)
    assert len(model.pages.free) == 20
    ctx.close()
