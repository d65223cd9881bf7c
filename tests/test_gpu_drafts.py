"""The decoder stack with 4-bit weights, capped scores, a bias by distance, and steps that check trees of drafted
tokens, on the GPU against a plain 64-bit model that rounds to bf16 where the stack hands bf16 from one operator
to the next."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


def _b(t):
    return t.to(torch.bfloat16).double()


def _weights(sp, model, bf16, group):
    """Each layer's matrices in 64 bits; with `group` the quantised ones of the bf16 model's."""
    out = []
    for layer in bf16.layers:
        m = {}
        for k in ("qkv", "o", "w1", "w2"):
            w = layer[k].cpu().float()
            if group:
                codes, scales, _ = sp.w4_quantise(layer[k], group)
                codes, scales = codes.cpu(), scales.cpu()
                c = torch.stack([codes & 15, codes >> 4], -1).view(w.shape).double() - 8
                m[k] = c * scales.double().repeat_interleave(group, 1)
            else:
                m[k] = w.double()
        m["g1"], m["g2"] = layer["g1"].cpu().double(), layer["g2"].cpu().double()
        out.append(m)
    return out


def _plain(model, w, tokens, cap=0.0, slopes=None):
    """Logits [n, vocab] of one sequence, all tokens at once."""
    def norm(v, n):
        return _b(v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * n.weight.cpu().double())

    H, KH, D = model.heads, model.kv_heads, model.head_dim
    n = len(tokens)
    x = model.embed.cpu()[tokens].double()
    at = torch.arange(n, dtype=torch.float64)
    ang = at[:, None] * 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    for i, m in enumerate(w):
        y = norm(x, model.layers[i]["n1"])
        qkv = _b(y @ m["qkv"].t()).view(n, H + 2 * KH, D)
        qk = qkv[:, :H + KH]
        if slopes is None:
            lo, hi = qk[..., :D // 2], qk[..., D // 2:]
            qk = _b(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))
        q, k = qk[:, :H].transpose(0, 1), qk[:, H:].repeat_interleave(H // KH, 1).transpose(0, 1)
        v = qkv[:, H + KH:].repeat_interleave(H // KH, 1).transpose(0, 1)
        s = q @ k.transpose(1, 2) / D ** 0.5
        if cap:
            s = cap * torch.tanh(s / cap)
        if slopes is not None:
            s = s - slopes.double()[:, None, None] * (at[:, None] - at[None]).abs()
        p = torch.softmax(s.masked_fill(~torch.ones(n, n, dtype=torch.bool).tril(), float("-inf")), -1)
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


def _models(sp, ctx, group=None, cap=0.0, slopes=None, **kw):
    from paper_2511_19457_gb300.decoder import Decoder
    size = dict(layers=2, dim=256, heads=8, kv_heads=2, head_dim=64, hidden=512, vocab=504, pages=96, page_size=16, **kw)
    model = Decoder(ctx, group=group, cap=cap, slopes=slopes, **size)
    return model, _weights(sp, model, model if group is None else Decoder(ctx, **size), group)


CONFIGS = [dict(), dict(group=64), dict(cap=3.0), dict(slopes=True), dict(group=128, cap=2.0, slopes=True)]


def _config(c):
    c = dict(c)
    if c.get("slopes"):
        c["slopes"] = torch.exp2(-torch.arange(1.0, 9.0))
    return c


@pytest.mark.parametrize("config", CONFIGS)
def test_logits(sp, config):
    """Chunks of a prompt, then single tokens."""
    c = _config(config)
    ctx = sp.Context(0)
    model, w = _models(sp, ctx, **c)
    tokens = torch.randint(0, 504, (150,), generator=torch.Generator().manual_seed(3)).tolist()
    want = _plain(model, w, tokens, c.get("cap", 0.0), c.get("slopes"))
    at = 0
    for n in (90, 40, 17, 1, 1, 1):
        got = model.forward(torch.tensor(tokens[at:at + n]).cuda(), ["s"], [n])
        _close(got, want[at:at + n], f"tokens {at} to {at + n}")
        at += n
    ctx.sync()
    ctx.close()


def _tree(rng, n, vocab):
    parents = [-1] + [rng.randint(max(0, i - 5), i - 1) for i in range(1, n)]
    return [rng.randrange(vocab) for _ in range(n)], parents


def _way(parents, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i]
    return out[::-1]


@pytest.mark.parametrize("config", CONFIGS)
def test_trees_are_their_paths(sp, config):
    """Every node's logits are those of its path behind the prompt, as one text."""
    from paper_2511_19457_gb300.decoder import ancestors
    c = _config(config)
    ctx = sp.Context(0)
    model, w = _models(sp, ctx, **c)
    rng = random.Random(5)
    prompts = [[rng.randrange(504) for _ in range(n)] for n in (37, 5, 130)]
    seqs = ["a", "b", "c"]
    model.forward(torch.tensor([t for p in prompts for t in p]).cuda(), seqs, [len(p) for p in prompts])
    trees = [_tree(rng, n, 504) for n in (12, 1, 30)]
    new = [len(t) for t, _ in trees]
    before = [model.pages.length[s] for s in seqs]
    model.pages.grow_all(seqs, new)
    bits = [b for _, p in trees for b in ancestors(p)]
    pos = [L + bin(b).count("1") - 1 for (_, p), L in zip(trees, before) for b in ancestors(p)]
    flat = torch.tensor([t for tokens, _ in trees for t in tokens]).cuda()
    got = model._layers(flat, model.pages.batch(seqs, new), torch.tensor(bits).cuda(), torch.tensor(pos, dtype=torch.int32).cuda())
    ctx.sync()
    row = 0
    for prompt, (tokens, parents) in zip(prompts, trees):
        for i in range(len(tokens)):
            text = prompt + [tokens[j] for j in _way(parents, i)]
            _close(got[row:row + 1], _plain(model, w, text, c.get("cap", 0.0), c.get("slopes"))[-1:], f"node {i} of {len(tokens)}")
            row += 1
    ctx.close()


def test_check_keeps_the_confirmed_path(sp):
    """The step's own choices: drafts that hold them are kept, the cache goes on as if the tokens had come one by
    one, and pages behind what is settled come back."""
    ctx = sp.Context(0)
    model, w = _models(sp, ctx)
    rng = random.Random(7)
    prompts = [[rng.randrange(504) for _ in range(n)] for n in (45, 16, 3)]
    seqs = ["a", "b", "c"]
    logits = model.forward(torch.tensor([t for p in prompts for t in p]).cuda(), seqs, [len(p) for p in prompts])
    ends = torch.tensor([len(p) for p in prompts]).cumsum(0) - 1
    texts = [p + [t] for p, t in zip(prompts, logits[ends.cuda()].argmax(-1).tolist())]
    for step in range(4):
        drafts, hidden = [], []
        for i, text in enumerate(texts):
            # the plain model's next tokens, hidden among others
            ahead, t = [], list(text)
            for _ in range(rng.choice([0, 1, 3])):
                ahead.append(int(_plain(model, w, t)[-1].argmax()))
                t.append(ahead[-1])
            tokens, parents, at = [text[-1]], [-1], 0
            for token in ahead:
                for _ in range(rng.choice([0, 2])):
                    tokens.append((token + rng.randrange(1, 500)) % 504); parents.append(rng.choice([at, len(tokens) - 2]))
                tokens.append(token); parents.append(at)
                at = len(tokens) - 1
            drafts.append((tokens, parents))
            hidden.append(ahead)
        got = model.check(drafts, seqs)
        for text, more, ahead, s in zip(texts, got, hidden, seqs):
            top = _plain(model, w, text + more[:-1])
            for k, token in enumerate(more):
                row = top[len(text) - 1 + k]
                # (a choice within what the tolerance of the logits leaves open)
                assert row[token] >= row.max() - 4e-2 * row.norm() / 504 ** 0.5 * 6, f"step {step}"
            assert len(more) >= 1
            text += more
            assert model.pages.length[s] == len(text) - 1 and len(model.pages.held[s]) == -(-(len(text) - 1) // 16)
    got = model.forward(torch.tensor([t[-1] for t in texts]).cuda(), seqs, [1, 1, 1])
    for row, text in zip(got, texts):
        _close(row[None], _plain(model, w, text)[-1:], "the token after")
    ctx.close()


def test_generate_with_drafts(sp):
    """Drafts from the text and drafts that are nonsense: as many tokens as asked for, pages come back, and the same
    tokens as one by one wherever the two best logits are further apart than the logits may be off."""
    from paper_2511_19457_gb300.decoder import repeats
    ctx = sp.Context(0)
    model, w = _models(sp, ctx)
    rng = random.Random(9)
    prompts = [[1, 2, 3] * 20, [5], [rng.randrange(504) for _ in range(33)]]
    plain = model.generate(prompts, 12, chunk=32)
    for draft in (repeats, lambda text: ([7, 8, 9], [-1, 0, -1]), lambda text: ([], [])):
        got = model.generate(prompts, 12, chunk=32, draft=draft)
        assert len(model.pages.free) == 96 and [len(t) for t in got] == [12] * 3
        for p, a, b in zip(prompts, plain, got):
            k = next((k for k in range(12) if a[k] != b[k]), None)
            if k is not None:
                row = _plain(model, w, p + a[:k])[-1]
                assert (row[a[k]] - row[b[k]]).abs() <= 4e-2 * row.norm() / 504 ** 0.5 * 6, "another token without need"
    ctx.close()


def test_generate_with_rules(sp):
    """A presence penalty above every difference forbids a token to come twice; a mask leaves what it leaves; a
    bias brings its token; a mask without tokens is an error."""
    ctx = sp.Context(0)
    model, _ = _models(sp, ctx)
    prompts = [[1, 2, 3], list(range(100, 140))]
    got = model.generate(prompts, 30, penalties=(1.0, 1e4, 0.0, 1.0))
    for p, t in zip(prompts, got):
        assert len(set(p + t)) == len(p) + 30
    def odd(text):
        return torch.full((16,), 0x2AAAAAAA, dtype=torch.int32)
    assert all(v % 2 for t in model.generate(prompts, 9, allowed=odd) for v in t)
    bias = torch.zeros(504, device="cuda")
    bias[77] = 1e4
    assert model.generate(prompts, 3, bias=bias) == [[77] * 3] * 2
    with pytest.raises(ValueError):
        model.generate(prompts, 3, allowed=lambda text: torch.zeros(16, dtype=torch.int32))
    assert len(model.pages.free) == 96
    ctx.close()
