"""Steps that check drafted tokens keep what the model would have said itself: texts are chosen so that the plain
64-bit model's best token is ahead of the next by more than the logits may be off, and then every token of its
continuation has to be kept, however it is hidden among others."""
import random

import pytest
import torch

from test_gpu_drafts import CONFIGS, _config, _models, _plain, sp  # noqa: F401

pytestmark = pytest.mark.gpu


def _sure(row):
    """The best token, if it is ahead by more than two logits may be off (4e-2 of the row's norm would be all of the
    error in these two, as in test_gpu_drafts)."""
    top = row.topk(2)
    return int(top.indices[0]) if top.values[0] - top.values[1] > 4e-2 * row.norm() / 504 ** 0.5 * 6 else None


def _continued(plain, text, n):
    """The model's next n tokens, or None where it is not sure of one."""
    out = []
    for _ in range(n):
        t = _sure(plain(text + out)[-1])
        if t is None:
            return None
        out.append(t)
    return out


def _texts(plain, rng, lengths, n):
    """A text of each length that the model is sure to go on with for n tokens, and these."""
    out = []
    for length in lengths:
        for _ in range(2000):
            text = [rng.randrange(504) for _ in range(length)]
            ahead = _continued(plain, text, n)
            if ahead:
                break
        out.append((text, ahead))
    return out


@pytest.mark.parametrize("config", CONFIGS)
def test_what_the_model_would_say_is_kept(sp, config):  # noqa: F811
    c = _config(config)
    ctx = sp.Context(0)
    model, w = _models(sp, ctx, **c)

    def plain(text):
        return _plain(model, w, text, c.get("cap", 0.0), c.get("slopes"))

    rng = random.Random(11)
    texts = _texts(plain, rng, (6, 17, 30), 4)
    assert all(ahead for _, ahead in texts)
    seqs = ["a", "b", "c"]
    model.forward(torch.tensor([t for text, _ in texts for t in text[:-1]]).cuda(), seqs, [len(text) - 1 for text, _ in texts])
    drafts = []
    for text, ahead in texts:
        tokens, parents, at = [text[-1]], [-1], 0
        for token in ahead[:3]:
            for _ in range(rng.choice([0, 1, 4])):  # another token in its place, or behind one of those
                tokens.append((token + rng.randrange(1, 500)) % 504)
                parents.append(rng.choice([at, len(tokens) - 2]))
            tokens.append(token)
            parents.append(at)
            at = len(tokens) - 1
        drafts.append((tokens, parents))
    got = model.check(drafts, seqs)
    assert got == [ahead for _, ahead in texts]
    # and in the cache: a second check goes on from there
    drafts = [([a[-1], 7], [-1, 0]) for a in got]
    more = model.check(drafts, seqs)
    for (text, ahead), m in zip(texts, more):
        sure = _sure(plain(text + ahead)[-1])
        assert sure is None or m[0] == sure
    ctx.close()


def test_generate_takes_fewer_steps_than_tokens(sp):  # noqa: F811
    """where the drafts are the model's own continuation; and as many as tokens where they are nonsense."""
    ctx = sp.Context(0)
    model, w = _models(sp, ctx)
    texts = _texts(lambda t: _plain(model, w, t), random.Random(12), (9, 20), 3)
    assert all(ahead for _, ahead in texts)
    steps, check = [], model.check

    def counted(drafts, seqs):
        steps.append(len(drafts))
        return check(drafts, seqs)

    model.check = counted

    def knows(text):
        out = []
        for _ in range(3):
            out.append(int(_plain(model, w, text + out)[-1].argmax()))
        return out, [-1, 0, 1]

    got = model.generate([t for t, _ in texts], 12, draft=knows)
    assert [t[:3] for t in got] == [ahead for _, ahead in texts]
    # (four tokens a step where all is confirmed: three steps for the eleven behind the first; one that two near
    # logits end early costs one more each)
    assert len(steps) <= 6
    steps.clear()
    model.generate([t for t, _ in texts], 12, draft=lambda text: ([(knows(text)[0][0] + 1) % 504], [-1]))
    assert len(steps) >= 9
    ctx.close()


def test_a_model_without_numbers(sp):  # noqa: F811
    """says nothing: an error, and the cache as it was."""
    ctx = sp.Context(0)
    model, _ = _models(sp, ctx)
    model.forward(torch.tensor([1, 2, 3]).cuda(), ["a"], [3])
    ctx.sync()
    model.last.weight[0] = float("nan")
    with pytest.raises(ValueError):
        model.check([([4, 5], [-1, 0])], ["a"])
    assert model.pages.length == {"a": 3}
    model.last.weight[0] = 1.0
    assert len(model.check([([4, 5], [-1, 0])], ["a"])[0]) in (1, 2)
    assert len(model.pages.held["a"]) == 1
    ctx.close()
