"""The decoder's check of drafted tokens with stand-ins for its operators (no GPU): what it keeps, hands back and
refuses."""
import copy
from types import SimpleNamespace

import pytest
import torch

from paper_2511_19457_gb300 import build

build.build()

from paper_2511_19457_gb300 import decoder  # noqa: E402
from paper_2511_19457_gb300.decoder import Decoder, Pages  # noqa: E402


def _accept(ctx, tokens, best, tree, caches, batch, path, count, following, length):
    """sparoa_tree_accept's lists, from its definition."""
    start, kv = batch.start, batch.kv
    path.fill_(-1)
    for b, L in enumerate(kv):
        q0, n = start[b], start[b + 1] - start[b]
        bits = [int(tree[q0 + i]) & ((1 << i) - 1) for i in range(n)]
        at, way = 0, [0]
        while True:
            want = bits[at] | 1 << at
            to = [i for i in range(n) if bits[i] == want and int(best[q0 + at]) >= 0 and int(tokens[q0 + i]) == int(best[q0 + at])]
            if not to:
                break
            at = to[0]
            way.append(at)
        path[q0:q0 + len(way)] = torch.tensor(way, dtype=torch.int32)
        count[b], following[b], length[b] = len(way), best[q0 + at], L - n + len(way)


class _Batch:
    def __init__(self, start, kv, table, max_q):
        self.start, self.kv, self.table, self.max_q = start.tolist(), kv.tolist(), table, max_q


@pytest.fixture
def model(monkeypatch):
    """A model of 10 tokens that says t + 1 after t, and nothing (best -1) after 8."""
    ops = SimpleNamespace(PagedBatch=_Batch, sparoa_tree_accept=_accept)

    def choose(ctx, logits, rules=None, best=None):
        best.copy_(torch.where(logits.isnan().all(1), -1, logits.nan_to_num(-1.0).argmax(1)))

    ops.sparoa_shape_logits = choose
    monkeypatch.setattr(decoder, "sp", ops)
    m = Decoder.__new__(Decoder)  # (its weights would be on the GPU)
    m.pages, m.embed, m.layers, m.ctx = Pages(6, 16), torch.zeros(10, 8), [], SimpleNamespace(sync=lambda: None)

    def layers(tokens, batch, tree=None, positions=None):
        out = torch.nn.functional.one_hot((tokens + 1) % 10, 10).float()
        out[tokens == 8] = float("nan")
        return out

    m._layers = layers
    return m


def test_confirmed_drafts_are_kept(model):
    model.pages.grow("a", 15); model.pages.grow("b", 16)
    got = model.check([([1, 5, 2, 3, 3, 9], [-1, 0, 0, 1, 2, 4]), ([4], [-1])], ["a", "b"])
    assert got == [[2, 3, 4], [5]] and model.pages.length == {"a": 18, "b": 17}


def test_a_choice_of_nothing_is_an_error(model):
    """as it is without drafts; the sequences are left as they were."""
    model.pages.grow("a", 15); model.pages.grow("b", 16)
    before = copy.deepcopy((model.pages.free, model.pages.held, model.pages.length))
    for drafts in ([([8], [-1]), ([1, 2], [-1, 0])], [([1, 2], [-1, 0]), ([6, 7, 8], [-1, 0, 1])]):
        with pytest.raises(ValueError):
            model.check(drafts, ["a", "b"])
        assert (model.pages.free, model.pages.held, model.pages.length) == before
    assert model.check([([1, 8], [-1, 0]), ([1], [-1])], ["a", "b"]) == [[2], [2]]  # (nothing follows a draft that is not kept)
    with pytest.raises(ValueError):
        model.generate([[1, 2], [3]], 12, draft=lambda text: ([(text[-1] + 1) % 10], [-1]))
    assert len(model.pages.free) == 3  # ("a" and "b" hold theirs)


def test_tokens_outside_the_vocabulary(model):
    """are refused on the host: the embedding's rows are looked up on the GPU."""
    model.pages.grow("a", 15)
    before = copy.deepcopy((sorted(model.pages.free), model.pages.held, model.pages.length))
    for bad in (10, -1, 1 << 40):
        for tokens, parents in (([1, bad], [-1, 0]), ([bad], [-1])):
            with pytest.raises(ValueError):
                model.check([(tokens, parents)], ["a"])
        with pytest.raises(ValueError):
            model.generate([[1], [2, bad, 3]], 2)
        with pytest.raises(ValueError):
            model.generate([[1], [2]], 4, draft=lambda text: ([bad], [-1]))
    assert (sorted(model.pages.free), model.pages.held, model.pages.length) == before


def test_nothing_to_check(model):
    assert model.check([], []) == []
