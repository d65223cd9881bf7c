"""Steps of the decoder stack that fail leave its sequences as they were (no GPU)."""
import copy

import pytest
import torch

from paper_2511_19457_gb300 import build

build.build()

from paper_2511_19457_gb300.decoder import Decoder, Pages  # noqa: E402


def _state(p):
    return copy.deepcopy((p.free, p.held, p.length))


def _decoder(pages):
    model = Decoder.__new__(Decoder)  # (its weights are on the GPU)
    model.pages = pages
    model.embed = torch.zeros(4, 8)
    return model


def test_a_step_that_does_not_fit():
    p = Pages(4, 16)
    p.grow("a", 16); p.grow("b", 16)
    before = _state(p)
    with pytest.raises(RuntimeError):
        _decoder(p).forward(torch.zeros(57, dtype=torch.int64), ["a", "b"], [17, 40])
    assert _state(p) == before
    with pytest.raises(RuntimeError):
        p.grow_all(["a", "c", "b"], [1, 1, 1])
    assert _state(p) == before
    p.grow_all(["a", "b"], [1, 1])  # what fits, fits still
    assert p.length == {"a": 17, "b": 17} and not p.free


def test_a_step_that_raises():
    """Anything that goes wrong after the sequences have grown: here there are no operators at all."""
    p = Pages(9, 16)
    p.grow("a", 5); p.grow("b", 32)
    before = _state(p)
    with pytest.raises(Exception):
        _decoder(p).forward(torch.zeros(60, dtype=torch.int64), ["a", "new", "b"], [40, 17, 3])
    assert _state(p) == before


def test_grow_all_and_back():
    p = Pages(8, 16)
    p.grow("a", 10)
    before = _state(p)
    p.grow_all(["a", "b", "a"], [30, 16, 1])
    assert p.length == {"a": 41, "b": 16} and len(p.held["a"]) == 3 and len(p.free) == 4
    p.shrink_all(["a", "b", "a"], [30, 16, 1])
    assert _state(p) == before


def test_prompts_without_tokens():
    p = Pages(4, 16)
    model = _decoder(p)
    assert model.generate([], 3) == []
    for prompts in ([[]], [[1, 2], []], [[], [1]]):
        with pytest.raises(ValueError):
            model.generate(prompts, 3)
    assert len(p.free) == 4 and not p.held
