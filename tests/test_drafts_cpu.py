"""Host side of the operators that check drafted tokens (no GPU): struct layouts, sizes of packed weights,
refusals, trees, pages, and drafts from the text."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

from paper_2511_19457_gb300 import build

build.build()

from paper_2511_19457_gb300 import sparoa as sp  # noqa: E402
from paper_2511_19457_gb300.decoder import Decoder, Pages, ancestors, repeats  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts(tmp_path):
    prog = tmp_path / "layout.c"
    prog.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "sparoa.h"
int main(void) {
  printf("%zu %zu %zu\\n", sizeof(sparoa_w4), sizeof(sparoa_logit_rules), sizeof(sparoa_score_rules));
  printf("%zu %zu %zu %zu %zu %zu\\n", offsetof(sparoa_w4, group), offsetof(sparoa_w4, zeros), offsetof(sparoa_logit_rules, penalties),
         offsetof(sparoa_logit_rules, ld_allowed), offsetof(sparoa_score_rules, slopes), offsetof(sparoa_score_rules, tree));
  return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(c) for c in (sp.W4Desc, sp.LogitRulesDesc, sp.ScoreRulesDesc)] + [
        sp.W4Desc.group.offset, sp.W4Desc.zeros.offset, sp.LogitRulesDesc.penalties.offset, sp.LogitRulesDesc.ld_allowed.offset,
        sp.ScoreRulesDesc.slopes.offset, sp.ScoreRulesDesc.tree.offset]


def test_packed_sizes():
    """Tiles of 16 rows x 128 columns: 1024 bytes of codes, 32 of scales and 16 of zeros for each group."""
    size = sp._lib.sparoa_w4_bytes
    assert size(16, 128, 128, 0) == 1024 + 32 and size(16, 128, 128, 1) == 1024 + 48
    assert size(8, 32, 32, 0) == 1024 + 4 * 32 and size(24, 160, 32, 1) == 4 * (1024 + 4 * 48)
    assert size(4096, 14336, 64, 0) == 256 * 112 * (1024 + 64)
    for bad in ((12, 128, 128, 0), (16, 100, 32, 0), (16, 128, 16, 0), (0, 128, 128, 0), (16, -128, 128, 0), (1 << 21, 128, 128, 0),
                (16, 1 << 21, 128, 0), (16, 96, 64, 0)):
        assert size(*bad) == 0, bad


def test_refusals_without_a_gpu():
    """Tensors that are not on a GPU, of other types and sizes, are refused before anything is launched."""
    f, i, l = torch.zeros(4, 4), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    u, b = torch.zeros(16, 64, dtype=torch.uint8), torch.zeros(16, 1, dtype=torch.bfloat16)
    cases = [lambda: sp.W4(None, u, b), lambda: sp.LogitRules(seen_start=i, seen=i), lambda: sp.LogitRules(seen=i),
             lambda: sp.LogitRules(penalties=f), lambda: sp.ScoreRules(slopes=f[0]), lambda: sp.ScoreRules(tree=l),
             lambda: sp.ScoreRules(prefix=i), lambda: sp.sparoa_shape_logits(None, f, best=i)]
    for k, call in enumerate(cases):
        with pytest.raises(sp.SparoaError) as e:
            call()
            raise AssertionError(f"call {k} was taken")
        assert e.value.status == sp.ERR_INVALID_ARG


def test_null_contexts():
    """Every new entry refuses a NULL context."""
    lib, n = sp._lib, None
    assert lib.sparoa_w4_pack(n, n, n, n, 16, 128, 128, n) == sp.ERR_INVALID_ARG
    assert lib.sparoa_gemm_w4(n, n, 1, n, n, n, 0, n) == sp.ERR_INVALID_ARG
    assert lib.sparoa_shape_logits(n, n, 1, 1, 1, 1, n, n, 1, n, n) == sp.ERR_INVALID_ARG
    assert lib.sparoa_tree_accept(n, n, n, n, 1, n, 1, n, n, n, n, n) == sp.ERR_INVALID_ARG
    assert lib.sparoa_ruled_attention(n, n, 1, 1, 1, 1.0, 1, 0, n, n, n, n, n, n) == sp.ERR_INVALID_ARG


def test_ancestors():
    assert ancestors([-1, 0, 0, 2, 1]) == [1, 0b11, 0b101, 0b1101, 0b10011]
    assert ancestors([]) == [] and ancestors(list(range(-1, 63)))[63] == (1 << 64) - 1
    for bad in ([0], [-1, 1], [-1, -2], [-1] * 65):
        with pytest.raises(ValueError):
            ancestors(bad)


def test_pages_cut():
    p = Pages(8, 16)
    p.grow("a", 50); p.grow("b", 16)
    held = list(p.held["a"])
    p.cut("a", 33)
    assert p.held["a"] == held[:3] and p.length["a"] == 33 and len(p.free) == 4
    p.cut("a", 32)
    assert p.held["a"] == held[:2] and len(p.free) == 5
    p.grow("a", 1)
    assert p.held["a"] == held[:3]  # (the page given back last is taken first)
    p.release("a"); p.release("b")
    assert sorted(p.free) == list(range(8))


def test_repeats():
    tokens, parents = repeats([1, 2, 3, 9, 1, 2, 4, 7, 1], tokens=3, ways=2)
    assert tokens == [2, 4, 7, 2, 3, 9] and parents == [-1, 0, 1, -1, 3, 4]
    assert repeats([5]) == ([], []) and repeats([5, 6]) == ([], [])
    assert repeats([3, 3, 3], tokens=4, ways=1) == ([3], [-1])


def test_trees_that_are_none():
    model = Decoder.__new__(Decoder)  # (its weights are on the GPU)
    model.pages, model.embed = Pages(4, 16), torch.zeros(4, 8)
    for drafts in ([([], [])], [([1, 2], [-1])], [([1, 2], [0, 0])], [([1, 2], [-1, 1])], [(list(range(65)), [-1] + list(range(64)))]):
        with pytest.raises(ValueError):
            model.check(drafts, ["a"])
    one = ([1], [-1])
    for drafts, seqs in (([one, one], ["a", "a"]), ([one], ["a", "b"]), ([one, one], ["a"])):
        with pytest.raises(ValueError):
            model.check(drafts, seqs)
    with pytest.raises(ValueError):
        model.generate([[1]], 2, draft=repeats, penalties=(1.0, 0.0, 0.0, 1.0))
    assert len(model.pages.free) == 4 and not model.pages.held


def test_a_check_that_raises():
    """leaves the sequence as it was (there are no operators at all here)."""
    model = Decoder.__new__(Decoder)
    model.pages, model.embed = Pages(4, 16), torch.zeros(4, 8)
    model.pages.grow("a", 5)
    with pytest.raises(Exception):
        model.check([([1, 2, 3], [-1, 0, 0])], ["a"])
    assert model.pages.length == {"a": 5} and len(model.pages.held["a"]) == 1


def test_quantised_weights():
    """Codes, scales and zeros of each group by its range; off by a step at most (half a step, and the rounding of
    the scale to bf16, 2^-8 of up to 15 steps)."""
    g = torch.Generator().manual_seed(1)
    rng = random.Random(1)
    for zeros in (False, True):
        w = torch.randn(24, 256, generator=g) * torch.tensor([rng.choice([0.0, 1e-3, 1.0, 50.0]) for _ in range(24)])[:, None]
        codes, scales, points = sp.w4_quantise(w, 64, zeros)
        assert codes.shape == (24, 128) and codes.dtype == torch.uint8 and scales.shape == (24, 4) and (points is None) != zeros
        c = torch.stack([codes & 15, codes >> 4], -1).view(24, 256).double()
        z = points.double().repeat_interleave(64, 1) if zeros else 8.0
        s = scales.double().repeat_interleave(64, 1)
        assert (((c - z) * s - w.double()).abs() <= s + 1e-12).all()
