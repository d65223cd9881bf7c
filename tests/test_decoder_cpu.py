"""Host side of the decoder operators (no GPU): struct layouts, rotary frequencies, the page table's
bookkeeping, and the arithmetic by which the attention kernels cut their work, restated."""
import ctypes
import math
import os
import random
import subprocess
from decimal import Decimal, getcontext

import pytest

from paper_2511_19457_gb300 import build

build.build()

from paper_2511_19457_gb300 import sparoa as sp  # noqa: E402
from paper_2511_19457_gb300.decoder import Pages  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts(tmp_path):
    prog = tmp_path / "layout.c"
    prog.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "sparoa.h"
int main(void) {
  printf("%zu %zu %zu %zu\\n", sizeof(sparoa_norm_spec), sizeof(sparoa_kv_cache), sizeof(sparoa_paged_batch), sizeof(sparoa_rope));
  printf("%zu %zu %zu %zu %zu\\n", offsetof(sparoa_norm_spec, bias), offsetof(sparoa_kv_cache, head_dim),
         offsetof(sparoa_paged_batch, table_stride), offsetof(sparoa_paged_batch, max_q), offsetof(sparoa_rope, scale));
  return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(c) for c in (sp.NormSpec, sp.KvCacheDesc, sp.PagedBatchDesc, sp.RopeDesc)] + [
        sp.NormSpec.bias.offset, sp.KvCacheDesc.head_dim.offset, sp.PagedBatchDesc.table_stride.offset,
        sp.PagedBatchDesc.max_q.offset, sp.RopeDesc.scale.offset]


def _freqs(rot, base, scaling, factor, context, low, high):
    """Frequencies in 50 digits."""
    base = Decimal(repr(float(base)))
    if scaling == "base":
        base = base * (Decimal(rot) / Decimal(rot - 2) * Decimal(factor).ln()).exp()
    out = []
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510")
    for i in range(rot // 2):
        f = (Decimal(-2 * i) / Decimal(rot) * base.ln()).exp()
        if scaling == "linear":
            f /= Decimal(factor)
        if scaling == "parts":
            keep = (Decimal(context) * f / two_pi - Decimal(low)) / (Decimal(high) - Decimal(low))
            keep = min(max(keep, Decimal(0)), Decimal(1))
            f *= keep + (1 - keep) / Decimal(factor)
        out.append(f / two_pi)
    return out


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
@pytest.mark.parametrize("rot,base", [(16, 10000.0), (64, 500000.0), (128, 10000.0)])
def test_rope_turns(scaling, rot, base):
    """Double precision and one rounding to 2^-64 of a turn: within 2^-48 of the frequency itself."""
    getcontext().prec = 50
    kw = dict(factor=8.0, context=8192.0, low=1.0, high=32.0)
    got = sp.sparoa_rope_turns(rot, base, scaling, **kw)
    want = _freqs(rot, base, scaling, **kw)
    assert len(got) == len(want) == rot // 2
    for g, w in zip(got, want):
        assert abs(Decimal(int(g)) / 2 ** 64 - w) <= w * Decimal(2) ** -48 + Decimal(2) ** -64


def test_rope_turns_refusals():
    for rot, base, scaling, kw in ((8, 1e4, "none", {}), (-16, 1e4, "none", {}), (16, 1.0, "none", {}), (16, math.nan, "none", {}),
                                   (16, 1e4, "linear", dict(factor=0.9)), (16, 1e4, "base", dict(factor=math.inf)),
                                   (16, 1e4, "parts", dict(factor=2.0)), (16, 1e4, "parts", dict(factor=2.0, context=10.0, low=3.0, high=2.0))):
        with pytest.raises(sp.SparoaError):
            sp.sparoa_rope_turns(rot, base, scaling, **kw)
    assert sp.sparoa_rope_turns(0).size == 0


def test_pages():
    p = Pages(6, 16)
    p.grow("a", 16)
    p.grow("b", 17)
    assert len(p.held["a"]) == 1 and len(p.held["b"]) == 2 and p.length == {"a": 16, "b": 17}
    p.grow("a", 1)
    with pytest.raises(RuntimeError):
        p.grow("b", 48)
    assert p.length["b"] == 17 and len(p.free) == 2
    held = p.held["a"] + p.held["b"]
    assert len(set(held)) == 4 and set(held) | set(p.free) == set(range(6))
    p.release("a")
    p.release("a")
    assert len(p.free) == 4 and "a" not in p.length


def _cut(extra, least, whole_share, whole_more, items, grid):
    """Who has which units of the items (units, weight), as csrc/paged.cuh cuts them."""
    cost = [u * w + extra for u, w in items]
    total = sum(cost)
    ctas = int(total > 0) if total < least else min(grid, total // least)
    whole = total // ctas + whole_more if total < whole_share * ctas else 0
    start = [0]
    for c in cost:
        start.append(start[-1] + c)
    owner = lambda u: ((u + 1) * ctas - 1) // total  # noqa: E731
    got: list = [[] for _ in items]
    for c in range(ctas):
        p0, left = total * c // ctas, total * (c + 1) // ctas - total * c // ctas
        i = max(k for k in range(len(items)) if start[k] <= p0)
        pos, slots = p0 - start[i], []
        while left > 0:
            units, weight = items[i]
            if cost[i] <= whole:
                first, end = (0 if pos == 0 else units), units
            else:
                first, end = (max(0, at - extra + weight - 1) // weight for at in (pos, pos + left))
                end = min(units, end)
            if first < end:
                got[i].append((c, first, end))
                if first > 0 or end < units:
                    slots.append(first == 0)
            left -= cost[i] - pos
            i, pos = i + 1, 0
        assert len(slots) == len(set(slots))  # a CTA's parts have places of their own
    for i, (units, weight) in enumerate(items):
        parts = got[i]
        assert parts and parts[0][1] == 0 and parts[-1][2] == units
        # every unit once, and no CTA between the parts' CTAs without one: the last to arrive is known
        assert all(a[2] == b[1] and b[0] == a[0] + 1 for a, b in zip(parts, parts[1:]))
        if len(parts) > 1:
            at = start[i] + extra
            assert owner(at) == parts[0][0] and owner(at + (units - 1) * weight) == parts[-1][0]


def test_cut_of_the_work():
    rng = random.Random(1)
    for _ in range(1500):
        grid = rng.choice([1, 2, 7, 152])
        n, top = rng.randint(1, rng.choice([3, 50, 400])), rng.choice([1, 5, 100, 3000])
        _cut(2, 2, 8, 8, [(rng.randint(1, top), 1) for _ in range(n)], grid)            # few rows
        _cut(9, 16, 0, 0, [(rng.randint(1, top), rng.choice([4, 5])) for _ in range(n)], grid)  # chunks


def test_group_multiplier():
    """n / group as the kernels take it: umulhi(n, mul) >> shift for n below 2^31."""
    rng = random.Random(2)
    for d in list(range(2, 130)) + [255, 4097, 32769, 65535, 65536]:
        s = (d - 1).bit_length()
        mul = (1 << (31 + s)) // d + 1
        assert mul < 1 << 32
        for n in [0, 1, d - 1, d, 2 ** 31 - 1] + [rng.randrange(2 ** 31) for _ in range(50)] + [
                d * rng.randrange(1, 2 ** 31 // d) - 1 for _ in range(50)]:
            assert ((n * mul) >> 32) >> (s - 1) == n // d
