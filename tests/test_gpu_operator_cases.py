"""The measurable cases of perf/operators.py: what the framework's calls give for them against the file's own definition in
64 bits, the small fixed ones and a few drawn ones.

Every output is rounded to bf16 (2^-8 of an element at most, so 2^-8 of the norm) or fp32, and all else that the kernels
add is below a tenth of that; what a cache stands for is equal."""
import random

import pytest
import torch

import perf.operators as P
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

SMALL = 6e7      # bytes of a pass
FIXED = [c for c in P.listed() if P.work(c)["bytes"] < SMALL]


def _drawn(kind, seed):
    rng = random.Random(f"{kind} {seed}")
    while True:
        c = P.draw(rng)
        if c["kind"] == kind and P.work(c)["bytes"] < SMALL:
            return c


def _check(case, monkeypatch):
    say(f"operator case {case}")
    want = P.exact(case, 5)
    monkeypatch.setattr(P, "own", True)
    state = P.prepare(case, 5)
    for _ in range(2):
        got = P.run(state)
    torch.cuda.synchronize()
    assert len(got) == len(want)
    for g, w in zip(got, want):
        g = g.double()
        assert g.shape == w.shape
        if case["kind"] == "pack":
            assert torch.equal(g, w)
            continue
        same = g == w                                    # (infinities among them: rows of no keys)
        diff, size = torch.where(same, 0.0, g - w), torch.where(torch.isfinite(w), w, 0.0)
        assert torch.isfinite(diff).all()
        assert diff.norm() <= 2.0 ** -8 * 1.1 * size.norm()


@pytest.mark.parametrize("case", FIXED, ids=lambda c: c["name"])
def test_fixed_cases(case, monkeypatch):
    _check(case, monkeypatch)


@pytest.mark.parametrize("kind", ["pack", "unpack", "attend", "norm"])
@pytest.mark.parametrize("seed", range(3))
def test_drawn_cases(kind, seed, monkeypatch):
    _check(_drawn(kind, seed), monkeypatch)
