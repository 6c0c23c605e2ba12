"""How near the totals of a selection by log softmax are to 64 bits (tests/test_select.py allows what exponentials in fp32 would be off by).

A term is exp(d) with d taken in fp64, off by less than 2^-34 of it; sums and the logarithm are fp64.  So a logarithm of a probability is off
by 2^-34 and some units of fp64, 2^-33 in all, and by half a unit of fp32, 2^-24 of the total, once it is rounded."""
import os

import numpy as np
import pytest

gpu = pytest.mark.gpu
TURN = 16384  # scores that a workgroup reads at once; a thread has 8 in a row of them, in each quarter


@pytest.fixture(scope="module")
def gv():
    import paper_1903_00757_amd as gv

    if not os.path.exists(gv.LIB_PATH):
        from paper_1903_00757_amd import build

        build.build()
    gv.load()
    return gv


def logs_of(torch, scores):
    """(scores, logarithms of their probabilities) in 64 bits"""
    s = scores.double()
    return s, s - torch.logsumexp(s, 1, keepdim=True)


def near(torch, got, want):
    got = got.double()
    off = (got - want).abs() - want.abs() * 2.0 ** -24 - 2.0 ** -33
    assert (off <= 0).all(), off.max().item()


@gpu
@pytest.mark.parametrize("beams", [1, 8])
@pytest.mark.parametrize("turns", [2, 3])
def test_a_late_score_that_is_nearly_certain(gv, beams, turns):
    """One thread sees a score in its first turn and a larger one, by 0 to 80, in its last; all others are far below.  A probability is
    at most 1."""
    import torch

    queries = 1024  # so many that one workgroup goes through all of a query's turns
    d = torch.linspace(0, 80, queries, device="cuda")
    for low in (-60.0, -9.3):
        s = torch.full((queries, turns * TURN - 5), low, device="cuda")
        s[:, 3] = 0.37
        s[:, (turns - 1) * TURN + 4] = 0.37 + d
        got = gv.gv_select_rows(s, 1, beams=beams)
        logs = logs_of(torch, s)[1].view(queries // beams, -1).amax(1, keepdim=True)
        assert (got.total <= 0).all(), got.total.max().item()
        near(torch, got.total, logs)


@gpu
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_many_equal_scores_below_the_best(gv, kind):
    """Equal terms are all off by the same, so nothing averages out."""
    import torch

    d = torch.linspace(-20, 0, 64, device="cuda").to(getattr(torch, kind))
    s = d.view(-1, 1).repeat(1, 300_001)
    s[:, 200_000] = 0.0
    got = gv.gv_select_rows(s, 3)
    near(torch, got.total, torch.topk(logs_of(torch, s)[1], 3, dim=1).values)


@gpu
def test_scores_of_all_sizes(gv):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(5)
    for scale in (0.01, 1.0, 7.0, 300.0):
        s = scale * torch.randn(9, 100_003, device="cuda", generator=gen)
        s[:, ::7] = -float("inf")
        got = gv.gv_select_rows(s, 5, log_softmax=True)
        near(torch, got.total, torch.topk(logs_of(torch, s)[1], 5, dim=1).values)
        rising = torch.sort(s, dim=1).values
        near(torch, gv.gv_select_rows(rising, 5).total, torch.topk(logs_of(torch, s)[1], 5, dim=1).values)


@gpu
@pytest.mark.parametrize("first", [0, 1])
def test_beams_a_unit_apart(gv, first):
    """Two beams have the same scores in another order, so the same sum, and totals a unit of fp32 apart: that decides."""
    import torch

    groups, rows = 512, 3 * TURN
    gen = torch.Generator(device="cuda").manual_seed(6)
    s = 2 * torch.randn(groups, rows, device="cuda", generator=gen)
    s[:, -TURN:] += torch.linspace(0, 18, groups, device="cuda").view(-1, 1)  # the last turn has the best
    both = torch.stack([s, s.flip(1)], 1).view(2 * groups, rows)
    totals = torch.full((groups, 2), -0.5, device="cuda")
    totals[:, first] += 2.0 ** -25
    got = gv.gv_select_rows(both, 2, beams=2, totals=totals.view(-1))
    order = torch.topk(s, 1, dim=1).indices.view(-1)
    want = torch.stack([order, rows - 1 - order], 1)
    groups_first = 2 * torch.arange(groups, device="cuda")
    assert torch.equal(got.parent[:, 0], groups_first + first) and torch.equal(got.row[:, 0], want[:, first])
    assert torch.equal(got.parent[:, 1], groups_first + 1 - first) and torch.equal(got.row[:, 1], want[:, 1 - first])


def test_the_polynomial_of_the_exponentials():
    """What csrc/gv_select.hip computes, in numpy: within 2^-34 of exp(d), and 1 of 0."""
    import re

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1903_00757_amd", "csrc", "gv_select.hip")
    with open(path) as f:
        body = re.search(r"double exp_of\(double d\) \{(.*?)\n\}", f.read(), re.S).group(1)
    c = [float(x) for x in re.findall(r"\d\.\d{9,}(?:e-\d+)?", body)]
    log2_e, c = c[0], c[1:]
    assert abs(log2_e * np.log(2) - 1) < 2.0 ** -52 and len(c) == 7
    d = np.concatenate([np.linspace(-40, 21, 2_000_001), [0.0]])
    n = np.rint(d * log2_e)
    f = d * log2_e - n
    p = np.zeros_like(f)
    for x in c:
        p = p * f + x
    p = p * f + 1
    assert np.abs(np.ldexp(p, n.astype(int)) / np.exp(d) - 1).max() < 2.0 ** -34 and p[-1] == 1
