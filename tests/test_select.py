"""The selection of the best rows over the scores of beams, against plain float64 arithmetic and a full sort.

Parents and rows are compared exactly: within a beam the order is that of the scores, and where beams compete the inputs either are
multiples of 1/8 (every sum exact, ties everywhere) or lie far further apart than the error of a total.  A total is rounded to fp32
(2^-24 of it); with log_softmax, the sum's terms are exponentials in fp32 of differences d from a score that is at most 20 below the
largest one that its thread has seen: a term is off by (|d| + 4) 2^-23 of it (the difference, its product with log2 e, and two units of the
instruction), so the logarithm of their sum by the mean of that, weighted as the terms are."""
import ctypes
import os

import numpy as np
import pytest

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def gv():
    import paper_1903_00757_amd as gv

    if not os.path.exists(gv.LIB_PATH):
        from paper_1903_00757_amd import build

        build.build()
    gv.load()
    return gv


def best_of(scores, best, beams, totals, done, end, log):
    """(parent, row, total, bound of the error) in 64 bits"""
    s = scores.astype(np.float64)
    queries, rows = s.shape
    s[np.isnan(s)] = -np.inf
    base = np.zeros(queries) if totals is None else totals.astype(np.float64)
    parent, row = np.full((queries // beams, best), -1), np.full((queries // beams, best), -1)
    total, bound = np.full((queries // beams, best), -np.inf), np.zeros((queries // beams, best))
    for group in range(queries // beams):
        every = []
        for b in range(group * beams, (group + 1) * beams):
            if not np.isfinite(base[b]):
                continue
            if done is not None and done[b]:
                every.append((np.array([base[b]]), np.array([b]), np.array([np.inf]), np.array([end]), np.zeros(1)))
                continue
            at = np.nonzero(s[b] > -np.inf)[0]
            if not at.size:
                continue
            v, off = s[b, at], 0.0
            count = base[b] + v
            if log:
                top = v.max()
                d = np.where(v == top, 0.0, np.where(v < np.inf, v, 0.0) - top)
                e = np.exp(d)
                count = base[b] + d - np.log(e.sum())
                off = (e * (np.minimum(-d, 110) + 24)).sum() / e.sum() * 2.0 ** -23
            every.append((count, np.full(at.size, b), v, at, np.full(at.size, off)))
        if not every:
            continue
        t, b, v, r, off = (np.concatenate(x) for x in zip(*every))
        some = t > -np.inf
        t, b, v, r, off = t[some], b[some], v[some], r[some], off[some]
        order = np.lexsort((r, -v, b, -t))[:best]
        n = order.size
        parent[group, :n], row[group, :n], total[group, :n], bound[group, :n] = b[order], r[order], t[order], off[order]
    return parent, row, total, bound


def check(gv, scores, best, beams=1, totals=None, done=None, end=0, log=True, order=True):
    import torch

    got = gv.gv_select_rows(scores, best, beams=beams, totals=totals, done=done, end=end, log_softmax=log)
    host = [None if x is None else x.cpu().numpy() for x in (totals, done)]
    parent, row, total, off = best_of(scores.double().cpu().numpy(), best, beams, host[0], host[1], end, log)
    assert got.parent.dtype is torch.int64 and got.row.dtype is torch.int64 and got.total.dtype is torch.float32
    if order:
        for name, x, want in (("parent", got.parent, parent), ("row", got.row, row)):
            off_at = np.argwhere(x.cpu().numpy() != want)
            assert not off_at.size, (name, off_at[:5].tolist(), total[tuple(off_at[0])])
    t = got.total.double().cpu().numpy()
    same = (t == total) | (np.abs(t - np.where(np.isfinite(total), total, 0)) <= off + np.abs(np.where(np.isfinite(total), total, 0)) * 2.0 ** -24 * 1.01 + 2.0 ** -140)
    assert same.all(), (t[~same][:5], total[~same][:5])
    return got


# ------------------------------------------------------------------------------------------------ refusals, on the CPU


def test_refusals_need_no_device(gv):
    L = gv.load()
    at = ctypes.c_void_p(1 << 20)
    ok = dict(queries=4, rows=10, type=gv.GV_F32, scores=at, stride=10, beams=2, totals=None, done=None, end=0, log=1, best=3, parent=at, row=at,
              total=at, workspace=at, bytes=1 << 30, stream=None)
    for bad, word in [(dict(queries=65538), "2^16"), (dict(rows=2**31 + 1), "2^31"), (dict(beams=0), "beams"), (dict(beams=513), "beams"),
                      (dict(beams=3), "groups"), (dict(best=0), "best"), (dict(best=1025), "best"), (dict(type=gv.GV_I8), "type"),
                      (dict(scores=None), "null scores"), (dict(scores=ctypes.c_void_p(2)), "aligned"), (dict(stride=9), "stride"),
                      (dict(stride=2**41), "stride"), (dict(totals=ctypes.c_void_p(2)), "aligned"), (dict(done=at, end=10), "end"),
                      (dict(parent=None), "null parent"), (dict(row=ctypes.c_void_p(4)), "aligned"), (dict(total=None), "null total"),
                      (dict(workspace=None), "workspace"), (dict(bytes=100), "needed")]:
        assert L.gv_select_rows(*{**ok, **bad}.values()) == gv.GV_EINVAL, bad
        assert word in L.gv_last_error(None).decode(), (bad, L.gv_last_error(None))
    assert L.gv_select_rows(*{**ok, "queries": 0, "scores": None, "workspace": None, "bytes": 0}.values()) == gv.GV_OK
    assert gv.gv_select_rows_workspace(1, 5000, 1, 10) == 0 and gv.gv_select_rows_workspace(0, 5000, 1, 10) == 0
    with pytest.raises(gv.GvError):
        gv.gv_select_rows_workspace(5, 100, 2, 10)


@gpu
def test_refusals_of_tensors(gv):
    import torch

    s = torch.zeros(4, 10, device="cuda")
    for call in (lambda: gv.gv_select_rows(s.cpu(), 3), lambda: gv.gv_select_rows(s.int(), 3), lambda: gv.gv_select_rows(s[0], 3),
                 lambda: gv.gv_select_rows(s.t(), 3), lambda: gv.gv_select_rows(s, 3, totals=torch.zeros(3, device="cuda")),
                 lambda: gv.gv_select_rows(s, 3, done=torch.zeros(4, device="cuda")), lambda: gv.gv_select_rows(s.requires_grad_(), 3)):
        with pytest.raises(ValueError):
            call()
    s = s.detach()
    for call in (lambda: gv.gv_select_rows(s, 0), lambda: gv.gv_select_rows(s, 2000), lambda: gv.gv_select_rows(s, 3, beams=3), lambda: gv.gv_select_rows(s, 3, beams=0),
                 lambda: gv.gv_select_rows(s, 3, done=torch.zeros(4, dtype=torch.bool, device="cuda"), end=10)):
        with pytest.raises(gv.GvError):
            call()


# ------------------------------------------------------------------------------------------------ values


@gpu
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("queries,rows,best", [(1, 1, 1), (1, 1, 5), (3, 7, 7), (2, 100, 1), (1, 8191, 10), (5, 8193, 64), (2, 20_000, 65), (3, 16_384, 128),
                                               (1, 300_001, 100), (7, 70_000, 300), (2, 100_000, 1024), (1, 5000, 1024), (40, 30_011, 512), (2000, 333, 9)])
def test_one_beam(gv, kind, queries, rows, best):
    """The order is that of the scores, ties by row; short types tie often."""
    import torch

    rng = np.random.default_rng(rows + best)
    wide = torch.from_numpy(3 * rng.standard_normal((queries, rows + 3)).astype(np.float32)).cuda().to(getattr(torch, kind))
    check(gv, wide[:, 1:rows + 1], best, log=True)
    check(gv, wide[:, :rows], best, log=False)


@gpu
@pytest.mark.parametrize("rows,best", [(9000, 10), (100_000, 100), (50_000, 1000)])
@pytest.mark.parametrize("shape", ["equal", "rising", "falling", "few values", "hidden", "zeros of both signs", "one block"])
def test_scores_in_a_special_order(gv, rows, best, shape):
    import torch

    rng = np.random.default_rng(2)
    s = {"equal": np.zeros(rows), "rising": np.arange(rows), "falling": -np.arange(rows), "few values": rng.integers(0, 3, rows),
         "hidden": np.where(rng.random(rows) < 0.001, rng.random(rows), -np.inf), "zeros of both signs": rng.choice([-0.0, 0.0], rows),
         "one block": np.where((np.arange(rows) >= 8200) & (np.arange(rows) < 8200 + 64), 1 + rng.random(rows), rng.random(rows))}[shape]
    two = torch.from_numpy(np.stack([s, np.roll(s, 4097)]).astype(np.float32)).cuda()
    check(gv, two, best, log=False)
    check(gv, two, best, log=True)


@gpu
@pytest.mark.parametrize("groups,beams,rows,best", [(1, 2, 5, 4), (3, 8, 1000, 8), (2, 5, 40_000, 5), (1, 16, 300_000, 16), (1, 512, 700, 100), (2, 300, 20_000, 1024),
                                                    (20, 4, 2011, 3), (1, 3, 100, 500)])
def test_beams_with_ties_everywhere(gv, groups, beams, rows, best):
    """Multiples of 1/8 without the softmax: every total is exact."""
    import torch

    rng = np.random.default_rng(beams)
    n = groups * beams
    scores = torch.from_numpy((rng.integers(-40, 41, (n, rows)) / 8).astype(np.float32)).cuda()
    totals = torch.from_numpy((-rng.integers(0, 20, n) / 8).astype(np.float32)).cuda()
    done = torch.from_numpy(rng.random(n) < 0.2).cuda()
    check(gv, scores, best, beams, totals, None, log=False)
    check(gv, scores, best, beams, totals, done, end=rows - 1, log=False)
    check(gv, scores.half(), best, beams, None, done, end=0, log=False)


@gpu
@pytest.mark.parametrize("groups,beams,rows,best", [(1, 2, 9, 3), (4, 4, 3001, 4), (2, 8, 100_003, 8), (1, 32, 20_000, 32), (16, 5, 777, 5)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_beams_with_softmax(gv, groups, beams, rows, best, kind):
    import torch

    rng = np.random.default_rng(rows)
    n = groups * beams
    scores = torch.from_numpy((3 * rng.standard_normal((n, rows))).astype(np.float32)).cuda().to(getattr(torch, kind))
    scores[torch.from_numpy(rng.random((n, rows)) < 0.1).cuda()] = -np.inf
    totals = torch.from_numpy((-20 * rng.random(n)).astype(np.float32)).cuda()
    done = torch.from_numpy(rng.random(n) < 0.2).cuda()
    check(gv, scores, best, beams, totals, done, end=rows // 2)


@gpu
def test_beams_that_begin_alike(gv):
    """All beams of a group have the same scores and totals: the lowest beam's go first, exactly."""
    import torch

    scores = torch.randn(1, 50_001, device="cuda").repeat(6, 1)
    got = gv.gv_select_rows(scores, 9, beams=6, totals=torch.full((6,), -2.5, device="cuda"))
    assert got.parent.view(-1).tolist() == [0, 1, 2, 3, 4, 5, 0, 1, 2]
    top = torch.topk(scores[0], 2).indices.tolist()
    assert got.row.view(-1).tolist() == [top[0]] * 6 + [top[1]] * 3


@gpu
@pytest.mark.parametrize("log", [False, True])
@pytest.mark.parametrize("rows", [50, 30_000])
def test_what_is_masked_and_what_is_not_finite(gv, log, rows):
    import torch

    inf, nan = float("inf"), float("nan")
    low = torch.finfo(torch.float32).min
    s = torch.randn(12, rows, device="cuda")
    s[0] = -inf                       # nothing left
    s[1] = nan
    s[2, 5:] = -inf                   # less than best
    s[3, ::2] = nan
    s[4] = low                        # the lowest value is a score
    s[4, 3] = 0.0
    s[5, 7], s[5, 9] = inf, inf
    s[6, :] = -inf
    s[6, rows - 1] = inf
    s[7] = 3e38
    s[8] *= 1e-30
    s[9, 1], s[9, 2] = 88.0, -3e38
    totals = torch.zeros(12, device="cuda")
    totals[10], totals[11] = -inf, nan
    check(gv, s, 20, 1, totals, log=log)
    if not log:
        check(gv, s, 20, 12, totals, log=log)
    got = gv.gv_select_rows(s[:2], 3, log_softmax=log)
    assert (got.parent == -1).all() and (got.row == -1).all() and (got.total == -inf).all()


@gpu
def test_scores_of_no_rows_and_no_queries(gv):
    import torch

    got = gv.gv_select_rows(torch.zeros(4, 0, device="cuda"), 3, beams=2)
    assert got.row.shape == (2, 3) and (got.row == -1).all() and (got.parent == -1).all()
    got = gv.gv_select_rows(torch.zeros(0, 10, device="cuda"), 3)
    assert got.row.shape == (0, 3)


@gpu
def test_far_offsets(gv):
    """A group's scores take more than 2^32 values, and a beam's rows more than a part's."""
    import torch

    rows = 1 << 28
    s = torch.zeros(17, rows, dtype=torch.bfloat16, device="cuda")
    s[16, rows - 1], s[16, 77], s[3, rows // 2], s[0, 0] = 4.0, 3.0, 5.0, 1.0
    got = gv.gv_select_rows(s, 5, beams=17, log_softmax=False)
    assert got.parent.tolist() == [[3, 16, 16, 0, 0]] and got.row.tolist() == [[rows // 2, rows - 1, 77, 0, 1]]
    assert got.total.tolist() == [[5.0, 4.0, 3.0, 1.0, 0.0]]
    got = gv.gv_select_rows(s[16:], 2)
    sure = np.log(rows + np.exp(4.0) + np.exp(3.0) - 2)
    assert got.row.tolist() == [[rows - 1, 77]]
    assert np.abs(got.total.double().cpu().numpy() - (np.array([[4.0, 3.0]]) - sure)).max() < 28 * 2.0 ** -23 + sure * 2.0 ** -24


@gpu
@pytest.mark.parametrize("log", [False, True])
def test_as_many_rows_as_there_may_be(gv, log):
    """2^31 rows, the last of which is the best; of the equal ones the lowest."""
    import torch

    rows = 1 << 31
    s = torch.zeros(1, rows, dtype=torch.bfloat16, device="cuda")
    s[0, rows - 1], s[0, rows // 2] = 4.0, 3.0
    done = torch.zeros(1, dtype=torch.bool, device="cuda")
    got = gv.gv_select_rows(s, 4, done=done, end=rows - 1, log_softmax=log)
    assert got.row.tolist() == [[rows - 1, rows // 2, 0, 1]] and got.parent.tolist() == [[0, 0, 0, 0]]
    assert log or got.total.tolist() == [[4.0, 3.0, 0.0, 0.0]]
    got = gv.gv_select_rows(s, 2, done=~done, end=rows - 1, totals=torch.tensor([-2.5], device="cuda"), log_softmax=log)
    assert got.row.tolist() == [[rows - 1, -1]] and got.total.tolist() == [[-2.5, -np.inf]]


@gpu
@pytest.mark.parametrize("rows", [3000, 200_000])
def test_captured_and_replayed(gv, rows):
    """A step of a search, with the states reordered, replayed on other scores; eager work and another stream in between."""
    import torch

    rng = np.random.default_rng(3)
    beams, n = 4, 12
    scores, states = torch.zeros(n, rows, device="cuda"), torch.randn(n, 33, device="cuda")
    totals = torch.zeros(n, device="cuda")

    def step():
        got = gv.gv_select_rows(scores, beams, beams=beams, totals=totals)
        return got, gv.gv_lookup_rows(states, got.parent.view(-1))

    step()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, *step()))
    graphs = [(g, *rest) for g, *rest in graphs]
    for _ in range(4):
        scores.copy_(torch.from_numpy(rng.standard_normal((n, rows)).astype(np.float32)))
        totals.copy_(torch.from_numpy(-5 * rng.random(n).astype(np.float32)))
        for g, *_ in graphs:
            g.replay()
        want = check(gv, scores, beams, beams, totals)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = step()
        torch.cuda.current_stream().wait_stream(side)
        for got, moved in [eager] + [rest for _, *rest in graphs]:
            assert torch.equal(got.parent, want.parent) and torch.equal(got.row, want.row) and torch.equal(got.total, want.total)
            assert torch.equal(moved, states[want.parent.view(-1)])


@gpu
@pytest.mark.parametrize("log", [False, True])
@pytest.mark.parametrize("rows,share", [(70_000, 1.0), (70_000, 0.2), (200_000, 0.05)])
def test_many_scores_of_infinity(gv, log, rows, share):
    """More of them than a workgroup keeps, over several of its turns: the lowest rows, each with an equal share."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(7)
    s = torch.randn(3, rows, device="cuda", generator=gen)
    s[torch.rand(3, rows, device="cuda", generator=gen) < share] = float("inf")
    check(gv, s, 100, log=log)
    check(gv, s.half(), 700, beams=3, log=log)


@gpu
def test_scores_of_infinity_take_no_longer_than_other_equal_ones(gv):
    """Once `best` of them are kept none of the others is of interest.  (Taken up in every turn they took nine times as long.)"""
    import torch

    def least_time(s):
        times = []
        for _ in range(6):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            gv.gv_select_rows(s, 10, log_softmax=False)
            end.record()
            end.synchronize()
            times.append(begin.elapsed_time(end))
        return min(times)

    zeros = torch.zeros(1024, 40 * 16384, dtype=torch.float16, device="cuda")
    assert least_time(torch.full_like(zeros, float("inf"))) < 2 * least_time(zeros)
