"""The operators on rows at the ends of their ranges: values near the ends of fp32, rows without values, tables and batches past
the sizes at which the kernels change their layout, and what a program around the calls has a right to.

Tolerances (u = 2^-24) are derived as those of test_rows.py are; powers of two that are taken out and put back round nothing."""
import ctypes

import numpy as np
import pytest

from test_rows import (U, check, grads_in_64_bits, gv, in_8_bits, keep_mask, make_rows, norm_in_64_bits,  # noqa: F401
                       norm_tolerance, packed, rounding, scores_in_64_bits)

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ scores near fp32's ends

# powers of two of the table's scales and of the queries (8-bit queries: of their scales); every score stays inside fp32
REACHES = {"f32": [(88, 0), (105, -10), (124, -60), (126, -85), (-100, 60), (-132, 80), (-20, 115), (-60, 123), (0, 100)],
           "f16": [(88, 0), (110, -8), (120, -12), (-100, 8), (-132, 8)],
           "i8": [(88, 0), (112, -20), (126, -60), (126, -140), (40, -140), (-100, 100), (-132, 126), (0, 98)]}
REACHES["bf16"] = REACHES["f32"]


@gpu
@pytest.mark.parametrize("rows, cols, group", [(300, 32, 32), (300, 60, 32), (300, 64, 64), (300, 128, 32), (301, 200, 64),
                                               (200, 544, 128), (40, 2100, 64)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "i8"])
def test_scores_reach_as_far_as_their_results(gv, rows, cols, group, kind):
    import torch

    rng = np.random.default_rng(rows + cols + group)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8}[kind]
    codes = rng.integers(-8, 8, (rows, cols))
    codes_t = torch.from_numpy(packed(codes)).cuda()
    for of_table, of_query in REACHES[kind]:
        scale_t = torch.from_numpy(np.ldexp(rng.uniform(1, 2, (rows, -(-cols // group))), of_table).astype(np.float32)).to(torch.bfloat16)
        scales = scale_t.double().numpy()
        for queries in (1, 2, 4, 7, 20, 40):
            if kind == "i8":
                t = torch.from_numpy(rng.integers(-127, 128, (queries, cols)).astype(np.int8))
                x_scale = torch.from_numpy(np.ldexp(rng.uniform(1, 2, queries), of_query).astype(np.float32))
                x = t.double().numpy() * x_scale.double().numpy()[:, None]
                x_scale = x_scale.cuda()
            else:
                t = torch.from_numpy(np.ldexp(rng.standard_normal((queries, cols)), of_query)).to(dtype)
                x, x_scale = t.double().numpy(), None
            want, sums, weights = scores_in_64_bits(codes, scales, group, x)
            tolerance = (scales.shape[1] + 8) * U * sums + 2.0 ** -28 * np.abs(x).max(1, keepdims=True) * weights[None, :]
            # no sum leaves fp32, and terms that are subnormal (off by 2^-150) stay inside one of the roundings of the tolerance
            assert sums.max() < 2.0 ** 127 and scales.shape[1] * 2.0 ** -150 < U * sums.min()
            got = gv.gv_score_rows(codes_t, scale_t.cuda(), t.cuda(), group=group, scale=x_scale)
            check(got, want, tolerance, (of_table, of_query, queries))


@gpu
def test_scores_of_a_table_of_large_rows(gv):
    import torch

    codes = torch.full((50, 16), 0x77, dtype=torch.uint8, device="cuda")
    scales = torch.full((50, 1), 2.0 ** 88, dtype=torch.bfloat16, device="cuda")
    for queries in (1, 3, 20):
        got = gv.gv_score_rows(codes, scales, torch.ones(queries, 32, device="cuda"))
        assert (got == 7.0 * 32 * 2.0 ** 88).all()
    rows = torch.from_numpy(np.random.default_rng(4).standard_normal((400, 512)).astype(np.float32)).cuda()
    x = torch.from_numpy(np.random.default_rng(5).standard_normal((9, 512)).astype(np.float32)).cuda()
    small, large = gv.gv_quantize_rows(rows), gv.gv_quantize_rows(rows * 2.0 ** 93)  # up to 3e28
    assert torch.equal(small[0], large[0])
    for queries in (1, 9):
        got = gv.gv_score_rows(*large, x[:queries])
        assert torch.isfinite(got).all() and torch.equal(got * 2.0 ** -93, gv.gv_score_rows(*small, x[:queries]))


@gpu
@pytest.mark.parametrize("kind", ["f32", "i8"])
def test_scores_of_large_rows_beside_rows_that_are_not_finite(gv, kind):
    """A row that is not finite, an ordinary one and one whose joined groups leave fp32 do not change each other's scores."""
    import torch

    rng = np.random.default_rng(12)
    rows, cols, group = 150, 200, 32
    codes = torch.from_numpy(packed(rng.integers(-8, 8, (rows, cols)))).cuda()
    scales = torch.from_numpy(np.exp(rng.standard_normal((rows, 7))).astype(np.float32)).to(torch.bfloat16).cuda()
    for queries in (1, 4, 16, 20, 40):
        x = torch.from_numpy(rng.integers(-127, 128, (queries, cols)).astype(np.int8 if kind == "i8" else np.float32)).cuda()
        x_scale = torch.from_numpy(np.exp(rng.standard_normal(queries) - 20).astype(np.float32)).cuda() if kind == "i8" else None
        x = x if kind == "i8" else x * 2.0 ** -30
        plain = gv.gv_score_rows(codes, scales, x, group=group, scale=x_scale)
        mixed = scales.clone()
        mixed[3::7] *= 2.0 ** 110
        mixed[5::7, 4] = float("nan")
        mixed[6::14, 2] = float("inf")
        got = gv.gv_score_rows(codes, mixed, x, group=group, scale=x_scale)
        assert torch.isfinite(plain).all() and torch.isnan(got[:, 5::7]).all() and not torch.isfinite(got[:, 6::14]).any()
        assert torch.equal(got[:, 3::7] * 2.0 ** -110, plain[:, 3::7])
        for lo in (0, 1, 2, 4):
            assert torch.equal(got[:, lo::7], plain[:, lo::7])


# ------------------------------------------------------------------------------------------------ rows without values


@gpu
@pytest.mark.parametrize("cols", [8, 31, 130, 700, 1500, 3000, 9000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_empty_rows_without_eps(gv, cols, kind):
    """A row whose values are all 0 (where dropout left none, too) gives 0 with any eps, and does not spoil the gain's gradient."""
    import torch

    rng = np.random.default_rng(cols)
    rows, p = (1500, 0.6) if cols == 8 else (9, 0.25)
    t, x = make_rows(torch, rng, rows, cols, kind)
    grad_t, grad = make_rows(torch, rng, rows, cols, kind)
    more_t, more = make_rows(torch, rng, rows, cols, kind)
    t[[0, rows - 2]] = 0
    x[[0, rows - 2]] = 0
    gain = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).cuda()
    g = gain.double().cpu().numpy()
    kept = keep_mask(rows, cols, p, 31, 7)
    h = np.where(kept[0], x * kept[1], 0.0)
    empty = ~h.any(1)
    assert empty.sum() >= (10 if cols == 8 else 2) and not empty.all()
    args = dict(drop=p, seed=31, first_row=7)
    got = gv.gv_norm_rows(t, gain, eps=0.0, keep_rstd=True, **args)
    rstd = got.rstd.double().cpu().numpy()
    assert (rstd[empty] == 0).all() and (got.out[torch.from_numpy(empty).cuda()] == 0).all() and torch.isfinite(got.out).all()
    some = h[~empty]
    want = 1 / np.sqrt((some * some).mean(1))
    assert np.all(np.abs(rstd[~empty] - want) <= 48 * U * want)
    rel, least = rounding(kind)
    kept_h = got.sum.double().cpu().numpy()
    rs = rstd[:, None]
    dx, dh, dg = grads_in_64_bits(grad, kept_h, g, rs, more, kept)
    grads = gv.gv_norm_rows_backward(grad_t, got.sum, gain, got.rstd, grad_sum=more_t, **args)
    n, u = kept_h * rs, grad * g
    off = rs * (4 * U * np.abs(u) + 88 * U * np.abs(n) * np.abs(u * n).mean(1, keepdims=True)) + 3 * U * np.abs(dh)
    off += 1.01 * rel * (np.abs(dh) + off) + least
    if kind == "f16":  # the gradient of a row of one small value may pass half's largest
        off[np.abs(dh) > 65000] = np.inf
    check(grads.residual, dh, off, "residual")
    check(grads.gain, dg, (min(rows, 1100) + 4) * U * np.abs(grad * n).sum(0), "gain")
    assert torch.equal(grads.residual[0], more_t[0])
    codes = gv.gv_norm_rows(t, gain, eps=0.0, out_type=torch.int8, **args)
    assert (codes.out[torch.from_numpy(empty).cuda()] == 0).all() and (codes.scale[torch.from_numpy(empty).cuda()] == 0).all()


# ------------------------------------------------------------------------------------------------ rows whose squares leave fp32


@gpu
@pytest.mark.parametrize("cols", [1, 8, 31, 130, 700, 1500, 3000, 9000, 16384])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norm_of_rows_whose_squares_leave_the_range(gv, cols, kind):
    import torch

    rng = np.random.default_rng(cols + 1)
    exponents = [70, 0, 122, 63, -40, -75, -110, -60, 90, 55]
    rows = len(exponents)
    t, x = make_rows(torch, rng, rows, cols, kind)
    x = np.ldexp(np.clip(x, -8, 8) + 2.0 ** -6, np.array(exponents)[:, None])
    t.copy_(torch.from_numpy(x))
    grad_t, grad = make_rows(torch, rng, rows, cols, kind)
    x = t.double().cpu().numpy()
    gain = torch.from_numpy(rng.uniform(0.5, 1, cols).astype(np.float32)).cuda()
    g = gain.double().cpu().numpy()
    for eps in (0.0, 1e-6):
        _, rstd, y = norm_in_64_bits(x, None, g, float(np.float32(eps)), None)
        got = gv.gv_norm_rows(t, gain, eps=eps, keep_rstd=True)
        check(got.rstd, rstd[:, 0], 48 * U * rstd[:, 0], "rstd")
        check(got.out, y, norm_tolerance(kind, y, x, g, rstd, None) + 2.0 ** -126, "out")
        codes, step = in_8_bits(x, None, gain.cpu().numpy())
        eighth = gv.gv_norm_rows(t, gain, eps=eps, out_type=torch.int8)
        assert np.array_equal(eighth.out.cpu().numpy(), codes)
        check(eighth.scale, step * rstd[:, 0], 50 * U * step * rstd[:, 0] + 2.0 ** -126, "scale")
    # back through the rows whose gradients are inside fp32
    some = [i for i, e in enumerate(exponents) if -80 < e]
    rs = rstd[some].astype(np.float32).astype(np.float64)
    _, dh, dg = grads_in_64_bits(grad[some], x[some], g, rs, None, None)
    back = gv.gv_norm_rows_backward(grad_t[some], t[some], gain, torch.from_numpy(rs[:, 0].astype(np.float32)).cuda())
    n, u = x[some] * rs, grad[some] * g
    off = rs * (4 * U * np.abs(u) + 88 * U * np.abs(n) * np.abs(u * n).mean(1, keepdims=True)) + 3 * U * np.abs(dh)
    check(back.x, dh, off + 1.01 * rounding(kind)[0] * (np.abs(dh) + off) + 2.0 ** -126, "x")
    check(back.gain, dg, (rows + 4) * U * np.abs(grad[some] * n).sum(0), "gain")


@gpu
def test_norm_of_rows_that_are_too_small_for_their_inverse(gv):
    """1 / sqrt(mean(h^2)) has no float below 2^-128: such a row counts as empty."""
    import torch

    for cols in (8, 700, 3000):
        x = torch.full((3, cols), 2.0 ** -140, device="cuda")
        x[1] = 1.0
        got = gv.gv_norm_rows(x, torch.ones(cols, device="cuda"), eps=0.0, keep_rstd=True)
        assert (got.out[[0, 2]] == 0).all() and (got.rstd[[0, 2]] == 0).all() and (got.out[1] == 1).all()
        x[2] = float("nan")
        x[0, 0] = float("inf")
        got = gv.gv_norm_rows(x, torch.ones(cols, device="cuda"), eps=0.0, keep_rstd=True)
        assert torch.isnan(got.rstd[2]) and torch.isnan(got.out[2]).all() and torch.isnan(got.out[0, 0]) and (got.out[1] == 1).all()


# ------------------------------------------------------------------------------------------------ in a program with autograd


@gpu
def test_inputs_that_ask_for_gradients_are_refused(gv):
    """The calls record no graph: where torch would have to, they refuse instead of dropping the gradient."""
    import torch

    x, r = torch.randn(6, 32, device="cuda"), torch.randn(6, 32, device="cuda")
    gain = torch.nn.Parameter(torch.ones(32, device="cuda"))
    plain = gain.detach()
    wants = torch.randn(6, 32, device="cuda", requires_grad=True)
    later = wants * 2
    codes, scales = gv.gv_quantize_rows(torch.randn(40, 32, device="cuda"))
    y = gv.gv_norm_rows(x, plain, r, keep_rstd=True)
    for call in (lambda: gv.gv_norm_rows(x, gain), lambda: gv.gv_norm_rows(wants, plain), lambda: gv.gv_norm_rows(x, plain, later),
                 lambda: gv.gv_norm_rows(x, plain, out=wants), lambda: gv.gv_norm_rows(x, plain, r, sum=wants),
                 lambda: gv.gv_drop_rows(later, 0.1, 1), lambda: gv.gv_drop_rows(x, 0.1, 1, out=wants),
                 lambda: gv.gv_norm_rows_backward(later, y.sum, plain, y.rstd), lambda: gv.gv_norm_rows_backward(x, y.sum, gain, y.rstd),
                 lambda: gv.gv_norm_rows_backward(x, wants, plain, y.rstd),
                 lambda: gv.gv_norm_rows_backward(x, y.sum, plain, y.rstd, grad_sum=later),
                 lambda: gv.gv_score_rows(codes, scales, later)):
        with pytest.raises(ValueError, match="no_grad"):
            call()
    with torch.no_grad():
        assert torch.equal(gv.gv_norm_rows(x, gain, r).out, y.out) and gv.gv_drop_rows(later, 0.1, 1).shape == x.shape
        assert gv.gv_score_rows(codes, scales, later).shape == (6, 40)
        assert gv.gv_norm_rows_backward(x, y.sum, gain, y.rstd).gain.shape == (32,)
    # codes are constants, as every whole number of torch is
    assert not gv.gv_norm_rows(x, gain, out_type=torch.int8).scale.requires_grad
    assert torch.equal(gv.gv_quantize_rows(later)[0], gv.gv_quantize_rows(later.detach())[0])


@gpu
def test_autograd_sees_what_is_overwritten(gv):
    import torch

    x, gain = torch.randn(6, 32, device="cuda"), torch.ones(32, device="cuda")

    def fails_after(write):
        """A saved tensor that `write` goes over makes the backward pass raise."""
        saved, leaf = torch.randn(6, 32, device="cuda"), torch.ones(6, 32, device="cuda", requires_grad=True)
        loss = (leaf * saved).sum()
        write(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()

    fails_after(lambda s: gv.gv_drop_rows(s, 0.5, 1, out=s))
    fails_after(lambda s: gv.gv_norm_rows(x, gain, out=s))
    fails_after(lambda s: gv.gv_norm_rows(x, gain, s, sum=s))
    fails_after(lambda s: gv.gv_score_rows(*gv.gv_quantize_rows(torch.randn(32, 32, device="cuda")), x, out=s))
    scale = torch.empty(6, device="cuda")
    before = scale._version
    codes = gv.gv_norm_rows(x, gain, out_type=torch.int8, scale=scale)
    assert scale._version > before and codes.scale is scale
    assert gv.gv_norm_rows(x, gain).out._version == 0 and x._version == 0  # inputs and new results are not touched


# ------------------------------------------------------------------------------------------------ the package and the runtime around it


def test_the_package_is_imported_without_torch(gv):
    """Constants, the list of exports and the build need no torch; the names of rows.py are there all the same."""
    import os
    import subprocess
    import sys

    from paper_1903_00757_amd import rows

    code = ("import sys; sys.modules['torch'] = None\n"  # an import of torch raises
            "import paper_1903_00757_amd as gv, paper_1903_00757_amd.build as b\n"
            "assert gv.GV_BF16 == 1 and 'gv_drop_rows' in gv.EXPORTS and b.SOURCES\n"
            "assert 'gv_drop_rows' in dir(gv)\n"
            "try: gv.gv_norm_rows\n"
            "except ImportError: print('needs torch')\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(gv.__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout == "needs torch\n", done.stderr
    names = {}
    exec("from paper_1903_00757_amd import *", names)
    for name in rows.__all__:
        assert getattr(gv, name) is getattr(rows, name) and names[name] is getattr(rows, name)
    assert names["gv_create"] is gv.gv_create and gv.rows is rows and not hasattr(gv, "gv_no_such_call")


def runtime():
    """The HIP runtime of this process."""
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64.so" in line)
    return ctypes.CDLL(path)


@gpu
def test_errors_of_others_stay_with_them(gv):
    """An error that a call before left in the thread is neither reported by these calls nor taken from its owner."""
    import torch

    lib, hip = gv.load(), runtime()
    x, out, gain = torch.ones(8, 32, device="cuda"), torch.empty(8, 32, device="cuda"), torch.ones(32, device="cuda")
    rstd, grad_gain, space = torch.ones(5000, device="cuda"), torch.empty(32, device="cuda"), torch.empty(1 << 16, device="cuda")
    long, back = torch.ones(5000, 32, device="cuda"), torch.empty(5000, 32, device="cuda")
    codes, scales = torch.empty(8, 16, dtype=torch.uint8, device="cuda"), torch.empty(8, 1, dtype=torch.bfloat16, device="cuda")
    scores = torch.empty(8, 8, device="cuda")
    torch.cuda.synchronize()
    x_at, out_at = x.data_ptr(), out.data_ptr()
    calls = [
        lambda: lib.gv_drop_rows(8, 32, gv.GV_F32, x_at, 32, 0.0, 1, 0, out_at, 32, None),
        lambda: lib.gv_norm_rows(8, 32, gv.GV_F32, x_at, 32, None, 0, gain.data_ptr(), 0.0, 0.0, 0, 0, None, 0, gv.GV_F32, out_at, 32,
                                 None, None, None),
        lambda: lib.gv_norm_rows_backward(5000, 32, gv.GV_F32, long.data_ptr(), 32, long.data_ptr(), 32, gain.data_ptr(), rstd.data_ptr(),
                                          None, 0, 0.0, 0, 0, back.data_ptr(), 32, None, 0, grad_gain.data_ptr(), space.data_ptr(),
                                          space.nbytes, None),
        lambda: lib.gv_quantize_rows(8, 32, gv.GV_F32, x_at, 32, 32, codes.data_ptr(), scales.data_ptr(), None),
        lambda: lib.gv_score_rows(8, 32, 32, codes.data_ptr(), scales.data_ptr(), 1, gv.GV_F32, x_at, 32, None, scores.data_ptr(), 8, None),
        lambda: lib.gv_score_rows(8, 32, 32, codes.data_ptr(), scales.data_ptr(), 8, gv.GV_F32, x_at, 32, None, scores.data_ptr(), 8, None),
    ]
    hip.hipGetLastError()
    results = []
    try:
        for call in calls:
            refused = hip.hipSetDevice(1 << 20)  # there is no such GPU
            results.append((refused != 0, call(), hip.hipGetLastError() == refused))
    finally:
        hip.hipGetLastError()
    assert results == [(True, gv.GV_OK, True)] * len(calls), results
    torch.cuda.synchronize()
    seventh = torch.tensor(1 / 7).to(torch.bfloat16).float()  # the scale of a row of ones in 4 bits, whose codes are 7
    assert (out == 1).all() and (grad_gain == 5000).all() and (scores == 32 * 7 * seventh.cuda()).all()


class KernelNode(ctypes.Structure):
    """hipKernelNodeParams"""
    _fields_ = [("block", ctypes.c_uint32 * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p),
                ("grid", ctypes.c_uint32 * 3), ("params", ctypes.c_void_p), ("shared", ctypes.c_uint32)]


def launches_of(work):
    """(workgroups, threads) of every kernel that `work` launches, in order."""
    import torch

    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        held = work()
    hip, count, found = runtime(), ctypes.c_size_t(), []
    raw = ctypes.c_void_p(graph.raw_cuda_graph())
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    for node in nodes:
        kind, params = ctypes.c_int(), KernelNode()
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0 and kind.value == 0
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(params)) == 0
        found.append((params.grid[0], params.block[0]))
    del held
    return found


@gpu
def test_gradients_without_the_gains_spread_their_rows(gv):
    """One workgroup takes a few turns of rows where that saves the launch that joins the gain's gradient, and only there."""
    import torch

    x, gain, rstd = torch.randn(256, 128, device="cuda"), torch.ones(128, device="cuda"), torch.ones(256, device="cuda")
    both = gv.gv_norm_rows_backward(x, x, gain, rstd)
    without = gv.gv_norm_rows_backward(x, x, gain, rstd, keep_gain=False)
    assert torch.equal(both.x, without.x) and without.gain is None
    assert launches_of(lambda: gv.gv_norm_rows_backward(x, x, gain, rstd)) == [(1, 512)]
    assert launches_of(lambda: gv.gv_norm_rows_backward(x, x, gain, rstd, keep_gain=False)) == [(4, 512)]


# ------------------------------------------------------------------------------------------------ past the sizes where layouts change

# just past them, with odd remainders: four loads a wave of the few-query kernels (4096 waves; 64 to 1 rows each), two row tiles of
# the others (65536 rows), workgroups that take a second block, and digits that are staged again for it
LARGE = [(70_001, 128, 32, (1, 2, 4, 5, 16, 17, 40)), (70_001, 96, 32, (1, 3, 4, 9, 16, 17)), (70_003, 160, 64, (1, 2, 6)),
         (70_003, 256, 128, (2, 16)), (270_001, 32, 32, (1, 2, 4, 5, 20)), (270_001, 20, 64, (1, 5, 33)), (140_001, 64, 64, (1, 3, 5, 20)),
         (140_001, 50, 32, (1, 4, 17, 40)), (36_001, 256, 32, (1, 2, 4)), (17_001, 512, 128, (1, 2, 4)), (9_001, 1024, 64, (1, 2, 4)),
         (4_101, 2048, 32, (1, 4)), (4_101, 2100, 32, (1, 2, 4)), (70_001, 544, 64, (4, 20, 33)), (70_001, 1056, 32, (5, 40))]


@gpu
@pytest.mark.parametrize("rows, cols, group, batches", LARGE)
@pytest.mark.parametrize("kind", ["f32", "bf16", "i8"])
def test_scores_of_large_tables(gv, rows, cols, group, batches, kind):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    groups, parts = -(-cols // group), -(-cols // 32)
    q = torch.randint(-8, 8, (rows, cols), device="cuda", generator=gen, dtype=torch.int8)
    wide = torch.nn.functional.pad(q, (0, 32 * parts - cols))
    codes = ((wide[:, 0::2] & 15) | (wide[:, 1::2] << 4)).view(torch.uint8).contiguous()
    scales = torch.exp(torch.randn(rows, groups, device="cuda", generator=gen)).to(torch.bfloat16)
    w = q.double() * scales.double().repeat_interleave(group, dim=1)[:, :cols]
    for queries in batches:
        if kind == "i8":
            t = torch.randint(-128, 128, (queries, cols), device="cuda", generator=gen, dtype=torch.int8)
            x_scale = torch.exp(torch.randn(queries, device="cuda", generator=gen))
            x = t.double() * x_scale.double()[:, None]
        else:
            t = torch.randn(queries, cols, device="cuda", generator=gen).to(torch.float32 if kind == "f32" else torch.bfloat16)
            x, x_scale = t.double(), None
        got = gv.gv_score_rows(codes, scales, t, group=group, scale=x_scale)
        sums, weights = torch.matmul(x.abs(), w.abs().t()), w.abs().sum(1)
        tolerance = (groups + 8) * U * sums + 2.0 ** -28 * x.abs().amax(1, keepdim=True) * weights
        off = (got.double() - torch.matmul(x, w.t())).abs()
        assert (off <= tolerance).all(), (queries, (off / tolerance).max().item(), (off > tolerance).sum().item())
        for lo in (0, rows // 2 - 17, rows - 35):  # the same bits as from a small table
            part = gv.gv_score_rows(codes[lo:lo + 35], scales[lo:lo + 35], t, group=group, scale=x_scale)
            assert torch.equal(part, got[:, lo:lo + 35]), (queries, lo)


# several workgroups for every number of lanes that hold a row (1, 2, 4, 8, 16, 32, 64, 256 and 512), so that the gain's gradient
# is joined from parts; 520 and 1100 rows are more than the parts that there may be
JOINED = [(3000, 8), (1100, 16), (600, 31), (900, 100), (130, 257), (200, 200), (37, 1000), (9, 1025), (1100, 2048), (9, 4099), (520, 8192),
          (6, 16383)]


@gpu
@pytest.mark.parametrize("rows, cols", JOINED)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradient_of_the_gain_from_several_workgroups(gv, rows, cols, kind):
    import torch

    assert gv.gv_norm_rows_workspace(rows, cols) > 4 * cols
    rng = np.random.default_rng(rows + cols)
    for pad, shift in [(0, 0), (3, 1)]:
        st, h = make_rows(torch, rng, rows, cols, kind, pad, shift)
        gt, grad = make_rows(torch, rng, rows, cols, kind, pad, shift)
        gain = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).cuda()
        rstd = (1 / np.sqrt((h * h).mean(1) + 1e-5)).astype(np.float32)
        rs = rstd.astype(np.float64)[:, None]
        dx, _, dg = grads_in_64_bits(grad, h, gain.double().cpu().numpy(), rs, None, None)
        got = gv.gv_norm_rows_backward(gt, st, gain, torch.from_numpy(rstd).cuda())
        # h rstd rounds once; a product passes through at most 2 additions in its lane, 6 across lanes, 8 across waves, 32 in a
        # thread of the join and 5 across its lanes
        n, u = h * rs, grad * gain.double().cpu().numpy()
        check(got.gain, dg, 54 * U * np.abs(grad * n).sum(0), ("gain", pad))
        # a lane holds up to 32 values of a row; with the lanes and waves a mean passes through at most 46 additions
        off = rs * (4 * U * np.abs(u) + 54 * U * np.abs(n) * np.abs(u * n).mean(1, keepdims=True)) + 3 * U * np.abs(dx)
        rel, least = rounding(kind)
        check(got.x, dx, off + 1.01 * rel * (np.abs(dx) + off) + least, ("x", pad))


@gpu
@pytest.mark.parametrize("rows, cols, group, queries", [(3001, 128, 32, 300), (20_003, 160, 64, 1000), (500, 40, 32, 5000),
                                                        (40, 96, 128, 1 << 16), (33, 2100, 32, 257)])
@pytest.mark.parametrize("kind", ["f32", "i8"])
def test_scores_of_more_queries_than_a_pass_takes(gv, rows, cols, group, queries, kind):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(rows + queries)
    codes, scales = gv.gv_quantize_rows(torch.randn(rows, cols, device="cuda", generator=gen), group=group)
    if kind == "i8":
        t = torch.randint(-128, 128, (queries, cols), device="cuda", generator=gen, dtype=torch.int8)
        x_scale = torch.exp(torch.randn(queries, device="cuda", generator=gen))
        x = t.double() * x_scale.double()[:, None]
    else:
        t = torch.randn(queries, cols, device="cuda", generator=gen)
        x, x_scale = t.double(), None
    q = torch.stack([codes & 15, codes >> 4], -1).view(rows, -1)[:, :cols].to(torch.int8)
    w = torch.where(q > 7, q - 16, q).double() * scales.double().repeat_interleave(group, dim=1)[:, :cols]
    got = gv.gv_score_rows(codes, scales, t, group=group, scale=x_scale)
    tolerance = ((scales.shape[1] + 8) * U * torch.matmul(x.abs(), w.abs().t())
                 + 2.0 ** -28 * x.abs().amax(1, keepdim=True) * w.abs().sum(1))
    off = (got.double() - torch.matmul(x, w.t())).abs()
    assert (off <= tolerance).all(), ((off / tolerance).max().item(), (off > tolerance).sum().item())
