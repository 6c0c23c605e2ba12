"""A layer and its gradients, against plain float64 arithmetic.

Tolerances (u = 2^-24).  A sum of n products of inputs passes through n additions, each off by at most one unit (2 u, whether rounded or
cut off) of what it adds up to: 2 n u of the sum of the products' sizes.  The activations' slopes are at most 1.13; they and
the activations are off by a few units of the exponential or error function and by the rounding of its argument, (|z| + 8) 2 u of |z| (of
1 for the slopes) at most.  A result is rounded once, to its type (2^-8, 2^-11; 2^-25 near half's smallest); the gradients' products take gz
rounded to its type, which the bound counts for each of their terms."""
import ctypes
import os

import numpy as np
import pytest

U = 2.0 ** -24
gpu = pytest.mark.gpu
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


@pytest.fixture(scope="module")
def gv():
    import paper_1903_00757_amd as gv

    if not os.path.exists(gv.LIB_PATH):
        from paper_1903_00757_amd import build

        build.build()
    gv.load()
    return gv


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rounding(kind):
    return {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}[kind]


def make_rows(torch, rng, rows, cols, kind, pad=0, shift=0, scale=1.0):
    """(tensor on the GPU whose rows lie `pad` values apart and start `shift` values after an allocation, float64 tensor there)"""
    x = torch.from_numpy((scale * rng.standard_normal((rows, cols))).astype(np.float32))
    flat = torch.full((shift + rows * (cols + pad) + 1,), float("nan"), dtype=types(torch)[kind], device="cuda")  # nothing between counts
    t = torch.as_strided(flat, (rows, cols), (cols + pad, 1), shift)
    t.copy_(x)
    return t, t.double()


def act_of(torch, z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / np.sqrt(2))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def slope_of(torch, z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / np.sqrt(2)) + z * torch.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)


def product(torch, a, b):
    """a b^T of float64 matrices on the GPU."""
    return torch.matmul(a, b.t().contiguous())


def within(got, want, bound):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), ((got - want).abs() - bound)[bad].max().item()


def forward(torch, x, w, bias, residual, act, kind):
    """(z, out, bound of z, bound of out) in 64 bits"""
    rel, least = rounding(kind)
    z, size = product(torch, x, w), product(torch, x.abs(), w.abs())
    if bias is not None:
        z, size = z + bias, size + bias.abs()
    off = (x.shape[1] + 1) * 2 * U * size
    y = act_of(torch, z, act)
    off_y = 1.13 * off
    if act != "none":
        off_y = off_y + (z.abs() + 8) * 2 * U * z.abs()
    if residual is not None:
        y = y + residual
        off_y = off_y + U * y.abs()
    return z, y, off + (z.abs() + off) * rel + least, off_y + (y.abs() + off_y) * rel + least


# ------------------------------------------------------------------------------------------------ on the CPU


def test_slopes_are_those_of_the_activations():
    """The plain forms against differences."""
    import torch

    z, h = torch.linspace(-6, 6, 401, dtype=torch.float64) + 0.003, 1e-5
    for act in ACTS:
        difference = (act_of(torch, z + h, act) - act_of(torch, z - h, act)) / (2 * h)
        assert (difference - slope_of(torch, z, act)).abs().max() < 1e-8, act


def test_refusals_need_no_device(gv):
    L = gv.load()
    P = ctypes.c_void_p
    at, far, to = P(1 << 20), P(1 << 30), P(1 << 34)
    ok = dict(rows=100, cols=8, outs=16, type=gv.GV_F32, x=at, x_stride=8, weight=far, weight_stride=8, bias=None, act=0, residual=None, residual_stride=0,
              pre=None, pre_stride=0, out=to, out_stride=16, workspace=None, bytes=0, stream=None)
    for bad, word in [(dict(rows=2**31 + 1), "2^31"), (dict(cols=0), "columns"), (dict(cols=16385), "columns"), (dict(outs=0), "out"), (dict(outs=16385), "out"),
                      (dict(type=gv.GV_I8), "type"), (dict(act=4), "activation"), (dict(act=-1), "activation"), (dict(x=None), "null x"),
                      (dict(weight=None), "null weight"), (dict(out=None), "null out"), (dict(x_stride=7), "stride"), (dict(weight_stride=7), "stride"),
                      (dict(out_stride=15), "stride"), (dict(bias=P(2)), "aligned"), (dict(residual=to, residual_stride=15), "stride"),
                      (dict(pre=P(1 << 35), pre_stride=15), "stride"), (dict(out=at), "overlaps x"), (dict(out=P((1 << 30) + 480)), "overlaps weight"),
                      (dict(pre=at, pre_stride=16), "overlaps x"),
                      (dict(pre=to, pre_stride=16), "pre overlaps out"), (dict(pre=P(1 << 35), pre_stride=16, residual=P(1 << 35), residual_stride=16), "overlaps residual"),
                      (dict(cols=16384, outs=8, x_stride=16384, weight_stride=16384), "workspace")]:
        assert L.gv_dense_rows(*{**ok, **bad}.values()) == gv.GV_EINVAL, bad
        assert word in L.gv_last_error(None).decode(), (bad, L.gv_last_error(None))
    assert L.gv_dense_rows(*{**ok, "rows": 0, "x": None}.values()) == gv.GV_OK
    ok = dict(rows=100, cols=8, outs=16, type=gv.GV_F32, grad=to, grad_stride=16, x=at, x_stride=8, weight=far, weight_stride=8, act=0, pre=None, pre_stride=0,
              grad_x=P(1 << 35), grad_x_stride=8, grad_weight=P(1 << 36), grad_weight_stride=8, grad_bias=None, workspace=None, bytes=0, stream=None)
    for bad, word in [(dict(grad=None), "null grad"), (dict(x=None), "null x"), (dict(weight=None), "null weight"), (dict(act=2), "null pre"), (dict(grad_x_stride=7), "stride"),
                      (dict(grad_weight_stride=7), "stride"), (dict(grad_bias=P(2)), "aligned"), (dict(grad_x=to), "overlaps grad_out"),
                      (dict(grad_weight=at), "overlaps x"), (dict(grad_x=P(1 << 36)), "overlaps grad_weight"),
                      (dict(grad_bias=to), "workspace"), (dict(grad_bias=to, workspace=P(1 << 38), bytes=16), "needed"),
                      (dict(act=3, pre=P(1 << 33), pre_stride=16), "workspace")]:
        assert L.gv_dense_rows_backward(*{**ok, **bad}.values()) == gv.GV_EINVAL, bad
        assert word in L.gv_last_error(None).decode(), (bad, L.gv_last_error(None))
    with pytest.raises(gv.GvError):
        gv.gv_dense_rows_workspace(1, 0, 10, gv.GV_F32)
    with pytest.raises(gv.GvError):
        gv.gv_dense_rows_backward_workspace(1, 10, 10, gv.GV_F32, 9)
    assert gv.gv_dense_rows_workspace(16, 4096, 4096, gv.GV_BF16) == 0


def test_products_keep_their_sums_in_registers(gv):
    """The tiles on matrix instructions have all registers of a lane, and a spilled one would be read back in every step."""
    from test_kernel_registers import code_objects, kernels_of

    with open(gv.LIB_PATH, "rb") as f:
        data = f.read()
    found = {k[".name"]: k for elf in code_objects(data) for k in kernels_of(elf) if "k_product" in k[".name"] or "k_sum_runs" in k[".name"]}
    assert len([n for n in found if "k_product_wide" in n]) == 2 * 2 * 3
    for name, k in found.items():
        if "k_product_wide" in name or "small" in name or "few" in name or "k_sum_runs" in name:
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


@gpu
def test_refusals_of_tensors(gv):
    import torch

    x, w, g = (torch.zeros(*s, device="cuda") for s in ((5, 8), (6, 8), (5, 6)))
    for call in (lambda: gv.gv_dense_rows(x, w.half()), lambda: gv.gv_dense_rows(x, w[:, :7]), lambda: gv.gv_dense_rows(x, w.cpu()), lambda: gv.gv_dense_rows(x[0], w),
                 lambda: gv.gv_dense_rows(x, w, torch.zeros(5, device="cuda")), lambda: gv.gv_dense_rows(x, w, None, x), lambda: gv.gv_dense_rows(x, w.clone().requires_grad_()),
                 lambda: gv.gv_dense_rows(x, w, out=x), lambda: gv.gv_dense_rows_backward(g, x, w, act=gv.GV_ACT_GELU), lambda: gv.gv_dense_rows_backward(g, x, w[:5]),
                 lambda: gv.gv_dense_rows_backward(g, x[:4], w), lambda: gv.gv_dense_rows_backward(g.clone().requires_grad_(), x, w)):
        with pytest.raises(ValueError):
            call()
    square = torch.zeros(5, 5, device="cuda")
    with pytest.raises(gv.GvError):
        gv.gv_dense_rows(square, torch.zeros(5, 5, device="cuda"), out=square)
    with pytest.raises(gv.GvError):
        gv.gv_dense_rows(x, w, act=7)


# ------------------------------------------------------------------------------------------------ values

SHAPES = [(1, 1, 1, 0, 0), (1, 512, 2048, 0, 0), (3, 77, 19, 1, 1), (16, 4096, 100, 0, 0), (17, 130, 33, 3, 1), (33, 1001, 65, 0, 0), (64, 357, 500, 2, 0),
          (65, 357, 501, 0, 0), (100, 64, 64, 8, 0), (257, 40, 300, 1, 1), (1021, 357, 500, 0, 0), (2, 16384, 3, 0, 0), (130, 5, 16384, 0, 0),
          (300, 8200, 130, 0, 0), (2048, 256, 1100, 0, 0), (4100, 33, 4100, 0, 0),
          # whole pieces, in all kinds of whole and broken steps, with few and many tiles
          (4104, 520, 1032, 0, 0), (8200, 72, 2056, 0, 0), (1000, 2056, 2048, 8, 8), (3000, 136, 3000, 0, 0), (4100, 200, 4104, 24, 0), (70, 8, 16384, 0, 0)]


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,outs,pad,shift", SHAPES)
def test_layer(gv, kind, rows, cols, outs, pad, shift):
    import torch

    rng = np.random.default_rng(rows + outs)
    x, x64 = make_rows(torch, rng, rows, cols, kind, pad, shift)
    w, w64 = make_rows(torch, rng, outs, cols, kind, pad, shift, cols ** -0.5)
    b, b64 = make_rows(torch, rng, 1, outs, kind, 0, shift)
    r, r64 = make_rows(torch, rng, rows, outs, kind, pad, shift)
    b, b64 = b[0], b64[0]
    for act, bias, residual in (("none", False, False), ("relu", True, False), ("gelu", True, True), ("silu", False, True)):
        args = dict(act=ACTS[act], keep_pre=act != "none")
        got = gv.gv_dense_rows(x, w, b if bias else None, r if residual else None, **args)
        z, y, off_z, off_y = forward(torch, x64, w64, b64 if bias else None, r64 if residual else None, act, kind)
        within(got.out, y, off_y)
        if act != "none":
            within(got.pre, z, off_z)
        wide = torch.full((rows, outs + 3), 7.0, dtype=x.dtype, device="cuda")
        again = gv.gv_dense_rows(x, w, b if bias else None, r if residual else None, act=ACTS[act], out=wide[:, 1:outs + 1])
        assert torch.equal(again.out, got.out) and (wide[:, 0] == 7).all() and (wide[:, outs + 1:] == 7).all()  # the same bits, and no more
        if residual:
            mine = r.clone()
            assert torch.equal(gv.gv_dense_rows(x, w, b if bias else None, mine, act=ACTS[act], out=mine).out, got.out)


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,outs,pad,shift", SHAPES + [(5000, 17, 9, 0, 0), (40_000, 64, 96, 0, 0), (300, 33, 515, 1, 1), (90, 20, 1031, 0, 0)])
def test_gradients(gv, kind, rows, cols, outs, pad, shift):
    import torch

    rng = np.random.default_rng(rows + outs)
    rel, least = rounding(kind)
    x, x64 = make_rows(torch, rng, rows, cols, kind, pad, shift)
    w, w64 = make_rows(torch, rng, outs, cols, kind, pad, shift, cols ** -0.5)
    g, g64 = make_rows(torch, rng, rows, outs, kind, pad, shift)
    for act in ACTS:
        pre, pre64 = make_rows(torch, rng, rows, outs, kind, pad, shift) if act != "none" else (None, torch.zeros_like(g64))
        slope = slope_of(torch, pre64, act)
        gz = g64 * slope
        off = torch.zeros_like(gz) if act in ("none", "relu") else g64.abs() * ((pre64.abs() + 8) * 2 * U) + U * gz.abs()
        off_t = off if act in ("none", "relu") else off + (gz.abs() + off) * rel + least
        got = gv.gv_dense_rows_backward(g, x, w, pre, act=ACTS[act], keep_bias=True)
        want = product(torch, gz, w64.t())
        bound = product(torch, off_t, w64.t().abs()) + outs * 2 * U * product(torch, gz.abs() + off_t, w64.t().abs())
        within(got.x, want, bound + (want.abs() + bound) * rel + least)
        want = product(torch, gz.t(), x64.t())
        bound = product(torch, off_t.t(), x64.t().abs()) + rows * 2 * U * product(torch, (gz.abs() + off_t).t(), x64.t().abs())
        within(got.weight, want, bound + (want.abs() + bound) * rel + least)
        bound = off.sum(0) + rows * U * (gz.abs() + off).sum(0)
        within(got.bias, gz.sum(0), bound + (gz.sum(0).abs() + bound) * rel + least)
        for keep in (dict(keep_x=False), dict(keep_weight=False), dict(keep_x=False, keep_weight=False)):
            some = gv.gv_dense_rows_backward(g, x, w, pre, act=ACTS[act], keep_bias=True, **keep)
            for name in ("x", "weight", "bias"):
                one = getattr(some, name)
                assert (one is None) == (not keep.get("keep_" + name, True))
                assert one is None or torch.equal(one, getattr(got, name))  # the same bits, alone or not


@gpu
def test_gradients_against_differences(gv):
    """The product is bilinear: in whole numbers <dense(x + d, w) - dense(x, w), g> = <d, grad_x> exactly, and likewise for weight and bias."""
    import torch

    rng = np.random.default_rng(4)
    whole = lambda *shape: torch.from_numpy(rng.integers(-3, 4, shape).astype(np.float32)).cuda()  # noqa: E731
    for rows, cols, outs in ((9, 30, 17), (700, 70, 300)):
        x, w, b, g, dx, dw, db = whole(rows, cols), whole(outs, cols), whole(outs), whole(rows, outs), whole(rows, cols), whole(outs, cols), whole(outs)
        grads = gv.gv_dense_rows_backward(g, x, w, keep_bias=True)
        base = gv.gv_dense_rows(x, w, b).out.double()
        dot = lambda a, b: (a.double() * b.double()).sum().item()  # noqa: E731
        assert dot(gv.gv_dense_rows(x + dx, w, b).out.double() - base, g) == dot(dx, grads.x)
        assert dot(gv.gv_dense_rows(x, w + dw, b).out.double() - base, g) == dot(dw, grads.weight)
        assert dot(gv.gv_dense_rows(x, w, b + db).out.double() - base, g) == dot(db, grads.bias)
    # and through an activation: central differences in fp32, steps of 2^-5 along a direction (terms of the second order cancel; the
    # third's share is below 2^-10 of the sizes, far above the rounding of the two results)
    rows, cols, outs = 40, 24, 50
    x, w, g, d = (torch.randn(*s, device="cuda") for s in ((rows, cols), (outs, cols), (rows, outs), (rows, cols)))
    w /= cols ** 0.5
    h = 2.0 ** -5
    for act in (2, 3):
        kept = gv.gv_dense_rows(x, w, act=act, keep_pre=True)
        grads = gv.gv_dense_rows_backward(g, x, w, kept.pre, act=act)
        up, down = (gv.gv_dense_rows(x + s * h * d, w, act=act).out.double() for s in (1, -1))
        moved = ((up - down) / (2 * h) * g.double()).sum().item()
        along = (d @ w.t()).double()
        third = (h * h / 6 * 3 * along.abs() ** 3 * g.double().abs()).sum().item()  # |act'''| < 3
        assert abs(moved - (d.double() * grads.x.double()).sum().item()) < third + 1e-4 * g.abs().sum().item()


@gpu
def test_no_rows(gv):
    import torch

    x, w, g = (torch.zeros(*s, device="cuda") for s in ((0, 8), (6, 8), (0, 6)))
    assert gv.gv_dense_rows(x, w).out.shape == (0, 6)
    grads = gv.gv_dense_rows_backward(g, x, w, torch.zeros(0, 6, device="cuda"), act=gv.GV_ACT_SILU, keep_bias=True)
    assert grads.x.shape == (0, 8) and not grads.weight.any() and not grads.bias.any()


@gpu
@pytest.mark.parametrize("rows", [5, 200])
def test_what_is_not_finite_stays_where_it_belongs(gv, rows):
    """inf and NaN of one row, column or k reach the results that they are part of, and no others; what lies behind a row's end reaches none."""
    import torch

    cols, outs = 45, 70
    flat = torch.full((rows, 64), float("nan"), device="cuda")
    x = flat[:, :cols]
    x.copy_(torch.randn(rows, cols))
    w = torch.randn(outs, cols, device="cuda")
    x[2, 3], w[7, 5] = float("inf"), float("nan")
    got = gv.gv_dense_rows(x, w, act=gv.GV_ACT_RELU, keep_pre=True)
    bad = ~torch.isfinite(got.pre)
    want = torch.zeros(rows, outs, dtype=torch.bool, device="cuda")
    want[2], want[:, 7] = True, True
    assert torch.equal(bad, want)
    g = torch.randn(rows, outs, device="cuda")
    g[1, 4] = float("nan")
    grads = gv.gv_dense_rows_backward(g, x[:, :].nan_to_num(posinf=1.0), w.nan_to_num(), keep_bias=True)
    assert torch.equal(torch.isnan(grads.x).any(1).nonzero().view(-1), torch.tensor([1], device="cuda"))
    assert torch.equal(torch.isnan(grads.weight).any(1).nonzero().view(-1), torch.tensor([4], device="cuda"))
    assert torch.equal(torch.isnan(grads.bias).nonzero().view(-1), torch.tensor([4], device="cuda"))


@gpu
def test_far_offsets(gv):
    """Rows that take more than 2^32 values."""
    import torch

    rows, cols = (1 << 22) + 77, 1024
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[rows - 1] = 1
    x[rows - 200, 5] = 2
    w = torch.eye(8, cols, dtype=torch.bfloat16, device="cuda") * 3
    out = gv.gv_dense_rows(x, w).out
    assert out[rows - 1].tolist() == [3.0] * 8 and out[rows - 200].tolist() == [0.0] * 5 + [6.0] + [0.0] * 2 and out.float().sum().item() == 30
    g = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    g[rows - 1, 1], g[0, 0] = 1, 1
    grads = gv.gv_dense_rows_backward(g, x, w, keep_bias=True)
    assert grads.x[rows - 1, 1].item() == 3 and grads.x[0, 0].item() == 3 and grads.x.float().abs().sum().item() == 6
    assert (grads.weight[1] == 1).all() and grads.weight.float().sum().item() == cols and grads.bias.tolist() == [1.0, 1.0] + [0.0] * 6


@gpu
def test_as_many_rows_as_there_may_be(gv):
    """2^31 rows of one column, of whole numbers: what is rounded is exact in fp32, here and there."""
    import torch

    rows, piece = 1 << 31, 1 << 20
    x = torch.arange(piece, device="cuda").remainder(251).to(torch.bfloat16).repeat(rows // piece).view(rows, 1)
    w = torch.full((1, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    out = gv.gv_dense_rows(x, w, residual=x, act=gv.GV_ACT_RELU).out
    assert all(torch.equal(o, 3 * i) for o, i in zip(out.chunk(64), x.chunk(64)))
    out.zero_()
    out[rows - 1], out[rows // 2], out[5] = 1.0, 2.0, 4.0
    grads = gv.gv_dense_rows_backward(out, x, w, keep_weight=False, keep_bias=True)
    assert grads.bias.item() == 7.0 and sum(int(g.count_nonzero()) for g in grads.x.chunk(64)) == 3
    assert [grads.x[i, 0].item() for i in (5, rows // 2, rows - 1)] == [8.0, 4.0, 2.0]


@gpu
def test_many_rows_of_few_results(gv):
    """More tiles of 32 x 64 than one launch takes, of whole numbers: every sum is exact."""
    import torch

    rows, cols, piece = (1 << 29) + 3, 33, 1 << 16
    some = torch.randint(-3, 4, (piece, cols), device="cuda").float()
    x, w = some.repeat(rows // piece + 1, 1)[:rows], torch.arange(1.0, cols + 1, device="cuda").view(1, cols)
    want = product(torch, some.double(), w.double()).float()
    out = gv.gv_dense_rows(x, w, residual=x[:, 5:6]).out
    want += some[:, 5:6]
    assert all(torch.equal(o, want[:o.shape[0]]) for o in out.split(piece))
    grads = gv.gv_dense_rows_backward(out, x, w, keep_weight=False)
    assert all(torch.equal(g, want[:g.shape[0]] * w) for g in grads.x.split(piece))


@gpu
@pytest.mark.parametrize("rows", [7, 300, 3000])
def test_captured_and_replayed(gv, rows):
    import torch

    rng = np.random.default_rng(1)
    cols, outs = 600, 90
    x, w, g = (torch.zeros(*s, device="cuda") for s in ((rows, cols), (outs, cols), (rows, outs)))

    def step():
        got = gv.gv_dense_rows(x, w, act=gv.GV_ACT_GELU, keep_pre=True)
        return got.out, *gv.gv_dense_rows_backward(g, x, w, got.pre, act=gv.GV_ACT_GELU, keep_bias=True)

    step()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs_of = step()
        graphs.append((graph, outs_of))
    for _ in range(4):
        for t in (x, w, g):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32)))
        for graph, _ in graphs:
            graph.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = step()
        torch.cuda.current_stream().wait_stream(side)
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, eager))


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,outs", [(1, 40, 24), (33, 40, 24), (700, 96, 160), (5000, 64, 264)])
def test_slices_of_one_buffer(gv, kind, rows, cols, outs):
    """A layer's result and what it is taken of side by side in one buffer: the same bits as apart, and nothing else is written."""
    import torch

    rng = np.random.default_rng(rows)
    buf, _ = make_rows(torch, rng, rows, 2 * cols + 2 * outs, kind)
    before = buf.clone()
    w, _ = make_rows(torch, rng, outs, cols, kind, 0, 0, cols ** -0.5)
    x, grad_x, out, g = buf.split([cols, cols, outs, outs], 1)
    want = gv.gv_dense_rows(x.clone(), w, residual=g.clone(), act=gv.GV_ACT_SILU).out
    assert torch.equal(gv.gv_dense_rows(x, w, residual=g, act=gv.GV_ACT_SILU, out=out).out, want)
    assert torch.equal(buf[:, :2 * cols], before[:, :2 * cols]) and torch.equal(g, before[:, 2 * cols + outs:])
    index = torch.arange(rows, device="cuda").flip(0)
    assert torch.equal(gv.gv_lookup_rows(x, index, out=grad_x), before[:, :cols].flip(0))
    back = gv.gv_lookup_rows_backward(g, index, rows, out=out)
    assert torch.equal(back, before[:, 2 * cols + outs:].flip(0)) and torch.equal(x, before[:, :cols])


@gpu
@pytest.mark.parametrize("rows", [60, 2000, 70_000])
def test_gelu_in_full_precision(gv, rows):
    """Of one column and a weight of 1 z is x itself, so what is off is gelu.  Below |z| = 1/4 its second factor is 1/2 and a small part, a
    sum rounded once (u of it) whose part is off by some units, 6 u of a fifth of it; the product is rounded once more: 3.2 u.  Elsewhere the
    factor's tail passes through a power of 2 (2 u and the rounding of what makes it exact, u), a reciprocal (2 u, which the
    polynomial passes on) and three products and sums with coefficients of both signs (6 u): 12 u, with the last rounding 13.  The
    slope, at most 1.13, adds up the factor and z times the bell curve, at most 0.25: 4 u."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.cat([s * torch.randn(rows // 4 + 1, 1, device="cuda", generator=gen) for s in (0.05, 0.5, 2.0, 5.0)])[:rows]
    z.clamp_(min=-13.0)
    z[:7, 0] = torch.tensor([0.0, -0.0, 1.0, -1.0, 0.99999994, 1e-30, -13.0])
    z[7:10, 0] = torch.tensor([20.0, 1e30, -12.999])
    one, z64 = torch.ones(1, 1, device="cuda"), z.double()
    got, want = gv.gv_dense_rows(z, one, act=gv.GV_ACT_GELU).out, act_of(torch, z64, "gelu")
    within(got, want, want.abs() * torch.where(z64.abs() <= 0.25, 3.2, 13.0) * U + 2.0 ** -126)
    grads = gv.gv_dense_rows_backward(torch.ones_like(z), z, one, z, act=gv.GV_ACT_GELU, keep_weight=False)
    within(grads.x, slope_of(torch, z64, "gelu"), torch.full_like(z64, 4 * U))
    wild = torch.tensor([[float("inf")], [float("nan")], [-1e30], [-40.0]], device="cuda")
    assert torch.equal(gv.gv_dense_rows(wild, one, act=gv.GV_ACT_GELU).out.nan_to_num(nan=5.0, posinf=7.0).abs(), torch.tensor([[7.0], [5.0], [0.0], [0.0]], device="cuda"))


def test_no_kernel_of_these_operators_spills(gv):
    """Those whose operands pass through registers (k_product) included: every kernel of a layer, of rows by index and of the selection."""
    from test_kernel_registers import code_objects, kernels_of

    with open(gv.LIB_PATH, "rb") as f:
        data = f.read()
    of = ("k_product", "k_join_product", "k_slope", "k_join_bias", "k_lookup", "k_copy_rows", "k_grad_few", "k_rank", "_digits", "k_sum_runs", "k_join_runs", "k_select")
    found = {k[".name"]: k for elf in code_objects(data) for k in kernels_of(elf) if any(name in k[".name"] for name in of)}
    assert sum("9k_productI" in name for name in found) == 3 * 2 * 3  # along or turned operands, tiles of 256 and 128, three types
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
