"""Rows by index and their gradient, against plain float64 arithmetic.

Tolerances (u = 2^-24, half a unit in the last place of fp32).  A looked-up value is one product in fp32 (u), rounded once more
where the result's type is shorter (2^-8 or 2^-11; 2^-25 near half's smallest).  A sum of n rows passes through at most
n additions in fp32, each off by at most u of what it adds up to: n u of the sum of the values' sizes; then a product, an
addition of what was there, and the rounding of the result's type."""
import ctypes
import os

import numpy as np
import pytest

U = 2.0 ** -24
gpu = pytest.mark.gpu


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
    return {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}[kind]


def make_rows(torch, rng, rows, cols, kind, pad=0, shift=0):
    """(tensor on the GPU whose rows lie `pad` values apart and start `shift` values after an allocation, float64 copy)"""
    x = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32))
    flat = torch.zeros(shift + rows * (cols + pad) + 1, dtype=types(torch)[kind], device="cuda")
    t = torch.as_strided(flat, (rows, cols), (cols + pad, 1), shift)
    t.copy_(x)
    return t, t.double().cpu().numpy()


def make_index(torch, rng, count, rows, form, none=0.05):
    """(tensor on the GPU, int64 copy); every twentieth names no row, one way or another"""
    i = (rows * rng.random(count) ** 3).astype(np.int64) if rows else np.zeros(count, np.int64)
    i = np.minimum(i, max(0, rows - 1))
    out = rng.random(count) < none if rows else np.ones(count, bool)
    i[out] = rng.choice([-1, rows, 2**31 - 1, -2**31] + ([2**32, 2**40, -2**63] if form == "i64" else []), out.sum())
    if form == "pair":
        pairs = torch.from_numpy(np.stack([rng.integers(0, max(1, rows), count), i], 1).astype(np.int32)).cuda()
        return pairs[:, 1], i
    return torch.from_numpy(i.astype(np.int64 if form == "i64" else np.int32)).cuda(), i


def looked_up(table, i, scale):
    named = (i >= 0) & (i < table.shape[0])
    out = np.zeros((i.size, table.shape[1]))
    out[named] = table[i[named]] * scale
    return out


def added_up(grad, i, rows, scale, there=None):
    """(sums, sums of sizes, number of rows in each)"""
    named = (i >= 0) & (i < rows)
    out, size, n = np.zeros((rows, grad.shape[1])), np.zeros((rows, grad.shape[1])), np.zeros(rows)
    np.add.at(out, i[named], grad[named])
    np.add.at(size, i[named], np.abs(grad[named]))
    np.add.at(n, i[named], 1)
    return out * scale + (0 if there is None else there), size * abs(scale), n


def within(got, want, bound):
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))


# ------------------------------------------------------------------------------------------------ refusals, on the CPU


def test_refusals_need_no_device(gv):
    import torch

    L = gv.load()
    at = ctypes.c_void_p(1 << 20)
    far = ctypes.c_void_p(1 << 30)
    ok = dict(count=4, index=at, index_stride=1, index_type=gv.GV_I32, rows=10, cols=8, type=gv.GV_F32, table=far, table_stride=8,
              scale=1.0, out_type=gv.GV_F32, out=ctypes.c_void_p(1 << 25), out_stride=8, stream=None)
    for bad, word in [(dict(count=2**31 + 1), "2^31"), (dict(rows=2**31 + 1), "2^31"), (dict(cols=0), "columns"), (dict(cols=16385), "columns"),
                      (dict(type=6), "type"), (dict(type=-1), "type"), (dict(out_type=gv.GV_I8), "out_type"), (dict(index_type=gv.GV_F32), "index_type"),
                      (dict(index=None), "null index"), (dict(index=ctypes.c_void_p(2)), "aligned"), (dict(table=None), "null table"),
                      (dict(out=None), "null out"), (dict(table_stride=7), "stride"), (dict(out_stride=7), "stride"), (dict(out=far), "overlaps"),
                      (dict(out=ctypes.c_void_p((1 << 30) + 9 * 32)), "overlaps"), (dict(type=gv.GV_I32, out_type=gv.GV_F32), "copied"),
                      (dict(type=gv.GV_I64, out_type=gv.GV_I64, scale=2.0), "copied"), (dict(index_stride=2**41), "stride")]:
        assert L.gv_lookup_rows(*{**ok, **bad}.values()) == gv.GV_EINVAL, bad
        assert word in L.gv_last_error(None).decode(), (bad, L.gv_last_error(None))
    assert L.gv_lookup_rows(*{**ok, "count": 0, "index": None}.values()) == gv.GV_OK
    ok = dict(count=4, index=at, index_stride=1, index_type=gv.GV_I64, rows=10, cols=8, type=gv.GV_F32, grad=far, grad_stride=8, scale=1.0,
              add=0, out_type=gv.GV_F32, out=ctypes.c_void_p(1 << 25), out_stride=8, workspace=None, bytes=0, stream=None)
    for bad, word in [(dict(count=2**31 + 1), "2^31"), (dict(cols=0), "columns"), (dict(type=gv.GV_I8), "type"), (dict(out_type=gv.GV_I32), "out_type"),
                      (dict(grad=None), "null grad"), (dict(out=None), "null out"), (dict(out=far), "overlaps"), (dict(index=ctypes.c_void_p(4)), "aligned"),
                      (dict(grad_stride=7), "stride"), (dict(out_stride=7), "stride"), (dict(count=5000), "workspace"),
                      (dict(count=5000, workspace=ctypes.c_void_p(1 << 34), bytes=1000), "needed")]:
        assert L.gv_lookup_rows_backward(*{**ok, **bad}.values()) == gv.GV_EINVAL, bad
        assert word in L.gv_last_error(None).decode(), (bad, L.gv_last_error(None))
    assert L.gv_lookup_rows_backward(*{**ok, "rows": 0}.values()) == gv.GV_OK
    assert L.gv_lookup_rows_backward(*{**ok, "count": 0, "add": 1}.values()) == gv.GV_OK
    with pytest.raises(gv.GvError):
        gv.gv_lookup_rows_workspace(2**31 + 1, 10, 10)
    assert gv.gv_lookup_rows_workspace(100, 10**6, 128) == 0
    if not torch.cuda.is_available():
        with pytest.raises(ValueError):
            gv.gv_lookup_rows(torch.zeros(3, 4), torch.zeros(2, dtype=torch.int64))


@gpu
def test_refusals_of_tensors(gv):
    import torch

    table, index = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call in (lambda: gv.gv_lookup_rows(table, index.float()), lambda: gv.gv_lookup_rows(table, index.cpu()), lambda: gv.gv_lookup_rows(table, index.view(2, 2)),
                 lambda: gv.gv_lookup_rows(table.t(), index), lambda: gv.gv_lookup_rows(table, index, out=torch.zeros(5, 8, device="cuda")),
                 lambda: gv.gv_lookup_rows(table, index, out_type=torch.int32), lambda: gv.gv_lookup_rows(table.int(), index, out_type=torch.float32),
                 lambda: gv.gv_lookup_rows(table.requires_grad_(), index), lambda: gv.gv_lookup_rows_backward(table[:4].detach(), index[:3], 10),
                 lambda: gv.gv_lookup_rows_backward(torch.zeros(4, 8, device="cuda"), index, 10, add=True),
                 lambda: gv.gv_lookup_rows_backward(torch.zeros(4, 8, device="cuda", requires_grad=True), index, 10),
                 lambda: gv.gv_lookup_rows_backward(torch.zeros(4, 8, device="cuda"), index, 10, out_type=torch.int8)):
        with pytest.raises(ValueError):
            call()
    table = table.detach()
    with pytest.raises(gv.GvError):
        gv.gv_lookup_rows(table, index, out=table[6:])
    with pytest.raises(gv.GvError):
        gv.gv_lookup_rows(table.int(), index, scale=2.0)
    out = torch.zeros(4, 8, device="cuda")
    version = out._version
    gv.gv_lookup_rows(table, index, out=out)
    assert out._version > version
    with torch.no_grad():
        gv.gv_lookup_rows(table.clone().requires_grad_(), index)


# ------------------------------------------------------------------------------------------------ values


@gpu
@pytest.mark.parametrize("kind,out_kind", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("count,rows,cols,form,pad,shift", [
    (1, 1, 1, "i64", 0, 0), (5, 3, 7, "i32", 0, 1), (64, 1000, 128, "pair", 0, 0), (0, 10, 16, "i32", 0, 0), (9, 0, 16, "i64", 0, 0),
    (1000, 77, 357, "i32", 5, 3), (333, 50, 1001, "pair", 1, 1), (3, 5, 16384, "i64", 0, 0), (20000, 4096, 32, "i64", 8, 0)])
def test_lookup(gv, kind, out_kind, count, rows, cols, form, pad, shift):
    import torch

    rng = np.random.default_rng(count + cols)
    table, t64 = make_rows(torch, rng, rows, cols, kind, pad, shift)
    index, i = make_index(torch, rng, count, rows, form)
    rel, least = rounding(out_kind)
    for scale in (1.0, 11.5):
        got = gv.gv_lookup_rows(table, index, scale=scale, out_type=types(torch)[out_kind])
        want = looked_up(t64, i, np.float64(np.float32(scale)))
        assert got.dtype is types(torch)[out_kind] and tuple(got.shape) == (count, cols)
        within(got.double().cpu().numpy(), want, np.abs(want) * (U + rel) * 1.01 + least)
        if kind == out_kind and scale == 1.0:
            assert np.array_equal(got.double().cpu().numpy(), want)


@gpu
@pytest.mark.parametrize("name", ["float32", "float16", "uint8", "int8", "bool", "int32", "int64"])
def test_lookup_copies_bits(gv, name):
    import torch

    rng = np.random.default_rng(5)
    dtype = getattr(torch, name)
    size = torch.empty((), dtype=dtype).element_size()
    raw = rng.integers(0, 2 if name == "bool" else 256, (50, 37 * size)).astype(np.uint8)  # NaNs with any bits among them
    table = torch.from_numpy(raw).cuda().view(dtype)
    index = torch.from_numpy(rng.integers(0, 50, 80)).cuda()
    wide = torch.zeros(80, 41, dtype=dtype, device="cuda")
    out = gv.gv_lookup_rows(table, index, out=wide[:, 2:39])
    assert torch.equal(out.contiguous().view(torch.uint8), table[index].view(torch.uint8))
    assert torch.equal(gv.gv_lookup_rows(table, index).view(torch.uint8), table[index].view(torch.uint8))
    assert not wide[:, :2].any() and not wide[:, 39:].any()
    missing = gv.gv_lookup_rows(table, torch.tensor([-1, 50], device="cuda"))
    assert not missing.view(torch.uint8).any()


GRADS = [(1, 1, 1, "i64", 0, 0), (7, 3, 5, "i32", 1, 1), (0, 100, 16, "i64", 0, 0), (50, 0, 16, "i32", 0, 0), (997, 5003, 353, "i64", 0, 0),
         (1024, 40000, 32, "pair", 0, 0), (1025, 17, 128, "i32", 0, 0), (3000, 100000, 64, "i64", 3, 1), (16384, 900, 600, "i32", 0, 0),
         (16385, 2047, 128, "pair", 0, 0), (20001, 2048, 40, "i64", 0, 0), (60000, 70000, 9, "i32", 0, 0), (40000, 1, 24, "i64", 0, 0),
         (30000, 5_000_000, 3, "i64", 0, 0), (1500, 40, 8200, "i32", 0, 0), (1024, 5, 1100, "i64", 7, 0),
         (700, 50, 515, "i64", 0, 0), (6000, 300, 1031, "i32", 1, 1), (17_000, 900, 519, "i64", 0, 0)]  # a last part of few columns


@gpu
@pytest.mark.parametrize("kind,out_kind", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("count,rows,cols,form,pad,shift", GRADS)
def test_gradient(gv, kind, out_kind, count, rows, cols, form, pad, shift):
    import torch

    rng = np.random.default_rng(count + 3 * cols)
    grad, g64 = make_rows(torch, rng, count, cols, kind, pad, shift)
    index, i = make_index(torch, rng, count, rows, form)
    rel, least = rounding(out_kind)
    scale = np.float64(np.float32(0.7))
    dtype = types(torch)[out_kind]
    # every row is written, whatever was there; nothing between the rows is
    wide = torch.full((rows, cols + pad), float("nan"), dtype=dtype, device="cuda")
    got = gv.gv_lookup_rows_backward(grad, index, rows, scale=scale, out=wide[:, :cols])
    want, size, n = added_up(g64, i, rows, scale)
    bound = size * (n[:, None] + 1) * U * 1.01 + np.abs(want) * rel * 1.01 + least
    within(got.double().cpu().numpy(), want, bound)
    assert torch.isnan(wide[:, cols:]).all()
    again = gv.gv_lookup_rows_backward(grad, index, rows, scale=scale, out_type=dtype)
    assert torch.equal(again, got)  # the same bits
    there, t64 = make_rows(torch, rng, rows, cols, out_kind, pad, shift)
    want, size, n = added_up(g64, i, rows, scale, t64)
    before = there.clone()
    out = gv.gv_lookup_rows_backward(grad, index, rows, scale=scale, out=there, add=True)
    assert out is there
    bound = size * (n[:, None] + 1) * U * 1.01 + np.abs(want) * (U + rel) * 1.01 + least
    bound[n == 0] = 0
    within(there.double().cpu().numpy(), want, bound)
    assert torch.equal(there[torch.from_numpy(n == 0).cuda()], before[torch.from_numpy(n == 0).cuda()])


@gpu
@pytest.mark.parametrize("count", [1000, 10_000, 200_000])
@pytest.mark.parametrize("shape", ["one row", "all different", "two hubs", "nothing", "runs of 7"])
def test_gradient_of_any_distribution(gv, count, shape):
    """Integers up to 8 in fp32: every sum below 2^24 is exact, so results are compared bit for bit."""
    import torch

    rng = np.random.default_rng(count)
    rows, cols = 250_000, 20
    i = {"one row": np.full(count, 249_999), "all different": rng.permutation(rows)[:count], "two hubs": rng.choice([5, 70_000], count),
         "nothing": np.full(count, -1), "runs of 7": rng.permutation(np.arange(count) // 7)}[shape]
    g = rng.integers(-8, 9, (count, cols)).astype(np.float32)
    index, grad = torch.from_numpy(i).cuda(), torch.from_numpy(g).cuda()
    want = added_up(g.astype(np.float64), i, rows, 1.0)[0]
    assert np.array_equal(gv.gv_lookup_rows_backward(grad, index, rows).double().cpu().numpy(), want)
    out = torch.ones(rows, cols, device="cuda")
    gv.gv_lookup_rows_backward(grad, index.int(), rows, scale=-1.0, out=out, add=True)
    assert np.array_equal(out.double().cpu().numpy(), 1 - want)


@gpu
def test_gradient_against_differences(gv):
    """<lookup(table + d) - lookup(table), g> = <d, gradient(g)>: the lookup is linear, so in whole numbers this is exact."""
    import torch

    rng = np.random.default_rng(8)
    table, d = (torch.from_numpy(rng.integers(-4, 5, (300, 33)).astype(np.float32)).cuda() for _ in range(2))
    g = torch.from_numpy(rng.integers(-4, 5, (2000, 33)).astype(np.float32)).cuda()
    index = torch.from_numpy(rng.integers(-3, 303, 2000)).cuda()
    moved = gv.gv_lookup_rows(table + d, index, scale=2.0) - gv.gv_lookup_rows(table, index, scale=2.0)
    back = gv.gv_lookup_rows_backward(g, index, 300, scale=2.0)
    assert (moved.double() * g.double()).sum().item() == (d.double() * back.double()).sum().item()


@gpu
def test_far_offsets(gv):
    """A table of more than 2^32 values, and rows that lie far apart."""
    import torch

    rows, cols = 1 << 21, 2049  # 4.3e9 values of 2 bytes
    table = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    index = torch.tensor([rows - 1, 0, rows - 1, rows // 2 + 1], device="cuda")
    grad = torch.ones(4, cols, dtype=torch.bfloat16, device="cuda")
    gv.gv_lookup_rows_backward(grad, index, rows, out=table, add=True)
    got = gv.gv_lookup_rows(table, index, out_type=torch.float32)
    assert torch.equal(got[:, 0], torch.tensor([2.0, 1.0, 2.0, 1.0], device="cuda")) and (got == got[:, :1]).all()
    many = torch.full((5000,), rows - 1, device="cuda")
    gv.gv_lookup_rows_backward(torch.ones(5000, cols, dtype=torch.bfloat16, device="cuda"), many, rows, out=table)
    assert (gv.gv_lookup_rows(table, index[:2], out_type=torch.float32) == torch.tensor([[4992.0], [0.0]], device="cuda")).all()
    del table
    wide = torch.empty((1 << 32) + 64, dtype=torch.float16, device="cuda")
    two = torch.as_strided(wide, (2, 16), (1 << 32, 1))
    two.copy_(torch.arange(32.0).view(2, 16))
    assert torch.equal(gv.gv_lookup_rows(two, torch.tensor([1, 0], device="cuda")), two.flip(0))


@gpu
def test_as_many_places_as_there_may_be(gv):
    """2^31 places: ones, whose sums stay below 2^24, so fp32 holds them."""
    import torch

    count, rows = 1 << 31, 1000
    index = torch.arange(count, dtype=torch.int32, device="cuda").remainder_(rows)
    table = torch.arange(rows, device="cuda").remainder(251).to(torch.bfloat16).view(rows, 1)
    out = gv.gv_lookup_rows(table, index)
    assert all(torch.equal(o, table[i]) for o, i in zip(out.chunk(64), index.chunk(64)))
    out.fill_(1)
    grad = gv.gv_lookup_rows_backward(out, index, rows, out_type=torch.float32)
    assert torch.equal(grad, torch.full((rows, 1), float(count // rows), device="cuda") + (torch.arange(rows, device="cuda").view(-1, 1) < count % rows))


@gpu
@pytest.mark.parametrize("count", [500, 5000, 50_000])
def test_captured_and_replayed(gv, count):
    """Replays with other inputs, eager work in between, two graphs at once and another stream than the default."""
    import torch

    rng = np.random.default_rng(1)
    rows, cols = 3000, 48
    grad, index = torch.empty(count, cols, device="cuda"), torch.zeros(count, dtype=torch.int64, device="cuda")
    table = torch.randn(rows, cols, device="cuda")
    graphs, outs = [], []
    gv.gv_lookup_rows_backward(gv.gv_lookup_rows(table, index), index, rows)
    for scale in (1.0, -2.0):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((gv.gv_lookup_rows(table, index), gv.gv_lookup_rows_backward(grad, index, rows, scale=scale)))
        graphs.append(g)
    for turn in range(4):
        grad.copy_(torch.from_numpy(rng.integers(-4, 5, (count, cols)).astype(np.float32)))
        index.copy_(torch.from_numpy(rng.integers(-1, rows, count)))
        for g in graphs:
            g.replay()
        i = index.cpu().numpy()
        want = added_up(grad.double().cpu().numpy(), i, rows, 1.0)[0]
        for (got, back), scale in zip(outs, (1.0, -2.0)):
            assert np.array_equal(back.double().cpu().numpy(), scale * want)
            assert np.array_equal(got.cpu().numpy(), looked_up(table.cpu().numpy(), i, 1.0))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = gv.gv_lookup_rows_backward(grad, index, rows)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(eager, outs[0][1])
