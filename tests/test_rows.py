"""The operators on rows: dropout, root-mean-square norm with residual and gradients, 4-bit tables and their scores, against
plain float64 arithmetic on the host.

Tolerances (u = 2^-24, half a unit in the last place of fp32) are sums of the roundings that a call makes:
a sum of squares or products over a row passes through at most 80 additions (64 in a lane, the rest across lanes), so its
square root's inverse is off by at most 40 u and a few roundings more; rounding to bfloat16 or half adds 2^-8 or 2^-11 of
the result (2^-25 near half's smallest).  8-bit and 4-bit codes are compared bit for bit."""
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


# ------------------------------------------------------------------------------------------------ plain forms


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 on arrays of words."""
    w = [np.asarray(c, dtype=np.uint64) for c in np.broadcast_arrays(c0, c1, c2, c3)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * w[0], np.uint64(0xCD9E8D57) * w[2]
        w = [(p1 >> np.uint64(32)) ^ w[1] ^ k[0], p1 & low, (p0 >> np.uint64(32)) ^ w[3] ^ k[1], p0 & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return w


def keep_mask(rows, cols, drop, seed, first_row):
    """(mask, factor)"""
    t = int(np.floor(65536 * drop + 0.5))
    row = (np.arange(rows, dtype=np.uint64) + np.uint64(first_row))[:, None]
    words = philox(row & np.uint64(0xFFFFFFFF), row >> np.uint64(32), np.arange(-(-cols // 8), dtype=np.uint64)[None, :], 5, seed)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    return halves.reshape(rows, -1)[:, :cols] >= t, 65536.0 / (65536 - t)


def test_the_generator_is_the_one_of_training():
    """Known answers of Philox4x32-10 (tests/golden), and the library's initial embeddings use the same words."""
    import oracle

    assert [int(w) for w in philox(0, 0, 0, 0, 0)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    vertex, _ = oracle.init_embeddings(77, 5, 32)
    words = philox(np.arange(5)[:, None], 0, np.arange(8)[None, :], 1, 77)
    want = ((np.stack(words, -1).reshape(5, 32) + 0.5) / 2.0 ** 32 - 0.5) / 32
    assert np.array_equal(vertex, want.astype(np.float32))


def test_dropped_share_is_the_probability():
    for p in (0.1, 0.5, 0.9):
        kept, factor = keep_mask(500, 200, p, 42, 7)
        sigma = np.sqrt(p * (1 - p) / kept.size)
        assert abs(kept.mean() - (1 - p)) < 5 * sigma + 2.0 ** -17
        assert abs(factor * (1 - p) - 1) < 2.0 ** -16 / (1 - p)


def rounding(kind):
    return {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}[kind]


def make_rows(torch, rng, rows, cols, kind, pad=0, shift=0):
    """(tensor on the GPU whose rows lie `pad` values apart and start `shift` values after an allocation, float64 copy)"""
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    x = torch.from_numpy((rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal((rows, 1)))).astype(np.float32))
    flat = torch.zeros(shift + rows * (cols + pad) + 1, dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (rows, cols), (cols + pad, 1), shift)
    t.copy_(x)
    return t, t.double().cpu().numpy()


def norm_in_64_bits(x, residual, gain, eps, kept):
    h = x if kept is None else np.where(kept[0], x * kept[1], 0.0)
    h = h if residual is None else residual + h
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h, rstd, h * rstd * gain


def grads_in_64_bits(grad, h, gain, rstd, grad_sum, kept):
    n = h * rstd
    u = grad * gain
    dh = rstd * (u - n * (u * n).mean(1, keepdims=True))
    dh = dh if grad_sum is None else dh + grad_sum
    return (dh if kept is None else np.where(kept[0], dh * kept[1], 0.0)), dh, (grad * n).sum(0)


def in_8_bits(x, residual, gain):
    """Codes in fp32 arithmetic, step by step, and the step."""
    h = x.astype(np.float32)
    h = h if residual is None else residual.astype(np.float32) + h
    v = h * gain.astype(np.float32)
    a = np.abs(v).max(1, keepdims=True)
    step = a * np.float32(1 / 127)
    up = np.where(a >= np.float32(2.0 ** -100), np.float32(1) / np.maximum(step, np.float32(2.0 ** -120)), np.float32(0))
    return np.rint(v * up).astype(np.int8), np.where(up > 0, step, np.float32(0))[:, 0]


def table_in_4_bits(x, group):
    """(codes int[rows][cols], scales float32[rows][groups]) in fp32 arithmetic, step by step."""
    import torch

    rows, cols = x.shape
    groups = -(-cols // group)
    w = np.zeros((rows, groups * group), dtype=np.float32)
    w[:, :cols] = x
    w = w.reshape(rows, groups, group)
    a = np.abs(w).max(2)
    scale = torch.from_numpy(np.where(a >= np.float32(2.0 ** -100), a * np.float32(1 / 7), np.float32(0))).to(torch.bfloat16)
    scale = scale.float().numpy()
    up = np.where(scale > 0, np.float32(1) / np.where(scale > 0, scale, np.float32(1)), np.float32(0))
    return np.clip(np.rint(w * up[:, :, None]), -7, 7).astype(int).reshape(rows, -1)[:, :cols], scale


def packed(codes):
    rows, cols = codes.shape
    wide = np.zeros((rows, 32 * (-(-cols // 32))), dtype=np.uint8)
    wide[:, :cols] = codes & 15
    return wide[:, 0::2] | (wide[:, 1::2] << 4)


def check(got, want, tolerance, what):
    off = np.abs(got.double().cpu().numpy() - want)
    assert np.all(off <= tolerance), (what, float((off / np.maximum(tolerance, 1e-300)).max()), int((off > tolerance).sum()))


# ------------------------------------------------------------------------------------------------ refusals, without a GPU


def test_refusals(gv):
    lib = gv.load()
    a = 1 << 20  # an address that is never followed: every call here is refused before its launch
    u64 = ctypes.c_uint64()

    def drop(rows=4, cols=8, type=0, x=a, xs=8, p=0.1, out=a, outs=8):
        return lib.gv_drop_rows(rows, cols, type, x, xs, p, 1, 0, out, outs, None)

    def norm(rows=4, cols=8, type=0, x=a, xs=8, r=a, rs=8, gain=a, eps=1e-6, p=0.1, s=a, ss=8, ot=0, out=a, outs=8, scale=a,
             rstd=a):
        return lib.gv_norm_rows(rows, cols, type, x, xs, r, rs, gain, eps, p, 1, 0, s, ss, ot, out, outs, scale, rstd, None)

    def back(rows=4, cols=8, type=0, g=a, gs=8, s=a, ss=8, gain=a, rstd=a, d=a, ds=8, p=0.1, x=a, xs=8, r=a, rs=8, gg=a, w=a,
             size=1 << 20):
        return lib.gv_norm_rows_backward(rows, cols, type, g, gs, s, ss, gain, rstd, d, ds, p, 1, 0, x, xs, r, rs, gg, w, size, None)

    def quantize(rows=4, cols=8, type=0, x=a, xs=8, group=32, codes=a, scales=a):
        return lib.gv_quantize_rows(rows, cols, type, x, xs, group, codes, scales, None)

    def score(rows=4, cols=8, group=32, codes=a, scales=a, q=2, type=0, x=a, xs=8, scale=None, out=a, outs=4):
        return lib.gv_score_rows(rows, cols, group, codes, scales, q, type, x, xs, scale, out, outs, None)

    shapes = [dict(cols=0), dict(cols=gv.GV_MAX_ROW_COLS + 1), dict(rows=(1 << 31) + 1), dict(type=-1), dict(type=4)]
    odd = [dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=float("inf"))]
    for call, bad in [
        (drop, shapes + odd + [dict(type=3), dict(x=None), dict(out=None), dict(xs=7), dict(outs=0), dict(xs=(1 << 40) + 1),
                               dict(x=a + 2), dict(out=a + 1)]),
        (norm, shapes + odd + [dict(type=3), dict(x=None), dict(out=None), dict(gain=None), dict(rs=7), dict(ss=7), dict(r=a + 2),
                               dict(ot=1), dict(ot=3, scale=None), dict(ot=3, scale=a + 2), dict(eps=-1.0), dict(rstd=a + 1),
                               dict(eps=float("nan")), dict(eps=float("inf")), dict(gain=a + 2), dict(type=1, x=a + 1, ot=1)]),
        (back, shapes + odd + [dict(type=3), dict(g=None), dict(s=None), dict(gain=None), dict(rstd=None), dict(gs=7), dict(ds=7),
                               dict(xs=7), dict(rs=7), dict(gg=a + 2), dict(rows=0, gg=a + 2), dict(rows=5000, w=None),
                               dict(rows=5000, w=a + 4), dict(rows=5000, size=64)]),
        (quantize, shapes + [dict(type=3), dict(group=0), dict(group=16), dict(group=96), dict(x=None), dict(codes=None),
                             dict(scales=None), dict(codes=a + 8), dict(scales=a + 1), dict(xs=7)]),
        (score, shapes + [dict(group=0), dict(group=48), dict(codes=None), dict(codes=a + 4), dict(scales=None), dict(x=None),
                          dict(out=None), dict(outs=3), dict(xs=7), dict(q=(1 << 16) + 1), dict(type=3, scale=None),
                          dict(type=0, scale=a), dict(type=3, scale=a + 1), dict(x=a + 2)]),
    ]:
        for kw in bad:
            assert call(**kw) == gv.GV_EINVAL, (call.__name__, kw)
            assert lib.gv_last_error(None).decode().startswith("gv_"), kw
    # empty calls need neither addresses nor a GPU
    assert drop(rows=0, x=None, out=None) == norm(rows=0, x=None, out=None, gain=None) == gv.GV_OK
    assert back(rows=0, g=None, s=None, gg=None) == quantize(rows=0, x=None) == gv.GV_OK
    assert score(rows=0, codes=None, outs=0) == score(q=0, x=None) == gv.GV_OK
    assert lib.gv_norm_rows_workspace(10, 0, ctypes.byref(u64)) == gv.GV_EINVAL
    assert lib.gv_norm_rows_workspace(10, 8, None) == gv.GV_EINVAL
    assert lib.gv_norm_rows_workspace(10, 8, ctypes.byref(u64)) == gv.GV_OK and u64.value == 0  # one workgroup: no parts
    assert lib.gv_norm_rows_workspace(5000, 8, ctypes.byref(u64)) == gv.GV_OK and u64.value > 64


def test_refusals_of_tensors(gv):
    import torch

    x = torch.zeros(4, 8)
    for call in (lambda: gv.gv_drop_rows(x, 0.1, 1), lambda: gv.gv_norm_rows(x, torch.ones(8)),
                 lambda: gv.gv_norm_rows_backward(x, x, torch.ones(8), torch.ones(4)), lambda: gv.gv_quantize_rows(x),
                 lambda: gv.gv_score_rows(torch.zeros(3, 16, dtype=torch.uint8), torch.zeros(3, 1, dtype=torch.bfloat16), x)):
        with pytest.raises(ValueError):
            call()


def test_row_kernels_keep_everything_in_registers(gv):
    from test_kernel_registers import code_objects, kernels_of

    with open(gv.LIB_PATH, "rb") as f:
        data = f.read()
    names = ("k_drop", "k_norm", "k_gain_join", "k_score_few", "k_score_many", "k_score_narrow", "k_quantize")
    found = {n: 0 for n in names}
    for elf in code_objects(data):
        for k in kernels_of(elf):
            for n in names:
                if n in k[".name"]:
                    found[n] += 1
                    assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, k[".name"]
    assert all(found.values()), found


# ------------------------------------------------------------------------------------------------ on the GPU

SHAPES = [(1, 1), (1, 128), (3, 7), (5, 8), (257, 31), (64, 32), (100, 64), (33, 96), (1001, 128), (17, 129), (50, 160), (9, 257),
          (12, 352), (300, 357), (7, 512), (5, 513), (6, 1000), (3, 1025), (4, 2048), (2, 2056), (3, 4096), (2, 4099), (2, 8192),
          (1, 8200), (2, 16384), (1, 16383)]


@gpu
@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_dropout(gv, rows, cols, kind):
    import torch

    rng = np.random.default_rng(rows * 131 + cols)
    for pad, shift, p, seed, first in [(0, 0, 0.1, 1, 0), (5, 3, 0.5, 2 ** 64 - 3, 2 ** 32 - 2), (8, 8, 0.0, 9, 2 ** 40), (1, 0, 0.99, 5, 3)]:
        t, x = make_rows(torch, rng, rows, cols, kind, pad, shift)
        got = gv.gv_drop_rows(t, p, seed, first_row=first)
        kept, factor = keep_mask(rows, cols, p, seed, first)
        # one product with a factor that is rounded itself
        want = np.where(kept, x * factor, 0.0)
        rel, least = rounding(kind)
        check(got, want, np.abs(want) * (2.1 * U + 1.01 * rel) + least, (rows, cols, kind, p))
        assert torch.equal(gv.gv_drop_rows(t, p, seed, first_row=first, out=t), got)  # in place


@gpu
def test_dropout_cut_differently_is_the_same(gv):
    import torch

    x = torch.randn(1000, 77, device="cuda")
    x[3, 5] = float("nan")
    x[:, 9] = float("inf")
    whole = gv.gv_drop_rows(x, 0.3, 11, first_row=2 ** 33 - 400)
    parts = [gv.gv_drop_rows(x[lo:lo + 250], 0.3, 11, first_row=2 ** 33 - 400 + lo) for lo in range(0, 1000, 250)]
    assert torch.equal(torch.cat(parts).nan_to_num(7.0), whole.nan_to_num(7.0))
    kept, factor = keep_mask(1000, 77, 0.3, 11, 2 ** 33 - 400)
    assert torch.equal(torch.isinf(whole[:, 9]).cpu(), torch.from_numpy(kept[:, 9]))  # what is dropped is 0, whatever it was
    assert not torch.isnan(whole[:, 9]).any()
    assert not torch.equal(gv.gv_drop_rows(x, 0.3, 12, first_row=2 ** 33 - 400).isinf(), whole.isinf())


def norm_tolerance(kind, want, x, gain, rstd, kept):
    """40 u of the root, six roundings on the way, and those of the addend before the residual may cancel it."""
    rel, least = rounding(kind)
    addend = 0.0 if kept is None else 3 * U * np.abs(x) * kept[1] * rstd * np.abs(gain)
    return np.abs(want) * (48 * U + 1.01 * rel) + addend + least


@gpu
@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_norm(gv, rows, cols, kind):
    import torch

    rng = np.random.default_rng(rows * 7 + cols)
    for pad, shift, residual, p in [(0, 0, True, 0.0), (3, 1, True, 0.25), (8, 8, False, 0.0), (1, 5, False, 0.5)]:
        t, x = make_rows(torch, rng, rows, cols, kind, pad, shift)
        rt, r = make_rows(torch, rng, rows, cols, kind, 2 * pad, shift) if residual else (None, None)
        gain = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).cuda()
        g = gain.double().cpu().numpy()
        kept = keep_mask(rows, cols, p, 17, 5) if p else None
        h, rstd, y = norm_in_64_bits(x, r, g, 1e-5, kept)
        got = gv.gv_norm_rows(t, gain, rt, eps=1e-5, drop=p, seed=17, first_row=5, keep_rstd=True)
        check(got.out, y, norm_tolerance(kind, y, x, g, rstd, kept), ("out", pad, residual, p))
        check(got.rstd, rstd[:, 0], 48 * U * rstd[:, 0], "rstd")
        assert (got.sum is None) == (not residual and not p) and got.scale is None
        if got.sum is not None:
            rel, least = rounding(kind)
            addend = 0.0 if kept is None else 3 * U * np.abs(x) * kept[1]
            check(got.sum, h, np.abs(h) * (2 * U + 1.01 * rel) + addend + least, "sum")
        again = gv.gv_norm_rows(t, gain, rt, eps=1e-5, drop=p, seed=17, first_row=5, keep_rstd=True)
        assert torch.equal(again.out, got.out) and torch.equal(again.rstd, got.rstd)
        if residual:  # the sum takes the residual's place, the result x's
            in_place = gv.gv_norm_rows(t, gain, rt, eps=1e-5, drop=p, seed=17, first_row=5, sum=rt, out=t)
            assert torch.equal(rt, got.sum) and torch.equal(t, got.out) and in_place.out is t


@gpu
@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_norm_in_8_bits(gv, rows, cols, kind):
    import torch

    rng = np.random.default_rng(rows * 3 + cols)
    for pad, shift, residual in [(0, 0, True), (7, 2, False), (8, 0, True)]:
        t, x = make_rows(torch, rng, rows, cols, kind, pad, shift)
        rt, r = make_rows(torch, rng, rows, cols, kind, pad, shift) if residual else (None, None)
        gain = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).cuda()
        codes, step = in_8_bits(x, r, gain.cpu().numpy())
        _, rstd, _ = norm_in_64_bits(x, r, gain.double().cpu().numpy(), 1e-6, None)
        got = gv.gv_norm_rows(t, gain, rt, out_type=torch.int8)
        assert np.array_equal(got.out.cpu().numpy(), codes)
        check(got.scale, step * rstd[:, 0], 50 * U * step * rstd[:, 0], "scale")


@gpu
def test_rows_without_values_and_rows_that_are_not_finite(gv):
    import torch

    for cols in (8, 130, 700, 3000, 9000):
        x = torch.randn(8, cols, device="cuda")
        x[0] = 0.0
        x[1] = 2.0 ** -110
        x[2, cols // 2] = float("inf")
        x[3, cols - 1] = float("nan")
        x[4] = 3e38  # overflows in the sum
        gain = torch.ones(cols, device="cuda")
        got = gv.gv_norm_rows(x, gain, x.clone(), out_type=torch.int8)
        assert (got.out[:5] == 0).all()
        assert got.scale[0] == 0 and got.scale[1] == 0 and torch.isnan(got.scale[2:5]).all()
        assert (got.out[5:].abs().amax(1) == 127).all() and torch.isfinite(got.scale[5:]).all()
        y = gv.gv_norm_rows(x, gain).out
        assert (y[0] == 0).all() and torch.isfinite(y[5:]).all() and torch.isnan(y[3]).all()


@gpu
@pytest.mark.parametrize("rows, cols", SHAPES + [(40_000, 128), (5000, 512), (3000, 357)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_norm_gradients(gv, rows, cols, kind):
    import torch

    rng = np.random.default_rng(rows * 11 + cols)
    rel, least = rounding(kind)
    for pad, shift, further, p in [(0, 0, True, 0.0), (3, 1, True, 0.25), (8, 8, False, 0.0), (1, 5, False, 0.5)]:
        if rows > 2000 and pad == 8:
            continue
        st, h = make_rows(torch, rng, rows, cols, kind, pad, shift)
        gt, grad = make_rows(torch, rng, rows, cols, kind, 2 * pad, shift)
        dt, grad_sum = make_rows(torch, rng, rows, cols, kind, pad, 0) if further else (None, None)
        gain = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).cuda()
        g = gain.double().cpu().numpy()
        rstd = (1 / np.sqrt((h * h).mean(1) + 1e-5)).astype(np.float32)
        kept = keep_mask(rows, cols, p, 23, 2 ** 35) if p else None
        rs = rstd.astype(np.float64)[:, None]
        dx, dh, dg = grads_in_64_bits(grad, h, g, rs, grad_sum, kept)
        args = dict(grad_sum=dt, drop=p, seed=23, first_row=2 ** 35, keep_residual=True)
        got = gv.gv_norm_rows_backward(gt, st, gain, torch.from_numpy(rstd).cuda(), **args)
        # the mean of u n is off by 80 u of the mean of |u n| and a few roundings
        n, u = h * rs, grad * g
        t = rs * (4 * U * np.abs(u) + 88 * U * np.abs(n) * np.abs(u * n).mean(1, keepdims=True)) + 3 * U * np.abs(dh)
        check(got.residual, dh, t + 1.01 * rel * (np.abs(dh) + t) + least, ("residual", pad, p))
        if p:
            t = np.where(kept[0], t * kept[1] + 2 * U * np.abs(dx), 0.0)
        check(got.x, dx, t + 1.01 * rel * (np.abs(dx) + t) + least, ("x", pad, p))
        # rows are added one after the other within parts, and the parts
        check(got.gain, dg, (min(rows, 1100) + 4) * U * np.abs(grad * n).sum(0), ("gain", pad, p))
        again = gv.gv_norm_rows_backward(gt, st, gain, torch.from_numpy(rstd).cuda(), **args)
        assert torch.equal(again.gain, got.gain) and torch.equal(again.x, got.x)
    if not rows % 2:
        only = gv.gv_norm_rows_backward(gt, st, gain, torch.from_numpy(rstd).cuda(), keep_gain=False)
        assert only.gain is None and only.residual is None and only.x.shape == (rows, cols)


@gpu
def test_gradients_against_differences(gv):
    """The change of a weighted sum of both results along a random direction, in float64 by central differences."""
    import torch

    rng = np.random.default_rng(5)
    rows, cols, p, eps, step = 40, 96, 0.3, 1e-3, 1e-5
    x, r, g, a, b, dx, dr, dg = (rng.standard_normal(s) for s in [(rows, cols), (rows, cols), cols] + [(rows, cols)] * 4 + [cols])
    x, r, g, a, b = (v.astype(np.float32).astype(np.float64) for v in (x, r, g, a, b))
    kept = keep_mask(rows, cols, p, 3, 0)

    def loss(s):
        h, _, y = norm_in_64_bits(x + s * dx, r + s * dr, g + s * dg, eps, kept)
        return (a * y).sum() + (b * h).sum()

    want = (loss(step) - loss(-step)) / (2 * step)
    xt, rt, gt, at, bt = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (x, r, g, a, b))
    got = gv.gv_norm_rows(xt, gt, rt, eps=eps, drop=p, seed=3, keep_rstd=True)
    grads = gv.gv_norm_rows_backward(at, got.sum, gt, got.rstd, grad_sum=bt, drop=p, seed=3)
    parts = [(grads.x.double().cpu().numpy(), dx), (grads.residual.double().cpu().numpy(), dr), (grads.gain.double().cpu().numpy(), dg)]
    # 100 u of what is added up; the differences themselves are off by step^2 and 2^-52 / step of it
    assert abs(sum((u * v).sum() for u, v in parts) - want) < (100 * U + 1e-9) * sum(np.abs(u * v).sum() for u, v in parts)


@gpu
def test_gradient_of_the_gain_without_rows(gv):
    import torch

    x, gain = torch.empty(0, 40, device="cuda"), torch.ones(40, device="cuda")
    assert gv.gv_norm_rows(x, gain).out.shape == (0, 40) and gv.gv_drop_rows(x, 0.1, 1).shape == (0, 40)
    grads = gv.gv_norm_rows_backward(x, x, gain, torch.empty(0, device="cuda"))
    assert grads.x.shape == (0, 40) and (grads.gain == 0).all()


TABLES = [(1, 1, 32), (3, 31, 32), (5, 32, 64), (1000, 33, 32), (70, 64, 64), (63, 70, 64), (65, 96, 32), (257, 128, 32),
          (129, 128, 128), (1023, 128, 64), (50, 130, 128), (31, 160, 32), (40, 257, 64), (300, 352, 32), (77, 500, 64),
          (200, 512, 128), (200, 512, 32), (17, 1000, 32), (16, 1024, 128), (9, 2048, 64), (6, 2050, 32), (5, 4096, 128),
          (2, 16384, 128), (3, 16383, 32)]


@gpu
@pytest.mark.parametrize("rows, cols, group", TABLES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_tables_in_4_bits(gv, rows, cols, group, kind):
    import torch

    rng = np.random.default_rng(rows + cols)
    for pad, shift in [(0, 0), (3, 1), (8, 8)]:
        t, x = make_rows(torch, rng, rows, cols, kind, pad, shift)
        if rows > 2:
            t[1] = 0
            x[1] = 0
        codes, scales = table_in_4_bits(x, group)
        got_codes, got_scales = gv.gv_quantize_rows(t, group=group)
        assert np.array_equal(got_scales.float().cpu().numpy(), scales)
        assert np.array_equal(got_codes.cpu().numpy(), packed(codes))
    if rows > 2:
        t[2, cols - 1] = float("nan")
        t[0, 0] = float("inf")
        got_codes, got_scales = gv.gv_quantize_rows(t, group=group)
        assert torch.isnan(got_scales[2, -1]) and torch.isnan(got_scales[0, 0])
        assert torch.isnan(got_scales).sum() == 2
        assert (got_codes[0, :min(group, cols) // 2] == 0).all()


def scores_in_64_bits(codes, scales, group, x):
    """(scores, sums of |w x|, sums of |w|)"""
    w = codes * np.repeat(scales.astype(np.float64), group, axis=1)[:, :codes.shape[1]]
    return x @ w.T, np.abs(x) @ np.abs(w).T, np.abs(w).sum(1)


@gpu
@pytest.mark.parametrize("rows, cols, group", TABLES + [(20_011, 128, 32), (5000, 512, 128), (3001, 32, 32), (9000, 64, 32)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "i8"])
def test_scores(gv, rows, cols, group, kind):
    import torch

    rng = np.random.default_rng(rows * 5 + cols)
    codes = rng.integers(-8, 8, (rows, cols))
    codes[rng.random(rows) < 0.05] = -8
    scale_t = torch.from_numpy(np.exp(rng.standard_normal((rows, -(-cols // group)))).astype(np.float32)).to(torch.bfloat16)
    scales = scale_t.double().numpy()
    codes_t, scale_t = torch.from_numpy(packed(codes)).cuda(), scale_t.cuda()
    for queries, pad, shift in [(1, 0, 0), (2, 3, 1), (3, 0, 0), (4, 0, 0), (5, 8, 8), (8, 1, 0), (16, 0, 4), (17, 0, 0), (40, 4, 4),
                                (64, 0, 0), (70, 1, 1)]:
        if kind == "i8":
            flat = torch.from_numpy(rng.integers(-128, 128, shift + queries * (cols + pad)).astype(np.int8)).cuda()
            t = torch.as_strided(flat, (queries, cols), (cols + pad, 1), shift)
            x_scale = torch.from_numpy(np.exp(rng.standard_normal(queries)).astype(np.float32)).cuda()
            x = t.double().cpu().numpy() * x_scale.double().cpu().numpy()[:, None]
        else:
            t, x = make_rows(torch, rng, queries, cols, kind, pad, shift)
            x_scale = None
        want, sums, weights = scores_in_64_bits(codes, scales, group, x)
        # every group's sum is exact for x in whole numbers (off by half of 2^-30 of twice the largest |x| at most); it is
        # scaled and added with one rounding each, and joined from parts of 8 bits and from lanes with a few more
        groups = scales.shape[1]
        tolerance = (groups + 8) * U * sums + 2.0 ** -28 * np.abs(x).max(1, keepdims=True) * weights[None, :]
        got = gv.gv_score_rows(codes_t, scale_t, t, group=group, scale=x_scale)
        check(got, want, tolerance, (queries, pad))
        wide = torch.full((queries, rows + 5), 7.0, device="cuda")
        assert torch.equal(gv.gv_score_rows(codes_t, scale_t, t, group=group, scale=x_scale, out=wide[:, 2:rows + 2]), got)
        assert (wide[:, :2] == 7).all() and (wide[:, rows + 2:] == 7).all()


@gpu
def test_scores_of_strange_queries_and_tables(gv):
    import torch

    rng = np.random.default_rng(8)
    for rows, cols, queries in [(500, 128, 1), (500, 128, 20), (300, 700, 3), (300, 700, 17)]:
        table = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda()
        table[5, cols - 1] = float("nan")
        table[7] = 0
        codes, scales = gv.gv_quantize_rows(table)
        x = torch.from_numpy(rng.standard_normal((queries, cols)).astype(np.float32)).cuda()
        got = gv.gv_score_rows(codes, scales, x)
        assert torch.isnan(got[:, 5]).all() and (got[:, 7] == 0).all() and torch.isnan(got).sum() == queries
        for q, v in [(0, float("inf")), (queries - 1, float("nan"))]:
            y = x.clone()
            y[q, cols - 1] = v
            bad = gv.gv_score_rows(codes, scales, y)
            assert torch.isnan(bad[q]).all()
            others = [i for i in range(queries) if i != q]
            assert torch.equal(bad[others].nan_to_num(0.0), got[others].nan_to_num(0.0))
        x[0] = 0
        assert (gv.gv_score_rows(codes, scales, x)[0].nan_to_num(0.0) == 0).all()
        x[0] = 1e30 * torch.sign(torch.randn(cols, device="cuda"))
        x[0, 0] = 1e-20
        assert torch.isfinite(gv.gv_score_rows(codes, scales, x)[0, 8:]).all()


@gpu
def test_rows_beyond_32_bits_of_offset(gv):
    """Matrices of more than 2^32 bytes and values: their last rows are those of a call on a slice."""
    import torch

    cols = 1024
    rows = (1 << 22) + 37
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.normal_()
    end = 1000
    tail = x[-end:].clone()
    dropped = gv.gv_drop_rows(x, 0.2, 5, out=torch.empty_like(x))
    assert torch.equal(dropped[-end:], gv.gv_drop_rows(tail, 0.2, 5, first_row=rows - end))
    gain = torch.rand(cols, device="cuda") + 0.5
    got = gv.gv_norm_rows(x, gain, dropped, keep_rstd=True, sum=dropped, out=torch.empty_like(x))
    want = gv.gv_norm_rows(tail, gain, gv.gv_drop_rows(tail, 0.2, 5, first_row=rows - end), keep_rstd=True)
    assert torch.equal(got.out[-end:], want.out) and torch.equal(got.rstd[-end:], want.rstd)
    grads = gv.gv_norm_rows_backward(x, got.sum, gain, got.rstd)
    assert torch.equal(grads.x[-end:], gv.gv_norm_rows_backward(tail, want.sum, gain, want.rstd).x)
    del dropped, got, grads
    codes, scales = gv.gv_quantize_rows(x.view(-1, 128))
    n = codes.shape[0]
    wide = torch.empty(140, dtype=torch.float32, device="cuda").normal_()[:128].view(1, 128)
    slice_codes, slice_scales = gv.gv_quantize_rows(x.view(-1, 128)[-end:])
    assert torch.equal(codes[-end:], slice_codes) and torch.equal(scales[-end:], slice_scales)
    del x
    # 2^25 rows three times over: more than 2^32 bytes of codes
    codes, scales = codes.repeat(3, 1), scales.repeat(3, 1)
    assert codes.numel() > 1 << 32
    for queries in (1, 20):
        q = wide.repeat(queries, 1)
        got = gv.gv_score_rows(codes, scales, q)
        want = gv.gv_score_rows(slice_codes, slice_scales, q)
        assert torch.equal(got[:, n - end:n], want) and torch.equal(got[:, -end:], want)
        assert torch.equal(got[:, :n], got[:, 2 * n:])
        del got


@gpu
def test_on_another_stream_and_in_a_graph(gv):
    import torch

    x, r = torch.randn(500, 128, device="cuda"), torch.randn(500, 128, device="cuda")
    table, gain = torch.randn(3000, 128, device="cuda"), torch.rand(128, device="cuda") + 0.5

    def work():
        codes, scales = gv.gv_quantize_rows(table)
        y = gv.gv_norm_rows(x, gain, r, drop=0.1, seed=4, keep_rstd=True)
        grads = gv.gv_norm_rows_backward(y.out, y.sum, gain, y.rstd, grad_sum=x, drop=0.1, seed=4)
        q = gv.gv_norm_rows(gv.gv_drop_rows(x, 0.5, 9), gain, out_type=torch.int8)
        scores = [gv.gv_score_rows(codes, scales, q.out[:k], scale=q.scale[:k]) for k in (1, 30)]
        return [y.out, y.sum, grads.x, grads.residual, grads.gain, *scores, gv.gv_score_rows(codes, scales, x[:3])]

    want = [t.clone() for t in work()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = work()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        x.mul_(1.5)  # new inputs for the same graph
        want = [t.clone() for t in work()]


@gpu
def test_example_answers_queries(gv):
    """examples/answer_queries.py on the small community graph: the head learns, and a shortlist of a hundred from the 4-bit
    table holds nearly all of the best ten (a table of random codes would hold 2 % of them)."""
    import importlib.util

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_queries.py")
    spec = importlib.util.spec_from_file_location("answer_queries", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run("c4-small", samples=4_000_000, steps=40, queries=4)
    assert r["last_loss"] < 0.9 * r["first_loss"]
    assert r["recall"] > 0.9 and r["table_mb"] * 7 < r["rows_mb"] * 1.01
