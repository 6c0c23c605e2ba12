"""What the operators on rows accept and launch, without a GPU: tests/host_rows_recorder.cpp stands in for the HIP runtime and keeps the
launches.  Addresses are made up and never read."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1903_00757_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc"

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")

F32, BF16, F16 = 0, 1, 2
EINVAL = -1
SIZE = {F32: 4, BF16: 2, F16: 2}
X, W, OUT, PRE, SPACE = (ctypes.c_void_p(i << 42) for i in range(1, 6))  # far apart


class Recorder:
    def __init__(self, path):
        import paper_1903_00757_amd as gv

        self.lib = ctypes.CDLL(path)
        known = gv.load()
        for name in gv.EXPORTS:
            if hasattr(self.lib, name):
                getattr(self.lib, name).argtypes = getattr(known, name).argtypes
                getattr(self.lib, name).restype = getattr(known, name).restype
        self.lib.recorded_kernel.restype = ctypes.c_char_p
        for name in ("count", "blocks", "threads", "rows", "out"):
            getattr(self.lib, "recorded_" + name).restype = ctypes.c_uint64
        for name in ("kernel", "blocks", "threads", "rows", "out", "cut"):
            getattr(self.lib, "recorded_" + name).argtypes = [ctypes.c_uint64]

    def call(self, name, *args):
        """(return code, text of a refusal, launches as dictionaries)"""
        self.lib.recorded_clear()
        rc = getattr(self.lib, name)(*args)
        ask = lambda what, i: getattr(self.lib, "recorded_" + what)(i)  # noqa: E731
        return rc, self.lib.gv_last_error(None).decode() if rc else "", [
            {what: ask(what, i) for what in ("kernel", "blocks", "threads", "rows", "out", "cut")} for i in range(self.lib.recorded_count())]

    def bytes(self, name, *args):
        n = ctypes.c_uint64()
        assert getattr(self.lib, name)(*args, ctypes.byref(n)) == 0
        return n.value


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    out = tmp_path_factory.mktemp("host_rows")
    objects, common = [], [HIPCC, "-std=c++17", "-O1", "-fPIC", "--offload-arch=gfx950", "--cuda-host-only", "-x", "hip", "-Wno-unused-command-line-argument",
                           "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    sources = [os.path.join(CSRC, f) for f in ("gv_rows_api.cpp", "gv_rows.hip", "gv_scores.hip", "gv_lookup.hip", "gv_dense.hip", "gv_select.hip")]
    for src in sources + [os.path.join(ROOT, "tests", "host_rows_recorder.cpp")]:
        objects.append(str(out / (os.path.basename(src) + ".o")))
        subprocess.run([*common, "-c", src, "-o", objects[-1]], check=True, capture_output=True, text=True)
    path = str(out / "rows.so")
    # the device code is left out: its place in the objects has a name, which is given an address that nobody looks at
    wanted = subprocess.run(["nm", "-u", *objects], check=True, capture_output=True, text=True).stdout.split()
    places = [f"-Wl,--defsym={name}=0" for name in wanted if name.startswith("__hip_fatbin")]
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", *places, *objects, "-o", path], check=True, capture_output=True, text=True)
    return Recorder(path)


def check_products(launches, type, rows, stride):
    """Every launch has fewer than 2^32 threads (a launch takes no more), and the products' rows follow one another, all of them."""
    for l in launches:
        assert 0 < l["blocks"] * l["threads"] < 2**32, l
    products = [l for l in launches if b"k_product" in l["kernel"]]
    at = products[0]["out"]
    for l in products:
        assert l["out"] == at, l
        at += l["rows"] * stride * SIZE[type]
    assert sum(l["rows"] for l in products) == rows


SIZES = [(rows, cols, outs) for rows in (65, 1 << 20, (1 << 28) + 5, (1 << 29) - 32, 1 << 29, (1 << 29) + 1, 1 << 30, (1 << 30) + 7, 1 << 31)
         for cols in (1, 8, 33, 64, 193, 256) for outs in (1, 8, 33, 64, 65, 300) if rows * (cols + outs) < 1 << 38]


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("apart", [0, 1])
def test_layers_of_many_rows_can_be_launched(calls, type, apart):
    for rows, cols, outs in SIZES:
        space = calls.bytes("gv_dense_rows_workspace", rows, cols, outs, type)
        rc, text, launches = calls.call("gv_dense_rows", rows, cols, outs, type, X, cols + apart, W, cols + apart, None, 0, None, 0, None, 0, OUT,
                                        outs + apart, SPACE if space else None, space, None)
        assert rc == 0, text
        check_products(launches, type, rows, outs + apart)
        assert rows < 1 << 26 or not space and not any(l["cut"] for l in launches)
        # its gradients: for x alone, then for the weight, whose product has few rows and many k's
        space = calls.bytes("gv_dense_rows_backward_workspace", rows, cols, outs, type, 0, 1, 0, 0)
        rc, text, launches = calls.call("gv_dense_rows_backward", rows, cols, outs, type, X, outs + apart, None, 0, W, cols + apart, 0, None, 0, OUT,
                                        cols + apart, None, 0, None, SPACE if space else None, space, None)
        assert rc == 0, text
        check_products(launches, type, rows, cols + apart)
        space = calls.bytes("gv_dense_rows_backward_workspace", rows, cols, outs, type, 2, 0, 1, 1)
        rc, text, launches = calls.call("gv_dense_rows_backward", rows, cols, outs, type, X, outs + apart, W, cols + apart, None, 0, 2, PRE, outs + apart,
                                        None, 0, OUT, cols + apart, SPACE, SPACE, space, None)
        assert rc == 0, text
        check_products(launches, type, outs, cols + apart)


def test_rows_by_index_and_selections_can_be_launched(calls):
    """At the ends of what they accept: every launch has fewer than 2^32 threads."""
    for count in (1024, 1025, 8192, 8193, 1 << 20, 1 << 31):
        for rows in (1, 1 << 20, 1 << 31):
            for cols in (1, 9, 512, 513, 16384):
                if max(count, rows) * cols > 1 << 38:
                    continue
                rc, text, launches = calls.call("gv_lookup_rows", count, W, 1, 4, rows, cols, BF16, X, cols, 1.0, BF16, OUT, cols, None)
                assert rc == 0 and len(launches) == 1, text
                for add in (0, 1):
                    space = calls.bytes("gv_lookup_rows_workspace", count, rows, cols, add)
                    rc, text, more = calls.call("gv_lookup_rows_backward", count, W, 1, 4, rows, cols, BF16, X, cols, 1.0, add, F32, OUT, cols,
                                                SPACE if space else None, space, None)
                    assert rc == 0, text
                    launches += more
                assert all(0 < l["blocks"] * l["threads"] < 2**32 for l in launches), launches
    for queries, beams in ((1, 1), (512, 512), (65536, 1), (65536, 512)):
        for rows in (0, 1, 1 << 20, 1 << 31):
            for best in (1, 1024):
                space = calls.bytes("gv_select_rows_workspace", queries, rows, beams, best)
                rc, text, launches = calls.call("gv_select_rows", queries, rows, BF16, X, max(1, rows), beams, None, None, 0, 1, best, OUT, PRE, W,
                                                SPACE if space else None, space, None)
                assert rc == 0 and all(0 < l["blocks"] * l["threads"] < 2**32 for l in launches), (text, launches)


def at(base, values, type=F32):
    """The address that lies so many values behind another."""
    return ctypes.c_void_p(base.value + values * SIZE[type])


def layer(x=X, x_stride=8, w=W, w_stride=8, bias=None, residual=None, residual_stride=16, pre=None, pre_stride=16, out=OUT, out_stride=16, rows=100):
    return "gv_dense_rows", rows, 8, 16, F32, x, x_stride, w, w_stride, bias, 0, residual, residual_stride, pre, pre_stride, out, out_stride, None, 0, None


def test_layers_beside_what_they_read(calls):
    """Column slices of one buffer, and rows between other rows, share no value; what shares one is refused."""
    for fine in [dict(x_stride=24, out=at(X, 8), out_stride=24), dict(x=at(X, 16), x_stride=24, out=X, out_stride=24),  # x and out side by side
                 dict(x_stride=48, out=at(X, 24), out_stride=96),          # beside every other row
                 dict(x_stride=64, out=at(X, 32), out_stride=64),          # every other row
                 dict(out_stride=32, pre=at(OUT, 16), pre_stride=32), dict(out_stride=32, residual=at(OUT, 16), residual_stride=32),
                 dict(out_stride=32, residual=at(OUT, -16), residual_stride=32), dict(residual=OUT), dict(residual=OUT, residual_stride=16, out_stride=16),
                 dict(rows=1, bias=OUT), dict(rows=1, bias=OUT, residual=OUT, residual_stride=99), dict(rows=1, pre=PRE, bias=PRE),
                 dict(rows=1, x_stride=999, out=at(X, 8)), dict(out=at(X, 100 * 8)), dict(out=at(X, 99 * 24 + 8), x_stride=24), dict(bias=at(OUT, -16))]:
        name, *args = layer(**fine)
        rc, text, launches = calls.call(name, *args)
        assert rc == 0 and launches, (fine, text)
    for bad, word in [(dict(x_stride=23, out=at(X, 8), out_stride=23), "out overlaps x"), (dict(x_stride=24, out=at(X, 7), out_stride=24), "out overlaps x"),
                      (dict(x_stride=24, out=at(X, 9), out_stride=24), "out overlaps x"), (dict(x_stride=24, out=at(X, 8), out_stride=25), "out overlaps x"),
                      (dict(out_stride=32, pre=at(OUT, 15), pre_stride=32), "pre overlaps out"), (dict(residual=at(OUT, 1)), "out overlaps residual"),
                      (dict(residual=OUT, residual_stride=17), "out overlaps residual"), (dict(bias=OUT), "out overlaps bias"), (dict(pre=PRE, bias=PRE), "pre overlaps bias"),
                      (dict(rows=1, bias=at(OUT, 1)), "out overlaps bias"), (dict(rows=1, x_stride=999, out=at(X, 7)), "out overlaps x"),
                      (dict(out=at(X, 99 * 24 + 7), x_stride=24), "out overlaps x"),
                      (dict(x_stride=48, out=at(X, 24), out_stride=24), "out overlaps x")]:  # out's second row lies on x's
        name, *args = layer(**bad)
        rc, text, launches = calls.call(name, *args)
        assert rc == EINVAL and word in text and not launches, (bad, text)


def gradients(g=OUT, g_stride=16, x=X, x_stride=8, w=W, w_stride=8, act=0, pre=None, grad_x=None, grad_x_stride=8, grad_w=None, grad_w_stride=8, grad_b=None):
    return ("gv_dense_rows_backward", 100, 8, 16, F32, g, g_stride, x, x_stride, w, w_stride, act, pre, 16, grad_x, grad_x_stride, grad_w, grad_w_stride,
            grad_b, SPACE, 1 << 30, None)


def test_gradients_beside_what_they_read(calls):
    """What a call does not read may be overwritten by it."""
    for fine in [dict(g_stride=24, grad_x=at(OUT, 16), grad_x_stride=24), dict(x_stride=16, grad_x=at(X, 8), grad_x_stride=16),
                 dict(w_stride=16, grad_w=at(W, 8), grad_w_stride=16), dict(grad_x=X), dict(grad_w=W), dict(pre=PRE, grad_x=PRE), dict(grad_b=X), dict(grad_b=W),
                 dict(grad_x=PRE, grad_x_stride=24, grad_b=at(PRE, 8))]:  # between two rows
        name, *args = gradients(**fine)
        rc, text, launches = calls.call(name, *args)
        assert rc == 0 and launches, (fine, text)
    for bad, word in [(dict(grad_x=OUT), "grad_x overlaps grad_out"), (dict(grad_x=X, grad_w=PRE), "grad_x overlaps x"), (dict(grad_w=W, grad_x=PRE), "grad_weight overlaps weight"),
                      (dict(act=1, pre=PRE, grad_x=PRE), "grad_x overlaps pre"), (dict(grad_b=at(OUT, 1599)), "grad_bias overlaps grad_out"),
                      (dict(grad_b=X, grad_w=PRE), "grad_bias overlaps x"), (dict(grad_b=W, grad_x=PRE), "grad_bias overlaps weight"),
                      (dict(act=1, pre=PRE, grad_b=PRE), "grad_bias overlaps pre"), (dict(grad_w=PRE, grad_b=at(PRE, 127)), "grad_bias overlaps grad_weight"),
                      (dict(grad_w=PRE, grad_x=at(PRE, 8), grad_x_stride=15), "grad_x overlaps grad_weight")]:
        name, *args = gradients(**bad)
        rc, text, launches = calls.call(name, *args)
        assert rc == EINVAL and word in text and not launches, (bad, text)


def test_rows_by_index_beside_what_they_read(calls):
    I32, I64 = 4, 5

    def lookup(index=W, index_stride=1, index_type=I32, cols=8, type=F32, table=X, table_stride=8, out=OUT, out_stride=8):
        return calls.call("gv_lookup_rows", 50, index, index_stride, index_type, 100, cols, type, table, table_stride, 1.0, type, out, out_stride, None)

    def backward(index=W, index_stride=1, grad=X, grad_stride=8, out=OUT, out_stride=8):
        return calls.call("gv_lookup_rows_backward", 50, index, index_stride, I32, 100, 8, F32, grad, grad_stride, 1.0, 0, F32, out, out_stride, None, 0, None)

    eight = ctypes.c_void_p(OUT.value + 8 * 8)
    for rc, text, launches in (lookup(table_stride=16, out=at(X, 8), out_stride=16), lookup(out_stride=9, index=at(OUT, 8), index_stride=9),
                               lookup(index=OUT, index_type=I64, cols=1, type=I64, out_stride=1), lookup(index=OUT, index_type=I64, index_stride=9, cols=1, type=I64, out_stride=9),
                               lookup(index=eight, index_type=I64, index_stride=9, type=I64, out_stride=9),
                               backward(grad_stride=16, out=at(X, 8), out_stride=16), backward(out_stride=9, index=at(OUT, 8), index_stride=9)):
        assert rc == 0 and launches, text
    for (rc, text, launches), word in ((lookup(table_stride=16, out=at(X, 7), out_stride=16), "overlaps the table"), (lookup(out_stride=9, index=at(OUT, 7), index_stride=9), "overlaps index"),
                                       (lookup(index=OUT, index_type=I64, cols=1, type=I64, out_stride=2), "overlaps index"), (lookup(index=OUT, cols=1), "overlaps index"),
                                       (lookup(index=OUT, index_stride=0), "overlaps index"), (backward(grad_stride=16, out=at(X, 9), out_stride=16), "overlaps grad"),
                                       (backward(index=OUT), "overlaps index")):
        assert rc == EINVAL and word in text and not launches, text


@pytest.mark.parametrize("type", [F32, BF16])
def test_the_way_of_few_rows(calls, type):
    """Layers of up to 64 rows: the way goes by the rule beside few_rows, and the workspace is enough for each of them, whatever the alignment."""
    for rows in (1, 15, 16, 17, 32, 33, 64, 65):
        for cols in (8, 1024, 1025, 2048, 2056, 4096, 4104, 16384):
            for outs in (1, 512, 4096, 4104, 16384):
                for apart in (0, 1):
                    space = calls.bytes("gv_dense_rows_workspace", rows, cols, outs, type)
                    stride = cols + apart + (-cols % 4 if apart == 0 else 0)
                    rc, text, launches = calls.call("gv_dense_rows", rows, cols, outs, type, X, stride, W, stride, None, 0, None, 0, None, 0, OUT, outs,
                                                    SPACE if space else None, space, None)
                    assert rc == 0, text
                    few = b"k_product_few" in launches[0]["kernel"]
                    whole = stride * SIZE[type] % 16 == 0
                    most = 4096 // SIZE[type] if rows > 32 else 4096 if whole else 2048
                    assert few == (rows <= 16 or rows <= 64 and outs <= 4096 and (whole or type == F32) and cols <= most), (rows, cols, outs, apart)
                    assert space or not any(l["cut"] for l in launches)
                    assert len(launches) == (1 if few or not launches[0]["cut"] else 2)
