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
