"""gvhot: GraphVite's GPU training hot path (arXiv 1903.00757) as hand-written HIP for MI355X,
behind a C boundary (include/gvhot.h), with this thin ctypes binding on top."""
import importlib

from .binding import *  # noqa: F401,F403
from .binding import EXPORTS, LIB_PATH, GvError, load  # noqa: F401

# of rows.py, which is imported with the first of them: it needs torch, which constants, the exports and the build do without
_ROWS = ("NormRows", "NormGrads", "gv_drop_rows", "gv_norm_rows", "gv_norm_rows_workspace", "gv_norm_rows_backward",
         "gv_quantize_rows", "gv_score_rows", "gv_lookup_rows", "gv_lookup_rows_workspace", "gv_lookup_rows_backward",
         "DenseRows", "DenseGrads", "gv_dense_rows", "gv_dense_rows_workspace", "gv_dense_rows_backward", "gv_dense_rows_backward_workspace",
         "Selection", "gv_select_rows", "gv_select_rows_workspace")
__all__ = [name for name in globals() if not name.startswith("_") and name != "importlib"] + ["rows", *_ROWS]


def __getattr__(name):
    if name != "rows" and name not in _ROWS:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    rows = importlib.import_module(".rows", __name__)
    globals().update((of, getattr(rows, of)) for of in _ROWS)
    return globals()[name]


def __dir__():
    return sorted(set(globals()) | set(_ROWS))
