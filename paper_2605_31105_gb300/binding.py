"""ctypes binding of libgrkv.so: the C ABI of include/grkv.h, same names.

Argument marshalling only: torch tensors are passed as device pointers, the
torch stream as a cudaStream_t.  Every step of the path runs in the CUDA
library; there is no fallback, and `load()` raises if the library is absent.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgrkv.so")

GRKV_OK = 0
GRKV_ERR_INVALID_ARG = -1
GRKV_ERR_UNSUPPORTED = -2
GRKV_ERR_WORKSPACE_TOO_SMALL = -3
GRKV_ERR_MISALIGNED = -4
GRKV_ERR_CUDA = -5
GRKV_ERR_NUMERIC = -6
GRKV_ERR_TIMEOUT = -7
GRKV_ERR_BOUNDS = -8
GRKV_ERR_NO_PAGES = -9

GRKV_F32 = 0
GRKV_BF16 = 1
GRKV_POOL_MAX = 0
GRKV_POOL_AVG = 1
GRKV_UPDATE_K = 0x1
GRKV_FORCE_SIMT = 0x2
GRKV_ONE_READ_SCORE = 0x4
GRKV_DETERMINISTIC = 0x8
GRKV_CHECKS = 0x10
GRKV_TEST_TIMEOUT = 0x80000000
GRKV_ROPE_HALF = 0
GRKV_ROPE_PAIRS = 1
GRKV_ROPE_PLAIN = 0
GRKV_ROPE_LINEAR = 1
GRKV_ROPE_NTK = 2
GRKV_ROPE_BANDS = 3
GRKV_ROPE_YARN = 4
GRKV_ROPE_TRANSPOSE = 0x1

EXPORTS = ("grkv_params_init", "grkv_workspace_size", "grkv_score", "grkv_select", "grkv_merge",
           "grkv_compress", "grkv_status", "grkv_strerror", "grkv_launch_count",
           "grkv_select_noalloc", "grkv_transfer_workspace_size", "grkv_transfer_check",
           "grkv_compress_ragged_workspace_size", "grkv_compress_ragged",
           "grkv_cache_params_init", "grkv_cache_workspace_size", "grkv_cache_reserve",
           "grkv_cache_fork", "grkv_cache_trim", "grkv_cache_append", "grkv_cache_compact",
           "grkv_attend", "grkv_attend_tree", "grkv_attend_cross", "grkv_cache_map",
           "grkv_rope_params_init", "grkv_rope_make", "grkv_rope_rows", "grkv_cache_append_rope",
           "grkv_cache_compact_rope")


class grkv_params(ctypes.Structure):
    _fields_ = [
        ("units", ctypes.c_int32), ("group", ctypes.c_int32), ("n", ctypes.c_int32),
        ("d", ctypes.c_int32), ("window", ctypes.c_int32), ("budget", ctypes.c_int32),
        ("pool_kernel", ctypes.c_int32), ("pool_type", ctypes.c_int32),
        ("n_sink", ctypes.c_int32), ("beta", ctypes.c_float), ("lambda_v", ctypes.c_float),
        ("lambda_k", ctypes.c_float), ("scale", ctypes.c_float), ("causal", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32), ("cg_iters", ctypes.c_int32),
        ("cg_tol", ctypes.c_float), ("steps", ctypes.c_int32), ("step_tol", ctypes.c_float),
    ]


class grkv_cache_params(ctypes.Structure):
    _fields_ = [
        ("units", ctypes.c_int32), ("group", ctypes.c_int32), ("d", ctypes.c_int32),
        ("pages", ctypes.c_int32), ("page", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("tokens", ctypes.c_int32), ("window", ctypes.c_int32), ("n_sink", ctypes.c_int32),
        ("scale", ctypes.c_float), ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class grkv_rope_params(ctypes.Structure):
    _fields_ = [
        ("d", ctypes.c_int32), ("rotary", ctypes.c_int32), ("layout", ctypes.c_int32),
        ("scaling", ctypes.c_int32), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
        ("low", ctypes.c_double), ("high", ctypes.c_double), ("original", ctypes.c_double),
        ("amplitude", ctypes.c_double),
    ]


class grkv_rope(ctypes.Structure):
    _fields_ = [
        ("rotary", ctypes.c_int32), ("layout", ctypes.c_int32), ("amplitude", ctypes.c_float),
        ("reserved", ctypes.c_int32), ("turns", ctypes.c_uint64 * 64),
    ]


class grkv_rows(ctypes.Structure):
    _fields_ = [
        ("seqs", ctypes.c_int32), ("heads", ctypes.c_int32), ("tokens", ctypes.c_int32),
        ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32),
        ("in_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
    ]


class GrkvError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


_lib = None
_P = ctypes.POINTER(grkv_params)
_vp = ctypes.c_void_p


def load():
    """Load the in-tree library (built by paper_2605_31105_gb300.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() first")
    lib = ctypes.CDLL(LIB_PATH)
    lib.grkv_params_init.argtypes = [_P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_int32, ctypes.c_int32]
    lib.grkv_params_init.restype = None
    lib.grkv_workspace_size.argtypes = [_P, ctypes.POINTER(ctypes.c_size_t)]
    lib.grkv_score.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.grkv_select.argtypes = [_P, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.grkv_merge.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                               ctypes.c_size_t, _vp]
    lib.grkv_compress.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
    lib.grkv_status.argtypes = [_vp, ctypes.POINTER(ctypes.c_int), _vp]
    lib.grkv_strerror.argtypes = [ctypes.c_int]
    lib.grkv_strerror.restype = ctypes.c_char_p
    lib.grkv_select_noalloc.argtypes = [_P, _vp, _vp, _vp]
    lib.grkv_select_noalloc.restype = ctypes.c_int
    lib.grkv_launch_count.argtypes = []
    lib.grkv_launch_count.restype = ctypes.c_uint64
    lib.grkv_transfer_workspace_size.argtypes = [_P, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.grkv_transfer_check.argtypes = [_P, ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _vp, ctypes.c_size_t, _vp]
    _ip = ctypes.POINTER(ctypes.c_int32)
    lib.grkv_compress_ragged_workspace_size.argtypes = [_P, _ip, ctypes.POINTER(ctypes.c_size_t)]
    lib.grkv_compress_ragged.argtypes = [_P, _ip, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                         ctypes.c_size_t, _vp]
    for name in ("grkv_workspace_size", "grkv_score", "grkv_select", "grkv_merge",
                 "grkv_compress", "grkv_status", "grkv_transfer_workspace_size",
                 "grkv_transfer_check", "grkv_compress_ragged_workspace_size",
                 "grkv_compress_ragged"):
        getattr(lib, name).restype = ctypes.c_int
    _cp, _sz, _i = ctypes.POINTER(grkv_cache_params), ctypes.c_size_t, ctypes.c_int32
    _rp, _pp = ctypes.POINTER(grkv_rope), ctypes.POINTER(grkv_rope_params)
    lib.grkv_rope_params_init.argtypes = [_pp]
    lib.grkv_rope_params_init.restype = None
    lib.grkv_rope_make.argtypes = [_pp, ctypes.POINTER(ctypes.c_double), _rp]
    lib.grkv_rope_rows.argtypes = [_rp, ctypes.POINTER(grkv_rows), _vp, _vp, _vp, _vp, _vp]
    lib.grkv_rope_make.restype = lib.grkv_rope_rows.restype = ctypes.c_int
    lib.grkv_cache_params_init.argtypes = [_cp, _i, _i, _i, _i, _i]
    lib.grkv_cache_params_init.restype = None
    lib.grkv_cache_workspace_size.argtypes = [_cp, ctypes.POINTER(_sz)]
    for name, lead in (("grkv_cache_reserve", [_vp] * 6), ("grkv_cache_trim", [_vp] * 3),
                       ("grkv_cache_fork", [_i] + [_vp] * 6),
                       ("grkv_cache_append", [_vp] * 3 + [ctypes.c_int64] + [_vp] * 5),
                       ("grkv_cache_compact", [_vp] * 8), ("grkv_attend", [_vp] * 8),
                       ("grkv_attend_tree", [_vp] * 9), ("grkv_attend_cross", [_vp] * 8),
                       ("grkv_cache_map", [_vp] * 8),
                       ("grkv_cache_append_rope", [_rp] + [_vp] * 3 + [ctypes.c_int64] + [_vp] * 9),
                       ("grkv_cache_compact_rope", [_rp] + [_vp] * 9)):
        getattr(lib, name).argtypes = [_cp, *lead, _vp, _sz, _vp]
        getattr(lib, name).restype = ctypes.c_int
    lib.grkv_cache_workspace_size.restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load().grkv_strerror(code).decode()


def params(units, group, n, window, budget, **kw) -> grkv_params:
    """grkv_params with the library defaults, then any field overridden by name
    (dtype may be given as "bf16" / "f32")."""
    p = grkv_params()
    load().grkv_params_init(ctypes.byref(p), units, group, n, window, budget)
    for key, val in kw.items():
        if key == "dtype" and isinstance(val, str):
            val = {"bf16": GRKV_BF16, "f32": GRKV_F32}[val]
        if key == "pool_type" and isinstance(val, str):
            val = {"max": GRKV_POOL_MAX, "avg": GRKV_POOL_AVG}[val]
        if key == "lambda_v" and val == math.inf:
            val = float("inf")
        setattr(p, key, val)
    return p


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(rc: int, what: str, raise_on_error: bool):
    if rc != GRKV_OK and raise_on_error:
        raise GrkvError(rc, what)
    return rc


def grkv_workspace_size(p: grkv_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load().grkv_workspace_size(ctypes.byref(p), ctypes.byref(n)), "grkv_workspace_size",
           True)
    return n.value


def grkv_score(p, q, k, v, scores, y, row_stats, ws, ws_bytes=None, stream=None, check=True):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_score(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(scores), _ptr(y),
                           _ptr(row_stats), _ptr(ws), ws_bytes, _stream(stream))
    return _check(rc, "grkv_score", check)


def grkv_select(p, scores, idx, ws, ws_bytes=None, stream=None, check=True):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_select(ctypes.byref(p), _ptr(scores), _ptr(idx), _ptr(ws), ws_bytes,
                            _stream(stream))
    return _check(rc, "grkv_select", check)


def grkv_merge(p, q, k, v, scores, y, idx, k_out, v_out, ws, ws_bytes=None, stream=None,
               check=True, row_stats=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_merge(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(scores), _ptr(y),
                           _ptr(row_stats), _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(ws),
                           ws_bytes, _stream(stream))
    return _check(rc, "grkv_merge", check)


def grkv_compress(p, q, k, v, k_out, v_out, idx, ws, ws_bytes=None, stream=None, check=True):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_compress(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(k_out),
                              _ptr(v_out), _ptr(idx), _ptr(ws), ws_bytes, _stream(stream))
    return _check(rc, "grkv_compress", check)


def grkv_select_noalloc(p, scores, idx, stream=None, check=True):
    """grkv_select with the library's built-in scratch array (no workspace)."""
    rc = load().grkv_select_noalloc(ctypes.byref(p), _ptr(scores), _ptr(idx), _stream(stream))
    return _check(rc, "grkv_select_noalloc", check)


def grkv_transfer_workspace_size(p, held: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().grkv_transfer_workspace_size(ctypes.byref(p), held, ctypes.byref(n)),
           "grkv_transfer_workspace_size", True)
    return n.value


def grkv_transfer_check(p, held, q_win, q_held, k, v, idx, k_out, v_out, report, ws,
                        ws_bytes=None, stream=None, check=True):
    """Decode-side transfer check: report [U][8] fp32 (see include/grkv.h)."""
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_transfer_check(ctypes.byref(p), held, _ptr(q_win), _ptr(q_held), _ptr(k),
                                    _ptr(v), _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(report),
                                    _ptr(ws), ws_bytes, _stream(stream))
    return _check(rc, "grkv_transfer_check", check)


def _budgets(budgets):
    arr = (ctypes.c_int32 * len(budgets))(*[int(x) for x in budgets])
    return arr


def grkv_compress_ragged_workspace_size(p, budgets) -> int:
    n = ctypes.c_size_t(0)
    _check(load().grkv_compress_ragged_workspace_size(ctypes.byref(p), _budgets(budgets),
                                                      ctypes.byref(n)),
           "grkv_compress_ragged_workspace_size", True)
    return n.value


def grkv_compress_ragged(p, budgets, q, k, v, k_out, v_out, idx, ws, ws_bytes=None,
                         stream=None, check=True):
    """grkv_compress with one budget per unit (host list); packed outputs."""
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    rc = load().grkv_compress_ragged(ctypes.byref(p), _budgets(budgets), _ptr(q), _ptr(k),
                                     _ptr(v), _ptr(k_out), _ptr(v_out), _ptr(idx), _ptr(ws),
                                     ws_bytes, _stream(stream))
    return _check(rc, "grkv_compress_ragged", check)


# ------------------------------------------------------------------ paged cache
def cache_params(units, group, pages, page, max_pages, **kw) -> grkv_cache_params:
    """grkv_cache_params with the library defaults, then any field overridden by name
    (dtype may be given as "bf16" / "f32")."""
    p = grkv_cache_params()
    load().grkv_cache_params_init(ctypes.byref(p), units, group, pages, page, max_pages)
    for key, val in kw.items():
        if key == "dtype" and isinstance(val, str):
            val = {"bf16": GRKV_BF16, "f32": GRKV_F32}[val]
        setattr(p, key, val)
    return p


# The tensors of the calls, in the order of _addresses' arguments, each with its kind: r for row
# data of the call's type, i for 32-bit integers, l for 64-bit ones, f for fp32.
_CALLS = {
    "attend": "q:r k_pages:r v_pages:r out:r table:i lens:i q_lens:i lse:f",
    "attend_tree": "q:r k_pages:r v_pages:r out:r table:i lens:i q_lens:i parent:i lse:f",
    "reserve": "k_pages:r v_pages:r table:i lens:i want:i refs:i",
    "fork": "src:i table_in:i lens_in:i table_out:i lens_out:i refs:i",
    "trim": "table:i lens:i refs:i",
    "append": "k_new:r v_new:r k_pages:r v_pages:r table:i lens:i count:i first_row:l",
    "compact": "k_pages:r v_pages:r idx:i table_in:i lens_in:i table_out:i keep:i first:i",
    "map": "table:i lens:i pos:i slot:l count:i parent:i offset:i first_row:l",
    "append_rope": "k_new:r v_new:r k_pages:r v_pages:r table:i lens:i q:r q_out:r pos:i offset:i "
                   "count:i first_row:l",
    "compact_rope": "k_pages:r v_pages:r idx:i table_in:i lens_in:i table_out:i keep:i first:i turn:i",
}
_dtypes = {}   # (call, p.dtype) -> the tensors' types


def _types_of(call, dtype):
    import torch
    kinds = {"r": torch.bfloat16 if dtype == GRKV_BF16 else torch.float32, "i": torch.int32,
             "l": torch.int64, "f": torch.float32}
    types = tuple(kinds[x.split(":")[1]] for x in _CALLS[call].split())
    _dtypes[call, dtype] = types
    return types


def _fault(call, at, t, want, need):
    import torch
    name = _CALLS[call].split()[at].split(":")[0]
    if t.dtype != want:
        return f"{name} is {t.dtype}, the call takes {want}"
    if not t.is_contiguous():
        return f"{name} is not contiguous"
    if t.numel() < need:
        return f"{name} holds {t.numel()} elements, the call takes {need}"
    where = "a CUDA device" if t.get_device() < 0 else f"device {torch.cuda.current_device()}"
    return f"{name} is on {t.device}, the call runs on {where}"


def _addresses(call, p, ws, ws_bytes, stream, tensors, needs):
    """The addresses of a cache call's tensors, the workspace's address and bytes, and the
    stream.  Tensors are checked: types, contiguous, on the current device like the workspace, as
    large as the call reads or writes.  Addresses given as ints pass as they are, None where the
    call allows it.  (A call's checks are most of its time on the host: 4 us for 8 tensors.)"""
    import torch
    if type(ws) is int:
        dev = None
    else:
        dev = ws.get_device()
        if dev < 0 or dev != torch.cuda.current_device():
            raise ValueError("the workspace is not on the current CUDA device")
        if not ws.is_contiguous():
            raise ValueError("the workspace is not contiguous")
        if ws_bytes is None:
            ws_bytes = ws.numel() * ws.element_size()
        ws = ws.data_ptr()
    dtype = p.dtype
    types = _dtypes.get((call, dtype)) or _types_of(call, dtype)
    out = []
    for t, want, need in zip(tensors, types, needs):
        if t is not None and type(t) is not int:
            at = t.get_device()
            if (t.dtype is not want or at < 0 or t.numel() < need or not t.is_contiguous()
                    or (at != dev and (dev is not None or at != torch.cuda.current_device()))):
                raise ValueError(_fault(call, len(out), t, want, need))
            t = t.data_ptr()
        out.append(t)
    if stream is None:
        stream = _raw_stream(torch.cuda.current_device() if dev is None else dev)
    elif type(stream) is not int:
        stream = stream.cuda_stream
    return out, ws, ws_bytes, stream


def _raw_stream(dev):
    """The current stream of a device, without the Stream object (3 us a call)."""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(dev) if get else torch.cuda.current_stream(dev).cuda_stream


def grkv_cache_workspace_size(p: grkv_cache_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load().grkv_cache_workspace_size(ctypes.byref(p), ctypes.byref(n)),
           "grkv_cache_workspace_size", True)
    return n.value


def grkv_cache_reserve(p, table, lens, want, refs, k_pages, v_pages, ws, ws_bytes=None,
                       stream=None, check=True):
    """Own pages for slots [lens, want) of every unit."""
    u, pages = p.units, p.pages
    n = pages * p.page * p.d
    (k, v, t, le, wa, r), w, nb, st = _addresses(
        "reserve", p, ws, ws_bytes, stream, (k_pages, v_pages, table, lens, want, refs),
        (n, n, u * p.max_pages, u, u, pages))
    rc = load().grkv_cache_reserve(p, t, le, wa, r, k, v, w, nb, st)
    return _check(rc, "grkv_cache_reserve", check)


def grkv_cache_fork(p, src, table_in, lens_in, table_out, lens_out, refs, ws, units_in=None,
                    ws_bytes=None, stream=None, check=True):
    """Unit u of table_out shares the pages of unit src[u] of table_in (-1: none)."""
    if units_in is None:
        units_in = lens_in.numel()
    u, m = p.units, p.max_pages
    (s, ti, li, to, lo, r), w, nb, st = _addresses(
        "fork", p, ws, ws_bytes, stream, (src, table_in, lens_in, table_out, lens_out, refs),
        (u, units_in * m, units_in, u * m, u, p.pages))
    rc = load().grkv_cache_fork(p, units_in, s, ti, li, to, lo, r, w, nb, st)
    return _check(rc, "grkv_cache_fork", check)


def grkv_cache_trim(p, table, lens, refs, ws, ws_bytes=None, stream=None, check=True):
    """Gives back the pages behind lens."""
    u = p.units
    (t, le, r), w, nb, st = _addresses("trim", p, ws, ws_bytes, stream, (table, lens, refs),
                                       (u * p.max_pages, u, p.pages))
    rc = load().grkv_cache_trim(p, t, le, r, w, nb, st)
    return _check(rc, "grkv_cache_trim", check)


def grkv_cache_append(p, k_new, v_new, k_pages, v_pages, table, lens, ws, count=None,
                      first_row=None, ws_bytes=None, stream=None, check=True, new_rows=None):
    """New rows to the last `count` of the `lens` slots of every unit.  With first_row the rows
    are packed: unit u's start at row first_row[u] of k_new and v_new, which hold new_rows of them
    (to be given where one of the two is an address; else what both hold)."""
    u, d = p.units, p.d
    n, need = p.pages * p.page * d, u * p.tokens * d
    if first_row is None:
        new_rows = 0
    else:
        if new_rows is None:
            if type(k_new) is int or type(v_new) is int:
                raise ValueError("new_rows is not given: packed rows at an address have no size")
            new_rows = min(k_new.numel(), v_new.numel()) // d
        need = new_rows * d
    (kn, vn, k, v, t, le, c, f), w, nb, st = _addresses(
        "append", p, ws, ws_bytes, stream,
        (k_new, v_new, k_pages, v_pages, table, lens, count, first_row),
        (need, need, n, n, u * p.max_pages, u, u, u))
    rc = load().grkv_cache_append(p, kn, vn, f, new_rows, c, t, le, k, v, w, nb, st)
    return _check(rc, "grkv_cache_append", check)


def grkv_cache_compact(p, idx, k_pages, v_pages, table_in, lens_in, table_out, ws, keep=None,
                       first=None, ws_bytes=None, stream=None, check=True):
    """Slot first + i of table_out takes slot idx[u][i] of table_in."""
    u = p.units
    n, m = p.pages * p.page * p.d, u * p.max_pages
    (k, v, i, ti, li, to, ke, f), w, nb, st = _addresses(
        "compact", p, ws, ws_bytes, stream,
        (k_pages, v_pages, idx, table_in, lens_in, table_out, keep, first),
        (n, n, u * p.tokens, m, u, m, u, u))
    rc = load().grkv_cache_compact(p, i, ke, f, ti, li, to, k, v, w, nb, st)
    return _check(rc, "grkv_cache_compact", check)


def grkv_attend(p, q, k_pages, v_pages, table, lens, out, ws, q_lens=None, lse=None,
                ws_bytes=None, stream=None, check=True):
    """Attention of the last q_lens slots of every unit over its pages."""
    u, d = p.units, p.d
    n, rows = p.pages * p.page * d, u * p.group * p.tokens
    (q, k, v, o, t, le, ql, ls), w, nb, st = _addresses(
        "attend", p, ws, ws_bytes, stream, (q, k_pages, v_pages, out, table, lens, q_lens, lse),
        (rows * d, n, n, rows * d, u * p.max_pages, u, u, rows))
    rc = load().grkv_attend(p, q, k, v, t, le, ql, o, ls, w, nb, st)
    return _check(rc, "grkv_attend", check)


def grkv_attend_tree(p, q, k_pages, v_pages, table, lens, parent, out, ws, q_lens=None, lse=None,
                     ws_bytes=None, stream=None, check=True):
    """grkv_attend for trees of drafted tokens: parent [U][t], -1 for roots."""
    u, d, tokens = p.units, p.d, p.tokens
    n, rows = p.pages * p.page * d, u * p.group * tokens
    (q, k, v, o, t, le, ql, pa, ls), w, nb, st = _addresses(
        "attend_tree", p, ws, ws_bytes, stream,
        (q, k_pages, v_pages, out, table, lens, q_lens, parent, lse),
        (rows * d, n, n, rows * d, u * p.max_pages, u, u, u * tokens, rows))
    rc = load().grkv_attend_tree(p, q, k, v, t, le, ql, pa, o, ls, w, nb, st)
    return _check(rc, "grkv_attend_tree", check)


def grkv_attend_cross(p, q, k_pages, v_pages, table, lens, out, ws, q_lens=None, lse=None,
                      ws_bytes=None, stream=None, check=True):
    """Attention of q_lens rows of every unit over all of its lens slots."""
    u, d = p.units, p.d
    n, rows = p.pages * p.page * d, u * p.group * p.tokens
    (q, k, v, o, t, le, ql, ls), w, nb, st = _addresses(
        "attend", p, ws, ws_bytes, stream, (q, k_pages, v_pages, out, table, lens, q_lens, lse),
        (rows * d, n, n, rows * d, u * p.max_pages, u, u, rows))
    rc = load().grkv_attend_cross(p, q, k, v, t, le, ql, o, ls, w, nb, st)
    return _check(rc, "grkv_attend_cross", check)


def grkv_cache_map(p, table, lens, pos, slot, ws, count=None, parent=None, offset=None,
                   first_row=None, ws_bytes=None, stream=None, check=True):
    """Positions and slots of the last `count` of the `lens` slots of every unit; with first_row
    ([U + 1], written) packed."""
    u, rows = p.units, p.units * p.tokens
    (t, le, po, sl, c, pa, of, f), w, nb, st = _addresses(
        "map", p, ws, ws_bytes, stream, (table, lens, pos, slot, count, parent, offset, first_row),
        (u * p.max_pages, u, rows, rows, u, rows, u, u + 1))
    rc = load().grkv_cache_map(p, c, pa, of, t, le, f, po, sl, w, nb, st)
    return _check(rc, "grkv_cache_map", check)


# -------------------------------------------------------------- rotary positions
_ROPE_NAMES = {
    "layout": {"half": GRKV_ROPE_HALF, "pairs": GRKV_ROPE_PAIRS},
    "scaling": {"plain": GRKV_ROPE_PLAIN, "linear": GRKV_ROPE_LINEAR, "ntk": GRKV_ROPE_NTK,
                "bands": GRKV_ROPE_BANDS, "yarn": GRKV_ROPE_YARN},
}


def rope_params(**kw) -> grkv_rope_params:
    """grkv_rope_params with the library defaults, then any field overridden by name (layout and
    scaling may be given as "half", "pairs", "plain", "linear", "ntk", "bands", "yarn")."""
    p = grkv_rope_params()
    load().grkv_rope_params_init(ctypes.byref(p))
    for key, val in kw.items():
        if isinstance(val, str):
            val = _ROPE_NAMES[key][val]
        setattr(p, key, val)
    return p


def grkv_rope_make(p: grkv_rope_params, factors=None) -> grkv_rope:
    """The plan that the calls take; factors: [rotary / 2] by which frequencies are divided."""
    rope = grkv_rope()
    if factors is not None:
        if len(factors) != p.rotary // 2:
            raise ValueError(f"{len(factors)} factors, the plan has {p.rotary // 2} pairs")
        factors = (ctypes.c_double * len(factors))(*[float(x) for x in factors])
    _check(load().grkv_rope_make(ctypes.byref(p), factors, ctypes.byref(rope)), "grkv_rope_make", True)
    return rope


def grkv_rope_rows(rope, x, out, pos=None, start=None, transpose=False, stream=None, check=True):
    """Rotates rows x [S, H, t, 128] into out, both of any strides; pos [S, t] or start [S]."""
    import torch
    shape = x.shape
    if len(shape) != 4 or out.shape != shape:
        raise ValueError(f"x is {tuple(shape)}, out {tuple(out.shape)}: the call takes two [S, H, t, d]")
    s, h, t, d = shape
    dtype = x.dtype
    code = _ROW_TYPES.get(dtype) if _ROW_TYPES else _row_types().get(dtype)
    if code is None or out.dtype is not dtype:
        raise ValueError(f"x is {dtype}, out {out.dtype}: the call takes bfloat16 or float32")
    a, b, c, e = x.stride()
    oa, ob, oc, oe = out.stride()
    if x.numel() and (e != 1 or oe != 1):
        raise ValueError("the rows of x and out are not contiguous")
    dev = x.get_device()
    if dev < 0 or dev != torch.cuda.current_device() or out.get_device() != dev:
        raise ValueError(f"x is on {x.device}, out on {out.device}, the call runs on the current CUDA device")
    where = []
    for name, i, need in (("pos", pos, s * t), ("start", start, s)):
        if i is not None and type(i) is not int:
            if (i.dtype is not torch.int32 or i.get_device() != dev or i.numel() < need
                    or not i.is_contiguous()):
                raise ValueError(f"{name} is {i.dtype} {tuple(i.shape)} on {i.device}: the call takes {need} "
                                 f"contiguous int32 on {x.device}")
            i = i.data_ptr()
        where.append(i)
    rows = _rows(s, h, t, d, code, GRKV_ROPE_TRANSPOSE if transpose else 0, a, b, c, oa, ob, oc)
    if stream is None:
        stream = _raw_stream(dev)
    elif type(stream) is not int:
        stream = stream.cuda_stream
    rc = load().grkv_rope_rows(rope, rows, x.data_ptr(), out.data_ptr(), where[0], where[1], stream)
    return _check(rc, "grkv_rope_rows", check)


@functools.lru_cache(1024)
def _rows(s, h, t, d, dtype, flags, a, b, c, oa, ob, oc):   # 1.2 us a structure
    return grkv_rows(s, h, t, d, dtype, flags, (a, b, c), (oa, ob, oc))


_ROW_TYPES = {}


def _row_types():
    import torch
    _ROW_TYPES.update({torch.bfloat16: GRKV_BF16, torch.float32: GRKV_F32})
    return _ROW_TYPES


def grkv_cache_append_rope(p, rope, k_new, v_new, k_pages, v_pages, table, lens, ws, q=None,
                           q_out=None, pos=None, offset=None, count=None, first_row=None,
                           ws_bytes=None, stream=None, check=True, new_rows=None):
    """grkv_cache_append with rotated keys, and the same tokens' queries rotated into q_out."""
    u, d = p.units, p.d
    n, need = p.pages * p.page * d, u * p.tokens * d
    if first_row is None:
        new_rows = 0
    else:
        if new_rows is None:
            if type(k_new) is int or type(v_new) is int:
                raise ValueError("new_rows is not given: packed rows at an address have no size")
            new_rows = min(k_new.numel(), v_new.numel()) // d
        need = new_rows * d
    queries = u * p.group * p.tokens * d
    (kn, vn, k, v, t, le, qi, qo, po, of, c, f), w, nb, st = _addresses(
        "append_rope", p, ws, ws_bytes, stream,
        (k_new, v_new, k_pages, v_pages, table, lens, q, q_out, pos, offset, count, first_row),
        (need, need, n, n, u * p.max_pages, u, queries, queries, need // d, u, u, u))
    rc = load().grkv_cache_append_rope(p, rope, kn, vn, f, new_rows, c, po, of, qi, qo, t, le, k, v,
                                       w, nb, st)
    return _check(rc, "grkv_cache_append_rope", check)


def grkv_cache_compact_rope(p, rope, idx, k_pages, v_pages, table_in, lens_in, table_out, ws,
                            keep=None, first=None, turn=None, ws_bytes=None, stream=None, check=True):
    """grkv_cache_compact with keys turned by `turn` [U, t], or by what their slots change."""
    u = p.units
    n, m = p.pages * p.page * p.d, u * p.max_pages
    (k, v, i, ti, li, to, ke, f, tu), w, nb, st = _addresses(
        "compact_rope", p, ws, ws_bytes, stream,
        (k_pages, v_pages, idx, table_in, lens_in, table_out, keep, first, turn),
        (n, n, u * p.tokens, m, u, m, u, u, u * p.tokens))
    rc = load().grkv_cache_compact_rope(p, rope, i, ke, f, tu, ti, li, to, k, v, w, nb, st)
    return _check(rc, "grkv_cache_compact_rope", check)


def grkv_launch_count() -> int:
    return int(load().grkv_launch_count())


def grkv_status(ws, stream=None) -> int:
    st = ctypes.c_int(0)
    _check(load().grkv_status(_ptr(ws), ctypes.byref(st), _stream(stream)), "grkv_status", True)
    return st.value
