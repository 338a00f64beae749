"""Thin Python binding of ``libgptq2d.so`` (the C ABI in ``include/gptq2d.h``).

Argument marshalling only: every step of the factorisation and of the sweep
runs in the library's HIP kernels. PyTorch supplies device memory and the
current stream. The library must be built (``__graft_entry__.build()``); a
missing library is an error, never a fallback.

The functions named like the C entry points take and return the same things,
with torch tensors in place of device pointers and Python ints in place of
handles. ``Factors`` and ``round_matrix`` are conveniences built from them, and
``Blocks``, ``Cache``, ``block_*``, ``tree_masks`` and ``token_logprobs*`` those of
the eight-bit operators: they allocate outputs and workspaces as they go. Of these,
``block_linear`` (for X) and ``token_logprobs`` (for the logits) take part in autograd.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libgptq2d.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "gptq2d.h")

F32, F64, F16, BF16 = 0, 1, 2, 3
E4M3, INT8 = 0, 1
STATUS = {0: "OK", -1: "ERR_INVALID_ARG", -2: "ERR_SINGULAR", -3: "ERR_NONFINITE", -4: "ERR_OOM",
          -5: "ERR_HIP", -6: "ERR_WORKSPACE", -7: "ERR_OVERFLOW", -8: "ERR_TIMEOUT"}

_lib = None


class Gptq2dError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}: {detail}")


def declared_functions() -> list[str]:
    """Names of the functions declared in include/gptq2d.h."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(gptq2d_[a-z_]+)\s*\(", text)))


def load():
    """Load the built library (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    ip32 = ctypes.POINTER(ctypes.c_int32)
    sigs = {
        "gptq2d_factors_create": (i32, [i32, i32, ctypes.POINTER(vp)]),
        "gptq2d_factors_destroy": (None, [vp]),
        "gptq2d_factors_shape": (i32, [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]),
        "gptq2d_factors_set_order": (i32, [vp, i32]),
        "gptq2d_factor_compute": (i32, [vp, i32, vp, i64, vp, i64, vp]),
        "gptq2d_factor_check": (i32, [vp, vp]),
        "gptq2d_factor": (i32, [i32, i32, i32, vp, i64, vp, i64, vp, ctypes.POINTER(vp)]),
        "gptq2d_factor_batched_workspace_size": (sz, [i32]),
        "gptq2d_factor_batched": (i32, [i32, vp, i32, vp, vp, vp, vp, vp, sz, vp]),
        "gptq2d_factor_batched_check": (i32, [i32, vp, vp]),
        "gptq2d_factors_export": (i32, [vp, vp, i64, vp, i64, vp, vp, vp]),
        "gptq2d_factors_import": (i32, [vp, vp, i64, vp, i64, vp, vp, vp]),
        "gptq2d_round_workspace_size": (sz, [vp]),
        "gptq2d_round": (i32, [vp, i32, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]),
        "gptq2d_round_check": (i32, [vp, vp, vp]),
        "gptq2d_round_noalloc": (i32, [vp, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp]),
        "gptq2d_round_batched_workspace_size": (sz, [i32, vp]),
        "gptq2d_round_batched": (i32, [i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "gptq2d_round_batched_check": (i32, [vp, vp]),
        "gptq2d_block_quantize": (i32, [i64, i64, i32, vp, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]),
        "gptq2d_block_matmul_workspace_size": (sz, [i64, i64, i64]),
        "gptq2d_block_matmul": (i32, [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, vp, i64, vp, sz,
                                      vp]),
        "gptq2d_block_linear_workspace_size": (sz, [i64, i64, i64]),
        "gptq2d_block_linear": (i32, [i64, i64, i64, i32, vp, i64, vp, i64, vp, i64, i32, vp, i64, vp, sz, vp]),
        "gptq2d_block_linear_backward_workspace_size": (sz, [i64, i64, i64]),
        "gptq2d_block_linear_backward": (i32, [i64, i64, i64, i32, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, i64,
                                               vp, i64, vp, sz, vp]),
        "gptq2d_cache_append": (i32, [i64, i32, i32, i32, vp, i64, vp, i64, vp, i32, i64, i32, vp, vp, vp, vp, vp]),
        "gptq2d_cache_read": (i32, [i64, i32, i32, i32, vp, i32, i64, i32, vp, vp, vp, vp, vp, i64, vp, i64, vp]),
        "gptq2d_tree_masks": (i32, [i64, i32, vp, vp, vp]),
        "gptq2d_tree_attention_workspace_size": (sz, [i64, i32, i32, i32, i32]),
        "gptq2d_tree_attention": (i32, [i64, i32, i32, i32, i32, i32, vp, i64, i32, i64, i32, vp, vp, vp, vp, vp, i64,
                                        i64, vp, vp, vp, ctypes.c_float, vp, i64, vp, vp, sz, vp]),
        "gptq2d_token_logprobs_workspace_size": (sz, [i64, i64, i32]),
        "gptq2d_token_logprobs": (i32, [i64, i64, i32, vp, i64, ctypes.c_float, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "gptq2d_token_logprobs_backward": (i32, [i64, i64, i32, vp, i64, ctypes.c_float, vp, vp, vp, vp, vp, vp, i64,
                                                 vp]),
        "gptq2d_status_string": (ctypes.c_char_p, [i32]),
        "gptq2d_last_error": (ctypes.c_char_p, []),
        "gptq2d_version": (i32, []),
        "gptq2d_schedule_tasks": (i64, [i32, i32, i32, ip32, i64, ip32]),
        "gptq2d_schedule_sweeps": (i64, [i32, i32, ip32, i64]),
        "gptq2d_stage_timing": (i32, [vp, i32]),
        "gptq2d_stage_time": (i32, [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]),
    }
    for name, (res, args) in sigs.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(st: int, where: str):
    if st != 0:
        raise Gptq2dError(st, where, load().gptq2d_last_error().decode())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.float64:
        return F64
    raise TypeError(f"unsupported dtype {t.dtype}")


def _layout(t: torch.Tensor, rows: int, cols: int, what: str) -> int:
    """Leading dimension of a rows x cols row-major view, after checking that
    the library may read (or write) every row of it without touching memory
    outside the tensor or another row."""
    if t.dim() != 2 or tuple(t.shape) != (rows, cols):
        raise ValueError(f"{what} must be {rows} x {cols}, got {tuple(t.shape)}")
    if t.stride(1) != 1 and cols > 1:
        raise ValueError(f"{what} must be row-major with unit column stride")
    ld = t.stride(0) if rows > 1 else cols
    if rows > 1 and ld < cols:
        # an expanded or overlapping view: rows would alias each other
        raise ValueError(f"{what} has row stride {ld} < {cols} columns (expanded or overlapping view)")
    # the last element the library touches must lie inside the storage
    need = (t.storage_offset() + (rows - 1) * ld + cols) * t.element_size()
    if need > t.untyped_storage().nbytes():
        raise ValueError(f"{what}: rows x ld exceed the tensor's storage")
    return int(ld)


def _mat(t: torch.Tensor, rows: int, cols: int, what: str):
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    ld = _layout(t, rows, cols, what)
    return ctypes.c_void_p(t.data_ptr()), ld


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


# ---------------------------------------------------------------------------
# C entry points
# ---------------------------------------------------------------------------

def gptq2d_version() -> int:
    return int(load().gptq2d_version())


def gptq2d_status_string(st: int) -> str:
    return load().gptq2d_status_string(st).decode()


def gptq2d_last_error() -> str:
    return load().gptq2d_last_error().decode()


def gptq2d_factors_create(m: int, n: int) -> int:
    h = ctypes.c_void_p()
    _check(load().gptq2d_factors_create(m, n, ctypes.byref(h)), "gptq2d_factors_create")
    return h.value


def gptq2d_factors_destroy(h: int) -> None:
    load().gptq2d_factors_destroy(ctypes.c_void_p(h))


def gptq2d_factors_shape(h: int):
    m, n = ctypes.c_int(), ctypes.c_int()
    _check(load().gptq2d_factors_shape(ctypes.c_void_p(h), ctypes.byref(m), ctypes.byref(n)),
           "gptq2d_factors_shape")
    return m.value, n.value


def gptq2d_factors_set_order(h: int, reverse: bool) -> None:
    _check(load().gptq2d_factors_set_order(ctypes.c_void_p(h), int(bool(reverse))),
           "gptq2d_factors_set_order")


def gptq2d_factor_compute(h: int, A: torch.Tensor, B: torch.Tensor, stream=None) -> None:
    m, n = gptq2d_factors_shape(h)
    if A.dtype != B.dtype:
        raise TypeError("A and B must share a dtype")
    pa, lda = _mat(A, m, m, "A")
    pb, ldb = _mat(B, n, n, "B")
    _check(load().gptq2d_factor_compute(ctypes.c_void_p(h), _dt(A), pa, lda, pb, ldb, _stream(stream)),
           "gptq2d_factor_compute")


def gptq2d_factor_check(h: int, stream=None) -> None:
    _check(load().gptq2d_factor_check(ctypes.c_void_p(h), _stream(stream)), "gptq2d_factor_check")


def gptq2d_factor_batched_workspace_size(count: int) -> int:
    return int(load().gptq2d_factor_batched_workspace_size(count))


def gptq2d_factor_batched(handles, As, Bs, workspace: torch.Tensor, stream=None, shapes=None,
                          prepare=False):
    """Factorisations of len(handles) problems (distinct handles) in common
    launches per shape. prepare=True: as for gptq2d_round_batched."""
    count = len(handles)
    if count == 0 or len(As) != count or len(Bs) != count:
        raise ValueError("one A and one B per handle")
    dt = _dt(As[0])
    ap, al, bp, bl = [], [], [], []
    for p, h in enumerate(handles):
        m, n = shapes[p] if shapes is not None else gptq2d_factors_shape(h)
        if _dt(As[p]) != dt or _dt(Bs[p]) != dt:
            raise TypeError("every A and B of a batch must have the same dtype")
        a, la = _mat(As[p], m, m, f"A[{p}]")
        b, lb = _mat(Bs[p], n, n, f"B[{p}]")
        ap.append(a.value); al.append(la); bp.append(b.value); bl.append(lb)
    VP, I64 = ctypes.c_void_p * count, ctypes.c_int64 * count
    args = (count, _handles(handles), dt, VP(*ap), I64(*al), VP(*bp), I64(*bl), _ptr(workspace),
            workspace.numel() * workspace.element_size(), _stream(stream))
    fn = load().gptq2d_factor_batched

    def call():
        _check(fn(*args), "gptq2d_factor_batched")
    if prepare:
        return call
    call()


def gptq2d_factor_batched_check(handles, stream=None) -> None:
    _check(load().gptq2d_factor_batched_check(len(handles), _handles(handles), _stream(stream)),
           "gptq2d_factor_batched_check")


def gptq2d_factor(A: torch.Tensor, B: torch.Tensor, stream=None) -> int:
    if A.dtype != B.dtype:
        raise TypeError("A and B must share a dtype")
    m, n = A.shape[0], B.shape[0]
    pa, lda = _mat(A, m, m, "A")
    pb, ldb = _mat(B, n, n, "B")
    h = ctypes.c_void_p()
    _check(load().gptq2d_factor(m, n, _dt(A), pa, lda, pb, ldb, _stream(stream), ctypes.byref(h)),
           "gptq2d_factor")
    return h.value


def gptq2d_factors_export(h: int, stream=None):
    m, n = gptq2d_factors_shape(h)
    dev = torch.cuda.current_device()
    L = torch.empty((m, m), dtype=torch.float64, device=dev)
    U = torch.empty((n, n), dtype=torch.float64, device=dev)
    lamL = torch.empty(m, dtype=torch.float64, device=dev)
    lamU = torch.empty(n, dtype=torch.float64, device=dev)
    _check(load().gptq2d_factors_export(ctypes.c_void_p(h), _ptr(L), m, _ptr(U), n, _ptr(lamL),
                                        _ptr(lamU), _stream(stream)), "gptq2d_factors_export")
    return L, U, lamL, lamU


def gptq2d_factors_import(h: int, L, U, lamL, lamU, stream=None) -> None:
    m, n = gptq2d_factors_shape(h)
    for t in (L, U, lamL, lamU):
        if t.dtype != torch.float64 or not t.is_cuda:
            raise TypeError("factors must be float64 device tensors")
    pl, ldl = _mat(L, m, m, "L")
    pu, ldu = _mat(U, n, n, "U")
    if lamL.numel() != m or lamU.numel() != n or not lamL.is_contiguous() or not lamU.is_contiguous():
        raise ValueError("lamL / lamU have the wrong size or layout")
    _check(load().gptq2d_factors_import(ctypes.c_void_p(h), pl, ldl, pu, ldu, _ptr(lamL), _ptr(lamU),
                                        _stream(stream)), "gptq2d_factors_import")


def gptq2d_round_workspace_size(h: int) -> int:
    return int(load().gptq2d_round_workspace_size(ctypes.c_void_p(h)))


def gptq2d_round(h: int, X: torch.Tensor, Z: torch.Tensor, Y, objective, workspace: torch.Tensor,
                 stream=None) -> None:
    m, n = gptq2d_factors_shape(h)
    px, ldx = _mat(X, m, n, "X")
    if Z.dtype != torch.int32:
        raise TypeError("Z must be int32")
    pz, ldz = _mat(Z, m, n, "Z")
    if Y is not None:
        if Y.dtype != X.dtype:
            raise TypeError("Y must have X's dtype")
        py, ldy = _mat(Y, m, n, "Y")
    else:
        py, ldy = ctypes.c_void_p(0), n
    if objective is not None and (objective.dtype != torch.float64 or not objective.is_cuda):
        raise TypeError("objective must be a float64 device tensor")
    _check(load().gptq2d_round(ctypes.c_void_p(h), _dt(X), px, ldx, pz, ldz, py, ldy, _ptr(objective),
                               _ptr(workspace), workspace.numel() * workspace.element_size(),
                               _stream(stream)), "gptq2d_round")


def gptq2d_round_noalloc(h: int, X: torch.Tensor, Z: torch.Tensor, Y, objective, status_word: torch.Tensor,
                         stream=None) -> None:
    """gptq2d_round with the library's own fixed workspace; status_word is a
    one-element int32 device tensor (check it with gptq2d_round_check)."""
    m, n = gptq2d_factors_shape(h)
    px, ldx = _mat(X, m, n, "X")
    if Z.dtype != torch.int32:
        raise TypeError("Z must be int32")
    pz, ldz = _mat(Z, m, n, "Z")
    if Y is not None:
        if Y.dtype != X.dtype:
            raise TypeError("Y must have X's dtype")
        py, ldy = _mat(Y, m, n, "Y")
    else:
        py, ldy = ctypes.c_void_p(0), n
    if objective is not None and (objective.dtype != torch.float64 or not objective.is_cuda):
        raise TypeError("objective must be a float64 device tensor")
    if status_word.dtype != torch.int32 or not status_word.is_cuda or status_word.numel() < 1:
        raise TypeError("status_word must be an int32 device tensor")
    _check(load().gptq2d_round_noalloc(ctypes.c_void_p(h), _dt(X), px, ldx, pz, ldz, py, ldy,
                                       _ptr(objective), _ptr(status_word), _stream(stream)),
           "gptq2d_round_noalloc")


def gptq2d_round_check(h: int, workspace: torch.Tensor, stream=None) -> None:
    _check(load().gptq2d_round_check(ctypes.c_void_p(h), _ptr(workspace), _stream(stream)),
           "gptq2d_round_check")


def _handles(handles):
    arr = (ctypes.c_void_p * len(handles))(*[int(h) for h in handles])
    return arr


def gptq2d_round_batched_workspace_size(handles) -> int:
    return int(load().gptq2d_round_batched_workspace_size(len(handles), _handles(handles)))


def gptq2d_round_batched(handles, Xs, Zs, Ys, objective, workspace: torch.Tensor, stream=None,
                         shapes=None, prepare=False):
    """Problems p = 0 .. len(handles)-1 in common launches; Ys may be None (or
    hold None entries); objective None or a float64 device tensor of
    len(handles) entries. With prepare=True nothing is enqueued: the argument
    arrays are built once and a function of no arguments is returned that
    enqueues the call (for loops over the same tensors)."""
    count = len(handles)
    if not (len(Xs) == len(Zs) == count) or (Ys is not None and len(Ys) != count):
        raise ValueError("one X, Z (and Y) per handle")
    if count == 0:
        raise ValueError("empty batch")
    dt = _dt(Xs[0])
    xp, xl, zp, zl, yp, yl = [], [], [], [], [], []
    for p, h in enumerate(handles):
        m, n = shapes[p] if shapes is not None else gptq2d_factors_shape(h)
        if _dt(Xs[p]) != dt:
            raise TypeError("every X of a batch must have the same dtype")
        a, la = _mat(Xs[p], m, n, f"X[{p}]")
        if Zs[p].dtype != torch.int32:
            raise TypeError("Z must be int32")
        b, lb = _mat(Zs[p], m, n, f"Z[{p}]")
        xp.append(a.value); xl.append(la); zp.append(b.value); zl.append(lb)
        if Ys is not None:
            if Ys[p] is None:
                yp.append(None); yl.append(n)
            else:
                if Ys[p].dtype != Xs[p].dtype:
                    raise TypeError("Y must have X's dtype")
                c, lc = _mat(Ys[p], m, n, f"Y[{p}]")
                yp.append(c.value); yl.append(lc)
    if objective is not None and (objective.dtype != torch.float64 or not objective.is_cuda
                                  or objective.numel() < count or not objective.is_contiguous()):
        raise TypeError("objective must be a contiguous float64 device tensor of count entries")
    VP, I64 = ctypes.c_void_p * count, ctypes.c_int64 * count
    X_a, ldx_a, Z_a, ldz_a = VP(*xp), I64(*xl), VP(*zp), I64(*zl)
    Y_a = VP(*yp) if Ys is not None else None
    ldy_a = I64(*yl) if Ys is not None else None
    args = (count, _handles(handles), dt, X_a, ldx_a, Z_a, ldz_a, Y_a, ldy_a, _ptr(objective),
            _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    fn = load().gptq2d_round_batched

    def call():
        _check(fn(*args), "gptq2d_round_batched")
    if prepare:
        return call
    call()


def gptq2d_round_batched_check(workspace: torch.Tensor, stream=None) -> None:
    _check(load().gptq2d_round_batched_check(_ptr(workspace), _stream(stream)),
           "gptq2d_round_batched_check")


def gptq2d_stage_timing(h: int, enable: bool) -> None:
    _check(load().gptq2d_stage_timing(ctypes.c_void_p(h), int(bool(enable))), "gptq2d_stage_timing")


def gptq2d_stage_time(h: int):
    """(summed stage-kernel launch time in ms, launches) since the last read."""
    ms, cnt = ctypes.c_double(0.0), ctypes.c_int64(0)
    _check(load().gptq2d_stage_time(ctypes.c_void_p(h), ctypes.byref(ms), ctypes.byref(cnt)),
           "gptq2d_stage_time")
    return float(ms.value), int(cnt.value)


def gptq2d_schedule_tasks(m: int, n: int, g: int):
    """Host-only delivery plan: (tasks int32[T, 4], offsets int32[MT+NT])."""
    import numpy as np
    lib = load()
    total = lib.gptq2d_schedule_tasks(m, n, g, None, 0, None)
    if total < 0:
        raise ValueError(gptq2d_last_error())
    mt, nt = (m + 63) // 64, (n + 63) // 64
    offs = np.zeros(mt + nt, dtype=np.int32)
    tasks = np.zeros((max(total, 1), 4), dtype=np.int32)
    lib.gptq2d_schedule_tasks(m, n, g, tasks.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), total,
                              offs.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
    return tasks[:total], offs


def gptq2d_schedule_sweeps(m: int, n: int):
    """Host-only list of the tiles each sweep launch rounds: int32[S, 2] of
    (first, last) tile row; row I of launch k is tile (I, k - I)."""
    import numpy as np
    lib = load()
    total = lib.gptq2d_schedule_sweeps(m, n, None, 0)
    if total < 0:
        raise ValueError(gptq2d_last_error())
    rows = np.zeros((total, 2), dtype=np.int32)
    lib.gptq2d_schedule_sweeps(m, n, rows.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), total)
    return rows


# ---------------------------------------------------------------------------
# Eight-bit operators
#
# With prepare=True nothing is enqueued: the arguments are checked and laid out
# once and a function of no arguments is returned that enqueues the call on the
# stream given (or current) now, for loops over the same tensors.
# ---------------------------------------------------------------------------

_NARROW = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_CODES = {torch.float8_e4m3fn: E4M3, torch.int8: INT8}


def _narrow(*tensors) -> int:
    """The common dtype (float32, float16 or bfloat16) of the tensors given."""
    kinds = {t.dtype for t in tensors if t is not None}
    if len(kinds) != 1 or next(iter(kinds)) not in _NARROW:
        raise TypeError(f"need tensors of one dtype out of float32, float16 and bfloat16, got {sorted(map(str, kinds))}")
    return _NARROW[kinds.pop()]


def _codes(t: torch.Tensor, rows: int, cols: int, what: str):
    """Pointer and row stride of e4m3 codes, whose rows reach to a multiple of
    16 columns (the stride has to be one, also of a single row)."""
    if t.dtype != torch.float8_e4m3fn:
        raise TypeError(f"{what} must be float8_e4m3fn")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    ld = _layout(t, rows, cols, what)
    up = -(-cols // 16) * 16
    if rows == 1:
        ld = max(ld, up)
    if ld % 16 or t.data_ptr() % 16:
        raise ValueError(f"{what} needs rows on 16-byte boundaries, its row stride is {ld}")
    if t.storage_offset() + (rows - 1) * ld + up > t.untyped_storage().nbytes():
        raise ValueError(f"{what}: its rows must reach to a multiple of 16 columns")
    return ctypes.c_void_p(t.data_ptr()), ld


def _scales(t: torch.Tensor, rows: int, cols: int, what: str):
    if t.dtype != torch.float32:
        raise TypeError(f"{what} must be float32")
    return _mat(t, rows, cols, what)


def _space(workspace, need: int, what: str):
    if need == 0:
        return ctypes.c_void_p(0), 0
    if workspace is None or not workspace.is_cuda:
        raise ValueError(f"{what} needs a device workspace of {need} bytes")
    return _ptr(workspace), workspace.numel() * workspace.element_size()


def _blocks(v: int) -> int:
    return -(-v // 128)


def _one_device(name: str, tensors, stream) -> None:
    """The tensors and the stream (None: the current one) of a call have to be the
    current device's: a launch goes there, wherever its pointers lead."""
    device = torch.cuda.current_device()
    for t in (*tensors, stream):
        if t is not None and t.device.type == "cuda" and t.device.index != device:
            raise ValueError(f"{name}: a tensor or the stream is on {t.device}, the current device is cuda:{device}")


def _enqueue(name: str, args, keep, stream, prepare: bool):
    _one_device(name, keep, stream)
    fn = getattr(load(), name)

    def call(_keep=keep):  # the tensors live as long as the call can be made
        st = fn(*args)
        if st != 0:
            _check(st, name)
    if prepare:
        return call
    call()


def gptq2d_block_quantize(X, Q, S, QT=None, ST=None, block_rows: int = 1, pow2: bool = False, stream=None,
                          prepare=False):
    """e4m3 codes and scales of X (Q, S) and of its transpose (QT, ST); either
    pair may be None."""
    rows, cols = X.shape
    px, ldx = _mat(X, rows, cols, "X")
    tile = block_rows != 1
    q = s = qt = st = (ctypes.c_void_p(0), 0)
    if Q is not None:
        q = _codes(Q, rows, cols, "Q")
        s = _scales(S, _blocks(rows) if tile else _blocks(cols), _blocks(cols) if tile else rows, "S")
    if QT is not None:
        qt = _codes(QT, cols, rows, "QT")
        st = _scales(ST, _blocks(cols) if tile else _blocks(rows), _blocks(rows) if tile else cols, "ST")
    args = (rows, cols, _narrow(X), px, ldx, block_rows, int(bool(pow2)), *q, *s, *qt, *st, _stream(stream))
    return _enqueue("gptq2d_block_quantize", args, (X, Q, S, QT, ST), stream, prepare)


def gptq2d_block_matmul_workspace_size(M: int, N: int, K: int) -> int:
    return int(load().gptq2d_block_matmul_workspace_size(M, N, K))


def gptq2d_block_matmul(A, SA, B, SB, C, workspace=None, block_rows: int = 128, stream=None, prepare=False):
    """C = A B^T for e4m3 codes A (M x K; SA: blocks x M) and B (N x K; SB: the
    scales of blocks of block_rows x 128)."""
    (M, K), N = A.shape, B.shape[0]
    a, b = _codes(A, M, K, "A"), _codes(B, N, K, "B")
    sa = _scales(SA, _blocks(K), M, "SA")
    sb = _scales(SB, *((_blocks(K), N) if block_rows == 1 else (_blocks(N), _blocks(K))), "SB")
    c = _mat(C, M, N, "C")
    ws = _space(workspace, gptq2d_block_matmul_workspace_size(M, N, K), "gptq2d_block_matmul")
    args = (M, N, K, *a, *sa, *b, *sb, block_rows, _narrow(C), *c, *ws, _stream(stream))
    return _enqueue("gptq2d_block_matmul", args, (A, SA, B, SB, C, workspace), stream, prepare)


def gptq2d_block_linear_workspace_size(M: int, N: int, K: int) -> int:
    return int(load().gptq2d_block_linear_workspace_size(M, N, K))


def gptq2d_block_linear(X, W, SW, Y, workspace, pow2: bool = False, stream=None, prepare=False):
    """Y = X W^T: X (M x K) quantised on the way, W (N x K) e4m3 tiles of 128 x 128."""
    (M, K), N = X.shape, W.shape[0]
    x, w, y = _mat(X, M, K, "X"), _codes(W, N, K, "W"), _mat(Y, M, N, "Y")
    sw = _scales(SW, _blocks(N), _blocks(K), "SW")
    ws = _space(workspace, gptq2d_block_linear_workspace_size(M, N, K), "gptq2d_block_linear")
    args = (M, N, K, _narrow(X, Y), *x, *w, *sw, int(bool(pow2)), *y, *ws, _stream(stream))
    return _enqueue("gptq2d_block_linear", args, (X, W, SW, Y, workspace), stream, prepare)


def gptq2d_block_linear_backward_workspace_size(M: int, N: int, K: int) -> int:
    return int(load().gptq2d_block_linear_backward_workspace_size(M, N, K))


def gptq2d_block_linear_backward(dY, X, WT, SWT, dX, dW, workspace, pow2: bool = False, stream=None, prepare=False):
    """dX = dY W (dtype of dY) and dW = dY^T X (float32); either may be None. WT
    (K x N): the e4m3 tiles of W's transpose."""
    M, N = dY.shape
    if dX is None and dW is None:
        raise ValueError("neither dX nor dW is asked for")
    K = (dX if dX is not None else dW).shape[1]
    none = (ctypes.c_void_p(0), 0)
    dy = _mat(dY, M, N, "dY")
    x = wt = swt = dx = dw = none
    if dX is not None:
        wt, dx = _codes(WT, K, N, "WT"), _mat(dX, M, K, "dX")
        swt = _scales(SWT, _blocks(K), _blocks(N), "SWT")
    if dW is not None:
        x, dw = _mat(X, M, K, "X"), _scales(dW, N, K, "dW")
    dt = _narrow(dY, dX, X if dW is not None else None)
    ws = _space(workspace, gptq2d_block_linear_backward_workspace_size(M, N, K), "gptq2d_block_linear_backward")
    args = (M, N, K, dt, *dy, *x, *wt, *swt, int(bool(pow2)), *dx, *dw, *ws, _stream(stream))
    return _enqueue("gptq2d_block_linear_backward", args, (dY, X, WT, SWT, dX, dW, workspace), stream, prepare)


def _cache(KC, VC, KS, VS):
    """(code, pages, heads, page_size, dim) and the pointers of a cache."""
    if KC.dtype not in _CODES or VC.dtype != KC.dtype:
        raise TypeError("KC and VC must be float8_e4m3fn or both int8")
    if KC.dim() != 4 or VC.shape != KC.shape:
        raise ValueError("KC and VC must be [pages, heads, page_size, dim]")
    if KS.dtype != torch.float32 or VS.dtype != torch.float32:
        raise TypeError("KS and VS must be float32")
    if KS.shape != KC.shape[:3] or VS.shape != KC.shape[:3]:
        raise ValueError("KS and VS must be [pages, heads, page_size]")
    for t in (KC, VC, KS, VS):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("the cache's tensors must be contiguous device tensors")
    pages, heads, page, dim = KC.shape
    return _CODES[KC.dtype], pages, heads, page, dim, (_ptr(KC), _ptr(VC), _ptr(KS), _ptr(VS))


def _ints(t, shape, dtype, what: str):
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if not t.is_cuda or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor of shape {tuple(shape)}")
    return _ptr(t)


def gptq2d_cache_append(K, V, slots, KC, VC, KS, VS, stream=None, prepare=False):
    """K and V (tokens x (heads dim)) into the cache's slots (int64)."""
    code, pages, heads, page, dim, tensors = _cache(KC, VC, KS, VS)
    tokens = K.shape[0]
    k, v = _mat(K, tokens, heads * dim, "K"), _mat(V, tokens, heads * dim, "V")
    args = (tokens, heads, dim, _narrow(K, V), *k, *v, _ints(slots, (tokens,), torch.int64, "slots"), code, pages, page,
            *tensors, _stream(stream))
    return _enqueue("gptq2d_cache_append", args, (K, V, slots, KC, VC, KS, VS), stream, prepare)


def gptq2d_cache_read(slots, KC, VC, KS, VS, K, V, stream=None, prepare=False):
    """The values of the cache's slots into K and V (tokens x (heads dim))."""
    code, pages, heads, page, dim, tensors = _cache(KC, VC, KS, VS)
    tokens = K.shape[0]
    k, v = _mat(K, tokens, heads * dim, "K"), _mat(V, tokens, heads * dim, "V")
    args = (tokens, heads, dim, _narrow(K, V), _ints(slots, (tokens,), torch.int64, "slots"), code, pages, page,
            *tensors, *k, *v, _stream(stream))
    return _enqueue("gptq2d_cache_read", args, (slots, KC, VC, KS, VS, K, V), stream, prepare)


def gptq2d_tree_masks(parents, masks, stream=None, prepare=False):
    """masks (int64 bits, [seqs, width]) of the trees given by parents (int32)."""
    seqs, width = parents.shape
    args = (seqs, width, _ints(parents, (seqs, width), torch.int32, "parents"),
            _ints(masks, (seqs, width), torch.int64, "masks"), _stream(stream))
    return _enqueue("gptq2d_tree_masks", args, (parents, masks), stream, prepare)


def gptq2d_tree_attention_workspace_size(seqs: int, width: int, heads: int, kv_heads: int, dim: int) -> int:
    return int(load().gptq2d_tree_attention_workspace_size(seqs, width, heads, kv_heads, dim))


def gptq2d_tree_attention(Q, KC, VC, KS, VS, table, context, drafts, masks, scale: float, O, lse, workspace,
                          stream=None, prepare=False):
    """Attention of the drafted tokens (rows of Q and O, seqs * width x (heads
    dim)) over the pages table[b] (int32) of each sequence: context[b] (int32)
    tokens, then drafts[b] (int32; None: width) drafted ones, seen by masks
    (int64 bits, [seqs, width]; None: a chain). lse (float32, seqs * width x heads)
    may be None."""
    code, pages, kv, page, dim, tensors = _cache(KC, VC, KS, VS)
    seqs, rows = context.shape[0], Q.shape[0]
    if seqs < 1 or rows % seqs or Q.shape[1] % (kv * dim):
        raise ValueError(f"Q must be seqs * width x (heads dim) for {seqs} sequences and {kv} kv heads of {dim}")
    width, heads = rows // seqs, Q.shape[1] // dim
    q, o = _mat(Q, rows, heads * dim, "Q"), _mat(O, rows, heads * dim, "O")
    if table.dtype != torch.int32 or table.dim() != 2:
        raise TypeError("table must be an int32 matrix")
    tab = _mat(table, seqs, table.shape[1], "table")
    n = None if drafts is None else _ints(drafts, (seqs,), torch.int32, "drafts")
    m = None if masks is None else _ints(masks, (seqs, width), torch.int64, "masks")
    if lse is not None:
        _scales(lse, rows, heads, "lse")
        if not lse.is_contiguous():
            raise ValueError("lse must be contiguous")
    ws = _space(workspace, gptq2d_tree_attention_workspace_size(seqs, width, heads, kv, dim), "gptq2d_tree_attention")
    args = (seqs, width, heads, kv, dim, _narrow(Q, O), *q, code, pages, page, *tensors, *tab, table.shape[1],
            _ints(context, (seqs,), torch.int32, "context"), n, m, float(scale), *o, _ptr(lse), *ws, _stream(stream))
    return _enqueue("gptq2d_tree_attention", args, (Q, KC, VC, KS, VS, table, context, drafts, masks, O, lse, workspace),
                    stream, prepare)


def gptq2d_token_logprobs_workspace_size(rows: int, vocab: int, top: int) -> int:
    return int(load().gptq2d_token_logprobs_workspace_size(rows, vocab, top))


def gptq2d_token_logprobs(X, target, scale: float, logprob, entropy, lse, ids=None, tops=None, workspace=None,
                          stream=None, prepare=False):
    """Of every row of logits X: the log probability of target (int64; None: none
    given), entropy and log-sum-exp (float32) under scale X, and the largest
    logits' tokens ids (int32) with their log probabilities tops (float32), both
    rows x top or None."""
    rows, vocab = X.shape
    x = _mat(X, rows, vocab, "X")
    y = None if target is None else _ints(target, (rows,), torch.int64, "target")
    out = [_ints(t, (rows,), torch.float32, w) for t, w in ((logprob, "logprob"), (entropy, "entropy"), (lse, "lse"))]
    top, best = 0, [None, None]
    if ids is not None:
        top = ids.shape[1]
        best = [_ints(ids, (rows, top), torch.int32, "ids"), _ints(tops, (rows, top), torch.float32, "tops")]
    ws = _space(workspace, gptq2d_token_logprobs_workspace_size(rows, vocab, top), "gptq2d_token_logprobs")
    args = (rows, vocab, _narrow(X), *x, float(scale), y, top, *out, *best, *ws, _stream(stream))
    return _enqueue("gptq2d_token_logprobs", args, (X, target, logprob, entropy, lse, ids, tops, workspace), stream,
                    prepare)


def gptq2d_token_logprobs_backward(X, target, scale: float, lse, entropy, g_logprob, g_entropy, dX, stream=None,
                                   prepare=False):
    """dX (may be X) from the gradients of the log probabilities and of the
    entropies (float32; either may be None), with lse and entropy of the forward
    call."""
    rows, vocab = X.shape
    x, d = _mat(X, rows, vocab, "X"), _mat(dX, rows, vocab, "dX")
    y = None if target is None else _ints(target, (rows,), torch.int64, "target")
    v = [None if t is None else _ints(t, (rows,), torch.float32, w)
         for t, w in ((lse, "lse"), (entropy, "entropy"), (g_logprob, "g_logprob"), (g_entropy, "g_entropy"))]
    args = (rows, vocab, _narrow(X, dX), *x, float(scale), y, *v, *d, _stream(stream))
    return _enqueue("gptq2d_token_logprobs_backward", args, (X, target, lse, entropy, g_logprob, g_entropy, dX), stream,
                    prepare)


# ---------------------------------------------------------------------------
# Conveniences
# ---------------------------------------------------------------------------

class Factors:
    """Owning wrapper of a factor handle."""

    def __init__(self, m: int, n: int, reverse: bool = False):
        """reverse: round from the last row and column on (the factors are then
        those of the index-reversed problem)."""
        self.m, self.n = m, n
        self.handle = gptq2d_factors_create(m, n)
        self.reverse = bool(reverse)
        if self.reverse:
            gptq2d_factors_set_order(self.handle, True)

    @classmethod
    def from_bases(cls, A: torch.Tensor, B: torch.Tensor, check: bool = True, stream=None,
                   reverse: bool = False):
        f = cls(A.shape[0], B.shape[0], reverse)
        f.compute(A, B, stream)
        if check:
            gptq2d_factor_check(f.handle, stream)
        return f

    def compute(self, A, B, stream=None):
        gptq2d_factor_compute(self.handle, A, B, stream)

    def export(self, stream=None):
        return gptq2d_factors_export(self.handle, stream)

    def load(self, L, U, lamL, lamU, stream=None):
        gptq2d_factors_import(self.handle, L, U, lamL, lamU, stream)

    def workspace(self) -> torch.Tensor:
        return torch.empty(gptq2d_round_workspace_size(self.handle), dtype=torch.uint8,
                           device=torch.cuda.current_device())

    def close(self):
        if getattr(self, "handle", None):
            gptq2d_factors_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def round_matrix(f: Factors, X: torch.Tensor, want_y: bool = True, workspace=None, check=True,
                 stream=None):
    """Z (int32), Y (X's dtype or None) and the objective (float64 device scalar)."""
    m, n = f.m, f.n
    Z = torch.empty((m, n), dtype=torch.int32, device=X.device)
    Y = torch.empty((m, n), dtype=X.dtype, device=X.device) if want_y else None
    obj = torch.empty(1, dtype=torch.float64, device=X.device)
    ws = workspace if workspace is not None else f.workspace()
    gptq2d_round(f.handle, X, Z, Y, obj, ws, stream)
    if check:
        gptq2d_round_check(f.handle, ws, stream)
    return Z, Y, obj


def round_batched(factors, Xs, want_y: bool = True, workspace=None, check=True, stream=None):
    """Round problem p = X[p] with factors[p] (a Factors may repeat), all in
    common launches. Returns lists of Z, Y (or None) and the objectives as one
    float64 device tensor."""
    handles = [f.handle for f in factors]
    dev = Xs[0].device
    Zs = [torch.empty((f.m, f.n), dtype=torch.int32, device=dev) for f in factors]
    Ys = [torch.empty((f.m, f.n), dtype=X.dtype, device=dev) for f, X in zip(factors, Xs)] if want_y else None
    obj = torch.empty(len(factors), dtype=torch.float64, device=dev)
    ws = workspace if workspace is not None else torch.empty(
        gptq2d_round_batched_workspace_size(handles), dtype=torch.uint8, device=dev)
    gptq2d_round_batched(handles, Xs, Zs, Ys, obj, ws, stream, shapes=[(f.m, f.n) for f in factors])
    if check:
        gptq2d_round_batched_check(ws, stream)
    return Zs, Ys, obj


def factor_batched(factors, As, Bs, check=True, stream=None, workspace=None):
    """Compute the factors of every Factors in ``factors`` (distinct) from its
    bases As[p], Bs[p], in common launches per shape."""
    handles = [f.handle for f in factors]
    ws = workspace if workspace is not None else torch.empty(
        gptq2d_factor_batched_workspace_size(len(handles)), dtype=torch.uint8, device=As[0].device)
    gptq2d_factor_batched(handles, As, Bs, ws, stream, shapes=[(f.m, f.n) for f in factors])
    if check:
        gptq2d_factor_batched_check(handles, stream)


def _on(stream, t):
    """A call runs on `stream` or, without one, on the current stream of tensor t's
    device. Memory that it uses is taken for that stream, so that none of it goes to
    other work while the call may still run."""
    if stream is not None:
        return torch.cuda.stream(stream)
    return torch.cuda.device(t.device) if t.is_cuda else contextlib.nullcontext()


def _bytes(n: int) -> torch.Tensor:
    return torch.empty(max(n, 1), dtype=torch.uint8, device=torch.cuda.current_device())


class Blocks(NamedTuple):
    """A rows x cols matrix in e4m3 blocks of block_rows x 128: codes (rows on
    16-byte boundaries) and 32-bit scales (block_rows 1: [blocks, rows], 128:
    [row blocks, column blocks])."""
    codes: torch.Tensor
    scales: torch.Tensor
    block_rows: int

    @classmethod
    def empty(cls, rows: int, cols: int, block_rows: int = 128):
        dev = torch.cuda.current_device()
        codes = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.float8_e4m3fn, device=dev)[:, :cols]
        shape = (_blocks(cols), rows) if block_rows == 1 else (_blocks(rows), _blocks(cols))
        return cls(codes, torch.empty(shape, dtype=torch.float32, device=dev), block_rows)

    def transposed(self):
        """The transpose of a matrix in tiles of 128 x 128 (the same codes and scales)."""
        if self.block_rows != 128:
            raise ValueError("only tiles of 128 x 128 have a transpose")
        out = Blocks.empty(*self.codes.shape[::-1])
        out.codes.view(torch.uint8).copy_(self.codes.view(torch.uint8).T)
        return out._replace(scales=self.scales.T.contiguous())

    def values(self) -> torch.Tensor:
        """What the codes stand for, in 32 bits."""
        rows, cols = self.codes.shape
        s = self.scales.T if self.block_rows == 1 else self.scales.repeat_interleave(128, 0)[:rows]
        return self.codes.float() * s.repeat_interleave(128, 1)[:, :cols]


def block_quantize(X: torch.Tensor, block_rows: int = 128, pow2: bool = False, transposed: bool = False,
                   stream=None) -> Blocks:
    """X (or its transpose, whose blocks run along X's columns) in e4m3 blocks."""
    rows, cols = X.shape
    with _on(stream, X):
        out = Blocks.empty(*((cols, rows) if transposed else (rows, cols)), block_rows)
        pair = (None, None, out.codes, out.scales) if transposed else (out.codes, out.scales)
        gptq2d_block_quantize(X, *pair, block_rows=block_rows, pow2=pow2)
    return out


def block_matmul(A: Blocks, B: Blocks, dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """A B^T; A in blocks of 1 x 128."""
    if A.block_rows != 1:
        raise ValueError("A must be in blocks of 1 x 128")
    (M, K), N = A.codes.shape, B.codes.shape[0]
    with _on(stream, A.codes):
        C = torch.empty((M, N), dtype=dtype, device=A.codes.device)
        gptq2d_block_matmul(A.codes, A.scales, B.codes, B.scales, C,
                            _bytes(gptq2d_block_matmul_workspace_size(M, N, K)), block_rows=B.block_rows)
    return C


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, pow2, WT):
        ctx.W, ctx.WT, ctx.pow2 = W, WT, pow2
        return block_linear(X, W, pow2)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        N, K = ctx.W.codes.shape
        M, WT = dY.shape[0], ctx.W.transposed() if ctx.WT is None else ctx.WT
        dX = torch.empty((M, K), dtype=dY.dtype, device=dY.device)
        gptq2d_block_linear_backward(dY.contiguous(), None, WT.codes, WT.scales, dX, None,
                                     _bytes(gptq2d_block_linear_backward_workspace_size(M, N, K)), pow2=ctx.pow2)
        return dX, None, None, None


def block_linear(X: torch.Tensor, W: Blocks, pow2: bool = False, stream=None, WT=None) -> torch.Tensor:
    """X W^T for W in tiles of 128 x 128; X is quantised on the way. Where X requires
    a gradient it gets block_linear_backward's, by WT (block_quantize(W,
    transposed=True); None: W is turned there and then). W's own, of the weights that
    it holds, is block_linear_backward's dW."""
    (M, K), N = X.shape, W.codes.shape[0]
    for blocks in (W, WT):
        if blocks is not None and blocks.block_rows != 128:
            raise ValueError("W and WT must be in tiles of 128 x 128")
    if WT is not None and tuple(WT.codes.shape) != (K, N):
        raise ValueError(f"WT must be {K} x {N}, got {tuple(WT.codes.shape)}")
    with _on(stream, X):
        if X.requires_grad and torch.is_grad_enabled():
            return _Linear.apply(X, W, pow2, WT)
        Y = torch.empty((M, N), dtype=X.dtype, device=X.device)
        gptq2d_block_linear(X, W.codes, W.scales, Y, _bytes(gptq2d_block_linear_workspace_size(M, N, K)), pow2=pow2)
    return Y


def block_linear_backward(dY: torch.Tensor, X: torch.Tensor, WT: Blocks, pow2: bool = False, stream=None):
    """(dX, dW) of block_linear; WT: block_quantize(W, transposed=True)."""
    (M, N), K = dY.shape, X.shape[1]
    if WT.block_rows != 128:
        raise ValueError("WT must be in tiles of 128 x 128")
    with _on(stream, dY):
        dX = torch.empty((M, K), dtype=dY.dtype, device=dY.device)
        dW = torch.empty((N, K), dtype=torch.float32, device=dY.device)
        ws = _bytes(gptq2d_block_linear_backward_workspace_size(M, N, K))
        gptq2d_block_linear_backward(dY, X, WT.codes, WT.scales, dX, dW, ws, pow2=pow2)
    return dX, dW


class Cache:
    """A paged eight-bit cache of keys and values (code: torch.float8_e4m3fn or
    torch.int8). Pages are the caller's to hand out: table (int32, sequences x
    pages) names each sequence's."""

    def __init__(self, pages: int, heads: int, page_size: int, dim: int, code=torch.float8_e4m3fn):
        dev = torch.cuda.current_device()
        self.heads, self.page_size, self.dim = heads, page_size, dim
        self.KC, self.VC = (torch.zeros((pages, heads, page_size, dim), dtype=torch.uint8, device=dev).view(code)
                            for _ in range(2))
        self.KS, self.VS = (torch.ones((pages, heads, page_size), device=dev) for _ in range(2))

    @property
    def tensors(self):
        return self.KC, self.VC, self.KS, self.VS

    def slots(self, table: torch.Tensor, first: torch.Tensor, count: int) -> torch.Tensor:
        """The slots (int64, sequences * count) of positions first[b] .. first[b] +
        count - 1 of every sequence; -1 before the first token and past its pages."""
        at = first.long().unsqueeze(1) + torch.arange(count, device=table.device)
        page = at // self.page_size
        table = torch.nn.functional.pad(table.long(), (1, 1), value=-1)  # what lies outside names no page
        entry = table.gather(1, (page + 1).clamp(0, table.shape[1] - 1))
        return torch.where(entry >= 0, entry * self.page_size + at % self.page_size, -1).reshape(-1)

    def append(self, K, V, slots, stream=None) -> None:
        with _on(stream, self.KC):
            gptq2d_cache_append(K, V, slots, *self.tensors)

    def read(self, slots, dtype=torch.bfloat16, stream=None):
        with _on(stream, self.KC):
            K, V = (torch.empty((slots.shape[0], self.heads * self.dim), dtype=dtype, device=slots.device)
                    for _ in range(2))
            gptq2d_cache_read(slots, *self.tensors, K, V)
        return K, V

    def attend(self, Q, table, context, masks=None, drafts=None, scale=None, stream=None):
        """(O, lse) of gptq2d_tree_attention; scale defaults to dim^-1/2."""
        seqs, heads = context.shape[0], Q.shape[1] // self.dim
        with _on(stream, self.KC):
            O = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
            lse = torch.empty((Q.shape[0], heads), dtype=torch.float32, device=Q.device)
            ws = _bytes(gptq2d_tree_attention_workspace_size(seqs, Q.shape[0] // seqs, heads, self.heads, self.dim))
            gptq2d_tree_attention(Q, *self.tensors, table, context, drafts, masks,
                                  self.dim ** -0.5 if scale is None else scale, O, lse, ws)
        return O, lse


def tree_masks(parents: torch.Tensor, stream=None) -> torch.Tensor:
    """Masks (int64 bits) of trees of drafted tokens, from their parents (int32)."""
    with _on(stream, parents):
        masks = torch.empty(parents.shape, dtype=torch.int64, device=parents.device)
        gptq2d_tree_masks(parents, masks)
    return masks


class Scores(NamedTuple):
    logprob: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    ids: torch.Tensor | None
    tops: torch.Tensor | None


class _Scores(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, target, scale, top):
        ctx.set_materialize_grads(False)
        out = token_logprobs(X, target, scale, top)
        ctx.save_for_backward(X, target, out.lse, out.entropy)
        ctx.scale = scale
        if top:
            ctx.mark_non_differentiable(out.ids)
        return tuple(out)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logprob, g_entropy, g_lse, g_ids, g_tops):
        if g_lse is not None or g_tops is not None:
            raise RuntimeError("token_logprobs has gradients of the log probabilities and entropies only, not of lse or tops")
        X, target, lse, entropy = ctx.saved_tensors
        g_logprob, g_entropy = (None if g is None else g.contiguous() for g in (g_logprob, g_entropy))
        if target is None:
            g_logprob = None  # (of log probabilities that are 0 by convention)
        if g_logprob is None and g_entropy is None:
            return torch.zeros_like(X), None, None, None
        dX = torch.empty_like(X, memory_format=torch.contiguous_format)
        gptq2d_token_logprobs_backward(X, target, ctx.scale, lse, entropy, g_logprob, g_entropy, dX)
        return dX, None, None, None


def token_logprobs(X: torch.Tensor, target=None, scale: float = 1.0, top: int = 0, stream=None) -> Scores:
    """Scores of every row of logits X; ids and tops: the `top` largest. Where X
    requires a gradient, the log probabilities and entropies carry it."""
    rows, vocab = X.shape
    with _on(stream, X):
        if X.requires_grad and torch.is_grad_enabled():
            return Scores(*_Scores.apply(X, target, scale, top))
        out = [torch.empty(rows, dtype=torch.float32, device=X.device) for _ in range(3)]
        best = [torch.empty((rows, top), dtype=dt, device=X.device) if top else None
                for dt in (torch.int32, torch.float32)]
        gptq2d_token_logprobs(X, target, scale, *out, *best,
                              _bytes(gptq2d_token_logprobs_workspace_size(rows, vocab, top)))
    return Scores(*out, *best)


def token_logprobs_backward(X: torch.Tensor, target, scores: Scores, g_logprob=None, g_entropy=None, scale: float = 1.0,
                            stream=None) -> torch.Tensor:
    """The gradient of the logits from those of the log probabilities and entropies."""
    with _on(stream, X):
        dX = torch.empty_like(X, memory_format=torch.contiguous_format)
        gptq2d_token_logprobs_backward(X, target, scale, scores.lse, scores.entropy, g_logprob, g_entropy, dX)
    return dX
