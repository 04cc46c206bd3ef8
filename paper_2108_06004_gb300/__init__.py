"""Python binding of libgs_sketch, the GB300 gs-SGD gradient-compression library.

The functions below carry the names of the C ABI declared in ``include/gs_sketch.h`` and
only marshal arguments: tensors become device pointers (``tensor.data_ptr()``), lists of
tensors become host arrays of device pointers, and the stream defaults to PyTorch's
current stream.  Every step of the computation runs in the library's CUDA kernels; there
is no fallback.  A non-OK status raises ``GsError`` with the library's message.
"""

from __future__ import annotations

import ctypes
import functools
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgs_sketch.so")

GS_OK = 0
GS_ERR_INVALID_ARG = 1
GS_ERR_MISMATCH = 2
GS_ERR_OOM = 3
GS_ERR_CUDA = 4
GS_ERR_TIMEOUT = 5
GS_MAX_ROWS = 16
GS_MAX_COLS = 1 << 26
GS_MAX_WORKERS = 64
GS_MAX_DIM = (1 << 31) - 1
GS_NOALLOC_MAX_DIM = 1 << 30
GS_CEILING_WINDOW_FLOATS = 1 << 17
GS_F32 = 0
GS_F16 = 1
GS_BF16 = 2
GS_NORM_MAX_COLS = 16384

_lib = None

_vp = ctypes.c_void_p
_i32, _i64, _u64, _f32, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float, ctypes.c_size_t
_PP = ctypes.POINTER(ctypes.c_void_p)


class GsSeq(ctypes.Structure):
    """A [B][T][D] tensor: its address, batch and token strides in elements."""
    _fields_ = [("data", _vp), ("batch_stride", _i64), ("token_stride", _i64)]


_SEQ = ctypes.POINTER(GsSeq)

# name -> argument types (all return gs_status / int32 unless listed in _RESTYPES)
SIGNATURES = {
    "gs_sketch_create": [_i32, _i32, _u64, _i32, _i32, ctypes.POINTER(_vp)],
    "gs_sketch_destroy": [_vp],
    "gs_sketch_info": [_vp, ctypes.POINTER(_i32), ctypes.POINTER(_i32), ctypes.POINTER(_i32),
                       ctypes.POINTER(_i32), ctypes.POINTER(_i32)],
    "gs_sketch_coefficients": [_vp, ctypes.POINTER(_u64)],
    "gs_sketch_zero": [_vp, _vp],
    "gs_accumulate": [_vp, _vp, _vp, _i64, _f32, _vp],
    "gs_sketch_insert": [_vp, _i32, _vp, _i64, _vp],
    "gs_accumulate_insert": [_vp, _i32, _i32, _PP, _PP, _PP, _i64, _f32, _vp],
    "gs_accumulate_insert_staged": [_vp, _i32, _i32, _PP, _PP, _PP, _i64, _f32, _vp],
    "gs_sketch_merge_tree": [_vp, _i32, _vp],
    "gs_sketch_merge_sketches": [_PP, _i32, _vp],
    "gs_query_topk_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "gs_query_topk": [_vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp],
    "gs_query_topk_noalloc": [_vp, _i64, _i64, _vp, _vp, _vp],
    "gs_query_heavymix_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "gs_query_heavymix": [_vp, _i64, _i64, _u64, _vp, _vp, _vp, _vp, _sz, _vp],
    "gs_gather_and_zero": [_PP, _PP, _i32, _i64, _vp, _i64, _vp, _vp],
    "gs_apply_update": [_vp, _i64, _vp, _vp, _i64, _f32, _vp],
    "gs_gather_zero_update": [_PP, _PP, _i32, _i64, _vp, _i64, _vp, _vp, _f32, _vp],
    "gs_train_step": [_vp, _vp, _f32, _PP, _PP, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _vp, _sz, _vp],
    "gs_heavymix_step_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "gs_heavymix_step": [_vp, _PP, _PP, _PP, _i64, _f32, _i64, _u64, _vp, _vp, _vp, _vp, _sz, _vp],
    "gs_heavymix_step_plan_create": [_vp, _PP, _PP, _PP, _i64, _f32, _i64, _u64, _vp, _vp, _vp, _vp, _sz, _i32,
                                     ctypes.POINTER(_vp)],
    "gs_sketch_merged_table": [_vp, ctypes.POINTER(_vp)],
    "gs_sketch_query_at": [_vp, _vp, _i64, _vp, _vp],
    "gs_sketch_add_sparse": [_vp, _vp, _vp, _i64, _f32, _vp],
    "gs_sketched_state_step": [_vp, _vp, _vp, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _f32, _vp, _sz, _vp],
    "gs_step_plan_create": [_vp, _PP, _PP, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _vp, _f32, _vp, _sz, _i32,
                            ctypes.POINTER(_vp)],
    "gs_step_host_plan_create": [_vp, _PP, _PP, _PP, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _sz, _i32,
                                 ctypes.POINTER(_vp)],
    "gs_sketched_state_plan_create": [_vp, _vp, _vp, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _f32, _vp, _sz, _i32,
                                      ctypes.POINTER(_vp)],
    "gs_plan_launch": [_vp, _vp],
    "gs_plan_insert_times": [_vp, _vp, _i32, ctypes.POINTER(_i32)],
    "gs_plan_query_times": [_vp, _vp, _vp, _i32, ctypes.POINTER(_i32)],
    "gs_plan_destroy": [_vp],
    "gs_step_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "gs_step": [_vp, _PP, _PP, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _vp, _sz, _vp],
    "gs_step_host": [_vp, _PP, _PP, _PP, _PP, _i64, _f32, _i64, _vp, _vp, _vp, _sz, _vp],
    "gs_dropout": [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _i32, _f32, _u64, _u64, _vp],
    "gs_dropout_backward": [_vp, _i64, _vp, _i64, _i64, _i64, _i32, _f32, _u64, _u64, _vp],
    "gs_dropout_add_norm": [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _i32, _f32, _u64, _u64,
                            _f32, _vp],
    "gs_dropout_add_norm_workspace_size": [_i64, _i64, ctypes.POINTER(_sz)],
    "gs_dropout_add_norm_backward": [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _i64,
                                     _i32, _f32, _u64, _u64, _vp, _sz, _vp],
    "gs_recurrence_states_size": [_i64, _i64, _i64, ctypes.POINTER(_sz)],
    "gs_recurrence_workspace_size": [_i64, _i64, _i64, ctypes.POINTER(_sz)],
    "gs_recurrence_forward": [_SEQ, _SEQ, _SEQ, _vp, _vp, _vp, _vp, _SEQ, _vp, _vp, _i64, _i64, _i64, _i32, _f32, _vp],
    "gs_recurrence_backward": [_SEQ, _vp, _SEQ, _SEQ, _SEQ, _vp, _vp, _vp, _vp, _SEQ, _SEQ, _SEQ, _vp, _vp, _i64, _i64,
                               _i64, _i32, _f32, _vp, _sz, _vp],
    "gs_recurrence_wait_tries": [_i32, _i32],
    "gs_recurrence_step": [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _i32,
                           _f32, _vp],
    "gs_insert_request_ceiling_window_size": [_vp, ctypes.POINTER(_sz)],
    "gs_insert_request_ceiling": [_vp, _i64, _vp, _sz, ctypes.POINTER(_f32), _vp],
    "gs_query_request_ceiling": [_vp, _i64, _vp, _sz, ctypes.POINTER(_f32), _vp],
    "gs_hash_eval": [_vp, _vp, _i64, _vp, _vp, _vp],
    "gs_sketch_copy_to_host": [_vp, _i32, _vp],
    "gs_last_error": [],
}
_RESTYPES = {"gs_last_error": ctypes.c_char_p}


class GsError(RuntimeError):
    def __init__(self, status: int, func: str, msg: str):
        super().__init__(f"{func} failed with status {status}: {msg}")
        self.status = status


def load_library():
    """Load libgs_sketch.so (built by ``paper_2108_06004_gb300._build``); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -c \"import __graft_entry__ as g; g.build()\"` "
                "(the CUDA library is required; there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, args in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = _RESTYPES.get(name, _i32)
        _lib = lib
    return _lib


def _check(status: int, func: str):
    if status != GS_OK:
        msg = load_library().gs_last_error().decode(errors="replace")
        raise GsError(status, func, msg)


def _ptr(x) -> int | None:
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    return int(x)


def _ptr_array(xs):
    return (ctypes.c_void_p * len(xs))(*[_ptr(x) for x in xs])


def _stream(stream):
    if stream is not None:
        return _ptr(getattr(stream, "cuda_stream", stream))
    return _current_stream(_torch().cuda.current_device())


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _current_stream(device: int) -> int:
    """Handle of PyTorch's current stream.  The stream object that the public call makes costs
    more than a kernel launch, so the handle is taken from where that call takes it."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw is not None else torch.cuda.current_stream(device).cuda_stream


# ---- C ABI, same names ------------------------------------------------------------------

def gs_sketch_create(r: int, c: int, seed: int, workers: int, group_width: int = 0) -> int:
    out = _vp()
    _check(load_library().gs_sketch_create(r, c, seed, workers, group_width, ctypes.byref(out)),
           "gs_sketch_create")
    return out.value


def gs_sketch_destroy(sketch: int) -> None:
    _check(load_library().gs_sketch_destroy(sketch), "gs_sketch_destroy")


def gs_sketch_info(sketch: int) -> dict:
    r, c, w, g, rp = _i32(), _i32(), _i32(), _i32(), _i32()
    _check(load_library().gs_sketch_info(sketch, ctypes.byref(r), ctypes.byref(c), ctypes.byref(w),
                                         ctypes.byref(g), ctypes.byref(rp)), "gs_sketch_info")
    return {"r": r.value, "c": c.value, "workers": w.value, "group_width": g.value,
            "rows_per_pass": rp.value}


def gs_sketch_coefficients(sketch: int):
    """(a, b, a2, b2) lists of Python ints, one entry per row."""
    r = gs_sketch_info(sketch)["r"]
    buf = (_u64 * (4 * r))()
    _check(load_library().gs_sketch_coefficients(sketch, buf), "gs_sketch_coefficients")
    v = list(buf)
    return v[0::4], v[1::4], v[2::4], v[3::4]


def gs_sketch_zero(sketch: int, stream=None) -> None:
    _check(load_library().gs_sketch_zero(sketch, _stream(stream)), "gs_sketch_zero")


def gs_accumulate(momentum, error, grad, d: int, rho: float, stream=None) -> None:
    _check(load_library().gs_accumulate(_ptr(momentum), _ptr(error), _ptr(grad), d, rho,
                                        _stream(stream)), "gs_accumulate")


def gs_sketch_insert(sketch: int, worker: int, vec, d: int, stream=None) -> None:
    _check(load_library().gs_sketch_insert(sketch, worker, _ptr(vec), d, _stream(stream)),
           "gs_sketch_insert")


def gs_accumulate_insert(sketch: int, first_worker: int, momentum, error, grad, d: int,
                         rho: float, stream=None) -> None:
    n = len(grad)
    _check(load_library().gs_accumulate_insert(sketch, first_worker, n, _ptr_array(momentum),
                                               _ptr_array(error), _ptr_array(grad), d, rho,
                                               _stream(stream)), "gs_accumulate_insert")


def gs_accumulate_insert_staged(sketch: int, first_worker: int, momentum, error, grad, d: int,
                                rho: float, stream=None) -> None:
    n = len(grad)
    _check(load_library().gs_accumulate_insert_staged(sketch, first_worker, n, _ptr_array(momentum),
                                                      _ptr_array(error), _ptr_array(grad), d, rho,
                                                      _stream(stream)), "gs_accumulate_insert_staged")


def gs_sketch_merge_tree(sketch: int, P: int, stream=None) -> None:
    _check(load_library().gs_sketch_merge_tree(sketch, P, _stream(stream)), "gs_sketch_merge_tree")


def gs_sketch_merge_sketches(sketches, stream=None) -> None:
    """Tree merge of separately created sketches into the merged table of sketches[0]."""
    arr = (ctypes.c_void_p * len(sketches))(*sketches)
    _check(load_library().gs_sketch_merge_sketches(arr, len(sketches), _stream(stream)), "gs_sketch_merge_sketches")


def gs_query_topk_workspace_size(d: int, k: int) -> int:
    out = _sz()
    _check(load_library().gs_query_topk_workspace_size(d, k, ctypes.byref(out)),
           "gs_query_topk_workspace_size")
    return out.value


def gs_query_topk(sketch: int, d: int, k: int, idx_out, est_out, workspace, workspace_bytes=None,
                  stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_query_topk(sketch, d, k, _ptr(idx_out), _ptr(est_out), _ptr(workspace),
                                        workspace_bytes, _stream(stream)), "gs_query_topk")


def gs_query_heavymix_workspace_size(d: int, k: int) -> int:
    out = _sz()
    _check(load_library().gs_query_heavymix_workspace_size(d, k, ctypes.byref(out)),
           "gs_query_heavymix_workspace_size")
    return out.value


def gs_query_heavymix(sketch: int, d: int, k: int, fill_seed: int, idx_out, est_out, l2sq_out, workspace,
                      workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_query_heavymix(sketch, d, k, fill_seed, _ptr(idx_out), _ptr(est_out), _ptr(l2sq_out),
                                            _ptr(workspace), workspace_bytes, _stream(stream)), "gs_query_heavymix")


def gs_query_topk_noalloc(sketch: int, d: int, k: int, idx_out, est_out, stream=None) -> None:
    """gs_query_topk without a caller workspace: the library's fixed device scratch is used
    (for hosts that cannot allocate device memory; est_out is required)."""
    _check(load_library().gs_query_topk_noalloc(sketch, d, k, _ptr(idx_out), _ptr(est_out), _stream(stream)),
           "gs_query_topk_noalloc")


def gs_gather_and_zero(momentum, error, d: int, idx, k: int, vals_out, stream=None) -> None:
    P = len(momentum)
    _check(load_library().gs_gather_and_zero(_ptr_array(momentum), _ptr_array(error), P, d, _ptr(idx), k,
                                             _ptr(vals_out), _stream(stream)), "gs_gather_and_zero")


def gs_apply_update(weights, d: int, idx, vals, k: int, lr: float, stream=None) -> None:
    _check(load_library().gs_apply_update(_ptr(weights), d, _ptr(idx), _ptr(vals), k, lr, _stream(stream)),
           "gs_apply_update")


def gs_gather_zero_update(momentum, error, d: int, idx, k: int, vals_out, weights, lr: float,
                          stream=None) -> None:
    P = len(momentum)
    _check(load_library().gs_gather_zero_update(_ptr_array(momentum), _ptr_array(error), P, d, _ptr(idx), k,
                                                _ptr(vals_out), _ptr(weights), lr, _stream(stream)),
           "gs_gather_zero_update")


def gs_train_step(sketch: int, weights, lr: float, momentum, error, grad, d: int, rho: float, k: int,
                  idx_out, vals_out, est_out, workspace, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_train_step(sketch, _ptr(weights), lr, _ptr_array(momentum), _ptr_array(error),
                                        _ptr_array(grad), d, rho, k, _ptr(idx_out), _ptr(vals_out), _ptr(est_out),
                                        _ptr(workspace), workspace_bytes, _stream(stream)), "gs_train_step")


def gs_sketch_merged_table(sketch: int) -> int:
    out = _vp()
    _check(load_library().gs_sketch_merged_table(sketch, ctypes.byref(out)), "gs_sketch_merged_table")
    return out.value


def gs_sketch_query_at(sketch: int, idx, k: int, est_out, stream=None) -> None:
    _check(load_library().gs_sketch_query_at(sketch, _ptr(idx), k, _ptr(est_out), _stream(stream)),
           "gs_sketch_query_at")


def gs_sketch_add_sparse(sketch: int, idx, vals, k: int, scale: float, stream=None) -> None:
    _check(load_library().gs_sketch_add_sparse(sketch, _ptr(idx), _ptr(vals), k, scale, _stream(stream)),
           "gs_sketch_add_sparse")


def gs_sketched_state_step(workers: int, momentum: int, error: int, grad, d: int, rho: float, k: int, idx_out,
                           vals_out, weights, lr: float, workspace, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_sketched_state_step(workers, momentum, error, _ptr_array(grad), d, rho, k, _ptr(idx_out),
                                                 _ptr(vals_out), _ptr(weights), lr, _ptr(workspace), workspace_bytes,
                                                 _stream(stream)), "gs_sketched_state_step")


def gs_step_workspace_size(d: int, k: int) -> int:
    out = _sz()
    _check(load_library().gs_step_workspace_size(d, k, ctypes.byref(out)), "gs_step_workspace_size")
    return out.value


def gs_step(sketch: int, momentum, error, grad, d: int, rho: float, k: int, idx_out, vals_out,
            est_out, workspace, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_step(sketch, _ptr_array(momentum), _ptr_array(error), _ptr_array(grad), d, rho, k,
                                  _ptr(idx_out), _ptr(vals_out), _ptr(est_out), _ptr(workspace),
                                  workspace_bytes, _stream(stream)), "gs_step")


def gs_step_host(sketch: int, momentum, error, grad_host, grad_dev, d: int, rho: float, k: int,
                 idx_host, vals_host, workspace, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(load_library().gs_step_host(sketch, _ptr_array(momentum), _ptr_array(error), _ptr_array(grad_host),
                                       _ptr_array(grad_dev), d, rho, k, _ptr(idx_host), _ptr(vals_host),
                                       _ptr(workspace), workspace_bytes, _stream(stream)), "gs_step_host")


GS_PLAN_TIME_INSERT = 1
GS_PLAN_TIME_QUERY = 2


def _nbytes(workspace, workspace_bytes):
    return workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes


def gs_heavymix_step_workspace_size(d: int, k: int) -> int:
    out = _sz()
    _check(load_library().gs_heavymix_step_workspace_size(d, k, ctypes.byref(out)), "gs_heavymix_step_workspace_size")
    return out.value


def gs_heavymix_step(sketch: int, momentum, error, grad, d: int, rho: float, k: int, fill_seed: int, idx_out,
                     vals_out, l2sq_out, workspace, workspace_bytes=None, stream=None) -> None:
    _check(load_library().gs_heavymix_step(sketch, _ptr_array(momentum), _ptr_array(error), _ptr_array(grad), d, rho,
                                           k, fill_seed, _ptr(idx_out), _ptr(vals_out), _ptr(l2sq_out),
                                           _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)),
           "gs_heavymix_step")


def gs_heavymix_step_plan_create(sketch: int, momentum, error, grad, d: int, rho: float, k: int, fill_seed: int,
                                 idx_out, vals_out, l2sq_out, workspace, workspace_bytes=None, flags: int = 0) -> int:
    out = _vp()
    _check(load_library().gs_heavymix_step_plan_create(sketch, _ptr_array(momentum), _ptr_array(error),
                                                       _ptr_array(grad), d, rho, k, fill_seed, _ptr(idx_out),
                                                       _ptr(vals_out), _ptr(l2sq_out), _ptr(workspace),
                                                       _nbytes(workspace, workspace_bytes), flags,
                                                       ctypes.byref(out)), "gs_heavymix_step_plan_create")
    return out.value


def gs_step_plan_create(sketch: int, momentum, error, grad, d: int, rho: float, k: int, idx_out, vals_out,
                        est_out=None, weights=None, lr: float = 0.0, workspace=None, workspace_bytes=None,
                        flags: int = 0) -> int:
    out = _vp()
    _check(load_library().gs_step_plan_create(sketch, _ptr_array(momentum), _ptr_array(error), _ptr_array(grad), d,
                                              rho, k, _ptr(idx_out), _ptr(vals_out), _ptr(est_out), _ptr(weights), lr,
                                              _ptr(workspace), _nbytes(workspace, workspace_bytes), flags,
                                              ctypes.byref(out)), "gs_step_plan_create")
    return out.value


def gs_step_host_plan_create(sketch: int, momentum, error, grad_host, grad_dev, d: int, rho: float, k: int,
                             idx_host, vals_host, workspace, workspace_bytes=None, flags: int = 0) -> int:
    out = _vp()
    _check(load_library().gs_step_host_plan_create(sketch, _ptr_array(momentum), _ptr_array(error),
                                                   _ptr_array(grad_host), _ptr_array(grad_dev), d, rho, k,
                                                   _ptr(idx_host), _ptr(vals_host), _ptr(workspace),
                                                   _nbytes(workspace, workspace_bytes), flags, ctypes.byref(out)),
           "gs_step_host_plan_create")
    return out.value


def gs_sketched_state_plan_create(workers: int, momentum: int, error: int, grad, d: int, rho: float, k: int,
                                  idx_out, vals_out, weights, lr: float, workspace, workspace_bytes=None,
                                  flags: int = 0) -> int:
    out = _vp()
    _check(load_library().gs_sketched_state_plan_create(workers, momentum, error, _ptr_array(grad), d, rho, k,
                                                        _ptr(idx_out), _ptr(vals_out), _ptr(weights), lr,
                                                        _ptr(workspace), _nbytes(workspace, workspace_bytes), flags,
                                                        ctypes.byref(out)), "gs_sketched_state_plan_create")
    return out.value


def gs_plan_launch(plan: int, stream=None) -> None:
    _check(load_library().gs_plan_launch(plan, _stream(stream)), "gs_plan_launch")


def gs_plan_insert_times(plan: int, n: int = 1024) -> list:
    buf = (ctypes.c_float * max(n, 1))()
    got = _i32()
    _check(load_library().gs_plan_insert_times(plan, ctypes.cast(buf, _vp), n, ctypes.byref(got)),
           "gs_plan_insert_times")
    return [float(buf[i]) for i in range(got.value)]


def gs_plan_query_times(plan: int, n: int = 1024) -> tuple:
    """(query_ms, select_ms): lists over the last launches, oldest first."""
    q = (ctypes.c_float * max(n, 1))()
    sel = (ctypes.c_float * max(n, 1))()
    got = _i32()
    _check(load_library().gs_plan_query_times(plan, ctypes.cast(q, _vp), ctypes.cast(sel, _vp), n,
                                              ctypes.byref(got)), "gs_plan_query_times")
    return [float(q[i]) for i in range(got.value)], [float(sel[i]) for i in range(got.value)]


def gs_plan_destroy(plan: int) -> None:
    _check(load_library().gs_plan_destroy(plan), "gs_plan_destroy")


# ---- operators of a recurrent layer -------------------------------------------------------
# Tensors are torch tensors on the GPU; shapes, strides and types are read from them, and what
# the C ABI cannot see of them is checked here.

_CODES = {}


def _refuse(func: str, msg: str):
    raise GsError(GS_ERR_INVALID_ARG, func, msg)


def _dtype(func: str, t) -> int:
    if t is None:
        _refuse(func, "the first tensor is missing")
    if not _CODES:
        torch = _torch()
        _CODES.update({torch.float32: GS_F32, torch.float16: GS_F16, torch.bfloat16: GS_BF16})
    code = _CODES.get(t.dtype)
    if code is None:
        _refuse(func, f"dtype {t.dtype} is none of float32, float16, bfloat16")
    return code


def _unlike(func: str, name: str, t, shape, dtype, device):
    """Refuses a tensor that is not of this shape and type on this device."""
    if t.shape != shape:
        _refuse(func, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        _refuse(func, f"{name} has type {t.dtype}, expected {dtype}")
    _refuse(func, f"{name} is on {t.device}, expected {device}")


def _launch_stream(func: str, t, stream):
    """The stream to launch on; the tensors have to be on the current device."""
    if not t.is_cuda:
        _refuse(func, f"the tensors are on {t.device}, expected a CUDA device")
    device = _torch().cuda.current_device()
    if t.get_device() != device:
        _refuse(func, f"the tensors are on {t.device}, the current device is {device}")
    return _current_stream(device) if stream is None else _stream(stream)


def _dense(func: str, name: str, t, shape, dtype, device):
    """Address of a contiguous tensor, or None for an absent one."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        _unlike(func, name, t, shape, dtype, device)
    if not t.is_contiguous():
        _refuse(func, f"{name} must be contiguous")
    return t.data_ptr()


def _matrix(func: str, name: str, t, shape, dtype, device):
    """(address, row stride) of a tensor whose last dimension is adjacent and whose others can be
    walked with one stride; (None, 0) for an absent one."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        _unlike(func, name, t, shape, dtype, device)
    if t.is_contiguous():
        return t.data_ptr(), shape[-1]
    stride = t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        _refuse(func, f"{name}: the last dimension must be adjacent")
    row, span = None, None   # of the innermost leading dimension with more than one entry, outwards
    for size, st in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if size == 1:
            continue
        if row is None:
            row, span = st, st * size
        elif st != span:
            _refuse(func, f"{name}: the rows cannot be walked with one stride")
        else:
            span = st * size
    return t.data_ptr(), shape[-1] if row is None else row


def _room(func: str, name: str, t, device, size=None):
    """(address, bytes) of a workspace: a contiguous tensor, of which `size` bytes may be used, or an
    address with its size."""
    if not hasattr(t, "data_ptr"):
        return _ptr(t), size or 0
    if t.device != device:
        _refuse(func, f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        _refuse(func, f"{name} must be contiguous")
    have = t.numel() * t.element_size()
    if size is not None and size > have:
        _refuse(func, f"{name} holds {have} bytes, not {size}")
    return t.data_ptr(), have if size is None else size


def _rows_cols(func: str, t):
    if t.dim() < 1:
        _refuse(func, "a tensor of at least one dimension is expected")
    cols = t.shape[-1]
    if cols:
        return t.numel() // cols, cols
    rows = 1
    for n in t.shape[:-1]:
        rows *= n
    return rows, cols


def gs_dropout(x, out, p: float, seed: int, offset: int, residual=None, stream=None) -> None:
    """out = dropout(x) (+ residual); any shape, the mask indexed by the element's flat position."""
    f = "gs_dropout"
    code = _dtype(f, x)
    stream = _launch_stream(f, x, stream)
    rows, cols = _rows_cols(f, x)
    shape, dtype, dev = x.shape, x.dtype, x.device
    xp, xs = _matrix(f, "x", x, shape, dtype, dev)
    rp, rs = _matrix(f, "residual", residual, shape, dtype, dev)
    op, os_ = _matrix(f, "out", out, shape, dtype, dev)
    _check(load_library().gs_dropout(xp, xs, rp, rs, op, os_, rows, cols, code, p, seed, offset, stream), f)


def gs_dropout_backward(dout, dx, p: float, seed: int, offset: int, stream=None) -> None:
    """dx = the gradient of gs_dropout's x from that of its out."""
    f = "gs_dropout_backward"
    code = _dtype(f, dout)
    stream = _launch_stream(f, dout, stream)
    rows, cols = _rows_cols(f, dout)
    shape, dtype, dev = dout.shape, dout.dtype, dout.device
    gp, gstride = _matrix(f, "dout", dout, shape, dtype, dev)
    op, os_ = _matrix(f, "dx", dx, shape, dtype, dev)
    _check(load_library().gs_dropout_backward(gp, gstride, op, os_, rows, cols, code, p, seed, offset, stream), f)


def gs_dropout_add_norm(x, residual, weight, y, z, rstd, p: float, seed: int, offset: int, eps: float = 1e-6,
                        stream=None) -> None:
    """y = residual + dropout(x), z = RMS norm of y times weight, over the last dimension."""
    f = "gs_dropout_add_norm"
    code = _dtype(f, x)
    stream = _launch_stream(f, x, stream)
    rows, cols = _rows_cols(f, x)
    shape, dtype, dev, f32 = x.shape, x.dtype, x.device, _torch().float32
    xp, xs = _matrix(f, "x", x, shape, dtype, dev)
    rp, rs = _matrix(f, "residual", residual, shape, dtype, dev)
    yp, ys = _matrix(f, "y", y, shape, dtype, dev)
    zp, zs = _matrix(f, "z", z, shape, dtype, dev)
    _check(load_library().gs_dropout_add_norm(
        xp, xs, rp, rs, _dense(f, "weight", weight, (cols,), f32, dev), yp, ys, zp, zs,
        _dense(f, "rstd", rstd, shape[:-1], f32, dev), rows, cols, code, p, seed, offset, eps, stream), f)


def gs_dropout_add_norm_workspace_size(rows: int, cols: int) -> int:
    out = _sz()
    _check(load_library().gs_dropout_add_norm_workspace_size(rows, cols, ctypes.byref(out)),
           "gs_dropout_add_norm_workspace_size")
    return out.value


def gs_dropout_add_norm_backward(dz, dy, y, weight, rstd, dx, dresidual, dweight, p: float, seed: int, offset: int,
                                 workspace, workspace_bytes=None, stream=None) -> None:
    """Gradients of gs_dropout_add_norm; dy, dx and dresidual may be None."""
    f = "gs_dropout_add_norm_backward"
    code = _dtype(f, dz)
    stream = _launch_stream(f, dz, stream)
    rows, cols = _rows_cols(f, dz)
    shape, dtype, dev, f32 = dz.shape, dz.dtype, dz.device, _torch().float32
    gp, gstride = _matrix(f, "dz", dz, shape, dtype, dev)
    dp, ds = _matrix(f, "dy", dy, shape, dtype, dev)
    yp, ys = _matrix(f, "y", y, shape, dtype, dev)
    xp, xs = _matrix(f, "dx", dx, shape, dtype, dev)
    rp, rs = _matrix(f, "dresidual", dresidual, shape, dtype, dev)
    wp, wn = _room(f, "workspace", workspace, dev, workspace_bytes)
    _check(load_library().gs_dropout_add_norm_backward(
        gp, gstride, dp, ds, yp, ys, _dense(f, "weight", weight, (cols,), f32, dev),
        _dense(f, "rstd", rstd, shape[:-1], f32, dev), xp, xs, rp, rs, _dense(f, "dweight", dweight, (cols,), f32, dev),
        rows, cols, code, p, seed, offset, wp, wn, stream), f)


def _seq(func: str, name: str, t, shape, dtype, device):
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        _unlike(func, name, t, shape, dtype, device)
    b, s, d = t.stride()
    if d != 1 and shape[2] > 1:
        _refuse(func, f"{name}: the channels must be adjacent")
    return GsSeq(t.data_ptr(), b, s)


def _resets(func: str, t, shape, device):
    if t is None:
        return None
    torch = _torch()
    return _dense(func, "reset", t.view(torch.uint8) if t.dtype == torch.bool else t, shape, torch.uint8, device)


def _whole(func: str, name: str, t, shape, device):
    return None if t is None else _dense(func, name, t, shape, _torch().int32, device)


def _sequence(func: str, t):
    if t.dim() != 3:
        _refuse(func, f"tensors of [B][T][D] are expected, got {t.dim()} dimensions")
    return t.shape


def gs_recurrence_states_size(B: int, T: int, D: int) -> int:
    out = _sz()
    _check(load_library().gs_recurrence_states_size(B, T, D, ctypes.byref(out)), "gs_recurrence_states_size")
    return out.value


def gs_recurrence_workspace_size(B: int, T: int, D: int) -> int:
    out = _sz()
    _check(load_library().gs_recurrence_workspace_size(B, T, D, ctypes.byref(out)), "gs_recurrence_workspace_size")
    return out.value


_states_size = functools.lru_cache(maxsize=256)(gs_recurrence_states_size)   # a function of the sizes alone


def _states_fit(func: str, states, B: int, T: int, D: int, device=None) -> None:
    if states is None:
        return   # the library knows whether it needs them
    if device is not None and states.device != device:
        _refuse(func, f"states is on {states.device}, expected {device}")
    if states.numel() * states.element_size() < _states_size(B, T, D) or not states.is_contiguous():
        _refuse(func, "states must be contiguous and hold gs_recurrence_states_size(B, T, D) bytes")


def gs_recurrence_forward(x, r, i, decay, y, h0=None, reset=None, lengths=None, h_last=None, states=None,
                          c: float = 8.0, stream=None) -> None:
    """y_t = h_t of the gated linear recurrence over [B][T][D]; states keeps what the backward
    pass needs (None when there is none)."""
    f = "gs_recurrence_forward"
    code = _dtype(f, x)
    shape = B, T, D = _sequence(f, x)
    stream = _launch_stream(f, x, stream)
    dtype, dev, f32 = x.dtype, x.device, _torch().float32
    _states_fit(f, states, B, T, D, dev)
    _check(load_library().gs_recurrence_forward(
        _seq(f, "x", x, shape, dtype, dev), _seq(f, "r", r, shape, dtype, dev), _seq(f, "i", i, shape, dtype, dev),
        _dense(f, "decay", decay, (D,), f32, dev), _dense(f, "h0", h0, (B, D), f32, dev),
        _resets(f, reset, (B, T), dev), _whole(f, "lengths", lengths, (B,), dev),
        _seq(f, "y", y, shape, dtype, dev), _dense(f, "h_last", h_last, (B, D), f32, dev), _ptr(states), B, T, D, code,
        c, stream), f)


def gs_recurrence_backward(dy, x, r, i, decay, states, dx, dr, di, ddecay, workspace, dh_last=None, reset=None,
                           lengths=None, dh0=None, c: float = 8.0, workspace_bytes=None, stream=None) -> None:
    """Gradients of gs_recurrence_forward from dy and dh_last, its inputs and the states it filled."""
    f = "gs_recurrence_backward"
    code = _dtype(f, x)
    shape = B, T, D = _sequence(f, x)
    stream = _launch_stream(f, x, stream)
    dtype, dev, f32 = x.dtype, x.device, _torch().float32
    _states_fit(f, states, B, T, D, dev)
    wp, wn = _room(f, "workspace", workspace, dev, workspace_bytes)
    _check(load_library().gs_recurrence_backward(
        _seq(f, "dy", dy, shape, dtype, dev), _dense(f, "dh_last", dh_last, (B, D), f32, dev),
        _seq(f, "x", x, shape, dtype, dev), _seq(f, "r", r, shape, dtype, dev), _seq(f, "i", i, shape, dtype, dev),
        _dense(f, "decay", decay, (D,), f32, dev), _resets(f, reset, (B, T), dev),
        _whole(f, "lengths", lengths, (B,), dev), _ptr(states), _seq(f, "dx", dx, shape, dtype, dev),
        _seq(f, "dr", dr, shape, dtype, dev), _seq(f, "di", di, shape, dtype, dev),
        _dense(f, "ddecay", ddecay, (D,), f32, dev), _dense(f, "dh0", dh0, (B, D), f32, dev), B, T, D, code, c,
        wp, wn, stream), f)


def gs_recurrence_wait_tries(tiles: int = 1 << 20, messages: int = 1 << 20) -> None:
    """Tries of the sequence kernels' waits in later calls of this thread, for tests of waits that run out."""
    _check(load_library().gs_recurrence_wait_tries(tiles, messages), "gs_recurrence_wait_tries")


def gs_recurrence_step(x, r, i, decay, state, y, slots=None, c: float = 8.0, stream=None) -> None:
    """One token of each of B streams: state rows (fp32, one per slot) in place, y = the new state."""
    f = "gs_recurrence_step"
    code = _dtype(f, x)
    stream = _launch_stream(f, x, stream)
    B, D = _rows_cols(f, x)
    shape, dtype, dev, f32 = x.shape, x.dtype, x.device, _torch().float32
    xp, xs = _matrix(f, "x", x, shape, dtype, dev)
    rp, rs = _matrix(f, "r", r, shape, dtype, dev)
    ip, istride = _matrix(f, "i", i, shape, dtype, dev)
    yp, ys = _matrix(f, "y", y, shape, dtype, dev)
    if state is None or state.dim() != 2:
        _refuse(f, "state must have two dimensions")
    n = state.shape[0]
    sp, ss = _matrix(f, "state", state, (n, D), f32, dev)
    _check(load_library().gs_recurrence_step(
        xp, xs, rp, rs, ip, istride, _dense(f, "decay", decay, (D,), f32, dev), sp, ss, n,
        _whole(f, "slots", slots, (B,), dev), yp, ys, B, D, code, c, stream), f)


def gs_insert_request_ceiling_window_size(sketch: int) -> int:
    out = _sz()
    _check(load_library().gs_insert_request_ceiling_window_size(sketch, ctypes.byref(out)),
           "gs_insert_request_ceiling_window_size")
    return out.value


def gs_insert_request_ceiling(sketch: int, d: int, window, window_bytes=None, stream=None) -> float:
    """Milliseconds of one insert phase's request mix with the vectors held in L2."""
    ms = _f32()
    _check(load_library().gs_insert_request_ceiling(sketch, d, _ptr(window), _nbytes(window, window_bytes),
                                                    ctypes.byref(ms), _stream(stream)), "gs_insert_request_ceiling")
    return float(ms.value)


def gs_query_request_ceiling(sketch: int, d: int, window, window_bytes=None, stream=None) -> float:
    """Milliseconds of the median query's loads alone (all r rows) for d coordinates."""
    ms = _f32()
    _check(load_library().gs_query_request_ceiling(sketch, d, _ptr(window), _nbytes(window, window_bytes),
                                                   ctypes.byref(ms), _stream(stream)), "gs_query_request_ceiling")
    return float(ms.value)


def gs_hash_eval(sketch: int, coords, n: int, bucket_out, sign_out, stream=None) -> None:
    _check(load_library().gs_hash_eval(sketch, _ptr(coords), n, _ptr(bucket_out), _ptr(sign_out),
                                       _stream(stream)), "gs_hash_eval")


def gs_sketch_copy_to_host(sketch: int, worker: int, host_out) -> None:
    """host_out: a contiguous host fp32 buffer of r*c values (numpy array or tensor)."""
    ptr = host_out.ctypes.data if hasattr(host_out, "ctypes") else _ptr(host_out)
    _check(load_library().gs_sketch_copy_to_host(sketch, worker, ptr), "gs_sketch_copy_to_host")


def gs_last_error() -> str:
    return load_library().gs_last_error().decode(errors="replace")
