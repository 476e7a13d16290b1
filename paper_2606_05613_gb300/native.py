"""ctypes binding of the C ABI in include/bkmoo.h.

Argument marshalling only: every step of the resolve runs in the CUDA library
(libbkmoo.so, built in-tree by paper_2606_05613_gb300.build).  There is no
CPU or PyTorch fallback; if the library is missing or cannot be loaded, every
call raises.  Functions carry the C names; torch tensors supply device
pointers and the current CUDA stream.
"""
from __future__ import annotations

import array
import ctypes
import operator
import os
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbkmoo.so")

BKMOO_OK = 0
BKMOO_ERR_INVALID = 1
BKMOO_ERR_CUDA = 2
BKMOO_ERR_NONFINITE = 3
BKMOO_ERR_WORKSPACE = 4
BKMOO_ERR_TIMEOUT = 5
BKMOO_ERR_BUFFER_TOO_SMALL = 6
BKMOO_ERR_NOT_CONVERGED = 7

BKMOO_MGDA, BKMOO_PCGRAD, BKMOO_CAGRAD, BKMOO_MEAN = 0, 1, 2, 3
BKMOO_F32, BKMOO_BF16, BKMOO_E4M3 = 0, 1, 2
BKMOO_FLAG_CLOSED_FORM_K2 = 0x1
BKMOO_FLAG_POLISH = 0x2
BKMOO_FLAG_FUSED = 0x4
BKMOO_FLAG_THREE_PASS = 0x8
BKMOO_FLAG_TEST_WITHHOLD = 0x100
BKMOO_FLAG_TEST_WITHHOLD_EXCHANGE = 0x200
BKMOO_NORM_WS_BYTES = 16384
BKMOO_SILU, BKMOO_GELU, BKMOO_GELU_TANH = 0, 1, 2
BKMOO_NOALLOC_SCRATCH_BYTES = 32 << 20
BKMOO_NOALLOC_MAX_BUCKETS = 4096

RULES = {"mgda": BKMOO_MGDA, "pcgrad": BKMOO_PCGRAD, "cagrad": BKMOO_CAGRAD, "mean": BKMOO_MEAN}
ACTS = {"silu": BKMOO_SILU, "gelu": BKMOO_GELU, "gelu_tanh": BKMOO_GELU_TANH}

_lock = threading.Lock()
_lib = None


class BkmooError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (where, bkmoo_status_string(code), code))


class bkmoo_params(ctypes.Structure):
    _fields_ = [
        ("max_iter", ctypes.c_int32),
        ("tol", ctypes.c_double),
        ("cagrad_c", ctypes.c_double),
        ("seed", ctypes.c_uint64),
        ("step", ctypes.c_uint64),
        ("flags", ctypes.c_uint32),
        ("events", ctypes.c_void_p),
    ]


class bkmoo_adamw_params(ctypes.Structure):
    _fields_ = [
        ("lr", ctypes.c_double),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("max_norm", ctypes.c_double),
        ("step", ctypes.c_int64),
        ("seed", ctypes.c_uint64),
    ]


def load():
    """Load libbkmoo.so (raises if it is missing: there is no fallback)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libbkmoo.so is not built (%s); run "
                               "paper_2606_05613_gb300.build.build()" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        i32, i64, sz, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p
        lib.bkmoo_default_params.restype = None
        lib.bkmoo_default_params.argtypes = [ctypes.POINTER(bkmoo_params)]
        lib.bkmoo_plan.restype = ctypes.c_int
        lib.bkmoo_plan.argtypes = [vp, i32, i32, i64, vp, i64, ctypes.POINTER(i64)]
        lib.bkmoo_workspace_size.restype = ctypes.c_int
        lib.bkmoo_workspace_size.argtypes = [i32, i32, vp, i64, ctypes.POINTER(sz)]
        lib.bkmoo_workspace_init.restype = ctypes.c_int
        lib.bkmoo_workspace_init.argtypes = [i32, i32, vp, i64, vp, sz, vp]
        lib.bkmoo_gram.restype = ctypes.c_int
        lib.bkmoo_gram.argtypes = [vp, i32, i32, vp, i64, vp, vp, sz, vp]
        lib.bkmoo_conflicts.restype = ctypes.c_int
        lib.bkmoo_conflicts.argtypes = [vp, i32, i64, vp, vp, vp, vp]
        lib.bkmoo_gram_noalloc.restype = ctypes.c_int
        lib.bkmoo_gram_noalloc.argtypes = [vp, i32, i32, vp, i64, vp, vp]
        lib.bkmoo_resolve.restype = ctypes.c_int
        lib.bkmoo_resolve.argtypes = [vp, i32, i32, vp, i64, i32, ctypes.POINTER(bkmoo_params),
                                      vp, i32, vp, vp, vp, sz, vp]
        lib.bkmoo_resolve_buckets.restype = ctypes.c_int
        lib.bkmoo_resolve_buckets.argtypes = [vp, i32, i32, vp, i64, i64, i64, i32,
                                              ctypes.POINTER(bkmoo_params), vp, i32, vp, vp, vp,
                                              sz, vp]
        lib.bkmoo_host_staging_size.restype = ctypes.c_int
        lib.bkmoo_host_staging_size.argtypes = [i32, i32, i32, vp, i64, i64, ctypes.POINTER(sz)]
        lib.bkmoo_resolve_host.restype = ctypes.c_int
        lib.bkmoo_resolve_host.argtypes = [vp, i32, i32, vp, i64, i32,
                                           ctypes.POINTER(bkmoo_params), vp, i32, vp, vp, vp, sz,
                                           vp, sz, vp]
        lib.bkmoo_workspace_status.restype = ctypes.c_int
        lib.bkmoo_workspace_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        lib.bkmoo_status_string.restype = ctypes.c_char_p
        lib.bkmoo_status_string.argtypes = [i32]
        lib.bkmoo_version.restype = i32
        lib.bkmoo_version.argtypes = []
        lib.bkmoo_resolve_path.restype = ctypes.c_int
        lib.bkmoo_resolve_path.argtypes = [i32, i32, i32, vp, i64, ctypes.c_uint32,
                                           ctypes.POINTER(ctypes.c_int32)]
        lib.bkmoo_resolve_launches.restype = ctypes.c_int
        lib.bkmoo_resolve_launches.argtypes = [i32, i32, i32, vp, i64,
                                               ctypes.POINTER(bkmoo_params),
                                               ctypes.POINTER(ctypes.c_int32)]
        lib.bkmoo_selftest_fp64.restype = ctypes.c_int
        lib.bkmoo_selftest_fp64.argtypes = [i32, vp, vp, vp, i64, vp]
        lib.bkmoo_gate_forward.restype = ctypes.c_int
        lib.bkmoo_gate_forward.argtypes = [vp, i64, vp, vp, i64, i64, i64, i64, i32, vp, i64, vp,
                                           vp, i64, vp]
        lib.bkmoo_gate_backward_workspace_size.restype = ctypes.c_int
        lib.bkmoo_gate_backward_workspace_size.argtypes = [i64, i64, ctypes.POINTER(sz)]
        lib.bkmoo_gate_backward.restype = ctypes.c_int
        lib.bkmoo_gate_backward.argtypes = [vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, i64, i64,
                                            i64, i32, i32, vp, vp, i64, vp, vp, i32, i32, vp, sz,
                                            vp]
        lib.bkmoo_language_wgrad.restype = ctypes.c_int
        lib.bkmoo_language_wgrad.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32, vp, vp, i32,
                                             i32, vp]
        lib.bkmoo_op_status.restype = ctypes.c_int
        lib.bkmoo_op_status.argtypes = [vp, ctypes.POINTER(i32)]
        lib.bkmoo_op_status_copy.restype = ctypes.c_int
        lib.bkmoo_op_status_copy.argtypes = [vp, vp]
        lib.bkmoo_selftest_give_up.restype = ctypes.c_int
        lib.bkmoo_selftest_give_up.argtypes = [i32, vp]
        lib.bkmoo_grad_norm.restype = ctypes.c_int
        lib.bkmoo_grad_norm.argtypes = [vp, i32, i64, vp, vp, sz, vp]
        lib.bkmoo_adamw_default_params.restype = None
        lib.bkmoo_adamw_default_params.argtypes = [ctypes.POINTER(bkmoo_adamw_params)]
        lib.bkmoo_adamw.restype = ctypes.c_int
        lib.bkmoo_adamw.argtypes = [vp, vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, i32,
                                    ctypes.POINTER(bkmoo_adamw_params), vp, vp]
        _lib = lib
        return lib


def _check(code: int, where: str):
    if code != BKMOO_OK:
        raise BkmooError(code, where)


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return BKMOO_F32
    if t.dtype == torch.bfloat16:
        return BKMOO_BF16
    raise TypeError("gradients must be float32 or bfloat16, got %s" % t.dtype)


def _stream_handle(stream, device):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return ctypes.c_void_p(stream.cuda_stream)


def _offsets_array(offsets) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(offsets, dtype=np.int64))


def _grad_ptrs(grads):
    if not grads:
        raise ValueError("need at least one gradient")
    for g in grads:
        if not g.is_cuda or not g.is_contiguous():
            raise ValueError("gradients must be contiguous CUDA tensors")
    return (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])


def bkmoo_default_params() -> bkmoo_params:
    p = bkmoo_params()
    load().bkmoo_default_params(ctypes.byref(p))
    return p


def bkmoo_plan(param_sizes, elem_bytes: int, bucket_bytes: int) -> np.ndarray:
    lib = load()
    sizes = np.ascontiguousarray(np.asarray(param_sizes, dtype=np.int64))
    nb = ctypes.c_int64(0)
    _check(lib.bkmoo_plan(sizes.ctypes.data, len(sizes), elem_bytes, bucket_bytes, None, 0,
                          ctypes.byref(nb)), "bkmoo_plan")
    out = np.zeros(nb.value + 1, dtype=np.int64)
    _check(lib.bkmoo_plan(sizes.ctypes.data, len(sizes), elem_bytes, bucket_bytes,
                          out.ctypes.data, len(out), ctypes.byref(nb)), "bkmoo_plan")
    return out


def bkmoo_workspace_size(K: int, in_dtype: int, offsets) -> int:
    off = _offsets_array(offsets)
    n = ctypes.c_size_t(0)
    _check(load().bkmoo_workspace_size(K, in_dtype, off.ctypes.data, len(off) - 1,
                                       ctypes.byref(n)), "bkmoo_workspace_size")
    return int(n.value)


def bkmoo_workspace_init(K: int, in_dtype: int, offsets, ws, stream=None):
    off = _offsets_array(offsets)
    _check(load().bkmoo_workspace_init(K, in_dtype, off.ctypes.data, len(off) - 1,
                                       ws.data_ptr(), ws.numel() * ws.element_size(),
                                       _stream_handle(stream, ws.device)),
           "bkmoo_workspace_init")


def bkmoo_gram(grads, offsets, out_gram, ws, stream=None):
    off = _offsets_array(offsets)
    ptrs = _grad_ptrs(grads)
    _check(load().bkmoo_gram(ptrs, len(grads), _dtype_code(grads[0]), off.ctypes.data,
                             len(off) - 1, out_gram.data_ptr(), ws.data_ptr(),
                             ws.numel() * ws.element_size(),
                             _stream_handle(stream, grads[0].device)), "bkmoo_gram")


def bkmoo_conflicts(gram, out_cos=None, out_stats=None, out_conflict=None, stream=None):
    """Figure 1's conflict statistics from Gram matrices [B, K, K] (fp64, CUDA)."""
    B, K = int(gram.shape[0]), int(gram.shape[1])
    _check(load().bkmoo_conflicts(gram.data_ptr(), K, B,
                                  out_cos.data_ptr() if out_cos is not None else None,
                                  out_stats.data_ptr() if out_stats is not None else None,
                                  out_conflict.data_ptr() if out_conflict is not None else None,
                                  _stream_handle(stream, gram.device)), "bkmoo_conflicts")


def bkmoo_gram_noalloc(grads, offsets, out_gram, stream=None):
    """bkmoo_gram for callers that cannot allocate device memory: no
    workspace; the scratch is a static device array of the library (see
    include/bkmoo.h for its limits and the rule that overlapping calls race)."""
    off = _offsets_array(offsets)
    ptrs = _grad_ptrs(grads)
    _check(load().bkmoo_gram_noalloc(ptrs, len(grads), _dtype_code(grads[0]), off.ctypes.data,
                                     len(off) - 1, out_gram.data_ptr(),
                                     _stream_handle(stream, grads[0].device)),
           "bkmoo_gram_noalloc")


def bkmoo_resolve(grads, offsets, rule, out_dir, ws, params=None, out_weights=None,
                  out_status=None, stream=None):
    if isinstance(rule, str):
        rule = RULES[rule]
    off = _offsets_array(offsets)
    ptrs = _grad_ptrs(grads)
    p = params if params is not None else bkmoo_default_params()
    _check(load().bkmoo_resolve(ptrs, len(grads), _dtype_code(grads[0]), off.ctypes.data,
                                len(off) - 1, rule, ctypes.byref(p), out_dir.data_ptr(),
                                _dtype_code(out_dir),
                                out_weights.data_ptr() if out_weights is not None else None,
                                out_status.data_ptr() if out_status is not None else None,
                                ws.data_ptr(), ws.numel() * ws.element_size(),
                                _stream_handle(stream, grads[0].device)), "bkmoo_resolve")


def bkmoo_resolve_buckets(grads, offsets, b_lo, b_hi, rule, out_dir, ws, params=None,
                          out_weights=None, out_status=None, stream=None):
    if isinstance(rule, str):
        rule = RULES[rule]
    off = _offsets_array(offsets)
    ptrs = _grad_ptrs(grads)
    p = params if params is not None else bkmoo_default_params()
    _check(load().bkmoo_resolve_buckets(ptrs, len(grads), _dtype_code(grads[0]), off.ctypes.data,
                                        len(off) - 1, b_lo, b_hi, rule, ctypes.byref(p),
                                        out_dir.data_ptr(), _dtype_code(out_dir),
                                        out_weights.data_ptr() if out_weights is not None
                                        else None,
                                        out_status.data_ptr() if out_status is not None else None,
                                        ws.data_ptr(), ws.numel() * ws.element_size(),
                                        _stream_handle(stream, grads[0].device)),
           "bkmoo_resolve_buckets")


def bkmoo_host_staging_size(K: int, in_dtype: int, out_dtype: int, offsets,
                            window_elems: int = 0) -> int:
    off = _offsets_array(offsets)
    n = ctypes.c_size_t(0)
    _check(load().bkmoo_host_staging_size(K, in_dtype, out_dtype, off.ctypes.data, len(off) - 1,
                                          window_elems, ctypes.byref(n)),
           "bkmoo_host_staging_size")
    return int(n.value)


def bkmoo_resolve_host(host_grads, offsets, rule, host_out, ws, staging, params=None,
                       out_weights=None, out_status=None, stream=None):
    """host_grads / host_out: contiguous CPU tensors (page-locked for overlap);
    ws, staging, out_weights, out_status: CUDA tensors."""
    if isinstance(rule, str):
        rule = RULES[rule]
    if not host_grads:
        raise ValueError("need at least one gradient")
    for g in list(host_grads) + [host_out]:
        if g.is_cuda or not g.is_contiguous():
            raise ValueError("host_grads and host_out must be contiguous CPU tensors")
    off = _offsets_array(offsets)
    ptrs = (ctypes.c_void_p * len(host_grads))(*[g.data_ptr() for g in host_grads])
    p = params if params is not None else bkmoo_default_params()
    _check(load().bkmoo_resolve_host(ptrs, len(host_grads), _dtype_code(host_grads[0]),
                                     off.ctypes.data, len(off) - 1, rule, ctypes.byref(p),
                                     host_out.data_ptr(), _dtype_code(host_out),
                                     out_weights.data_ptr() if out_weights is not None else None,
                                     out_status.data_ptr() if out_status is not None else None,
                                     ws.data_ptr(), ws.numel() * ws.element_size(),
                                     staging.data_ptr(), staging.numel() * staging.element_size(),
                                     _stream_handle(stream, ws.device)), "bkmoo_resolve_host")


def bkmoo_workspace_status(ws, stream=None) -> int:
    st = ctypes.c_int32(0)
    _check(load().bkmoo_workspace_status(ws.data_ptr(), _stream_handle(stream, ws.device),
                                         ctypes.byref(st)), "bkmoo_workspace_status")
    return int(st.value)


def bkmoo_status_string(code: int) -> str:
    return load().bkmoo_status_string(code).decode()


def bkmoo_version() -> int:
    return int(load().bkmoo_version())


def bkmoo_resolve_launches(K: int, in_dtype: int, rule, offsets, params=None) -> int:
    """Kernels that bkmoo_resolve launches: 1 (the one launch), 3 or 4."""
    if isinstance(rule, str):
        rule = RULES[rule]
    off = _offsets_array(offsets)
    out = ctypes.c_int32(-1)
    _check(load().bkmoo_resolve_launches(K, in_dtype, rule, off.ctypes.data, len(off) - 1,
                                         ctypes.byref(params) if params is not None else None,
                                         ctypes.byref(out)), "bkmoo_resolve_launches")
    return int(out.value)


def bkmoo_resolve_path(K: int, in_dtype: int, rule, offsets, flags: int) -> int:
    """A classification of plans kept from earlier kernels; the launches of a
    call are bkmoo_resolve_launches' answer (see include/bkmoo.h)."""
    if isinstance(rule, str):
        rule = RULES[rule]
    off = _offsets_array(offsets)
    out = ctypes.c_int32(-1)
    _check(load().bkmoo_resolve_path(K, in_dtype, rule, off.ctypes.data, len(off) - 1, flags,
                                     ctypes.byref(out)), "bkmoo_resolve_path")
    return int(out.value)


def bkmoo_selftest_fp64(op: int, a, b, out, stream=None):
    """The solvers' fp64 division (op 0, out = a / b) or square root (op 1,
    out = sqrt(a)) element-wise on the device (fp64 CUDA tensors)."""
    _check(load().bkmoo_selftest_fp64(op, a.data_ptr(), b.data_ptr() if b is not None else None,
                                      out.data_ptr(), int(out.numel()),
                                      _stream_handle(stream, out.device)), "bkmoo_selftest_fp64")


def _matrix(t, rows: int, cols: int, dev: int, bf16, what: str):
    """(address, row stride) of a bf16 matrix the tile kernels take."""
    if t.dtype is not bf16 or t.get_device() != dev or t.shape != (rows, cols):
        raise ValueError("%s must be a bfloat16 matrix of %d x %d on cuda:%d, got %s %s on %s"
                         % (what, rows, cols, dev, t.dtype, tuple(t.shape), t.device))
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s must have contiguous rows" % what)
    if rows < 2:
        ld = (cols + 7) // 8 * 8         # no second row: any stride does
    p = t.data_ptr()
    if ld < cols or ld % 8 or p % 16:
        raise ValueError("%s: rows must start on 16 bytes (pad them to a multiple of 8 elements)"
                         % what)
    return p, ld


def _pair(t, u, rows: int, cols: int, dev: int, bf16, what: str):
    """Addresses and the one row stride of two matrices of a kind."""
    p, ld = _matrix(t, rows, cols, dev, bf16, what)
    q, lu = _matrix(u, rows, cols, dev, bf16, what)
    if ld != lu:
        raise ValueError("%s: both must have one row stride" % what)
    return p, q, ld


def _cuda_matrix(t, what: str):
    """(rows, columns, device index) of a CUDA matrix."""
    dev = t.get_device()
    if dev < 0 or t.dim() != 2:
        raise ValueError("%s must be a CUDA matrix" % what)
    rows, cols = t.shape
    return rows, cols, dev


def _act_code(act) -> int:
    return ACTS[act] if isinstance(act, str) else act


def _raw_stream(torch, stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


_op_devices = set()        # devices on which a gate or weight-gradient call has been made


def ops_called(dev: int) -> bool:
    """Whether the gate or weight-gradient calls have been used on device `dev`."""
    return dev in _op_devices


def _call(torch, dev: int, where: str, fn, *args):
    """fn(*args) with device `dev` current."""
    if torch.cuda.current_device() == dev:
        code = fn(*args)
    else:
        with torch.cuda.device(dev):
            code = fn(*args)
    if code != BKMOO_OK:
        raise BkmooError(code, where)


def _scratch(torch, nbytes: int, dev: int, stream):
    """A byte tensor for work on `stream` (None: the current one)."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)


def _workspace(ws, dev: int):
    """(address, bytes) of a workspace that a caller gave."""
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous tensor on cuda:%d" % dev)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _language_rows(rows, T: int):
    """(K, array) of the language bounds."""
    r = [int(i) for i in rows]
    last, ok = 0, 2 <= len(r) <= 17 and r[0] == 0 and r[-1] == T
    for i in r:
        ok = ok and i >= last
        last = i
    if not ok:
        raise ValueError("rows must be K + 1 bounds from 0 to the number of rows, 1 <= K <= 16")
    return len(r) - 1, (ctypes.c_int64 * len(r))(*r)


def _weight_grads(dw, K: int, rows: int, cols: int, dev: int, what: str):
    """(array of K addresses, dtype code) of a list of per-language gradients."""
    if len(dw) != K:
        raise ValueError("%s: one gradient per language, %d" % (what, K))
    dt, shape, at = dw[0].dtype, (rows, cols), []
    for g in dw:
        if g.dtype is not dt or g.get_device() != dev or g.shape != shape or not g.is_contiguous():
            raise ValueError("%s must be contiguous %d x %d matrices of one dtype on cuda:%d"
                             % (what, rows, cols, dev))
        at.append(g.data_ptr())
    return (ctypes.c_void_p * K)(*at), _dtype_code(dw[0])


def bkmoo_gate_forward(x, w_gate, w_up, act, h=None, a=None, b=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T), and a = x w_gate^T, b = x w_up^T for the
    backward pass where given.  x [T, D], weights [F, D], outputs [T, F], all
    bfloat16, rows on 16 bytes."""
    import torch
    bf16 = torch.bfloat16
    T, D, dev = _cuda_matrix(x, "x")
    F = w_gate.shape[0]
    px, ldx = _matrix(x, T, D, dev, bf16, "x")
    pg, pu, ldw = _pair(w_gate, w_up, F, D, dev, bf16, "w_gate and w_up")
    ph, ldh = _matrix(h, T, F, dev, bf16, "h") if h is not None else (None, 0)
    if (a is None) != (b is None):
        raise ValueError("a and b come together")
    pa, pb, ld_ab = _pair(a, b, T, F, dev, bf16, "a and b") if a is not None else (None, None, 0)
    _op_devices.add(dev)
    _call(torch, dev, "bkmoo_gate_forward", load().bkmoo_gate_forward, px, ldx, pg, pu, ldw, T, D,
          F, _act_code(act), ph, ldh, pa, pb, ld_ab, _raw_stream(torch, stream, dev))


def bkmoo_gate_backward_workspace_size(T: int, F: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().bkmoo_gate_backward_workspace_size(T, F, ctypes.byref(n)),
           "bkmoo_gate_backward_workspace_size")
    return int(n.value)


def bkmoo_gate_backward(dh, a, b, x, w_gate, w_up, act, rows, dx=None, dw_gate=None, dw_up=None,
                        accumulate=False, ws=None, stream=None):
    """From dh, with the forward pass's a and b: dx (may be None), and for every
    language k (rows[k] to rows[k + 1] of the batch) its own dw_gate[k], dw_up[k]
    (contiguous [F, D], float32 or bfloat16; both lists may be None).  ws: a CUDA
    byte tensor of bkmoo_gate_backward_workspace_size; allocated (torch, on
    `stream`) where None; the call leaves da and db in its halves (bkmoo.h)."""
    import torch
    bf16 = torch.bfloat16
    T, D, dev = _cuda_matrix(x, "x")
    F = w_gate.shape[0]
    K, r = _language_rows(rows, T)
    px, ldx = _matrix(x, T, D, dev, bf16, "x")
    pd, ldd = _matrix(dh, T, F, dev, bf16, "dh")
    pa, pb, ld_ab = _pair(a, b, T, F, dev, bf16, "a and b")
    pg, pu, ldw = _pair(w_gate, w_up, F, D, dev, bf16, "w_gate and w_up")
    pdx, lddx = _matrix(dx, T, D, dev, bf16, "dx") if dx is not None else (None, 0)
    gg = gu = None
    dt = BKMOO_BF16
    if (dw_gate is None) != (dw_up is None):
        raise ValueError("dw_gate and dw_up come together")
    if dw_gate is not None:
        gg, dt = _weight_grads(dw_gate, K, F, D, dev, "dw_gate")
        gu, du = _weight_grads(dw_up, K, F, D, dev, "dw_up")
        if dt != du:
            raise ValueError("dw_gate and dw_up must have one dtype")
    if ws is None:           # as bkmoo_gate_backward_workspace_size: da and db, rows on 16 bytes
        ws = _scratch(torch, 2 * -(-T * ((F + 7) // 8 * 16) // 256) * 256, dev, stream)
    pws, nws = _workspace(ws, dev)
    _op_devices.add(dev)
    _call(torch, dev, "bkmoo_gate_backward", load().bkmoo_gate_backward, pd, ldd, pa, pb, ld_ab,
          px, ldx, pg, pu, ldw, T, D, F, _act_code(act), K, r, pdx, lddx, gg, gu, dt,
          1 if accumulate else 0, pws, nws, _raw_stream(torch, stream, dev))


def bkmoo_language_wgrad(dy, x, rows, dw, accumulate=False, stream=None):
    """dw[k] = dy[rows[k]:rows[k + 1]]^T x[rows[k]:rows[k + 1]] for every language:
    dy [T, M] and x [T, N] bfloat16, dw[k] contiguous [M, N], float32 or bfloat16."""
    import torch
    bf16 = torch.bfloat16
    T, M, dev = _cuda_matrix(dy, "dy")
    N = x.shape[-1]
    K, r = _language_rows(rows, T)
    pd, ldd = _matrix(dy, T, M, dev, bf16, "dy")
    px, ldx = _matrix(x, T, N, dev, bf16, "x")
    g, dt = _weight_grads(dw, K, M, N, dev, "dw")
    _op_devices.add(dev)
    _call(torch, dev, "bkmoo_language_wgrad", load().bkmoo_language_wgrad, pd, ldd, px, ldx, T, M,
          N, K, r, g, dt, 1 if accumulate else 0, _raw_stream(torch, stream, dev))


def bkmoo_op_status(device=None, stream=None) -> int:
    """Status word of the gate and weight-gradient calls on `device`; cleared."""
    import torch
    st = ctypes.c_int32(0)
    with torch.cuda.device(device):
        _check(load().bkmoo_op_status(_stream_handle(stream, device), ctypes.byref(st)),
               "bkmoo_op_status")
    return int(st.value)


def bkmoo_op_status_copy(out, stream=None):
    """Queue a copy of that word into `out`, one int32 on a GPU or in pinned memory;
    neither waits nor clears it."""
    import torch
    dev = torch.cuda.current_device() if out.device.type == "cpu" else out.get_device()
    if out.dtype is not torch.int32 or out.numel() != 1 or (out.device.type == "cpu" and not out.is_pinned()):
        raise ValueError("out must be one int32 on a GPU or in pinned memory")
    _call(torch, dev, "bkmoo_op_status_copy", load().bkmoo_op_status_copy,
          _raw_stream(torch, stream, dev), out.data_ptr())


def bkmoo_selftest_give_up(device=None, what: int = 0, stream=None):
    """Queue a kernel that gives up: a wait alone of 1 ms (0), or the forward pass's
    kernel of one CTA or of a pair without its operands, 2 s (1, 2)."""
    import torch
    dev = torch.cuda.current_device() if device is None else torch.device(device).index
    _call(torch, dev, "bkmoo_selftest_give_up", load().bkmoo_selftest_give_up, what,
          _raw_stream(torch, stream, dev))


def bkmoo_grad_norm(grad, out_norm, ws=None, stream=None):
    """The 2-norm of a flat gradient into out_norm (a float32 CUDA tensor of one
    element).  ws: a CUDA byte tensor of BKMOO_NORM_WS_BYTES; allocated (torch,
    on `stream`) where None."""
    import torch
    dev = grad.get_device()
    if dev < 0 or not grad.is_contiguous():
        raise ValueError("the gradient must be a contiguous CUDA tensor")
    if out_norm.dtype is not torch.float32 or out_norm.numel() != 1 or out_norm.get_device() != dev:
        raise ValueError("out_norm must be one float32 on the gradient's device")
    if ws is None:
        ws = _scratch(torch, BKMOO_NORM_WS_BYTES, dev, stream)
    _call(torch, dev, "bkmoo_grad_norm", load().bkmoo_grad_norm, grad.data_ptr(), _dtype_code(grad),
          grad.numel(), out_norm.data_ptr(), *_workspace(ws, dev), _raw_stream(torch, stream, dev))


def bkmoo_adamw_default_params() -> bkmoo_adamw_params:
    p = bkmoo_adamw_params()
    load().bkmoo_adamw_default_params(ctypes.byref(p))
    return p


_DTYPE = operator.attrgetter("dtype")


class TensorList:
    """The tensors of bkmoo_adamw: contiguous CUDA tensors of one dtype, in the
    order of the flat buffers, and their weight decay (one number, one per
    tensor, or None).  Keeps the tensors, and their addresses for the call: a
    tensor whose storage is replaced (p.data = ...) is followed, one that
    changes its size, dtype or device is refused by the next call."""

    def __init__(self, tensors, weight_decay=None):
        self.tensors = list(tensors)
        n = len(self.tensors)
        if n == 0:
            raise ValueError("need at least one tensor")
        self.dtype, self.device = self.tensors[0].dtype, self.tensors[0].get_device()
        self._sizes, self._addresses = self._look()
        self.dtype_code = _dtype_code(self.tensors[0])
        self.n_elems = sum(self._sizes)
        self._decay = None
        if weight_decay is not None:
            self._decay = array.array("f", [weight_decay] * n if isinstance(weight_decay, (int, float))
                                      else weight_decay)
            if len(self._decay) != n:
                raise ValueError("weight_decay must be one number, or one per tensor")

    def _look(self):
        """(sizes, addresses) as they are now."""
        import torch
        T, tensors = torch.Tensor, self.tensors
        if self.device < 0 or set(map(T.get_device, tensors)) != {self.device} or \
                not all(map(T.is_contiguous, tensors)) or \
                set(map(_DTYPE, tensors)) != {self.dtype}:
            raise ValueError("the tensors must be contiguous CUDA tensors of one dtype on one device")
        return array.array("q", map(T.numel, tensors)), array.array("Q", map(T.data_ptr, tensors))

    def look_again(self) -> None:
        sizes, self._addresses = self._look()
        if sizes != self._sizes:
            raise ValueError("the tensors' sizes have changed")

    @property
    def args(self):
        """Addresses of the three arrays, as the C call takes them."""
        return (self._addresses.buffer_info()[0], self._sizes.buffer_info()[0],
                self._decay.buffer_info()[0] if self._decay is not None else None, len(self.tensors))


def bkmoo_adamw(tensors, grad, m, v, params=None, weight_decay=None, master=None, m_scale=None,
                v_scale=None, grad_norm=None, stream=None):
    """One AdamW step of `tensors` (a TensorList, or the tensors and weight_decay
    one would make it of) with the flat gradient.  m, v: flat float32, or flat
    float8_e4m3fn with one float32 scale per 256 elements (v then holds the root
    of the second moment); master: flat float32 weights of bfloat16 tensors, or
    None."""
    import torch
    if not isinstance(tensors, TensorList):
        tensors = TensorList(tensors, weight_decay)
    elif weight_decay is not None:
        raise ValueError("the TensorList has its own weight decay")
    else:
        tensors.look_again()
    dev, N = tensors.device, tensors.n_elems
    f32, eight = torch.float32, m.dtype is torch.float8_e4m3fn
    if master is not None and tensors.dtype is not torch.bfloat16:
        raise ValueError("a master copy goes with bfloat16 tensors")
    for name, t, want in (("grad", grad, grad.dtype), ("m", m, m.dtype if eight else f32),
                          ("v", v, m.dtype), ("master", master, f32)):
        if t is not None and (t.dtype is not want or t.get_device() != dev or t.numel() != N or
                              not t.is_contiguous()):
            raise ValueError("%s must be a flat tensor of the tensors' %d elements, %s, on cuda:%d"
                             % (name, N, want, dev))
    ms = vs = None
    if eight:
        for name, t in (("m_scale", m_scale), ("v_scale", v_scale)):
            if t is None or t.dtype is not f32 or t.get_device() != dev or \
                    t.numel() != (N + 255) // 256 or not t.is_contiguous():
                raise ValueError("%s must hold one float32 per 256 elements" % name)
        ms, vs = m_scale.data_ptr(), v_scale.data_ptr()
    if grad_norm is not None and (grad_norm.dtype is not f32 or grad_norm.get_device() != dev or
                                  grad_norm.numel() != 1):
        raise ValueError("grad_norm must be one float32 on the gradient's device")
    p = params if params is not None else bkmoo_adamw_default_params()
    _call(torch, dev, "bkmoo_adamw", load().bkmoo_adamw, *tensors.args, tensors.dtype_code,
          grad.data_ptr(), _dtype_code(grad), master.data_ptr() if master is not None else None,
          m.data_ptr(), v.data_ptr(), ms, vs, BKMOO_E4M3 if eight else BKMOO_F32, ctypes.byref(p),
          grad_norm.data_ptr() if grad_norm is not None else None,
          _raw_stream(torch, stream, dev))


class Resolver:
    """Holds the plan and the workspace of one (K, dtype, offsets) triple.

    Allocates the workspace once (torch, on `device`) and initialises it; each
    call to resolve() then queues Gram -> solve -> combine on the current
    stream without further allocation."""

    def __init__(self, K: int, in_dtype, offsets, device):
        import torch
        self.K = K
        self.in_dtype = in_dtype if isinstance(in_dtype, int) else (
            BKMOO_F32 if in_dtype == torch.float32 else BKMOO_BF16)
        self.offsets = _offsets_array(offsets)
        self.n_buckets = len(self.offsets) - 1
        self.device = torch.device(device)
        nbytes = bkmoo_workspace_size(K, self.in_dtype, self.offsets)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        bkmoo_workspace_init(K, self.in_dtype, self.offsets, self.ws)

    def resolve(self, grads, rule, out_dir, params=None, out_weights=None, out_status=None,
                stream=None):
        bkmoo_resolve(grads, self.offsets, rule, out_dir, self.ws, params, out_weights,
                      out_status, stream)

    def resolve_buckets(self, grads, b_lo, b_hi, rule, out_dir, params=None, out_weights=None,
                        out_status=None, stream=None):
        bkmoo_resolve_buckets(grads, self.offsets, b_lo, b_hi, rule, out_dir, self.ws, params,
                              out_weights, out_status, stream)

    def resolve_host(self, host_grads, rule, host_out, staging, params=None, out_weights=None,
                     out_status=None, stream=None):
        bkmoo_resolve_host(host_grads, self.offsets, rule, host_out, self.ws, staging, params,
                           out_weights, out_status, stream)

    def staging_size(self, out_dtype: int, window_elems: int = 0) -> int:
        return bkmoo_host_staging_size(self.K, self.in_dtype, out_dtype, self.offsets,
                                       window_elems)

    def gram(self, grads, out_gram, stream=None):
        bkmoo_gram(grads, self.offsets, out_gram, self.ws, stream)

    def status(self, stream=None) -> int:
        return bkmoo_workspace_status(self.ws, stream)
