"""ctypes binding of libbq (include/bq.h), with the C names.

Argument marshalling only: torch tensors are passed as device pointers and the
current torch stream as the HIP stream; every step of the path runs in the HIP
kernels of libbq.so.  There is no fallback: if the library is not built, or a
call returns an error, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import sys
import warnings

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# BQ_SANITIZE=1 selects the host-sanitized build (build.py --sanitize), for the
# CPU tests under AddressSanitizer / UndefinedBehaviorSanitizer only
LIB_PATH = (os.path.join(_PKG, "_build", "san", "libbq.so") if os.environ.get("BQ_SANITIZE") == "1"
            else os.path.join(_PKG, "libbq.so"))

BQ_OK, BQ_ERR_NULL, BQ_ERR_SIZE, BQ_ERR_BLOCKSIZE, BQ_ERR_ENUM = 0, 1, 2, 3, 4
BQ_ERR_DTYPE, BQ_ERR_ALIGN, BQ_ERR_HIP, BQ_ERR_ARG = 5, 6, 7, 8
BQ_SIGNED, BQ_UNSIGNED = 0, 1
BQ_INVERSE_SIGNED, BQ_INVERSE_UNSIGNED = 2, 3
BQ_LINEAR_SIGNED, BQ_LINEAR_UNSIGNED = 4, 5
CODEBOOKS = {"dynamic": (BQ_SIGNED, BQ_UNSIGNED),
             "inverse_dynamic": (BQ_INVERSE_SIGNED, BQ_INVERSE_UNSIGNED),
             "linear": (BQ_LINEAR_SIGNED, BQ_LINEAR_UNSIGNED)}
BQ_ADAM, BQ_ADAMW, BQ_MOMENTUM, BQ_ADAGRAD, BQ_LAMB, BQ_LARS = 0, 1, 2, 3, 4, 5
BQ_F32, BQ_F16, BQ_BF16 = 0, 1, 2
OPTIMIZERS = {"adam": BQ_ADAM, "adamw": BQ_ADAMW, "momentum": BQ_MOMENTUM,
              "adagrad": BQ_ADAGRAD, "lamb": BQ_LAMB, "lars": BQ_LARS}

EXPORTS = ("bq_make_dynamic_codebook", "bq_make_codebook", "bq_make_quantile_codebook",
           "bq_estimate_quantile_codebook", "bq_quantile_workspace_bytes",
           "bq_quantize_blockwise", "bq_dequantize_blockwise",
           "bq_optimizer8bit_step", "bq_optimizer8bit_step_static", "bq_optimizer32bit_step",
           "bq_prepare_codebook",
           "bq_quantize_blockwise_prepared",
           "bq_step_plan_create", "bq_step_plan_run", "bq_step_plan_run_prepared",
           "bq_step_plan_run_device", "bq_step_plan_destroy", "bq_status_string",
           "bq_layer_norm_forward", "bq_layer_norm_workspace_bytes", "bq_layer_norm_backward",
           "bq_embedding_forward", "bq_embedding_workspace_bytes", "bq_embedding_backward",
           "bq_stable_embedding_forward", "bq_stable_embedding_workspace_bytes",
           "bq_stable_embedding_backward", "bq_grad_norm_workspace_bytes", "bq_grad_norm",
           "bq_clip_grad_norm")
BQ_PREPARED_CODEBOOK_BYTES = 8720
BQ_QUANTILE_CHUNK = 4096
BQ_NORM_L2, BQ_NORM_INF = 0, 1
BQ_STABLE_EMBEDDING_MAX_DIM = 16384


class BQError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class bq_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("state1", ctypes.c_void_p), ("state2", ctypes.c_void_p),
                ("absmax1", ctypes.c_void_p), ("absmax2", ctypes.c_void_p),
                ("numel", ctypes.c_int64)]


class bq_tensor32(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("state1", ctypes.c_void_p), ("state2", ctypes.c_void_p),
                ("numel", ctypes.c_int64)]


class bq_hparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("step", ctypes.c_int64), ("trust_coeff", ctypes.c_float)]


class bq_grad(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libbq.so (built by ``__graft_entry__.build()``); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m "
                               "paper_2110_02861_amd.build` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, I = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int
        L.bq_make_dynamic_codebook.argtypes = [I, P]
        L.bq_make_dynamic_codebook.restype = I
        L.bq_make_codebook.argtypes = [I, P]
        L.bq_make_codebook.restype = I
        L.bq_make_quantile_codebook.argtypes = [P, I64, P]
        L.bq_make_quantile_codebook.restype = I
        L.bq_estimate_quantile_codebook.argtypes = [P, I64, P, P, P]
        L.bq_estimate_quantile_codebook.restype = I
        L.bq_quantile_workspace_bytes.argtypes = [I64]
        L.bq_quantile_workspace_bytes.restype = I64
        L.bq_quantize_blockwise.argtypes = [P, P, I64, I32, P, P, P]
        L.bq_quantize_blockwise.restype = I
        L.bq_dequantize_blockwise.argtypes = [P, P, P, I64, I32, P, P]
        L.bq_dequantize_blockwise.restype = I
        L.bq_optimizer8bit_step.argtypes = [I, I32, I, P, I32, P, P, P, P]
        L.bq_optimizer8bit_step.restype = I
        L.bq_optimizer8bit_step_static.argtypes = [I, I32, I, P, I32, P, P, P, P]
        L.bq_optimizer8bit_step_static.restype = I
        L.bq_optimizer32bit_step.argtypes = [I, I, P, I32, P, P]
        L.bq_optimizer32bit_step.restype = I
        L.bq_prepare_codebook.argtypes = [P, P, P]
        L.bq_prepare_codebook.restype = I
        L.bq_quantize_blockwise_prepared.argtypes = [P, P, I64, I32, P, P, P]
        L.bq_quantize_blockwise_prepared.restype = I
        L.bq_step_plan_create.argtypes = [I, I32, I, P, I32, ctypes.POINTER(ctypes.c_void_p)]
        L.bq_step_plan_create.restype = I
        L.bq_step_plan_run.argtypes = [P, P, P, P, P]
        L.bq_step_plan_run.restype = I
        L.bq_step_plan_run_prepared.argtypes = [P, P, P, P]
        L.bq_step_plan_run_prepared.restype = I
        L.bq_step_plan_run_device.argtypes = [P, P, I32, P, P]
        L.bq_step_plan_run_device.restype = I
        L.bq_step_plan_destroy.argtypes = [P]
        L.bq_step_plan_destroy.restype = I
        F, D = ctypes.c_float, ctypes.c_double
        L.bq_layer_norm_forward.argtypes = [I, I, P, I64, I64, I64, P, P, F, P, P, P, P]
        L.bq_layer_norm_workspace_bytes.argtypes = [I64, I64]
        L.bq_layer_norm_backward.argtypes = [I, I, P, I64, P, I64, I64, I64, P, P, P, P, P, P, P,
                                             P]
        L.bq_embedding_forward.argtypes = [I, I, P, I64, I64, P, I32, I64, F, P, P]
        L.bq_embedding_workspace_bytes.argtypes = [I64, I64, I64]
        L.bq_embedding_backward.argtypes = [I, I, P, P, I32, I64, I64, I64, I64, F, P, P, P]
        L.bq_stable_embedding_forward.argtypes = [I, I, P, I64, I64, P, I32, I64, P, P, F, P, P]
        L.bq_stable_embedding_workspace_bytes.argtypes = [I64, I64, I64]
        L.bq_stable_embedding_backward.argtypes = [I, I, P, P, I32, I64, P, I64, I64, I64, P, F, P,
                                                   P, P, P, P]
        L.bq_grad_norm_workspace_bytes.argtypes = [I32]
        L.bq_grad_norm.argtypes = [P, I32, I, P, P, P]
        L.bq_clip_grad_norm.argtypes = [P, I32, I, D, P, P, P]
        for name in ("bq_layer_norm", "bq_embedding", "bq_stable_embedding"):
            getattr(L, name + "_forward").restype = I
            getattr(L, name + "_backward").restype = I
            getattr(L, name + "_workspace_bytes").restype = I64
        L.bq_grad_norm_workspace_bytes.restype = I64
        L.bq_grad_norm.restype = I
        L.bq_clip_grad_norm.restype = I
        L.bq_status_string.argtypes = [I]
        L.bq_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


# csrc/bq_host*.cpp: the ordinary case of the calls below in native code.  Each of
# its functions returns None where the Python code after it is to run (errors,
# tensors of other classes, active torch modes).
_HOST_CALLS = ("bq_quantize_blockwise", "bq_quantize_blockwise_prepared",
               "bq_dequantize_blockwise", "bq_estimate_quantile_codebook",
               "bq_quantile_workspace_bytes", "bq_optimizer8bit_step", "bq_step_plan_run",
               "bq_step_plan_run_prepared")
_HOST_OPS = ("bq_layer_norm_forward", "bq_layer_norm_workspace_bytes", "bq_layer_norm_backward",
             "bq_embedding_forward", "bq_embedding_workspace_bytes", "bq_embedding_backward",
             "bq_stable_embedding_forward", "bq_stable_embedding_workspace_bytes",
             "bq_stable_embedding_backward", "bq_grad_norm_workspace_bytes", "bq_grad_norm",
             "bq_clip_grad_norm")
_host_module = None


class _PythonOnly:
    """Stands in for _bqhost where that is not built: every call runs in Python."""

    def __getattr__(self, name):
        return lambda *args: None


def host():
    """The module _bqhost, bound to lib().  It only saves host time, so where it is
    not built, or was built against another torch, the Python code runs alone."""
    global _host_module
    if _host_module is None:
        L = lib()
        import torch  # noqa: F401  (the module links against it)
        try:
            from . import _bqhost
            for bind, names in ((_bqhost.bind, _HOST_CALLS), (_bqhost.bind_ops, _HOST_OPS)):
                bind(tuple(ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in names))
            _host_module = _bqhost
        except (ImportError, AttributeError) as e:  # absent, or of other sources
            _host_module = _PythonOnly()
            warnings.warn(f"_bqhost is not available, calls take more host time ({e}); run "
                          "`python -m paper_2110_02861_amd.build`", RuntimeWarning, stacklevel=3)
    return _host_module


def status_string(s: int) -> str:
    return lib().bq_status_string(int(s)).decode()


def _check(status: int, where: str) -> None:
    if status != BQ_OK:
        raise BQError(status, where)


def _dev_ptr(t, name):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU torch tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != torch.cuda.current_device():
        # the C calls run on the current device
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")
    return t.data_ptr()


def _map_ptr(q, name):
    """A codebook: 256 fp32 values on the current device."""
    import torch
    if not isinstance(q, torch.Tensor) or q.dtype != torch.float32 or q.numel() != 256:
        raise TypeError(f"{name} must be a tensor of 256 fp32 values")
    return _dev_ptr(q, name)


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def bq_make_dynamic_codebook(kind: int) -> np.ndarray:
    """Host call: the 256-entry signed (0) or unsigned (1) dynamic codebook."""
    out = np.empty(256, np.float32)
    _check(lib().bq_make_dynamic_codebook(int(kind), out.ctypes.data), "bq_make_dynamic_codebook")
    return out


def bq_make_codebook(kind: int) -> np.ndarray:
    """Host call: any fixed codebook (BQ_SIGNED ... BQ_LINEAR_UNSIGNED)."""
    out = np.empty(256, np.float32)
    _check(lib().bq_make_codebook(int(kind), out.ctypes.data), "bq_make_codebook")
    return out


def bq_estimate_quantile_codebook(x, out=None, workspace=None, stream=None):
    """GPU quantile map of a device fp32 tensor (App. F.2, App. G); returns the
    device map (256 fp32).  The workspace (bq_quantile_workspace_bytes) is
    allocated here by torch unless given."""
    if out is not None and workspace is not None:
        r = host().estimate(x, out, workspace, stream)
        if r is out:
            return r
        if r is not None:
            _check(r, "bq_estimate_quantile_codebook")
    import torch
    n = x.numel()
    if x.dtype != torch.float32:
        raise TypeError("x must be fp32")
    nbytes = max(8, int(lib().bq_quantile_workspace_bytes(n)))
    if workspace is None:
        workspace = torch.empty(nbytes // 8, dtype=torch.float64, device=x.device)
    elif workspace.numel() * workspace.element_size() < nbytes:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} "
                         f"bytes, needs {nbytes}")
    if out is None:
        out = torch.empty(256, dtype=torch.float32, device=x.device)
    elif out.dtype != torch.float32 or out.numel() != 256:
        raise TypeError("out must be a tensor of 256 fp32 values")
    _check(lib().bq_estimate_quantile_codebook(_dev_ptr(x, "x") if n else None, n,
                                               _dev_ptr(workspace, "workspace"),
                                               _dev_ptr(out, "out"), _stream(stream)),
           "bq_estimate_quantile_codebook")
    return out


def bq_make_quantile_codebook(sample) -> np.ndarray:
    """Host call: the quantile map of a host fp32 sample (App. F.2)."""
    x = np.ascontiguousarray(sample, dtype=np.float32).ravel()
    out = np.empty(256, np.float32)
    _check(lib().bq_make_quantile_codebook(x.ctypes.data if x.size else None, x.size,
                                           out.ctypes.data), "bq_make_quantile_codebook")
    return out


def bq_quantize_blockwise(qmap, x, blocksize: int, codes=None, absmax=None, stream=None):
    """codes (uint8, like x) and absmax (fp32, ceil(n/B)) of the GPU tensor x."""
    r = host().quantize(False, qmap, x, blocksize, codes, absmax, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        _check(r, "bq_quantize_blockwise")
    import torch
    n = x.numel()
    if codes is None:
        codes = torch.empty(n, dtype=torch.uint8, device=x.device)
    if absmax is None:
        absmax = torch.empty((n + blocksize - 1) // blocksize, dtype=torch.float32,
                             device=x.device)
    if x.dtype != torch.float32 or codes.dtype != torch.uint8 or absmax.dtype != torch.float32:
        raise TypeError("x fp32, codes uint8, absmax fp32")
    if codes.numel() < n or absmax.numel() < (n + blocksize - 1) // blocksize:
        raise ValueError("output buffers too small")
    _check(lib().bq_quantize_blockwise(_map_ptr(qmap, "qmap"), _dev_ptr(x, "x"), n,
                                       int(blocksize), _dev_ptr(codes, "codes"),
                                       _dev_ptr(absmax, "absmax"), _stream(stream)),
           "bq_quantize_blockwise")
    return codes, absmax


def bq_dequantize_blockwise(qmap, codes, absmax, blocksize: int, out=None, stream=None):
    r = host().dequantize(qmap, codes, absmax, blocksize, out, stream)
    if r.__class__ is int:
        _check(r, "bq_dequantize_blockwise")
    if r is not None:
        return r
    import torch
    n = codes.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=codes.device)
    if codes.dtype != torch.uint8 or absmax.dtype != torch.float32 or out.dtype != torch.float32:
        raise TypeError("codes uint8, absmax fp32, out fp32")
    if out.numel() < n or absmax.numel() < (n + blocksize - 1) // blocksize:
        raise ValueError("buffers too small")
    _check(lib().bq_dequantize_blockwise(_map_ptr(qmap, "qmap"), _dev_ptr(codes, "codes"),
                                         _dev_ptr(absmax, "absmax"), n, int(blocksize),
                                         _dev_ptr(out, "out"), _stream(stream)),
           "bq_dequantize_blockwise")
    return out


def _grad_torch_dtype(grad_dtype):
    import torch
    return {BQ_F32: torch.float32, BQ_F16: torch.float16,
            BQ_BF16: torch.bfloat16}.get(int(grad_dtype))


def check_step_tensors(opt, blocksize: int, grad_dtype: int, tensors) -> None:
    """Sizes, dtypes and device of a step's (param, grad, state1, state2,
    absmax1, absmax2) tuples.  The C ABI takes plain pointers and cannot see
    them: a state or absmax array shorter than its param would be written
    past its end.  Raises ValueError / TypeError."""
    import torch
    if isinstance(opt, str):
        opt = OPTIMIZERS[opt]
    two = int(opt) in (BQ_ADAM, BQ_ADAMW, BQ_LAMB)
    gdt = _grad_torch_dtype(grad_dtype)
    cur = torch.cuda.current_device()
    B = int(blocksize)
    for i, (p, g, s1, s2, a1, a2) in enumerate(tensors):
        n = p.numel()
        want = [(p, "param", torch.float32, n), (g, "grad", gdt, n), (s1, "state1", torch.uint8, n)]
        if B > 0:
            want.append((a1, "absmax1", torch.float32, (n + B - 1) // B))
        if two:
            want.append((s2, "state2", torch.uint8, n))
            if B > 0:
                want.append((a2, "absmax2", torch.float32, (n + B - 1) // B))
        for t, name, dtype, size in want:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"tensor {i}: {name} must be a torch tensor")
            if dtype is not None and t.dtype != dtype:
                raise TypeError(f"tensor {i}: {name} must be {dtype}, got {t.dtype}")
            if t.numel() < size:
                raise ValueError(f"tensor {i}: {name} holds {t.numel()} elements, needs {size}")
            if t.is_cuda and t.get_device() != cur:
                raise ValueError(f"tensor {i}: {name} is on cuda:{t.get_device()}, the current "
                                 f"device is cuda:{cur}")


def make_tensor_array(tensors):
    """Pack (param, grad, state1, state2, absmax1, absmax2) tuples of GPU
    tensors (state2 / absmax2 may be None) into a ctypes bq_tensor array."""
    arr = (bq_tensor * max(1, len(tensors)))()
    for i, (p, g, s1, s2, a1, a2) in enumerate(tensors):
        arr[i].param = _dev_ptr(p, "param")
        arr[i].grad = _dev_ptr(g, "grad")
        arr[i].state1 = _dev_ptr(s1, "state1")
        arr[i].state2 = None if s2 is None else _dev_ptr(s2, "state2")
        arr[i].absmax1 = _dev_ptr(a1, "absmax1")
        arr[i].absmax2 = None if a2 is None else _dev_ptr(a2, "absmax2")
        arr[i].numel = p.numel()
    return arr


def bq_optimizer8bit_step(opt, blocksize: int, grad_dtype: int, tensors, hp: dict, qmap1,
                          qmap2=None, stream=None):
    """One fused 8-bit step over a list of tensors (see make_tensor_array), or
    over a prebuilt ``(bq_tensor array, count)`` pair."""
    if isinstance(opt, str):
        opt = OPTIMIZERS[opt]
    if isinstance(tensors, tuple) and len(tensors) == 2 and isinstance(tensors[1], int):
        arr, count = tensors  # prebuilt by the caller, who vouches for the sizes
    else:
        check_step_tensors(opt, blocksize, grad_dtype, tensors)
        arr, count = make_tensor_array(tensors), len(tensors)
    if isinstance(arr, ctypes.Array):
        r = host().step(opt, blocksize, grad_dtype, ctypes.addressof(arr), count, hp, qmap1,
                        qmap2, stream)
        if r is not None:
            return _check(r, "bq_optimizer8bit_step")
    h = _hparams(hp)
    _check(lib().bq_optimizer8bit_step(int(opt), int(blocksize), int(grad_dtype), arr, count,
                                       ctypes.byref(h), _map_ptr(qmap1, "qmap1"),
                                       None if qmap2 is None else _map_ptr(qmap2, "qmap2"),
                                       _stream(stream)),
           "bq_optimizer8bit_step")


def bq_optimizer8bit_step_static(opt, blocksize: int, grad_dtype: int, tensors, hp: dict,
                                 qmap1, qmap2=None, stream=None):
    """bq_optimizer8bit_step through the library's static device array (no
    allocation; calls on one GPU must not overlap)."""
    if isinstance(opt, str):
        opt = OPTIMIZERS[opt]
    if isinstance(tensors, tuple) and len(tensors) == 2 and isinstance(tensors[1], int):
        arr, count = tensors  # prebuilt by the caller, who vouches for the sizes
    else:
        check_step_tensors(opt, blocksize, grad_dtype, tensors)
        arr, count = make_tensor_array(tensors), len(tensors)
    h = _hparams(hp)
    _check(lib().bq_optimizer8bit_step_static(
        int(opt), int(blocksize), int(grad_dtype), arr, count, ctypes.byref(h),
        _map_ptr(qmap1, "qmap1"), None if qmap2 is None else _map_ptr(qmap2, "qmap2"),
        _stream(stream)), "bq_optimizer8bit_step_static")


def make_tensor32_array(tensors):
    """Pack (param, grad, state1, state2) tuples of GPU tensors (state2 may be
    None) into a ctypes bq_tensor32 array."""
    arr = (bq_tensor32 * max(1, len(tensors)))()
    for i, (p, g, m, v) in enumerate(tensors):
        arr[i].param = _dev_ptr(p, "param")
        arr[i].grad = _dev_ptr(g, "grad")
        arr[i].state1 = _dev_ptr(m, "state1")
        arr[i].state2 = None if v is None else _dev_ptr(v, "state2")
        arr[i].numel = p.numel()
    return arr


def bq_optimizer32bit_step(opt, grad_dtype: int, tensors, hp: dict, stream=None):
    """One step with fp32 states over (param, grad, state1, state2) tuples."""
    import torch
    if isinstance(opt, str):
        opt = OPTIMIZERS[opt]
    two = int(opt) in (BQ_ADAM, BQ_ADAMW)
    gdt = _grad_torch_dtype(grad_dtype)
    cur = torch.cuda.current_device()
    for i, (p, g, m, v) in enumerate(tensors):
        n = p.numel()
        want = [(p, "param", torch.float32), (g, "grad", gdt), (m, "state1", torch.float32)]
        if two:
            want.append((v, "state2", torch.float32))
        for t, name, dtype in want:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"tensor {i}: {name} must be a torch tensor")
            if dtype is not None and t.dtype != dtype:
                raise TypeError(f"tensor {i}: {name} must be {dtype}, got {t.dtype}")
            if t.numel() < n:
                raise ValueError(f"tensor {i}: {name} holds {t.numel()} elements, needs {n}")
            if t.is_cuda and t.get_device() != cur:
                raise ValueError(f"tensor {i}: {name} is on cuda:{t.get_device()}, the current "
                                 f"device is cuda:{cur}")
    arr = make_tensor32_array(tensors)
    h = _hparams(hp)
    _check(lib().bq_optimizer32bit_step(int(opt), int(grad_dtype), arr, len(tensors),
                                        ctypes.byref(h), _stream(stream)),
           "bq_optimizer32bit_step")


def _hparams(hp: dict) -> bq_hparams:
    return bq_hparams(hp["lr"], hp["beta1"], hp.get("beta2", 0.0), hp.get("eps", 0.0),
                      hp.get("wd", hp.get("weight_decay", 0.0)), int(hp["step"]),
                      hp.get("trust", 0.0))


def bq_prepare_codebook(qmap, prepared=None, stream=None):
    """Decision tables of a device codebook into a device uint8 buffer of
    BQ_PREPARED_CODEBOOK_BYTES (allocated here by torch if not given)."""
    import torch
    if prepared is None:
        prepared = torch.empty(BQ_PREPARED_CODEBOOK_BYTES, dtype=torch.uint8, device=qmap.device)
    if prepared.numel() < BQ_PREPARED_CODEBOOK_BYTES:
        raise ValueError("prepared buffer too small")
    _check(lib().bq_prepare_codebook(_map_ptr(qmap, "qmap"), _dev_ptr(prepared, "prepared"),
                                     _stream(stream)), "bq_prepare_codebook")
    return prepared


def bq_quantize_blockwise_prepared(prepared, x, blocksize: int, codes=None, absmax=None,
                                   stream=None):
    r = host().quantize(True, prepared, x, blocksize, codes, absmax, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        _check(r, "bq_quantize_blockwise_prepared")
    import torch
    n = x.numel()
    if codes is None:
        codes = torch.empty(n, dtype=torch.uint8, device=x.device)
    if absmax is None:
        absmax = torch.empty((n + blocksize - 1) // blocksize, dtype=torch.float32,
                             device=x.device)
    if x.dtype != torch.float32 or codes.dtype != torch.uint8 or absmax.dtype != torch.float32:
        raise TypeError("x fp32, codes uint8, absmax fp32")
    if codes.numel() < n or absmax.numel() < (n + blocksize - 1) // blocksize:
        raise ValueError("output buffers too small")
    if prepared.numel() * prepared.element_size() < BQ_PREPARED_CODEBOOK_BYTES:
        raise ValueError(f"prepared codebook: need {BQ_PREPARED_CODEBOOK_BYTES} bytes")
    _check(lib().bq_quantize_blockwise_prepared(_dev_ptr(prepared, "prepared"), _dev_ptr(x, "x"),
                                                n, int(blocksize), _dev_ptr(codes, "codes"),
                                                _dev_ptr(absmax, "absmax"), _stream(stream)),
           "bq_quantize_blockwise_prepared")
    return codes, absmax


def prepare_codebook_pair(qmap1, qmap2=None, stream=None):
    """Both codebooks of an optimizer prepared back to back in one device
    buffer (bq_prepare_codebook twice), as bq_step_plan_run_prepared reads
    them: map 1's tables, then map 2's (absent for one-state optimizers)."""
    import torch
    prepared = torch.empty(2 * BQ_PREPARED_CODEBOOK_BYTES, dtype=torch.uint8,
                           device=qmap1.device)
    bq_prepare_codebook(qmap1, prepared[:BQ_PREPARED_CODEBOOK_BYTES], stream)
    if qmap2 is not None:
        bq_prepare_codebook(qmap2, prepared[BQ_PREPARED_CODEBOOK_BYTES:], stream)
    return prepared


class StepPlan:
    """bq_step_plan_create / bq_step_plan_run / bq_step_plan_destroy.

    The plan holds device pointers to the given tensors.  By default this
    object keeps references to them, so they stay allocated while the plan
    lives.  keep=False drops those references: the caller must then check,
    before every run, that the same storages (pointers and sizes) are still
    the live tensors (the drop-in optimizers do)."""

    def __init__(self, opt, blocksize: int, grad_dtype: int, tensors, keep: bool = True):
        if isinstance(opt, str):
            opt = OPTIMIZERS[opt]
        self._keep = [t for row in tensors for t in row if t is not None] if keep else []
        check_step_tensors(opt, blocksize, grad_dtype, tensors)
        arr = make_tensor_array(tensors)
        h = ctypes.c_void_p()
        _check(lib().bq_step_plan_create(int(opt), int(blocksize), int(grad_dtype), arr,
                                         len(tensors), ctypes.byref(h)), "bq_step_plan_create")
        self._h = h
        self._two = opt in (BQ_ADAM, BQ_ADAMW, BQ_LAMB)

    def run(self, hp: dict, qmap1, qmap2=None, stream=None):
        r = host().run(self._address(), hp, qmap1, qmap2, stream)
        if r is not None:
            return _check(r, "bq_step_plan_run")
        h = _hparams(hp)
        _check(lib().bq_step_plan_run(self._h, ctypes.byref(h), _map_ptr(qmap1, "qmap1"),
                                      None if qmap2 is None else _map_ptr(qmap2, "qmap2"),
                                      _stream(stream)), "bq_step_plan_run")

    def run_prepared(self, hp: dict, prepared, stream=None):
        """One run with codebooks prepared beforehand (prepare_codebook_pair)."""
        need = (2 if self._two else 1) * BQ_PREPARED_CODEBOOK_BYTES
        r = host().run_prepared(self._address(), need, hp, prepared, stream)
        if r is not None:
            return _check(r, "bq_step_plan_run_prepared")
        import torch
        if prepared.dtype != torch.uint8 or prepared.numel() < need:
            raise ValueError(f"prepared codebooks: need {need} uint8 bytes")
        h = _hparams(hp)
        _check(lib().bq_step_plan_run_prepared(self._h, ctypes.byref(h),
                                               _dev_ptr(prepared, "prepared"), _stream(stream)),
               "bq_step_plan_run_prepared")

    def run_device(self, hp_device, prepared, advance: bool = True, stream=None):
        """One run whose hyperparameters are read from device memory when it
        executes (hp_device: device_hparams); capturable into a graph."""
        import torch
        need = (2 if self._two else 1) * BQ_PREPARED_CODEBOOK_BYTES
        if prepared.dtype != torch.uint8 or prepared.numel() < need:
            raise ValueError(f"prepared codebooks: need {need} uint8 bytes")
        if hp_device.dtype != torch.uint8 or hp_device.numel() != ctypes.sizeof(bq_hparams):
            raise ValueError("hp_device must come from device_hparams()")
        _check(lib().bq_step_plan_run_device(self._h, _dev_ptr(hp_device, "hp_device"),
                                             1 if advance else 0,
                                             _dev_ptr(prepared, "prepared"), _stream(stream)),
               "bq_step_plan_run_device")

    def _address(self) -> int:
        return 0 if self._h is None else self._h.value or 0

    def is_open(self) -> bool:
        return getattr(self, "_h", None) is not None and self._h.value is not None

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value is not None:
            lib().bq_step_plan_destroy(self._h)
        self._h = None
        self._keep = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def bq_step_plan_create(opt, blocksize, grad_dtype, tensors):
    return StepPlan(opt, blocksize, grad_dtype, tensors)


def bq_step_plan_run(plan: StepPlan, hp: dict, qmap1, qmap2=None, stream=None):
    plan.run(hp, qmap1, qmap2, stream)


def bq_step_plan_run_prepared(plan: StepPlan, hp: dict, prepared, stream=None):
    plan.run_prepared(hp, prepared, stream)


def bq_step_plan_run_device(plan: StepPlan, hp_device, prepared, advance=True, stream=None):
    plan.run_device(hp_device, prepared, advance, stream)


def device_hparams(hp: dict, device=None):
    """A bq_hparams packed into a device uint8 tensor, for run_device.  Start
    from step 0 with advance=True for a first step."""
    import torch
    h = _hparams(dict(hp, step=hp.get("step", 0)))
    raw = ctypes.string_at(ctypes.addressof(h), ctypes.sizeof(h))
    t = torch.frombuffer(bytearray(raw), dtype=torch.uint8)
    return t.to("cuda" if device is None else device)


def read_device_hparams(t) -> dict:
    """The fields of a device bq_hparams (as written by device_hparams)."""
    h = bq_hparams.from_buffer_copy(bytes(t.cpu().numpy().tobytes()))
    return dict(lr=h.lr, beta1=h.beta1, beta2=h.beta2, eps=h.eps, wd=h.weight_decay,
                step=h.step, trust=h.trust_coeff)


def bq_step_plan_destroy(plan: StepPlan):
    plan.close()


# ---------------------------------------------------------------------------
# Operators around the optimizer step
# ---------------------------------------------------------------------------

def _dtype_id(t, name):
    import torch
    d = {torch.float32: BQ_F32, torch.float16: BQ_F16, torch.bfloat16: BQ_BF16}.get(
        t if isinstance(t, torch.dtype) else getattr(t, "dtype", None))
    if d is None:
        raise TypeError(f"{name} must be fp32, fp16 or bf16")
    return d


def _eager():
    """Refuses a call that a tracer records: the kernels write through addresses, so the
    trace would hold the allocation of a result and nothing that fills it."""
    import torch
    fx = sys.modules.get("torch.fx.experimental.proxy_tensor")
    if torch.jit.is_tracing() or (fx is not None and fx.get_proxy_mode() is not None):
        raise NotImplementedError("libbq's kernels cannot be traced")


def _no_tangent(*tensors):
    """Refuses dual tensors of forward-mode differentiation: a result would come without a
    tangent, as if it did not depend on them."""
    import torch
    from torch.autograd import forward_ad
    if torch._C._is_fwd_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
                raise NotImplementedError("libbq's kernels have no forward-mode derivatives")


def _on_device(t, name):
    """t, a dense GPU tensor on the current device."""
    import torch
    _eager()
    _no_tangent(t)
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.layout is not torch.strided:
        raise TypeError(f"{name} must be a dense GPU torch tensor")
    if t.is_neg():
        raise TypeError(f"{name} is a view with a pending negation; pass {name}.resolve_neg()")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")
    # (a null pointer would stand for a parameter that was left out)
    if t.numel() and (t.untyped_storage().nbytes() == 0 or t.data_ptr() == 0):
        raise ValueError(f"{name} has no memory (an emptied storage, or a fake tensor)")
    return t


def _rows_of(t, name):
    """(rows, cols, elements between rows) of a GPU tensor whose last dimension is packed."""
    _on_device(t, name)
    if t.dim() == 0 or t.size(-1) == 0:
        raise ValueError(f"{name} needs a last dimension of at least one element")
    cols = t.size(-1)
    if t.is_contiguous():
        return t.numel() // cols, cols, cols
    if t.dim() == 2 and (t.stride(1) == 1 or cols == 1):
        return t.size(0), cols, t.stride(0)
    raise ValueError(f"{name} must be contiguous, or two-dimensional with packed rows")


def _vector(t, n, dtype, name):
    """Pointer of an optional parameter vector of n elements of dtype."""
    if t is None:
        return None
    _on_device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous elements")
    return t.data_ptr()


def _other(stream):
    """stream, where it is not the current one; else None."""
    import torch
    if stream is None:
        return None
    if stream.device_index != torch.cuda.current_device():
        # the C calls run on the current device
        raise ValueError(f"stream is on cuda:{stream.device_index}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")
    return None if stream == torch.cuda.current_stream() else stream


def _empty(shape, dtype, device, other):
    """A buffer for a call on stream `other` (None: the current one): it comes from that
    stream's memory, and is not given away while the current stream may use it."""
    import torch
    if other is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(other):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream())
    return t


def _used(other, *tensors):
    """Keeps the memory of a call's tensors until stream `other` has used them."""
    if other is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(other)


def _output(out, shape, dtype, device, other, name):
    if out is None:
        return _empty(shape, dtype, device, other)
    _on_device(out, name)
    if out.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {out.dtype}")
    if tuple(out.shape) != tuple(shape) or not out.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of shape {tuple(shape)}")
    _used(other, out)
    return out


def _workspace(workspace, nbytes, device, other):
    """A device buffer of at least nbytes."""
    import torch
    if workspace is None:
        return _empty((max(16, nbytes),), torch.uint8, device, other)
    _on_device(workspace, "workspace")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if workspace.numel() * workspace.element_size() < nbytes:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} bytes, "
                         f"needs {nbytes}")
    _used(other, workspace)
    return workspace


def _norm_params(x, weight, bias, cols):
    """(dtype of the parameters, pointer of weight, pointer of bias) of a layer norm."""
    import torch
    given = weight if weight is not None else bias
    dtype = x.dtype if given is None else given.dtype
    if dtype not in (torch.float32, x.dtype):
        raise TypeError(f"weight and bias must be fp32 or {x.dtype}, got {dtype}")
    return dtype, _vector(weight, cols, dtype, "weight"), _vector(bias, cols, dtype, "bias")


def bq_layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, stats: bool = False,
                          out=None, stream=None):
    """The layer norm of x over its last dimension; with stats, (y, mean, rstd), the
    fp32 statistics of every row that the backward pass takes.  weight and bias: of
    x's type or fp32, both alike, each may be None."""
    if not stats and out is None and stream is None:
        y = host().layer_norm(x, weight, bias, eps, False)
        if y is not None:
            return y
    import torch
    _no_tangent(x, weight, bias)
    rows, cols, stride = _rows_of(x, "x")
    xt = _dtype_id(x, "x")
    pdtype, w, b = _norm_params(x, weight, bias, cols)
    other = _other(stream)
    _used(other, x, weight, bias)
    y = _output(out, x.shape, x.dtype, x.device, other, "out")
    mean = rstd = None
    if stats:
        mean = _empty((rows,), torch.float32, x.device, other)
        rstd = _empty((rows,), torch.float32, x.device, other)
    _check(lib().bq_layer_norm_forward(xt, _dtype_id(pdtype, "weight"), x.data_ptr(), rows, cols,
                                       stride, w, b, eps, y.data_ptr(),
                                       mean.data_ptr() if stats else None,
                                       rstd.data_ptr() if stats else None, _stream(stream)),
           "bq_layer_norm_forward")
    return (y, mean, rstd) if stats else y


def bq_layer_norm_backward(dy, x, weight, mean, rstd, need_dx: bool = True,
                           need_params: bool = True, param_dtype=None, workspace=None,
                           stream=None):
    """(dx, dweight, dbias) of the layer norm of x, None where not needed; mean and rstd as
    bq_layer_norm_forward returned them.  The parameters' gradients have weight's type
    (param_dtype where weight is None)."""
    import torch
    _no_tangent(dy, x, weight, mean, rstd)
    rows, cols, stride = _rows_of(x, "x")
    xt = _dtype_id(x, "x")
    if not isinstance(dy, torch.Tensor) or dy.dtype != x.dtype or dy.shape != x.shape:
        raise TypeError("dy must have x's type and shape")
    _, _, dy_stride = _rows_of(dy, "dy")
    if weight is None and param_dtype is not None:
        if param_dtype not in (torch.float32, x.dtype):
            raise TypeError(f"param_dtype must be fp32 or {x.dtype}")
        pdtype, w = param_dtype, None
    else:
        pdtype, w, _ = _norm_params(x, weight, None, cols)
    m, r = (_vector(t, rows, torch.float32, n) for t, n in ((mean, "mean"), (rstd, "rstd")))
    if m is None or r is None:
        raise TypeError("mean and rstd are required")
    other = _other(stream)
    _used(other, dy, x, weight, mean, rstd)
    dx = _empty(x.shape, x.dtype, x.device, other) if need_dx else None
    dw = db = ws = None
    if need_params:
        dw = _empty((cols,), pdtype, x.device, other)
        db = _empty((cols,), pdtype, x.device, other)
        ws = _workspace(workspace, lib().bq_layer_norm_workspace_bytes(rows, cols), x.device, other)
    _check(lib().bq_layer_norm_backward(
        xt, _dtype_id(pdtype, "weight"), dy.data_ptr(), dy_stride, x.data_ptr(), stride, rows, cols,
        w, m, r, *(None if t is None else t.data_ptr() for t in (dx, dw, db, ws)),
        _stream(stream)), "bq_layer_norm_backward")
    return dx, dw, db


def _ids_of(ids):
    """(pointer, bits) of a GPU tensor of token ids."""
    import torch
    _on_device(ids, "ids")
    if ids.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"ids must be int64 or int32, got {ids.dtype}")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return ids.data_ptr(), 64 if ids.dtype == torch.int64 else 32


def _table_of(weight):
    """(dtype id, rows, dim) of an embedding table."""
    _on_device(weight, "weight")
    if weight.dim() != 2 or not weight.is_contiguous():
        raise ValueError("weight must be a contiguous matrix")
    return _dtype_id(weight, "weight"), weight.size(0), weight.size(1)


def _lookup_dtype(weight_dtype, out_dtype):
    import torch
    out = weight_dtype if out_dtype is None else out_dtype
    _dtype_id(out, "out_dtype")
    if weight_dtype not in (torch.float32, out):
        raise TypeError(f"a {weight_dtype} table gives {weight_dtype} rows, not {out}")
    return out


def _padding(padding_idx, num):
    """padding_idx as a row (negative ones count from the end), -1 for None."""
    if padding_idx is None:
        return -1
    if not -num <= padding_idx < num:
        raise ValueError(f"padding_idx {padding_idx} is outside of a table of {num} rows")
    return padding_idx % num


def bq_embedding_forward(weight, ids, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """scale * weight[ids]: rows of weight (num, dim) looked up by int64 or int32 ids of
    any shape, in out_dtype (weight's type, or any where weight is fp32).  An id outside
    of the table gives a row of NaN."""
    if out is None and stream is None:
        y = host().embedding(ids, weight, None, scale, out_dtype, False)
        if y is not None:
            return y
    wt, num, dim = _table_of(weight)
    ptr, bits = _ids_of(ids)
    dtype = _lookup_dtype(weight.dtype, out_dtype)
    other = _other(stream)
    _used(other, weight, ids)
    y = _output(out, (*ids.shape, dim), dtype, weight.device, other, "out")
    _check(lib().bq_embedding_forward(wt, _dtype_id(dtype, "out"), weight.data_ptr(), num, dim, ptr,
                                      bits, ids.numel(), scale, y.data_ptr(), _stream(stream)),
           "bq_embedding_forward")
    return y


def _lookup_grad(dout, ids, dim):
    _no_tangent(dout)
    ptr, bits = _ids_of(ids)
    _on_device(dout, "dout")
    if not dout.is_contiguous() or tuple(dout.shape) != (*ids.shape, dim):
        raise ValueError(f"dout must be contiguous, of shape {(*ids.shape, dim)}")
    return ptr, bits, _dtype_id(dout, "dout")


def bq_embedding_backward(dout, ids, num: int, padding_idx=None, scale: float = 1.0, dtype=None,
                          out=None, workspace=None, stream=None):
    """The gradient of a table of num rows whose rows were looked up by ids: scale times the
    sums of dout's rows by id, as a dense matrix of dtype (dout's type, or fp32)."""
    import torch
    dim = dout.size(-1) if isinstance(dout, torch.Tensor) and dout.dim() else 0
    ptr, bits, yt = _lookup_grad(dout, ids, dim)
    dtype = dout.dtype if dtype is None else dtype
    _lookup_dtype(dtype, dout.dtype)
    pad = _padding(padding_idx, num)
    other = _other(stream)
    _used(other, dout, ids)
    dw = _output(out, (num, dim), dtype, dout.device, other, "out")
    ws = _workspace(workspace, lib().bq_embedding_workspace_bytes(ids.numel(), num, dim),
                    dout.device, other)
    _check(lib().bq_embedding_backward(_dtype_id(dtype, "dtype"), yt, dout.data_ptr(), ptr, bits,
                                       ids.numel(), num, dim, pad, scale, dw.data_ptr(),
                                       ws.data_ptr(), _stream(stream)), "bq_embedding_backward")
    return dw


def bq_stable_embedding_forward(weight, ids, norm_weight=None, norm_bias=None, eps: float = 1e-5,
                                out_dtype=None, out=None, stream=None):
    """The layer norm of weight[ids] (as bq_embedding_forward looks it up) in one pass;
    norm_weight and norm_bias of weight's type, each may be None."""
    if out is None and stream is None:
        y = host().stable_embedding(ids, weight, norm_weight, norm_bias, eps, None, out_dtype,
                                    False)
        if y is not None:
            return y
    _no_tangent(weight, norm_weight, norm_bias)
    wt, num, dim = _table_of(weight)
    ptr, bits = _ids_of(ids)
    dtype = _lookup_dtype(weight.dtype, out_dtype)
    w = _vector(norm_weight, dim, weight.dtype, "norm_weight")
    b = _vector(norm_bias, dim, weight.dtype, "norm_bias")
    other = _other(stream)
    _used(other, weight, ids, norm_weight, norm_bias)
    y = _output(out, (*ids.shape, dim), dtype, weight.device, other, "out")
    _check(lib().bq_stable_embedding_forward(wt, _dtype_id(dtype, "out"), weight.data_ptr(), num,
                                             dim, ptr, bits, ids.numel(), w, b, eps, y.data_ptr(),
                                             _stream(stream)), "bq_stable_embedding_forward")
    return y


def bq_stable_embedding_backward(dout, ids, weight, norm_weight=None, eps: float = 1e-5,
                                 padding_idx=None, need_norm: bool = True, workspace=None,
                                 stream=None):
    """(dweight, dnorm_weight, dnorm_bias) of the stable embedding, in weight's type; the
    last two None without need_norm."""
    _no_tangent(dout, weight, norm_weight)
    wt, num, dim = _table_of(weight)
    ptr, bits, yt = _lookup_grad(dout, ids, dim)
    _lookup_dtype(weight.dtype, dout.dtype)
    w = _vector(norm_weight, dim, weight.dtype, "norm_weight")
    pad = _padding(padding_idx, num)
    other = _other(stream)
    _used(other, dout, ids, weight, norm_weight)
    dweight = _empty((num, dim), weight.dtype, weight.device, other)
    dw = db = None
    if need_norm:
        dw = _empty((dim,), weight.dtype, weight.device, other)
        db = _empty((dim,), weight.dtype, weight.device, other)
    ws = _workspace(workspace, lib().bq_stable_embedding_workspace_bytes(ids.numel(), num, dim),
                    weight.device, other)
    _check(lib().bq_stable_embedding_backward(
        wt, yt, dout.data_ptr(), ptr, bits, ids.numel(), weight.data_ptr(), num, dim, pad, w, eps,
        dweight.data_ptr(), *(None if t is None else t.data_ptr() for t in (dw, db)),
        ws.data_ptr(), _stream(stream)), "bq_stable_embedding_backward")
    return dweight, dw, db


def _norm_kind(norm_type):
    kind = {2.0: BQ_NORM_L2, float("inf"): BQ_NORM_INF}.get(float(norm_type))
    if kind is None:
        raise ValueError(f"norm_type must be 2 or inf, got {norm_type}")
    return kind


def _packed(t):
    """Whether the tensor's elements fill one range of memory, in any order."""
    if t.is_contiguous():
        return True
    want = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size > 1:
            if stride != want:
                return False
            want *= size
    return True


def make_grad_array(grads):
    """Pack gradients (GPU tensors that each fill one range of memory) into a ctypes bq_grad
    array."""
    arr = (bq_grad * max(1, len(grads)))()
    for i, g in enumerate(grads):
        _on_device(g, f"gradient {i}")
        if not _packed(g):
            raise ValueError(f"gradient {i} does not fill one range of memory")
        arr[i].data = g.data_ptr()
        arr[i].numel = g.numel()
        arr[i].dtype = _dtype_id(g, f"gradient {i}")
    return arr


def _grad_norm(grads, norm_type, max_norm, out, workspace, stream):
    import torch
    _eager()
    kind = _norm_kind(norm_type)
    grads = list(grads)
    arr = make_grad_array(grads)
    if max_norm is not None:
        places = [g.data_ptr() for g in grads if g.numel()]
        if len(set(places)) != len(places):
            raise ValueError("two gradients are in the same place")
    other = _other(stream)
    _used(other, *grads)
    device = torch.device("cuda", torch.cuda.current_device())
    norm = _output(out, (), torch.float32, device, other, "out")
    ws = _workspace(workspace, lib().bq_grad_norm_workspace_bytes(len(grads)), device, other)
    if max_norm is None:
        _check(lib().bq_grad_norm(arr, len(grads), kind, ws.data_ptr(), norm.data_ptr(),
                                  _stream(stream)), "bq_grad_norm")
    else:
        _check(lib().bq_clip_grad_norm(arr, len(grads), kind, max_norm, ws.data_ptr(),
                                       norm.data_ptr(), _stream(stream)), "bq_clip_grad_norm")
    return norm


def bq_grad_norm(grads, norm_type=2.0, out=None, workspace=None, stream=None):
    """The norm (2 or inf) of a list of gradients taken as one vector: an fp32 scalar on the
    GPU."""
    return _grad_norm(grads, norm_type, None, out, workspace, stream)


def bq_clip_grad_norm(grads, max_norm: float, norm_type=2.0, out=None, workspace=None,
                      stream=None):
    """The norm as bq_grad_norm; then every gradient times min(1, max_norm / (norm + 1e-6)),
    in place.  The gradients must not overlap.  Nothing is read back by the host."""
    return _grad_norm(grads, norm_type, float(max_norm), out, workspace, stream)
