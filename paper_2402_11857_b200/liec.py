"""ctypes binding of ``include/liec.h``: same names, argument marshalling only.

PyTorch appears here only as the owner of device memory and streams.  There is no
fallback: if ``libliec.so`` is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

import numpy as np

COMP_IDENTITY, COMP_SCALED_SIGN, COMP_TOPK, COMP_RANDK = 0, 1, 2, 3
SUMSQ_ERROR, SUMSQ_GRADS, SUMSQ_PARAMS = 0, 1, 2
F32, BF16 = 0, 1
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}
ACTIVATION_BLOCK = 32

STATUS_NAMES = {0: "LIEC_OK", 1: "LIEC_ERR_INVALID_ARG", 2: "LIEC_ERR_UNSUPPORTED", 3: "LIEC_ERR_WORKSPACE",
                4: "LIEC_ERR_STATE", 5: "LIEC_ERR_CUDA", 6: "LIEC_ERR_DEVICE_CHECK"}

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libliec.so")
_LIB: Optional[C.CDLL] = None


class LiecError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class liec_config(C.Structure):
    _fields_ = [("num_workers", C.c_int32), ("dim", C.c_int64), ("num_segments", C.c_int32),
                ("seg_offsets", C.POINTER(C.c_int64)), ("uplink", C.c_int32), ("downlink", C.c_int32),
                ("topk_k", C.POINTER(C.c_int64)), ("grad_dtype", C.c_int32)]


class liec_messages(C.Structure):
    _fields_ = [("up_words", C.c_void_p), ("up_scales", C.c_void_p), ("up_idx", C.c_void_p),
                ("up_val", C.c_void_p), ("down_words", C.c_void_p), ("down_scales", C.c_void_p),
                ("down_idx", C.c_void_p), ("down_val", C.c_void_p), ("v", C.c_void_p),
                ("num_words", C.c_int64), ("num_topk", C.c_int64)]


class liec_layer_norm_desc(C.Structure):
    _fields_ = [("groups", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("eps", C.c_float),
                ("x_row_stride", C.c_int64), ("x_group_stride", C.c_int64),
                ("y_row_stride", C.c_int64), ("y_group_stride", C.c_int64),
                ("dx_row_stride", C.c_int64), ("dx_group_stride", C.c_int64),
                ("weight_stride", C.c_int64), ("bias_stride", C.c_int64),
                ("dweight_stride", C.c_int64), ("dbias_stride", C.c_int64), ("shared_grads", C.c_int32)]


class liec_activation_desc(C.Structure):
    _fields_ = [("workers", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32),
                ("x_row_stride", C.c_int64), ("x_worker_stride", C.c_int64)]


class liec_group_norm_desc(C.Structure):
    _fields_ = [("workers", C.c_int32), ("samples", C.c_int32), ("pixels", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32),
                ("dtype", C.c_int32), ("grad_dtype", C.c_int32), ("activation", C.c_int32), ("eps", C.c_float),
                ("x_pixel_stride", C.c_int64), ("x_sample_stride", C.c_int64), ("x_worker_stride", C.c_int64),
                ("y_pixel_stride", C.c_int64), ("y_sample_stride", C.c_int64), ("y_worker_stride", C.c_int64),
                ("dx_pixel_stride", C.c_int64), ("dx_sample_stride", C.c_int64), ("dx_worker_stride", C.c_int64),
                ("weight_stride", C.c_int64), ("bias_stride", C.c_int64),
                ("dweight_stride", C.c_int64), ("dbias_stride", C.c_int64), ("shared_grads", C.c_int32)]


class liec_weight_grad_desc(C.Structure):
    _fields_ = [("workers", C.c_int32), ("rows", C.c_int64), ("in_", C.c_int32), ("out", C.c_int32), ("dtype", C.c_int32), ("grad_dtype", C.c_int32),
                ("dy_row_stride", C.c_int64), ("dy_worker_stride", C.c_int64),
                ("dweight_row_stride", C.c_int64), ("dweight_worker_stride", C.c_int64)]


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Loads libliec.so (built in-tree) and declares every entry point of liec.h."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(f"{p} not found: build it with `python -m paper_2402_11857_b200.build`")
    lib = C.CDLL(p)
    vp, cfgp = C.c_void_p, C.POINTER(liec_config)
    lib.liec_workspace_bytes.argtypes = [cfgp]
    lib.liec_workspace_bytes.restype = C.c_size_t
    lib.liec_wire_bytes.argtypes = [cfgp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    lib.liec_wire_bytes.restype = C.c_int
    lib.liec_down_message_bytes.argtypes = [cfgp]
    lib.liec_down_message_bytes.restype = C.c_size_t
    lib.liec_init.argtypes = [cfgp, vp, vp, vp, C.c_size_t, C.POINTER(vp)]
    lib.liec_init.restype = C.c_int
    lib.liec_uplink_compress.argtypes = [vp, vp, vp]
    lib.liec_uplink_compress.restype = C.c_int
    lib.liec_server_aggregate.argtypes = [vp, vp]
    lib.liec_server_aggregate.restype = C.c_int
    lib.liec_downlink_compress.argtypes = [vp, vp]
    lib.liec_downlink_compress.restype = C.c_int
    lib.liec_worker_update.argtypes = [vp, vp, C.c_float, vp]
    lib.liec_worker_update.restype = C.c_int
    lib.liec_set_subsets.argtypes = [vp, vp, vp]
    lib.liec_set_subsets.restype = C.c_int
    lib.liec_draw_subsets.argtypes = [vp, C.c_uint64, C.c_uint32, vp]
    lib.liec_draw_subsets.restype = C.c_int
    lib.liec_wire_bytes_seeded.argtypes = [cfgp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    lib.liec_wire_bytes_seeded.restype = C.c_int
    lib.liec_step.argtypes = [vp, vp, C.c_float, vp]
    lib.liec_step.restype = C.c_int
    lib.liec_topk_route_counts.argtypes = [vp, vp, C.c_int32, C.POINTER(C.c_int64), vp]
    lib.liec_topk_route_counts.restype = C.c_int
    lib.liec_abort_step.argtypes = [vp]
    lib.liec_abort_step.restype = C.c_int
    lib.liec_set_copy_wait.argtypes = [vp, C.c_uint32, C.c_uint32]
    lib.liec_set_copy_wait.restype = C.c_int
    lib.liec_set_norm_wait.argtypes = [vp, C.c_uint32, C.c_uint32]
    lib.liec_set_norm_wait.restype = C.c_int
    lib.liec_average_step.argtypes = [vp, vp, C.c_float, vp]
    lib.liec_average_step.restype = C.c_int
    lib.liec_mean_params.argtypes = [vp, vp, vp]
    lib.liec_mean_params.restype = C.c_int
    lib.liec_sumsq.argtypes = [vp, C.c_int32, vp, vp, vp]
    lib.liec_sumsq.restype = C.c_int
    lib.liec_set_telemetry.argtypes = [vp, C.c_int32]
    lib.liec_set_telemetry.restype = C.c_int
    lib.liec_get_telemetry.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.liec_get_telemetry.restype = C.c_int
    lib.liec_clip_grads.argtypes = [vp, vp, vp, C.c_float, C.c_int32, vp, vp]
    lib.liec_clip_grads.restype = C.c_int
    lib.liec_set_tensors.argtypes = [vp, vp, C.c_int32, vp]
    lib.liec_set_tensors.restype = C.c_int
    lib.liec_gather_grads.argtypes = [vp, vp, C.c_float, C.c_int32, vp, vp]
    lib.liec_gather_grads.restype = C.c_int
    lnp = C.POINTER(liec_layer_norm_desc)
    lib.liec_layer_norm_workspace_bytes.argtypes = [lnp]
    lib.liec_layer_norm_workspace_bytes.restype = C.c_size_t
    lib.liec_layer_norm_forward.argtypes = [lnp, vp, vp, vp, vp, vp, vp, vp]
    lib.liec_layer_norm_forward.restype = C.c_int
    lib.liec_layer_norm_backward.argtypes = [lnp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.liec_layer_norm_backward.restype = C.c_int
    acp, gnp, wgp = C.POINTER(liec_activation_desc), C.POINTER(liec_group_norm_desc), C.POINTER(liec_weight_grad_desc)
    lib.liec_activation_cols.argtypes = [C.c_int64]
    lib.liec_activation_cols.restype = C.c_int64
    lib.liec_activation_compress.argtypes = [acp, vp, vp, vp, vp]
    lib.liec_activation_compress.restype = C.c_int
    lib.liec_activation_restore.argtypes = [acp, vp, vp, vp, vp]
    lib.liec_activation_restore.restype = C.c_int
    lib.liec_group_norm_workspace_bytes.argtypes = [gnp, C.c_int32]
    lib.liec_group_norm_workspace_bytes.restype = C.c_size_t
    lib.liec_group_norm_forward.argtypes = [gnp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.liec_group_norm_forward.restype = C.c_int
    lib.liec_group_norm_backward.argtypes = [gnp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.liec_group_norm_backward.restype = C.c_int
    lib.liec_weight_grad_workspace_bytes.argtypes = [wgp, vp]
    lib.liec_weight_grad_workspace_bytes.restype = C.c_size_t
    lib.liec_weight_grad.argtypes = [wgp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.liec_weight_grad.restype = C.c_int
    lib.liec_step_host.argtypes = [vp, vp, vp, C.c_float, vp, vp]
    lib.liec_step_host.restype = C.c_int
    lib.liec_get_messages.argtypes = [vp, C.POINTER(liec_messages)]
    lib.liec_get_messages.restype = C.c_int
    lib.liec_device_status.argtypes = [vp, vp, C.POINTER(C.c_int32)]
    lib.liec_device_status.restype = C.c_int
    lib.liec_clear_status.argtypes = [vp, vp]
    lib.liec_clear_status.restype = C.c_int
    lib.liec_launch_count.argtypes = [vp]
    lib.liec_launch_count.restype = C.c_int64
    lib.liec_last_error.argtypes = [vp]
    lib.liec_last_error.restype = C.c_char_p
    lib.liec_destroy.argtypes = [vp]
    lib.liec_destroy.restype = None
    lib.liec_sign_compress_noalloc.argtypes = [vp, C.c_int32, C.c_int64, vp, vp, vp]
    lib.liec_sign_compress_noalloc.restype = C.c_int
    lib.liec_noalloc_last_error.argtypes = []
    lib.liec_noalloc_last_error.restype = C.c_char_p
    if path is None:
        _LIB = lib
    return lib


def make_config(num_workers: int, seg_offsets: Sequence[int], uplink: int, downlink: int,
                topk_k: Optional[Sequence[int]] = None, grad_dtype: int = F32):
    """Returns (liec_config, keepalive) - keepalive owns the host arrays the struct points to."""
    off = np.ascontiguousarray(seg_offsets, dtype=np.int64)
    k = None if topk_k is None else np.ascontiguousarray(topk_k, dtype=np.int64)
    cfg = liec_config()
    cfg.num_workers = int(num_workers)
    cfg.dim = int(off[-1]) if off.size else 0
    cfg.num_segments = int(off.size - 1)
    cfg.seg_offsets = off.ctypes.data_as(C.POINTER(C.c_int64))
    cfg.uplink, cfg.downlink = int(uplink), int(downlink)
    cfg.topk_k = k.ctypes.data_as(C.POINTER(C.c_int64)) if k is not None else None
    cfg.grad_dtype = int(grad_dtype)
    return cfg, (off, k)


def workspace_bytes(cfg: liec_config) -> int:
    return int(load_library().liec_workspace_bytes(C.byref(cfg)))


def liec_wire_bytes_seeded(cfg: liec_config):
    """As liec_wire_bytes when sender and receiver draw the random-k subsets from a shared seed."""
    return liec_wire_bytes(cfg, _seeded=True)


def liec_wire_bytes(cfg: liec_config, _seeded: bool = False):
    """(uplink, downlink, full-precision) bytes per worker and iteration."""
    lib = load_library()
    up, down, full = C.c_int64(0), C.c_int64(0), C.c_int64(0)
    fn = lib.liec_wire_bytes_seeded if _seeded else lib.liec_wire_bytes
    st = fn(C.byref(cfg), C.byref(up), C.byref(down), C.byref(full))
    if st != 0:
        raise LiecError(st, lib.liec_last_error(None).decode())
    return int(up.value), int(down.value), int(full.value)


def down_message_bytes(cfg: liec_config) -> int:
    return int(load_library().liec_down_message_bytes(C.byref(cfg)))


NOALLOC_MAX_ELEMENTS = 64 * 1024 * 1024


def liec_sign_compress_noalloc(x, words, scale, stream=None):
    """Scaled sign of one CUDA vector into caller-provided `words` (int32, ceil(n/32)) and `scale`
    (float32, 1 element) without any workspace or allocation; see liec.h for who needs this."""
    import torch
    lib = load_library()
    n = x.numel()
    if not (x.is_cuda and x.is_contiguous() and x.dtype in (torch.float32, torch.bfloat16)):
        raise ValueError("x must be a contiguous CUDA tensor of float32 or bfloat16")
    if not (words.is_cuda and words.is_contiguous() and words.dtype in (torch.int32, torch.uint32)
            and words.numel() == (n + 31) // 32 and words.device == x.device):
        raise ValueError("words must be a contiguous CUDA tensor of ceil(n/32) 32-bit integers on x's device")
    if not (scale.is_cuda and scale.dtype == torch.float32 and scale.numel() == 1 and scale.device == x.device):
        raise ValueError("scale must be a one-element float32 CUDA tensor on x's device")
    dtype = BF16 if x.dtype == torch.bfloat16 else F32
    s = (stream if stream is not None else torch.cuda.current_stream(x.device)).cuda_stream
    with torch.cuda.device(x.device):
        st = lib.liec_sign_compress_noalloc(x.data_ptr(), dtype, x.numel(), words.data_ptr(), scale.data_ptr(), s)
    if st != 0:
        raise LiecError(st, lib.liec_noalloc_last_error().decode())


# ---- layer normalisation over N workers -----------------------------------------------------------

def _device_of(name, t) -> int:
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be a CUDA tensor (there is no CPU path)")
    return index


def _launch(device: int, stream, fn, *args):
    """fn(raw stream, *args) on the caller's stream and the tensors' device; what fn allocates belongs to that stream."""
    import torch
    if stream is not None:
        with torch.cuda.stream(stream):
            return fn(stream.cuda_stream, *args)
    if device != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return fn(torch._C._cuda_getCurrentRawStream(device), *args)
    return fn(torch._C._cuda_getCurrentRawStream(device), *args)


def _layout(t):
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _ln_rows(name, t, x):
    """Row and group strides of [N, rows, h] or [rows, h] activations (N = 1), given as a layout."""
    shape, stride, dtype = t
    if shape != x[0] or dtype != x[2]:
        raise ValueError(f"{name} must have the shape and type of x")
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return stride[-2], (stride[0] if len(shape) == 3 else 0)


def _ln_vector(name, t, x, dtypes):
    """Stride from worker to worker of a weight-like [N, h] or [h] tensor (0: one vector for all workers)."""
    if t is None:
        return 0
    shape, stride, dtype = t
    h, N = x[0][-1], (x[0][0] if len(x[0]) == 3 else 1)
    if dtype not in dtypes:
        raise ValueError(f"{name} must be of type {' or '.join(str(d) for d in dtypes)}")
    if tuple(shape) not in ((h,), (N, h)) or (h > 1 and stride[-1] != 1):
        raise ValueError(f"{name} must be [h] or [N, h] with a contiguous last axis")
    return stride[0] if len(shape) == 2 else 0


@functools.lru_cache(maxsize=1024)
def _ln_desc(x, y, dx, weight, bias, dweight, dbias, eps):
    """Checks the layouts of a call and returns its descriptor and workspace size (both depend on sizes,
    strides and types alone, so calls of the same form share them)."""
    import torch
    both, f32 = (torch.float32, torch.bfloat16), (torch.float32,)
    shape = x[0]
    if x[2] not in both or len(shape) not in (2, 3):
        raise ValueError("x must be [N, rows, h] or [rows, h] of float32 or bfloat16")
    d = liec_layer_norm_desc()
    d.groups, d.rows, d.cols = (shape[0] if len(shape) == 3 else 1), shape[-2], shape[-1]
    d.dtype, d.eps = (BF16 if x[2] == torch.bfloat16 else F32), eps
    d.x_row_stride, d.x_group_stride = _ln_rows("x", x, x)
    d.y_row_stride, d.y_group_stride = _ln_rows("y" if dx is None else "dy", y, x)
    d.weight_stride, d.bias_stride = _ln_vector("weight", weight, x, f32), _ln_vector("bias", bias, x, f32)
    if dx is None:
        return d, C.byref(d), 0
    d.dx_row_stride, d.dx_group_stride = _ln_rows("dx", dx, x)
    d.dweight_stride, d.dbias_stride = _ln_vector("dweight", dweight, x, both), _ln_vector("dbias", dbias, x, both)
    if dweight[2] != dbias[2] or len(dweight[0]) != len(dbias[0]):
        raise ValueError("dweight and dbias must have the same type and number of axes")
    d.grad_dtype = BF16 if dweight[2] == torch.bfloat16 else F32
    if len(dweight[0]) == 1 and d.groups > 1:   # one vector for all workers: its gradient sums over their rows as well
        if d.weight_stride != 0:
            raise ValueError("workers with weights of their own need dweight and dbias [N, h]")
        if d.groups * d.rows < 1 << 31 and (d.rows <= 1 or all(t[1][0] == d.rows * t[1][1] for t in (x, y, dx))):
            # the workers' rows follow one another in all three: rows of one worker
            if d.rows == 1:
                d.x_row_stride, d.y_row_stride, d.dx_row_stride = x[1][0], y[1][0], dx[1][0]
            d.groups, d.rows = 1, d.groups * d.rows
        else:
            d.shared_grads = 1
    return d, C.byref(d), int(load_library().liec_layer_norm_workspace_bytes(C.byref(d)))


def liec_layer_norm_workspace_bytes(desc: liec_layer_norm_desc) -> int:
    return int(load_library().liec_layer_norm_workspace_bytes(C.byref(desc)))


def _ln_failed(lib, st):
    raise LiecError(st, lib.liec_last_error(None).decode())


@functools.lru_cache(maxsize=1024)
def _contiguous(shape):
    strides = [1]
    for n in reversed(shape[1:]):
        strides.append(strides[-1] * max(n, 1))
    return tuple(shape), tuple(reversed(strides))


def _empty(shape, dtype, device: int):
    """A contiguous tensor.  (torch.empty costs twice as much as empty_strided with plain tuples and a device's index.)"""
    import torch
    return torch.empty_strided(*_contiguous(shape), dtype=dtype, device=device)


def _empty_like(x):
    import torch
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _ln_forward(raw, device, x, weight, bias, eps, y):
    import torch
    if y is None:
        y = _empty_like(x)
    _, ref, _ = _ln_desc(_layout(x), _layout(y), None, _layout(weight), _layout(bias), None, None, eps)
    mean = _empty(x.shape[:-1], torch.float32, device)
    rstd = torch.empty_like(mean)
    lib = _LIB or load_library()
    st = lib.liec_layer_norm_forward(ref, x.data_ptr(), None if weight is None else weight.data_ptr(),
                                     None if bias is None else bias.data_ptr(), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), raw)
    if st != 0:
        _ln_failed(lib, st)
    return y, mean, rstd


def liec_layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, y=None, stream=None):
    """Layer norm of [N, rows, h] (or [rows, h]) activations with per-worker float32 weight and bias
    [N, h] (any stride between workers, e.g. ``params[:, a:a + h]``) or one [h] vector for all.
    Returns (y, mean, rstd); mean and rstd [N, rows] float32 are what the backward pass needs.  Automatic
    differentiation does not see the call: nothing that is returned requires a gradient, whatever x, weight and bias
    do; the gradients come from liec_layer_norm_backward."""
    device = _device_of("x", x)
    for name, t in (("weight", weight), ("bias", bias), ("y", y)):
        if t is not None and t.get_device() != device:
            raise ValueError(f"{name} must be on x's device")
    return _launch(device, stream, _ln_forward, device, x, weight, bias, eps, y)


def _ln_backward(raw, device, dy, x, mean, rstd, weight, dx, dweight, dbias, workspace):
    import torch
    if dx is None:
        dx = _empty_like(x)
    if dweight is None or dbias is None:
        like = weight if weight is not None else dweight if dweight is not None else dbias
        given = dweight if dweight is not None else dbias
        shape = given.shape if given is not None else like.shape if like is not None else x.shape[:-2] + x.shape[-1:]
        dtype = given.dtype if given is not None else torch.float32
        dweight = _empty(shape, dtype, device) if dweight is None else dweight
        dbias = _empty(shape, dtype, device) if dbias is None else dbias
    _, ref, need = _ln_desc(_layout(x), _layout(dy), _layout(dx), _layout(weight), None, _layout(dweight), _layout(dbias), 0.0)
    if workspace is None:
        workspace = _empty((need,), torch.uint8, device)
    lib = _LIB or load_library()
    st = lib.liec_layer_norm_backward(ref, dy.data_ptr(), x.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                      None if weight is None else weight.data_ptr(), dx.data_ptr(), dweight.data_ptr(),
                                      dbias.data_ptr(), workspace.data_ptr(), workspace.nbytes, raw)
    if st != 0:
        _ln_failed(lib, st)
    return dx, dweight, dbias


def liec_layer_norm_backward(dy, x, mean, rstd, weight=None, dx=None, dweight=None, dbias=None, workspace=None, stream=None):
    """Gradients of liec_layer_norm_forward.  dweight and dbias: [N, h] float32 or bfloat16 (any stride between
    workers, e.g. ``grads[:, a:a + h]``), or [h] for a vector that all workers share (its gradient is summed over
    the workers too, for any layout of x, dy and dx); allocated in float32, shaped like weight, where not given.  Returns (dx, dweight, dbias)."""
    import torch
    device = _device_of("x", x)
    for name, t in (("dy", dy), ("weight", weight), ("dx", dx), ("dweight", dweight), ("dbias", dbias), ("workspace", workspace)):
        if t is not None and t.get_device() != device:
            raise ValueError(f"{name} must be on x's device")
    rows = x.shape[:-1]
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or t.shape != rows or not t.is_contiguous() or t.get_device() != device:
            raise ValueError(f"{name} must be the contiguous float32 tensor that the forward pass returned")
    if workspace is not None and not workspace.is_contiguous():   # (its bytes are counted by its elements)
        raise ValueError("workspace must be contiguous")
    return _launch(device, stream, _ln_backward, device, dy, x, mean, rstd, weight, dx, dweight, dbias, workspace)


# ---- activations of N workers: 8-bit checkpoints, group normalisation, weight gradients -------------

def liec_activation_cols(cols: int) -> int:
    """Columns of a checkpoint's rows: cols rounded up to whole blocks of ACTIVATION_BLOCK."""
    return -(-int(cols) // ACTIVATION_BLOCK) * ACTIVATION_BLOCK


def _pointer(t):
    return None if t is None else t.data_ptr()


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.get_device() != device:
            raise ValueError(f"{name} must be on the device of the first argument")


def _below_2_31(*sizes):
    """Sizes of 32 bits in a descriptor: ctypes would cut them."""
    if max(sizes) >= 1 << 31:
        raise ValueError("workers, samples, channels and columns must be below 2^31")


def _dtype_code(name, dtype) -> int:
    import torch
    if dtype == torch.bfloat16:
        return BF16
    if dtype != torch.float32:
        raise ValueError(f"{name} must be float32 or bfloat16")
    return F32


@functools.lru_cache(maxsize=1024)
def _checkpoint_shapes(rows, cols):
    wide, rows = liec_activation_cols(cols), tuple(rows)
    return rows + (wide,), rows + (wide // ACTIVATION_BLOCK,)


def _check_checkpoint(q, scales, rows, cols):
    """q int8 [*rows, liec_activation_cols(cols)] and scales uint8 [*rows, the same / 32], both contiguous."""
    import torch
    wide, powers = _checkpoint_shapes(rows, cols)
    if q.shape != wide or q.dtype != torch.int8 or not q.is_contiguous():
        raise ValueError(f"q must be a contiguous int8 tensor {list(wide)}")
    if scales.shape != powers or scales.dtype != torch.uint8 or not scales.is_contiguous():
        raise ValueError(f"scales must be a contiguous uint8 tensor {list(powers)}")


def _new_checkpoint(rows, cols, q, scales, device):
    import torch
    wide, powers = _checkpoint_shapes(rows, cols)
    if q is None and scales is None:
        return _empty(wide, torch.int8, device), _empty(powers, torch.uint8, device)
    q = _empty(wide, torch.int8, device) if q is None else q
    scales = _empty(powers, torch.uint8, device) if scales is None else scales
    _check_checkpoint(q, scales, rows, cols)
    return q, scales


@functools.lru_cache(maxsize=1024)
def _rows_of(name, layout):
    """[..., cols] as (workers, rows, cols, row stride, worker stride): the axes in front of the columns, joined where
    they follow one another without a gap; two may remain."""
    shape, stride, _ = layout
    cols, axes = shape[-1], []
    if cols > 1 and stride[-1] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    for n, s in zip(shape[:-1], stride[:-1]):
        if n == 1:
            continue
        if axes and axes[-1][1] == n * s:
            axes[-1] = (axes[-1][0] * n, s)
        else:
            axes.append((n, s))
    if 0 in shape[:-1]:
        axes = [(0, cols)]
    if len(axes) > 2 or (len(axes) == 2 and axes[0][0] > 65535):
        raise ValueError(f"the axes of {name} in front of the last must join into at most two (the outer one of up to 65535 entries)")
    if any(s < 0 for _, s in axes):
        raise ValueError(f"{name} must not have negative strides")
    axes = [(1, 0)] * (2 - len(axes)) + axes
    _below_2_31(cols)
    return axes[0][0], axes[1][0], cols, axes[1][1], axes[0][1]


@functools.lru_cache(maxsize=1024)
def _activation_desc(name, layout):
    d = liec_activation_desc()
    d.workers, d.rows, d.cols, d.x_row_stride, d.x_worker_stride = _rows_of(name, layout)
    d.dtype = _dtype_code(name, layout[2])
    return d, C.byref(d)


def _activation_call(raw, device, compress, x, q, scales, shape, dtype):
    lib = _LIB or load_library()
    if compress:
        q, scales = _new_checkpoint(x.shape[:-1], x.shape[-1], q, scales, device)
    elif x is None:
        x = _empty(shape, dtype, device)
    ref = _activation_desc("x", _layout(x))[1]
    if compress:
        st = lib.liec_activation_compress(ref, x.data_ptr(), q.data_ptr(), scales.data_ptr(), raw)
    else:
        st = lib.liec_activation_restore(ref, q.data_ptr(), scales.data_ptr(), x.data_ptr(), raw)
    if st != 0:
        _ln_failed(lib, st)
    return (q, scales) if compress else x


def liec_activation_compress(x, q=None, scales=None, stream=None):
    """8-bit checkpoint of activations [..., h] (float32 or bfloat16, at least two axes): every 32 consecutive channels as
    signed bytes and one power of two, the last of a row filled up (so rows of a few channels only grow).  Returns (q, scales): int8 [..., liec_activation_cols(h)] and uint8 [..., the same / 32]."""
    device = _device_of("x", x)
    _same_device(device, q=q, scales=scales)
    if x.dim() < 2:
        raise ValueError("x must have at least two axes")
    return _launch(device, stream, _activation_call, device, True, x, q, scales, None, None)


def liec_activation_restore(q, scales, cols: int, dtype=None, x=None, stream=None):
    """What a checkpoint stands for, q 2^e, as [..., cols] of `dtype` (float32 where not given; exact in bfloat16 too), or into `x`."""
    import torch
    device = _device_of("q", q)
    _same_device(device, scales=scales, x=x)
    if q.dim() < 2:
        raise ValueError("q must have at least two axes")
    shape = tuple(q.shape[:-1]) + (int(cols),)
    _check_checkpoint(q, scales, shape[:-1], cols)
    if x is not None and (tuple(x.shape) != shape or (dtype is not None and x.dtype != dtype)):
        raise ValueError(f"x must be {list(shape)} of the given type")
    return _launch(device, stream, _activation_call, device, False, x, q, scales, shape, dtype or torch.float32)


def _gn_strides(name, t, x):
    """(pixel, sample, worker) strides of [N, samples, pixels, channels] or [samples, pixels, channels]."""
    shape, stride, dtype = t
    if shape != x[0] or dtype != x[2]:
        raise ValueError(f"{name} must have the shape and type of the activations")
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return stride[-2], stride[-3], (stride[0] if len(shape) == 4 else 0)


def _gn_vector(name, t, x, dtypes):
    if t is None:
        return 0
    shape, stride, dtype = t
    C_, N = x[0][-1], (x[0][0] if len(x[0]) == 4 else 1)
    if dtype not in dtypes:
        raise ValueError(f"{name} must be of type {' or '.join(str(d) for d in dtypes)}")
    if tuple(shape) not in ((C_,), (N, C_)) or (C_ > 1 and stride[-1] != 1):
        raise ValueError(f"{name} must be [channels] or [N, channels] with a contiguous last axis")
    return stride[0] if len(shape) == 2 else 0


@functools.lru_cache(maxsize=1024)
def _gn_desc(x, given, y, dx, weight, bias, dweight, dbias, groups, activation, eps):
    """Checks the layouts of a call and returns its descriptor and workspace size.  x: shape and type (and strides, where
    `given`) of the activations; dx None: forward."""
    import torch
    both, f32 = (torch.float32, torch.bfloat16), (torch.float32,)
    shape = x[0]
    if x[2] not in both or len(shape) not in (3, 4):
        raise ValueError("activations must be [N, samples, pixels, channels] or [samples, pixels, channels] of float32 or bfloat16")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    if groups < 1 or shape[-1] % groups:
        raise ValueError("groups must divide the channels")
    _below_2_31(shape[0], shape[-3], shape[-1])
    d = liec_group_norm_desc()
    d.workers, d.samples, d.pixels, d.channels = (shape[0] if len(shape) == 4 else 1), shape[-3], shape[-2], shape[-1]
    d.groups, d.dtype, d.activation, d.eps = groups, _dtype_code("x", x[2]), ACTIVATIONS[activation], eps
    if given:
        d.x_pixel_stride, d.x_sample_stride, d.x_worker_stride = _gn_strides("x", x, x)
    d.y_pixel_stride, d.y_sample_stride, d.y_worker_stride = _gn_strides("y" if dx is None else "dy", y, x)
    d.weight_stride, d.bias_stride = _gn_vector("weight", weight, x, f32), _gn_vector("bias", bias, x, f32)
    if dx is not None:
        d.dx_pixel_stride, d.dx_sample_stride, d.dx_worker_stride = _gn_strides("dx", dx, x)
        d.dweight_stride, d.dbias_stride = _gn_vector("dweight", dweight, x, both), _gn_vector("dbias", dbias, x, both)
        if dweight[2] != dbias[2] or len(dweight[0]) != len(dbias[0]):
            raise ValueError("dweight and dbias must have the same type and number of axes")
        d.grad_dtype = _dtype_code("dweight", dweight[2])
        if len(dweight[0]) == 1 and d.workers > 1:
            if d.weight_stride != 0 or d.bias_stride != 0:
                raise ValueError("workers with weights of their own need dweight and dbias [N, channels]")
            d.shared_grads = 1
    return d, C.byref(d), int(load_library().liec_group_norm_workspace_bytes(C.byref(d), 0 if dx is None else 1))


def liec_group_norm_workspace_bytes(desc: liec_group_norm_desc, backward: bool) -> int:
    return int(load_library().liec_group_norm_workspace_bytes(C.byref(desc), 1 if backward else 0))


def _gn_workspace(workspace, need, device):
    import torch
    if workspace is not None:
        if not workspace.is_contiguous():   # (its bytes are counted by its elements)
            raise ValueError("workspace must be contiguous")
        return workspace.data_ptr(), workspace.nbytes, workspace
    if need == 0:
        return None, 0, None
    workspace = _empty((need,), torch.uint8, device)
    return workspace.data_ptr(), need, workspace


def _gn_forward(raw, device, x, groups, weight, bias, eps, activation, compress, y, q, scales, workspace):
    import torch
    if y is None:
        y = _empty_like(x)
    _, ref, need = _gn_desc(_layout(x), True, _layout(y), None, _layout(weight), _layout(bias), None, None, groups, activation, eps)
    mean = _empty(x.shape[:-2] + (groups,), torch.float32, device)
    rstd = torch.empty_like(mean)
    if compress:
        q, scales = _new_checkpoint(x.shape[:-1], x.shape[-1], q, scales, device)
    ws, size, keep = _gn_workspace(workspace, need, device)
    lib = _LIB or load_library()
    st = lib.liec_group_norm_forward(ref, x.data_ptr(), _pointer(weight), _pointer(bias), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                     _pointer(q), _pointer(scales), ws, size, raw)
    if st != 0:
        _ln_failed(lib, st)
    return (y, mean, rstd, q, scales) if compress else (y, mean, rstd)


def liec_group_norm_forward(x, groups: int, weight=None, bias=None, eps: float = 1e-5, activation: str = "none", compress: bool = False,
                            y=None, q=None, scales=None, workspace=None, stream=None):
    """Group norm of [N, samples, pixels, channels] (or [samples, pixels, channels]) activations and an activation ("none",
    "relu", "silu"), with per-worker float32 weight and bias [N, channels] (any stride between workers, e.g.
    ``params[:, a:a + c]``) or one [channels] vector for all.  Returns (y, mean, rstd), mean and rstd [N, samples, groups]
    float32; with ``compress`` (or q and scales given) (y, mean, rstd, q, scales), the last two being x's 8-bit checkpoint.
    Automatic differentiation does not see the call; the gradients come from liec_group_norm_backward."""
    device = _device_of("x", x)
    _same_device(device, weight=weight, bias=bias, y=y, q=q, scales=scales, workspace=workspace)
    return _launch(device, stream, _gn_forward, device, x, int(groups), weight, bias, float(eps), activation,
                   bool(compress) or q is not None or scales is not None, y, q, scales, workspace)


def _gn_backward(raw, device, dy, x, q, scales, mean, rstd, weight, bias, activation, dx, dweight, dbias, workspace):
    import torch
    if dx is None:
        dx = _empty_like(dy)
    if dweight is None or dbias is None:
        # (a vector that all workers share beside one of their own: gradients per worker)
        like = next((t for t in (dweight, dbias) if t is not None), None)
        if like is None:
            like = max((t for t in (weight, bias) if t is not None), key=lambda t: t.dim(), default=None)
        shape = like.shape if like is not None else dy.shape[:-3] + dy.shape[-1:]
        dtype = next((t.dtype for t in (dweight, dbias) if t is not None), torch.float32)
        dweight = _empty(shape, dtype, device) if dweight is None else dweight
        dbias = _empty(shape, dtype, device) if dbias is None else dbias
    _, ref, need = _gn_desc(_layout(dy if x is None else x), x is not None, _layout(dy), _layout(dx), _layout(weight), _layout(bias),
                            _layout(dweight), _layout(dbias), mean.shape[-1], activation, 0.0)
    ws, size, keep = _gn_workspace(workspace, need, device)
    lib = _LIB or load_library()
    st = lib.liec_group_norm_backward(ref, dy.data_ptr(), _pointer(x), _pointer(q), _pointer(scales), mean.data_ptr(), rstd.data_ptr(),
                                      _pointer(weight), _pointer(bias), dx.data_ptr(), dweight.data_ptr(), dbias.data_ptr(), ws, size, raw)
    if st != 0:
        _ln_failed(lib, st)
    return dx, dweight, dbias


def liec_group_norm_backward(dy, x, mean, rstd, weight=None, bias=None, activation: str = "none", dx=None, dweight=None, dbias=None,
                             workspace=None, stream=None):
    """Gradients of liec_group_norm_forward.  x: the activations, or their checkpoint as a pair (q, scales).  dweight and
    dbias: [N, channels] float32 or bfloat16 (any stride between workers, e.g. ``grads[:, a:a + c]``), or [channels] for a
    vector that all workers share (its gradient is summed over the workers too); allocated in float32, shaped like weight and bias
    (per worker where one of them is), where not given.  Returns (dx, dweight, dbias)."""
    import torch
    device = _device_of("dy", dy)
    x, q, scales = (x, None, None) if torch.is_tensor(x) else (None, *x)
    _same_device(device, x=x, q=q, scales=scales, mean=mean, rstd=rstd, weight=weight, bias=bias, dx=dx, dweight=dweight, dbias=dbias, workspace=workspace)
    if dy.dim() not in (3, 4):
        raise ValueError("dy must be [N, samples, pixels, channels] or [samples, pixels, channels]")
    if x is None:
        _check_checkpoint(q, scales, dy.shape[:-1], dy.shape[-1])
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or t.dim() != dy.dim() - 1 or t.shape[:-1] != dy.shape[:-2] or t.shape != mean.shape or not t.is_contiguous():
            raise ValueError(f"{name} must be the contiguous float32 tensor that the forward pass returned")
    return _launch(device, stream, _gn_backward, device, dy, x, q, scales, mean, rstd, weight, bias, activation, dx, dweight, dbias, workspace)


@functools.lru_cache(maxsize=1024)
def _wg_desc(dy, dweight, cols, place):
    """place: dy's address within 16 bytes."""
    d = liec_weight_grad_desc()
    (shape, stride, dtype), (wshape, wstride, wdtype) = dy, dweight
    N = shape[0] if len(shape) == 3 else 1
    if (shape[-1] > 1 and stride[-1] != 1) or (cols > 1 and wstride[-1] != 1):
        raise ValueError("the last axes of dy and dweight must be contiguous")
    if tuple(wshape) != tuple(shape[:-2]) + (shape[-1], cols):
        raise ValueError("dweight must be [N, out, in] ([out, in] for one worker)")
    _below_2_31(N, shape[-1], cols)
    d.workers, d.rows, d.in_, d.out = N, shape[-2], cols, shape[-1]
    d.dtype, d.grad_dtype = _dtype_code("dy", dtype), _dtype_code("dweight", wdtype)
    d.dy_row_stride, d.dy_worker_stride = stride[-2], (stride[0] if len(shape) == 3 else 0)
    d.dweight_row_stride, d.dweight_worker_stride = wstride[-2], (wstride[0] if len(shape) == 3 else 0)
    return d, C.byref(d), int(load_library().liec_weight_grad_workspace_bytes(C.byref(d), 256 + place))


def liec_weight_grad_workspace_bytes(desc: liec_weight_grad_desc, dy) -> int:
    return int(load_library().liec_weight_grad_workspace_bytes(C.byref(desc), dy.data_ptr()))


def _weight_grad(raw, device, dy, q, scales, cols, dweight, workspace):
    import torch
    if dweight is None:
        dweight = _empty(tuple(dy.shape[:-2]) + (dy.shape[-1], cols), torch.float32, device)
    _, ref, need = _wg_desc(_layout(dy), _layout(dweight), cols, dy.data_ptr() % 16)
    ws, size, keep = _gn_workspace(workspace, need, device)
    lib = _LIB or load_library()
    st = lib.liec_weight_grad(ref, dy.data_ptr(), q.data_ptr(), scales.data_ptr(), dweight.data_ptr(), ws, size, raw)
    if st != 0:
        _ln_failed(lib, st)
    return dweight


def liec_weight_grad(dy, q, scales, cols: int, dweight=None, workspace=None, stream=None):
    """Weight gradient of linear layers from the 8-bit checkpoint (q, scales) of their input [N, rows, cols]: the sum over
    rows of dy[n, row, out] times the input.  dy: [N, rows, out] (or [rows, out]) float32 or bfloat16.  dweight: [N, out, cols]
    float32 or bfloat16 with any strides between workers and outputs, e.g. ``grads[:, a:a + out * cols].unflatten(1, (out, cols))``;
    allocated in float32 where not given.  Returns dweight."""
    device = _device_of("dy", dy)
    _same_device(device, q=q, scales=scales, dweight=dweight, workspace=workspace)
    if dy.dim() not in (2, 3):
        raise ValueError("dy must be [N, rows, out] or [rows, out]")
    _check_checkpoint(q, scales, dy.shape[:-1], cols)
    return _launch(device, stream, _weight_grad, device, dy, q, scales, int(cols), dweight, workspace)


class Context:
    """Owns a ``liec_ctx`` plus the torch tensors it points into (params, error, workspace)."""

    def __init__(self, params, error, seg_offsets, uplink, downlink, topk_k=None, grad_dtype=F32):
        import torch
        self._torch = torch
        self.lib = load_library()
        if not (params.is_cuda and error.is_cuda):
            raise ValueError("params and error must be CUDA tensors (there is no CPU path)")
        assert params.dtype == torch.float32 and error.dtype == torch.float32
        assert params.is_contiguous() and error.is_contiguous() and params.dim() == 2
        self.params, self.error = params, error
        self.N, self.d = params.shape
        self.cfg, self._keep = make_config(self.N, seg_offsets, uplink, downlink, topk_k, grad_dtype)
        if self.cfg.dim != self.d or error.numel() != self.d:
            raise ValueError("seg_offsets[-1], params.shape[1] and error.numel() must agree")
        nbytes = workspace_bytes(self.cfg)
        if nbytes == 0:
            # let liec_init produce the precise message
            nbytes = 256
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=params.device)
        self._ctx = C.c_void_p()
        with torch.cuda.device(params.device):
            st = self.lib.liec_init(C.byref(self.cfg), params.data_ptr(), error.data_ptr(),
                                    self.workspace.data_ptr(), nbytes, C.byref(self._ctx))
        if st != 0:
            raise LiecError(st, self.lib.liec_last_error(None).decode())
        self.grad_dtype = grad_dtype
        self.T = self.cfg.num_segments
        self._sizes = np.diff(self._keep[0]).tolist()
        self._device = params.get_device()

    # -- helpers ---------------------------------------------------------------------------
    def _stream(self, stream=None) -> int:
        s = stream if stream is not None else self._torch.cuda.current_stream(self.params.device)
        return s.cuda_stream

    def _check(self, st: int):
        if st != 0:
            raise LiecError(st, self.lib.liec_last_error(self._ctx).decode())

    def _check_grads(self, grads):
        t = self._torch
        want = t.bfloat16 if self.grad_dtype == BF16 else t.float32
        if not grads.is_cuda or grads.dtype != want or grads.shape != (self.N, self.d) or not grads.is_contiguous():
            raise ValueError("grads must be a contiguous CUDA tensor [N, d] of the configured dtype")

    # -- the C ABI, one method per entry point -----------------------------------------------
    def liec_uplink_compress(self, grads, stream=None):
        self._check_grads(grads)
        self._check(self.lib.liec_uplink_compress(self._ctx, grads.data_ptr(), self._stream(stream)))

    def liec_server_aggregate(self, stream=None):
        self._check(self.lib.liec_server_aggregate(self._ctx, self._stream(stream)))

    def liec_downlink_compress(self, stream=None):
        self._check(self.lib.liec_downlink_compress(self._ctx, self._stream(stream)))

    def liec_worker_update(self, grads, lr: float, stream=None):
        self._check_grads(grads)
        self._check(self.lib.liec_worker_update(self._ctx, grads.data_ptr(), float(lr), self._stream(stream)))

    def liec_set_subsets(self, up_sets=None, down_set=None):
        """Random-k: int32/uint32 CUDA tensors [N, K] / [K] of kept flat indices (ascending inside each
        segment).  The tensors are referenced, not copied; this object keeps them alive."""
        t = self._torch
        for name, s, shape in (("up_sets", up_sets, (self.N, -1)), ("down_set", down_set, (-1,))):
            if s is None:
                continue
            if not s.is_cuda or s.dtype not in (t.int32, t.uint32) or not s.is_contiguous() or s.dim() != len(shape):
                raise ValueError(f"{name} must be a contiguous CUDA tensor of 32-bit indices")
        self._subsets = (up_sets, down_set)
        self._check(self.lib.liec_set_subsets(self._ctx, None if up_sets is None else up_sets.data_ptr(),
                                              None if down_set is None else down_set.data_ptr()))

    def liec_draw_subsets(self, seed: int, epoch: int, stream=None):
        """Random-k: draws and installs the subsets of all workers and the server from (seed, epoch)."""
        self._subsets = None
        self._check(self.lib.liec_draw_subsets(self._ctx, int(seed), int(epoch), self._stream(stream)))

    def liec_step(self, grads, lr: float, stream=None):
        self._check_grads(grads)
        self._check(self.lib.liec_step(self._ctx, grads.data_ptr(), float(lr), self._stream(stream)))

    def liec_topk_route_counts(self, uplink: bool, stream=None, per_problem: bool = False) -> dict:
        """Counts of the routes taken by the last iteration's selections; with per_problem also a uint8
        array [rows, T] of flags (1 single pass, 2 second-digit pass, 4 dense one-CTA path, 8 single tile)."""
        out = (C.c_int64 * 5)()
        flags = np.zeros(((self.N if uplink else 1), self.T), np.uint8) if per_problem else None
        self._check(self.lib.liec_topk_route_counts(self._ctx, self._stream(stream), 1 if uplink else 0, out,
                                                    None if flags is None else flags.ctypes.data_as(C.c_void_p)))
        r = {"problems": int(out[0]), "single_pass": int(out[1]), "refined": int(out[2]), "slow": int(out[3]),
             "direct": int(out[4])}
        if flags is not None:
            r["flags"] = flags
        return r

    def liec_abort_step(self):
        self._check(self.lib.liec_abort_step(self._ctx))

    def liec_set_copy_wait(self, poll_limit: int = 0, expect_extra_bytes: int = 0):
        self._check(self.lib.liec_set_copy_wait(self._ctx, int(poll_limit), int(expect_extra_bytes)))

    def liec_set_norm_wait(self, poll_limit: int = 0, withhold: int = 0):
        self._check(self.lib.liec_set_norm_wait(self._ctx, int(poll_limit), int(withhold)))

    def liec_average_step(self, grads, lr: float, stream=None):
        self._check_grads(grads)
        self._check(self.lib.liec_average_step(self._ctx, grads.data_ptr(), float(lr), self._stream(stream)))

    def liec_mean_params(self, out, stream=None):
        assert out.is_cuda and out.dtype == self._torch.float32 and out.numel() == self.d and out.is_contiguous()
        self._check(self.lib.liec_mean_params(self._ctx, out.data_ptr(), self._stream(stream)))

    def liec_sumsq(self, which: int, out, grads=None, stream=None):
        """Per-segment squared norms (SUMSQ_ERROR / SUMSQ_GRADS / SUMSQ_PARAMS) into `out` [rows, T] float64."""
        rows = 1 if which == SUMSQ_ERROR else self.N
        assert out.is_cuda and out.dtype == self._torch.float64 and out.numel() == rows * self.T and out.is_contiguous()
        gptr = None
        if which == SUMSQ_GRADS:
            self._check_grads(grads)
            gptr = grads.data_ptr()
        self._check(self.lib.liec_sumsq(self._ctx, int(which), gptr, out.data_ptr(), self._stream(stream)))

    def _norms(self, norms):
        t = self._torch
        if norms is None:
            return t.empty(self.N, dtype=t.float32, device=self._device)
        if not norms.is_cuda or norms.dtype != t.float32 or norms.shape != (self.N,) or not norms.is_contiguous():
            raise ValueError("norms must be a contiguous float32 CUDA tensor [N]")
        return norms

    def _clip(self, raw, fn, args, max_norm, norms, zero_nonfinite):
        norms = self._norms(norms)
        self._check(fn(self._ctx, *args, max_norm, 1 if zero_nonfinite else 0, norms.data_ptr(), raw))
        return norms

    def liec_clip_grads(self, grads, max_norm: float, out=None, norms=None, zero_nonfinite: bool = False, stream=None):
        """Scales every worker's gradient row to at most max_norm, into `out` (default: in place).
        Returns the norms before clipping, [N] float32."""
        self._check_grads(grads)
        if out is None:
            out = grads
        else:
            self._check_grads(out)
        return _launch(self._device, stream, self._clip, self.lib.liec_clip_grads, (grads.data_ptr(), out.data_ptr()), max_norm, norms,
                       zero_nonfinite)

    def liec_set_tensors(self, tensors, stream=None):
        """The N*T gradient tensors of liec_gather_grads: N sequences of T contiguous CUDA tensors (None: no
        gradient) with the segments' element counts, all float32 or all bfloat16.  They are referenced, not
        copied; this object keeps them alive until the next call (a gather on another stream than the tensors'
        own has to be over by then, and a graph that captured this call needs them for as long as it is replayed).
        Every tensor is checked here, about 0.4 us of host time each: a program whose gradients stay in the
        same buffers calls this once, one whose backward pass leaves new tensors before every gather."""
        t = self._torch
        if len(tensors) != self.N or any(len(ts) != self.T for ts in tensors):
            raise ValueError("tensors must be N sequences of T tensors")
        sizes, device = self._sizes, self.params.device
        dtype, ptrs = None, np.zeros(self.N * self.T, np.uint64)
        q = 0
        for ts in tensors:
            for n, g in zip(sizes, ts):
                if g is not None:
                    dtype = g.dtype if dtype is None else dtype
                    if g.dtype != dtype or g.numel() != n or g.device != device or not g.is_contiguous():
                        raise ValueError("every tensor must be contiguous, on the context's device, of its segment's size and of one type")
                    ptrs[q] = g.data_ptr()
                q += 1
        if dtype not in (None, t.float32, t.bfloat16):
            raise ValueError("tensors must be float32 or bfloat16")
        self._check(self.lib.liec_set_tensors(self._ctx, ptrs.ctypes.data, BF16 if dtype == t.bfloat16 else F32, self._stream(stream)))
        self._tensors = [list(ts) for ts in tensors]

    def liec_gather_grads(self, out, max_norm: float = float("inf"), norms=None, zero_nonfinite: bool = False, stream=None):
        """Gradient rows from the tensors of liec_set_tensors, every worker's gradient scaled to at most
        max_norm.  Returns the norms before clipping, [N] float32."""
        self._check_grads(out)
        return _launch(self._device, stream, self._clip, self.lib.liec_gather_grads, (out.data_ptr(),), max_norm, norms, zero_nonfinite)

    def liec_set_telemetry(self, on: bool):
        self._check(self.lib.liec_set_telemetry(self._ctx, 1 if on else 0))

    def liec_get_telemetry(self, stream=None, kept: bool = True) -> dict:
        """Per-segment squared norms of the last iteration (float64 CUDA tensors, allocated here):
        e_sumsq [T], v_sumsq [T], g_sumsq [N, T] and, for sides with (index, value) messages and
        kept=True, up_kept_sumsq [N, T] / down_kept_sumsq [T]."""
        t = self._torch
        dev, f64 = self.params.device, t.float64
        sparse = (COMP_TOPK, COMP_RANDK)
        out = {"e_sumsq": t.empty(self.T, dtype=f64, device=dev), "v_sumsq": t.empty(self.T, dtype=f64, device=dev),
               "g_sumsq": t.empty(self.N, self.T, dtype=f64, device=dev),
               "up_kept_sumsq": t.empty(self.N, self.T, dtype=f64, device=dev) if kept and self.cfg.uplink in sparse else None,
               "down_kept_sumsq": t.empty(self.T, dtype=f64, device=dev) if kept and self.cfg.downlink in sparse else None}
        ptr = lambda name: None if out[name] is None else out[name].data_ptr()
        self._check(self.lib.liec_get_telemetry(self._ctx, ptr("e_sumsq"), ptr("v_sumsq"), ptr("g_sumsq"),
                                                ptr("up_kept_sumsq"), ptr("down_kept_sumsq"), self._stream(stream)))
        return out

    def liec_step_host(self, grads_host, grads_dev, lr: float, down_msg_host=None, stream=None):
        self._check_grads(grads_dev)
        assert not grads_host.is_cuda and grads_host.shape == grads_dev.shape and grads_host.dtype == grads_dev.dtype
        out_ptr = down_msg_host.data_ptr() if down_msg_host is not None else None
        self._check(self.lib.liec_step_host(self._ctx, grads_host.data_ptr(), grads_dev.data_ptr(), float(lr),
                                            out_ptr, self._stream(stream)))

    def liec_device_status(self, stream=None) -> int:
        out = C.c_int32(0)
        st = self.lib.liec_device_status(self._ctx, self._stream(stream), C.byref(out))
        if st not in (0, 6):
            self._check(st)
        return int(out.value)

    def liec_clear_status(self, stream=None):
        self._check(self.lib.liec_clear_status(self._ctx, self._stream(stream)))

    def liec_launch_count(self) -> int:
        return int(self.lib.liec_launch_count(self._ctx))

    def liec_get_messages(self) -> dict:
        """Device views (torch tensors aliasing the workspace) of the current messages."""
        t = self._torch
        m = liec_messages()
        self._check(self.lib.liec_get_messages(self._ctx, C.byref(m)))
        base = self.workspace.data_ptr()
        W, K, N, T = int(m.num_words), int(m.num_topk), self.N, self.T

        def view(ptr, count, dtype):
            if not ptr or count == 0:
                return None
            esz = 4
            off = ptr - base
            return self.workspace[off:off + count * esz].view(dtype)

        return {
            "up_words": _reshape(view(m.up_words, N * W, t.int32), (N, W)),
            "up_scales": _reshape(view(m.up_scales, N * T, t.float32), (N, T)),
            "up_idx": _reshape(view(m.up_idx, N * K, t.int32), (N, K)),
            "up_val": _reshape(view(m.up_val, N * K, t.float32), (N, K)),
            "down_words": view(m.down_words, W, t.int32),
            "down_scales": view(m.down_scales, T, t.float32),
            "down_idx": view(m.down_idx, K, t.int32),
            "down_val": view(m.down_val, K, t.float32),
            "v": self.error,
            "num_words": W, "num_topk": K,
        }

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self.lib.liec_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _reshape(t, shape):
    return None if t is None else t.view(*shape)
