"""Thin ctypes binding over libslidedp (same names as the C ABI in ``include/slidedp.h``).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
Tensors are torch tensors used purely as device / pinned-host memory; their
``data_ptr()`` and the raw ``cudaStream_t`` are what crosses the boundary. There is no CPU
fallback: if the shared library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import importlib
import os
import struct
from dataclasses import dataclass

import torch

from .build import marshal_name

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libslidedp.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2609_34162_b200.build` "
        "(nvcc, sm_100a). libslidedp has no CPU fallback.")

# The operators of the fine-tuning pass need the binding's C++ module; the paper's path does without it.
try:
    _marshal, _marshal_error = importlib.import_module("." + marshal_name(), __package__), None
except ImportError as e:
    _marshal, _marshal_error = None, e

_lib = ctypes.CDLL(LIB_PATH)

MAX_RANKS = 16
NORM_TILE = 16384
OK, ERR_INVALID_ARG, ERR_MISALIGNED, ERR_BUDGET, ERR_NOT_PINNED, ERR_CUDA, ERR_TIMEOUT, ERR_NO_NORM = (
    0, -1, -2, -3, -4, -5, -6, -7)
ERR_TOO_LARGE = -8
NOALLOC_MAX_ELEMS = 1 << 30
IPC_HANDLE_BYTES = 80


class _HParams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("inv_R", ctypes.c_double), ("max_norm", ctypes.c_double),
                ("step", ctypes.c_int64)]


class _Stats(ctypes.Structure):
    _fields_ = [("norm", ctypes.c_double), ("clip_coef", ctypes.c_double),
                ("ms_total", ctypes.c_double), ("ms_norm", ctypes.c_double),
                ("ms_h2d", ctypes.c_double), ("ms_kernel", ctypes.c_double),
                ("ms_d2h", ctypes.c_double), ("gbs_h2d", ctypes.c_double),
                ("gbs_d2h", ctypes.c_double), ("chunks", ctypes.c_int64),
                ("nonfinite", ctypes.c_int32), ("reserved", ctypes.c_int32)]


@dataclass
class HParams:
    lr: float = 1e-5
    beta1: float = 0.9
    beta2: float = 0.95
    eps: float = 1e-8
    weight_decay: float = 0.1
    inv_R: float = 1.0
    max_norm: float = 0.0
    step: int = 1

    def _c(self) -> _HParams:
        return _HParams(self.lr, self.beta1, self.beta2, self.eps, self.weight_decay,
                        self.inv_R, self.max_norm, int(self.step))


_vp, _pp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)
_lib.slidedp_create.restype = ctypes.c_int
_lib.slidedp_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_int, ctypes.c_size_t]
_lib.slidedp_destroy.restype = ctypes.c_int
_lib.slidedp_destroy.argtypes = [_vp]
_lib.slidedp_strerror.restype = ctypes.c_char_p
_lib.slidedp_strerror.argtypes = [ctypes.c_int]
_lib.slidedp_last_cuda_error.restype = ctypes.c_int
_lib.slidedp_last_cuda_error.argtypes = [_vp]
_lib.slidedp_state_bytes.restype = ctypes.c_size_t
_lib.slidedp_state_bytes.argtypes = [ctypes.c_int64]
_lib.slidedp_grad_norm.restype = ctypes.c_int
_lib.slidedp_grad_norm.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, ctypes.c_double,
                                   ctypes.c_int, _vp]
_lib.slidedp_grad_norm_finish.restype = ctypes.c_int
_lib.slidedp_grad_norm_finish.argtypes = [_vp, ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(ctypes.c_double), _vp]
_lib.slidedp_grad_norm_tiles.restype = ctypes.c_int
_lib.slidedp_grad_norm_tiles.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, ctypes.c_double, _vp, _vp]
_lib.slidedp_grad_norm_finish_from.restype = ctypes.c_int
_lib.slidedp_grad_norm_finish_from.argtypes = [_vp, _vp, ctypes.c_int64, ctypes.c_double,
                                               ctypes.POINTER(ctypes.c_double),
                                               ctypes.POINTER(ctypes.c_double), _vp]
_lib.slidedp_reduce_adamw_chunk.restype = ctypes.c_int
_lib.slidedp_reduce_adamw_chunk.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp,
                                            _vp, ctypes.POINTER(_HParams), _vp]
_lib.slidedp_stream_step.restype = ctypes.c_int
_lib.slidedp_stream_step.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                     ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                     ctypes.POINTER(_HParams), ctypes.POINTER(_Stats)]
_lib.slidedp_reduce_mean_bf16.restype = ctypes.c_int
_lib.slidedp_reduce_mean_bf16.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, ctypes.c_double, _vp, _vp]
_lib.slidedp_stream_step_async.restype = ctypes.c_int
_lib.slidedp_stream_step_async.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                           ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                           ctypes.POINTER(_HParams)]
class _Layer(ctypes.Structure):
    _fields_ = [("grads_bf16", _pp), ("n", ctypes.c_int64), ("host_master", _vp), ("host_m", _vp),
                ("host_v", _vp), ("param_bf16_out", _vp)]


_lib.slidedp_stream_layers.restype = ctypes.c_int
_lib.slidedp_stream_layers.argtypes = [_vp, ctypes.POINTER(_Layer), ctypes.c_int, ctypes.c_int,
                                       ctypes.c_int64, ctypes.c_int, ctypes.POINTER(_HParams),
                                       ctypes.POINTER(_Stats)]
_lib.slidedp_stream_wait.restype = ctypes.c_int
_lib.slidedp_stream_wait.argtypes = [_vp]
_lib.slidedp_deliver_params.restype = ctypes.c_int
_lib.slidedp_deliver_params.argtypes = [_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int64, ctypes.c_int,
                                        ctypes.POINTER(_Stats)]
_lib.slidedp_link_probe.restype = ctypes.c_int
_lib.slidedp_link_probe.argtypes = [_vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, ctypes.c_size_t,
                                    ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
_lib.slidedp_grad_norm_noalloc.restype = ctypes.c_int
_lib.slidedp_grad_norm_noalloc.argtypes = [_pp, ctypes.c_int, ctypes.c_int64, ctypes.c_double,
                                           ctypes.c_double, _vp, _vp]
_lib.slidedp_kernel_launches.restype = ctypes.c_int64
_lib.slidedp_kernel_launches.argtypes = [_vp]
_lib.slidedp_ipc_export.restype = ctypes.c_int
_lib.slidedp_ipc_export.argtypes = [_vp, _vp, ctypes.c_char_p]
_lib.slidedp_ipc_open.restype = ctypes.c_int
_lib.slidedp_ipc_open.argtypes = [_vp, ctypes.c_char_p, ctypes.POINTER(_vp)]
_lib.slidedp_ipc_close.restype = ctypes.c_int
_lib.slidedp_ipc_close.argtypes = [_vp, _vp]
_lib.slidedp_scatter_tile_sums.restype = ctypes.c_int
_lib.slidedp_scatter_tile_sums.argtypes = [_vp, _vp, ctypes.c_int64, _pp, ctypes.c_int, _vp]
_lib.slidedp_reduce_adamw_chunk_bcast.restype = ctypes.c_int
_lib.slidedp_reduce_adamw_chunk_bcast.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp,
                                                  _pp, ctypes.c_int, ctypes.POINTER(_HParams), _vp]
_lib.slidedp_hbm_mix_probe.restype = ctypes.c_int
_lib.slidedp_hbm_mix_probe.argtypes = [_vp, _pp, ctypes.c_int, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                       ctypes.c_int, ctypes.POINTER(ctypes.c_double), _vp]
_lib.slidedp_set_wait_seconds.restype = ctypes.c_int
_lib.slidedp_set_wait_seconds.argtypes = [_vp, ctypes.c_double]
_lib.slidedp_test_fail_nth_call.restype = ctypes.c_int
_lib.slidedp_test_fail_nth_call.argtypes = [_vp, ctypes.c_int64]
_lib.slidedp_test_wait_polls.restype = ctypes.c_int
_lib.slidedp_test_wait_polls.argtypes = [_vp, ctypes.c_int64]


class _Rates(ctypes.Structure):
    _fields_ = [("h2d_gbs", ctypes.c_double), ("d2h_gbs", ctypes.c_double),
                ("update_gparams_s", ctypes.c_double), ("norm_gbs", ctypes.c_double),
                ("per_copy_us", ctypes.c_double)]


_lib.slidedp_model_stream_step.restype = ctypes.c_int
_lib.slidedp_model_stream_step.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int64, ctypes.c_int,
                                           ctypes.POINTER(_Rates), ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_double)]


class _QkArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("heads_q", ctypes.c_int32), ("heads_k", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rope_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("table_rows", ctypes.c_int64), ("eps", ctypes.c_double)]


class _AttnArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32), ("docs", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("cu_docs", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("slopes", ctypes.c_void_p), ("scale", ctypes.c_double), ("softcap", ctypes.c_double)]


class _DistillArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("entries", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("logits_stride", ctypes.c_int64), ("d_logits_stride", ctypes.c_int64),
                ("temperature", ctypes.c_double), ("w_teacher", ctypes.c_double), ("w_label", ctypes.c_double)]


class _EmbeddingArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("vocab", ctypes.c_int64), ("hidden", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("accumulate", ctypes.c_int32), ("reserved", ctypes.c_int32), ("scale", ctypes.c_double)]


class _BlockNormArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("hidden", ctypes.c_int64), ("dtype", ctypes.c_int32), ("has_y", ctypes.c_int32),
                ("post_norm", ctypes.c_int32), ("pre_norm", ctypes.c_int32), ("gate_kind", ctypes.c_int32), ("gate_sigmoid", ctypes.c_int32),
                ("residual_scale", ctypes.c_double), ("eps", ctypes.c_double)]


class _PolicyArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("logits_stride", ctypes.c_int64), ("d_logits_stride", ctypes.c_int64), ("temperature", ctypes.c_double),
                ("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double), ("kl_weight", ctypes.c_double)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


# A call's views (slidedp_heads: an address and two strides, _V bytes each) are written to the calling thread's argument block
# and passed as addresses there; the scalar arguments go as the bytes of their struct (a ctypes object costs three times that).
# slidedp_rows (an address and a stride) take _R bytes.
_V, _R = 24, 16
_qk_bytes, _attn_bytes, _distill_bytes = (struct.Struct(f).pack for f in ("@qiiiiiiqd", "@qiiiiiiPPPdd", "@qqiiqqddd"))
_embedding_bytes, _block_norm_bytes, _policy_bytes = (struct.Struct(f).pack for f in ("@qqqiiiid", "@qqiiiiiidd", "@qqiiqqdddd"))
for _args, _pack in ((_QkArgs, _qk_bytes), (_AttnArgs, _attn_bytes), (_DistillArgs, _distill_bytes), (_EmbeddingArgs, _embedding_bytes),
                     (_BlockNormArgs, _block_norm_bytes), (_PolicyArgs, _policy_bytes)):
    assert len(_pack(*[0] * len(_args._fields_))) == ctypes.sizeof(_args)
for _name, _res, _args in (
        ("slidedp_qk_norm_rope", ctypes.c_int, [_vp, _vp] + [_vp] * 9),
        ("slidedp_qk_norm_rope_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 14),
        ("slidedp_qk_norm_rope_workspace", ctypes.c_size_t, [_vp]),
        ("slidedp_attention", ctypes.c_int, [_vp, _vp] + [_vp] * 6),
        ("slidedp_attention_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 11),
        ("slidedp_attention_workspace", ctypes.c_size_t, [_vp]),
        ("slidedp_distill_loss", ctypes.c_int, [_vp, _vp] + [_vp] * 7),
        ("slidedp_distill_loss_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 8),
        ("slidedp_distill_step", ctypes.c_int, [_vp, _vp] + [_vp] * 9),
        ("slidedp_embedding", ctypes.c_int, [_vp, _vp] + [_vp] * 4),
        ("slidedp_embedding_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 5),
        ("slidedp_embedding_workspace", ctypes.c_size_t, [_vp]),
        ("slidedp_block_norm", ctypes.c_int, [_vp, _vp] + [_vp] * 8),
        ("slidedp_block_norm_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 14),
        ("slidedp_block_norm_workspace", ctypes.c_size_t, [_vp]),
        ("slidedp_policy_loss", ctypes.c_int, [_vp, _vp] + [_vp] * 8),
        ("slidedp_policy_loss_backward", ctypes.c_int, [_vp, _vp] + [_vp] * 9),
        ("slidedp_policy_step", ctypes.c_int, [_vp, _vp] + [_vp] * 10),
        ("slidedp_clip_grad_norm", ctypes.c_int, [_vp, _vp, _vp, ctypes.c_int32, ctypes.c_double, ctypes.c_double] + [_vp] * 3),
        ("slidedp_clip_grad_norm_workspace", ctypes.c_size_t, [_vp, ctypes.c_int32])):
    getattr(_lib, _name).restype, getattr(_lib, _name).argtypes = _res, _args


class SlideDPError(RuntimeError):
    def __init__(self, status: int, cuda_error: int = 0):
        self.status, self.cuda_error = status, cuda_error
        msg = _lib.slidedp_strerror(status).decode()
        if status == ERR_CUDA:
            msg += f" (cudaError_t {cuda_error})"
        super().__init__(f"libslidedp: {msg} [{status}]")


def slidedp_strerror(status: int) -> str:
    return _lib.slidedp_strerror(status).decode()


def slidedp_state_bytes(n: int) -> int:
    return int(_lib.slidedp_state_bytes(n))


def _ptr(x) -> int:
    """Raw address of a tensor's first element (or an int passed through, or None)."""
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _grad_array(grads):
    return (ctypes.c_void_p * len(grads))(*[_ptr(g) for g in grads])


def _stream(stream, device: int = -1) -> int:
    """The handle of a stream; None: torch's current one, on `device` (-1: the current device)."""
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if _marshal is None else _marshal.current_stream(device)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_DTYPES = {torch.bfloat16: 0, torch.float32: 1}      # slidedp_dtype


def _refuse(x, what: str, dtype, shape):
    if not isinstance(x, torch.Tensor) or x.dtype != dtype or not x.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor of {dtype}")
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(x.shape)}")
    if x.get_device() != _marshal.device():
        raise ValueError(f"{what} must be on the context's device cuda:{_marshal.device()}, not {x.device}")
    raise ValueError(f"{what} must be contiguous")


# The library sees addresses only; these look at what it cannot: type, shape, device and layout. _marshal has their fast
# paths and calls them for tensors that need a second look.

def _as_tensor(x):
    return x.as_subclass(torch.Tensor) if isinstance(x, torch.Tensor) else x


def _careful_flat(x, what: str, dtype, shape=None) -> int:
    """Address of a contiguous tensor."""
    x = _as_tensor(x)
    if (not isinstance(x, torch.Tensor) or x.dtype is not dtype or not x.is_cuda or not x.is_contiguous()
            or x.get_device() != _marshal.device() or (shape is not None and x.shape != shape)):
        _refuse(x, what, dtype, shape)
    return x.data_ptr()


def _careful_heads(x, what: str, dtype, shape):
    """Address and strides of a [tokens, heads, head_dim] tensor whose last axis is contiguous."""
    x = _as_tensor(x)
    if (not isinstance(x, torch.Tensor) or x.dtype is not dtype or not x.is_cuda or x.shape != shape
            or x.get_device() != _marshal.device()):
        _refuse(x, what, dtype, shape)
    t, h, d = x.stride()
    if d != 1 and shape[2] > 1:
        raise ValueError(f"the last axis of {what} must be contiguous")
    return x.data_ptr(), t, h


def _matrix(x, what: str, dtype, shape) -> int:
    """Row stride of a [rows, columns] tensor whose last axis is contiguous."""
    if (not isinstance(x, torch.Tensor) or x.dtype is not dtype or not x.is_cuda or x.shape != shape
            or x.get_device() != _marshal.device()):
        _refuse(x, what, dtype, shape)
    t, c = x.stride()
    if c != 1 and shape[1] > 1:
        raise ValueError(f"the last axis of {what} must be contiguous")
    return t if shape[0] > 1 else shape[1]


def _careful_rows(x, what: str, dtype, shape):
    """Address and row stride of a [rows, columns] tensor whose last axis is contiguous."""
    x = _as_tensor(x)
    return (0 if not isinstance(x, torch.Tensor) else x.data_ptr()), _matrix(x, what, dtype, shape)


def _careful_tensor(x, what: str):
    """Address, size and type of one of many tensors."""
    x = _as_tensor(x)
    dtype = x.dtype if isinstance(x, torch.Tensor) else None
    if dtype not in _DTYPES:
        raise TypeError(f"{what} must be CUDA tensors of bfloat16 or float32")
    return _careful_flat(x, what, dtype), x.numel(), _DTYPES[dtype]


def _no_marshal(*_):
    raise ImportError("the operators need the binding's C++ module, built for this torch: `python -m paper_2609_34162_b200.build`") from _marshal_error


if _marshal is None:
    _flat = _heads = _rows = _tensors = _block = _no_marshal
else:
    _marshal.setup(_careful_flat, _careful_heads, _careful_rows, _careful_tensor)
    _flat, _heads, _rows, _tensors, _block = _marshal.flat, _marshal.heads, _marshal.rows, _marshal.tensors, _marshal.block


def _workspace(x, nbytes: int) -> int:
    if (x is None or not x.is_cuda or not x.is_contiguous() or x.numel() * x.element_size() < nbytes
            or x.get_device() != _marshal.device()):
        raise ValueError(f"workspace must be a contiguous tensor of at least {nbytes} bytes on cuda:{_marshal.device()}")
    return x.data_ptr()


def _two_sides(q, k):
    """Shapes of q and k, which must agree in tokens and head_dim."""
    qs, ks = q.shape, k.shape
    if len(qs) != 3 or len(ks) != 3 or qs[0] != ks[0] or qs[2] != ks[2]:
        raise ValueError("q and k must be [tokens, heads, head_dim] with the same tokens and head_dim")
    return qs, ks


class Context:
    """Owns a ``slidedp_ctx``. Methods carry the C entry points' names and argument order."""

    def __init__(self, device: int = 0, gpu_budget_bytes: int = 0):
        self._h = _vp()
        rc = _lib.slidedp_create(ctypes.byref(self._h), device, gpu_budget_bytes)
        if rc != OK:
            self._h = _vp()
            raise SlideDPError(rc)
        self.device = device

    def _check(self, rc: int):
        if rc != OK:
            raise SlideDPError(rc, _lib.slidedp_last_cuda_error(self._h))

    def slidedp_destroy(self):
        if self._h:
            rc = _lib.slidedp_destroy(self._h)
            self._h = _vp()
            if rc != OK:
                raise SlideDPError(rc)

    close = slidedp_destroy

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.slidedp_destroy()

    def __del__(self):
        try:
            if self._h:
                _lib.slidedp_destroy(self._h)
                self._h = _vp()
        except Exception:
            pass

    def slidedp_kernel_launches(self) -> int:
        return int(_lib.slidedp_kernel_launches(self._h))

    def slidedp_set_wait_seconds(self, seconds: float) -> None:
        self._check(_lib.slidedp_set_wait_seconds(self._h, seconds))

    def slidedp_test_fail_nth_call(self, nth: int) -> None:
        self._check(_lib.slidedp_test_fail_nth_call(self._h, nth))

    def slidedp_test_wait_polls(self, polls: int) -> None:
        self._check(_lib.slidedp_test_wait_polls(self._h, polls))

    def slidedp_last_cuda_error(self) -> int:
        return int(_lib.slidedp_last_cuda_error(self._h))

    def slidedp_grad_norm(self, grads, n: int, inv_R: float, first_chunk: bool = True,
                          stream=None) -> None:
        self._check(_lib.slidedp_grad_norm(self._h, _grad_array(grads), len(grads), n, inv_R,
                                           int(first_chunk), _stream(stream)))

    def slidedp_grad_norm_finish(self, max_norm: float, fetch: bool = False, stream=None):
        """Returns (norm, coef) if ``fetch`` (synchronises), else None."""
        if fetch:
            norm, coef = ctypes.c_double(), ctypes.c_double()
            self._check(_lib.slidedp_grad_norm_finish(self._h, max_norm, ctypes.byref(norm),
                                                      ctypes.byref(coef), _stream(stream)))
            return norm.value, coef.value
        self._check(_lib.slidedp_grad_norm_finish(self._h, max_norm, None, None, _stream(stream)))
        return None

    def slidedp_grad_norm_tiles(self, grads, n: int, inv_R: float, tile_sums_out, stream=None) -> None:
        self._check(_lib.slidedp_grad_norm_tiles(self._h, _grad_array(grads), len(grads), n, inv_R,
                                                 _ptr(tile_sums_out), _stream(stream)))

    def slidedp_grad_norm_finish_from(self, tile_sums, count: int, max_norm: float,
                                      fetch: bool = False, stream=None):
        if fetch:
            norm, coef = ctypes.c_double(), ctypes.c_double()
            self._check(_lib.slidedp_grad_norm_finish_from(
                self._h, _ptr(tile_sums), count, max_norm, ctypes.byref(norm), ctypes.byref(coef),
                _stream(stream)))
            return norm.value, coef.value
        self._check(_lib.slidedp_grad_norm_finish_from(self._h, _ptr(tile_sums), count, max_norm,
                                                       None, None, _stream(stream)))
        return None

    def slidedp_reduce_adamw_chunk(self, grads, n: int, master, m, v, param_bf16_out,
                                   hp: HParams, stream=None) -> None:
        c = hp._c()
        self._check(_lib.slidedp_reduce_adamw_chunk(
            self._h, _grad_array(grads), len(grads), n, _ptr(master), _ptr(m), _ptr(v),
            _ptr(param_bf16_out), ctypes.byref(c), _stream(stream)))

    def slidedp_reduce_adamw_chunk_bcast(self, grads, n: int, master, m, v, param_bf16_outs,
                                         hp: HParams, stream=None) -> None:
        c = hp._c()
        self._check(_lib.slidedp_reduce_adamw_chunk_bcast(
            self._h, _grad_array(grads), len(grads), n, _ptr(master), _ptr(m), _ptr(v),
            _grad_array(param_bf16_outs), len(param_bf16_outs), ctypes.byref(c), _stream(stream)))

    def slidedp_scatter_tile_sums(self, tile_sums, count: int, dsts, stream=None) -> None:
        self._check(_lib.slidedp_scatter_tile_sums(self._h, _ptr(tile_sums), count,
                                                   _grad_array(dsts), len(dsts), _stream(stream)))

    def slidedp_ipc_export(self, dev_ptr) -> bytes:
        """The 80-byte handle of a device buffer (tensor or address), to send to a peer process."""
        buf = ctypes.create_string_buffer(IPC_HANDLE_BYTES)
        self._check(_lib.slidedp_ipc_export(self._h, _ptr(dev_ptr), buf))
        return buf.raw

    def slidedp_ipc_open(self, handle: bytes) -> int:
        """Maps a peer's handle; returns the device address valid in this process."""
        if len(handle) != IPC_HANDLE_BYTES:
            raise ValueError("not a slidedp_ipc_handle")
        out = _vp()
        self._check(_lib.slidedp_ipc_open(self._h, handle, ctypes.byref(out)))
        return int(out.value)

    def slidedp_ipc_close(self, dev_ptr: int) -> None:
        self._check(_lib.slidedp_ipc_close(self._h, dev_ptr))

    def slidedp_reduce_mean_bf16(self, grads, n: int, inv_R: float, out_bf16, stream=None) -> None:
        self._check(_lib.slidedp_reduce_mean_bf16(self._h, _grad_array(grads), len(grads), n, inv_R,
                                                  _ptr(out_bf16), _stream(stream)))

    def slidedp_stream_step(self, grads, n_total: int, host_master, host_m, host_v,
                            param_bf16_out, chunk_elems: int, nbuf: int, hp: HParams,
                            norm_ready: bool = False, want_stats: bool = True):
        c = hp._c()
        st = _Stats()
        self._check(_lib.slidedp_stream_step(
            self._h, _grad_array(grads), len(grads), n_total, _ptr(host_master), _ptr(host_m),
            _ptr(host_v), _ptr(param_bf16_out), chunk_elems, nbuf, int(norm_ready),
            ctypes.byref(c), ctypes.byref(st) if want_stats else None))
        if not want_stats:
            return None
        return {f: getattr(st, f) for f, _ in _Stats._fields_ if f != "reserved"}

    def slidedp_stream_step_async(self, grads, n_total: int, host_master, host_m, host_v,
                                  param_bf16_out, chunk_elems: int, nbuf: int, hp: HParams,
                                  norm_ready: bool = False) -> None:
        c = hp._c()
        self._check(_lib.slidedp_stream_step_async(
            self._h, _grad_array(grads), len(grads), n_total, _ptr(host_master), _ptr(host_m),
            _ptr(host_v), _ptr(param_bf16_out), chunk_elems, nbuf, int(norm_ready),
            ctypes.byref(c)))

    def slidedp_stream_layers(self, layers, chunk_elems: int, nbuf: int, hp: HParams,
                              want_stats: bool = True):
        """``layers``: sequence of (grads, n, host_master, host_m, host_v, param_bf16_out), every
        ``grads`` a list of the same R device buffers' worth of rank gradients."""
        R = len(layers[0][0]) if layers else 1
        keep = [_grad_array(L[0]) for L in layers]              # the pointer arrays must outlive the call
        arr = (_Layer * max(len(layers), 1))()
        for i, (L, g) in enumerate(zip(layers, keep)):
            if len(L[0]) != R:
                raise ValueError("every layer needs the same number of rank gradients")
            arr[i] = _Layer(ctypes.cast(g, _pp), L[1], _ptr(L[2]), _ptr(L[3]), _ptr(L[4]), _ptr(L[5]))
        c, st = hp._c(), _Stats()
        self._check(_lib.slidedp_stream_layers(self._h, arr, len(layers), R, chunk_elems, nbuf,
                                               ctypes.byref(c), ctypes.byref(st) if want_stats else None))
        if not want_stats:
            return None
        return {f: getattr(st, f) for f, _ in _Stats._fields_ if f != "reserved"}

    def slidedp_stream_wait(self) -> None:
        self._check(_lib.slidedp_stream_wait(self._h))

    def slidedp_deliver_params(self, host_master, n_total: int, param_bf16_out, chunk_elems: int,
                               nbuf: int, want_stats: bool = True):
        st = _Stats()
        self._check(_lib.slidedp_deliver_params(
            self._h, _ptr(host_master), n_total, _ptr(param_bf16_out), chunk_elems, nbuf,
            ctypes.byref(st) if want_stats else None))
        if not want_stats:
            return None
        return {f: getattr(st, f) for f in ("ms_total", "ms_h2d", "gbs_h2d", "chunks")}

    def slidedp_hbm_mix_probe(self, grads, n: int, master, m, v, scratch_bf16_out, reps: int = 5,
                              stream=None) -> float:
        """GB/s of the update kernel's loads and stores with no arithmetic (state unchanged)."""
        out = ctypes.c_double()
        self._check(_lib.slidedp_hbm_mix_probe(self._h, _grad_array(grads), len(grads), n, _ptr(master),
                                               _ptr(m), _ptr(v), _ptr(scratch_bf16_out), reps,
                                               ctypes.byref(out), _stream(stream)))
        return out.value

    def slidedp_link_probe(self, host_a, host_b, dev_a, dev_b, nbytes: int, copy_bytes: int,
                           reps: int = 3):
        out = (ctypes.c_double * 4)()
        self._check(_lib.slidedp_link_probe(self._h, _ptr(host_a), _ptr(host_b), _ptr(dev_a),
                                            _ptr(dev_b), nbytes, copy_bytes, reps, out))
        return {"h2d": out[0], "d2h": out[1], "h2d_bidir": out[2], "d2h_bidir": out[3]}


    # ---- operators of the fine-tuning pass (include/slidedp_ops.h) ----------------------------

    @staticmethod
    def _qk_args(qs, ks, dtype, cos_sin, eps, interleaved):
        if dtype not in _DTYPES:
            raise TypeError("q and k must be bfloat16 or float32")
        rows, rope = cos_sin.shape if cos_sin is not None else (0, 0)
        return _qk_bytes(qs[0], qs[1], ks[1], qs[2], rope, bool(interleaved), _DTYPES[dtype], rows, eps)

    @staticmethod
    def _qk_tables(qs, dtype, w_q, w_k, cos_sin, positions):
        D = (qs[2],)
        return (None if w_q is None else _flat(w_q, "w_q", dtype, D), None if w_k is None else _flat(w_k, "w_k", dtype, D),
                None if cos_sin is None else _flat(cos_sin, "cos_sin", torch.float32),
                None if positions is None else _flat(positions, "positions", torch.int32, (qs[0],)))

    def slidedp_qk_norm_rope(self, q, k, w_q, w_k, cos_sin, positions, q_out, k_out, eps: float = 1e-6,
                             interleaved: bool = False, stream=None) -> None:
        """RMS norm of every head of ``q`` and ``k`` ([tokens, heads, head_dim]) and the rotation by
        ``cos_sin`` ([rows, rope_dim]: cosines, then sines; None: no rotation) at ``positions``
        (int32 per token; None: 0, 1, ..)."""
        (qs, ks), dt, at = _two_sides(q, k), q.dtype, _block(self.device)
        _heads(at, dt, qs, q, "q", q_out, "q_out")
        _heads(at + 2 * _V, dt, ks, k, "k", k_out, "k_out")
        rc = _lib.slidedp_qk_norm_rope(self._h, self._qk_args(qs, ks, dt, cos_sin, eps, interleaved), at, at + 2 * _V,
                                       *self._qk_tables(qs, dt, w_q, w_k, cos_sin, positions), at + _V, at + 3 * _V,
                                       _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_qk_norm_rope_workspace(self, q, k) -> int:
        """Bytes of workspace that ``slidedp_qk_norm_rope_backward`` needs for these heads."""
        return int(_lib.slidedp_qk_norm_rope_workspace(self._qk_args(*_two_sides(q, k), q.dtype, None, 0.0, False)))

    def slidedp_qk_norm_rope_backward(self, q, k, w_q, w_k, cos_sin, positions, dq_out, dk_out, dq, dk, dw_q,
                                      dw_k, workspace, eps: float = 1e-6, interleaved: bool = False,
                                      stream=None) -> None:
        """Gradients ``dq``, ``dk`` and (float32, may be None) ``dw_q``, ``dw_k`` from those of the outputs."""
        (qs, ks), dt, at = _two_sides(q, k), q.dtype, _block(self.device)
        a = self._qk_args(qs, ks, dt, cos_sin, eps, interleaved)
        D, f32, ws = (qs[2],), torch.float32, None
        if dw_q is not None or dw_k is not None:
            ws = _workspace(workspace, _lib.slidedp_qk_norm_rope_workspace(a))
        _heads(at, dt, qs, q, "q", dq_out, "dq_out", dq, "dq")
        ak = at + 3 * _V
        _heads(ak, dt, ks, k, "k", dk_out, "dk_out", dk, "dk")
        rc = _lib.slidedp_qk_norm_rope_backward(
            self._h, a, at, ak, *self._qk_tables(qs, dt, w_q, w_k, cos_sin, positions), at + _V, ak + _V, at + 2 * _V, ak + 2 * _V,
            None if dw_q is None else _flat(dw_q, "dw_q", f32, D), None if dw_k is None else _flat(dw_k, "dw_k", f32, D),
            ws, _stream(stream, self.device))
        if rc:
            self._check(rc)

    @staticmethod
    def _attn_args(qs, ks, cu_docs=None, prefix=None, slopes=None, causal=True, scale=None, softcap=0.0):
        T, H, D = qs
        docs, cu = 1, 0
        if cu_docs is not None:
            cu = _flat(cu_docs, "cu_docs", torch.int32)
            if cu_docs.dim() != 1 or cu_docs.numel() < 1:
                raise ValueError("cu_docs must hold docs + 1 offsets")
            docs = cu_docs.numel() - 1
        return _attn_bytes(T, H, ks[1], D, bool(causal), docs, 0, cu,
                           0 if prefix is None else _flat(prefix, "prefix", torch.int32, (docs,)),
                           0 if slopes is None else _flat(slopes, "slopes", torch.float32, (H,)),
                           D ** -0.5 if scale is None else scale, softcap)

    def slidedp_attention(self, q, k, v, out, lse, cu_docs=None, prefix=None, slopes=None, causal: bool = True,
                          scale: float | None = None, softcap: float = 0.0, stream=None) -> None:
        """Attention of ``q`` [tokens, heads_q, head_dim] over ``k``, ``v`` [tokens, heads_kv, head_dim] within
        packed documents (``cu_docs``: int32 offsets; None: one document). Fills ``out`` and ``lse``
        [heads_q, tokens]. ``scale`` defaults to head_dim ** -0.5."""
        (qs, ks), bf, at = _two_sides(q, k), torch.bfloat16, _block(self.device)
        a = self._attn_args(qs, ks, cu_docs, prefix, slopes, causal, scale, softcap)
        _heads(at, bf, qs, q, "q", out, "out")
        _heads(at + 2 * _V, bf, ks, k, "k", v, "v")
        rc = _lib.slidedp_attention(self._h, a, at, at + 2 * _V, at + 3 * _V, at + _V, _flat(lse, "lse", torch.float32, (qs[1], qs[0])),
                                    _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_attention_workspace(self, q, k) -> int:
        """Bytes of workspace that ``slidedp_attention_backward`` needs."""
        return int(_lib.slidedp_attention_workspace(self._attn_args(*_two_sides(q, k))))

    def slidedp_attention_backward(self, q, k, v, out, lse, d_out, dq, dk, dv, workspace, cu_docs=None, prefix=None,
                                   slopes=None, causal: bool = True, scale: float | None = None,
                                   softcap: float = 0.0, stream=None) -> None:
        """Gradients ``dq``, ``dk``, ``dv`` from ``d_out``, with the forward's ``out`` and ``lse``."""
        (qs, ks), bf, at = _two_sides(q, k), torch.bfloat16, _block(self.device)
        a = self._attn_args(qs, ks, cu_docs, prefix, slopes, causal, scale, softcap)
        ws = _workspace(workspace, _lib.slidedp_attention_workspace(a))
        _heads(at, bf, qs, q, "q", out, "out", d_out, "d_out", dq, "dq")
        ak = at + 4 * _V
        _heads(ak, bf, ks, k, "k", v, "v", dk, "dk", dv, "dv")
        rc = _lib.slidedp_attention_backward(
            self._h, a, at, ak, ak + _V, at + _V, _flat(lse, "lse", torch.float32, (qs[1], qs[0])), at + 2 * _V, at + 3 * _V,
            ak + 2 * _V, ak + 3 * _V, ws, _stream(stream, self.device))
        if rc:
            self._check(rc)

    def _distill_call(self, logits, teacher_ids, teacher_logits, labels, lse, row_grad, d_logits, temperature, w_teacher,
                      w_label):
        """The arguments that the three calls share: slidedp_distill_args and the addresses of the inputs, of
        lse and of the row gradients."""
        if logits.dtype not in _DTYPES or logits.dim() != 2:
            raise TypeError("logits must be [rows, vocab] of bfloat16 or float32")
        _block(self.device)
        dt, shape, f32, i32 = logits.dtype, logits.shape, torch.float32, torch.int32
        rows, vocab = shape
        entries = teacher_ids.shape[-1]
        a = _distill_bytes(rows, vocab, entries, _DTYPES[dt], _matrix(logits, "logits", dt, shape),
                           0 if d_logits is None else _matrix(d_logits, "d_logits", dt, shape), temperature, w_teacher, w_label)
        return (a, (logits.data_ptr(), _flat(teacher_ids, "teacher_ids", i32, (rows, entries)),
                    _flat(teacher_logits, "teacher_logits", f32, (rows, entries)),
                    None if labels is None else _flat(labels, "labels", i32, (rows,))),
                _flat(lse, "lse", f32, (2, rows)), None if row_grad is None else _flat(row_grad, "row_grad", f32, (rows,)))

    def slidedp_distill_loss(self, logits, teacher_ids, teacher_logits, labels, loss, lse, temperature: float = 1.0,
                             w_teacher: float = 1.0, w_label: float = 0.0, stream=None) -> None:
        """Per-row distillation ``loss`` and ``lse`` [2, rows] of ``logits`` [rows, vocab] against the teacher's
        stored entries (int32 ids, float32 logits, both [rows, entries]) and int32 ``labels`` (may be None)."""
        a, ins, l, _ = self._distill_call(logits, teacher_ids, teacher_logits, labels, lse, None, None, temperature,
                                          w_teacher, w_label)
        rc = _lib.slidedp_distill_loss(self._h, a, *ins, _flat(loss, "loss", torch.float32, logits.shape[:1]), l, _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_distill_loss_backward(self, logits, teacher_ids, teacher_logits, labels, lse, row_grad, d_logits,
                                      temperature: float = 1.0, w_teacher: float = 1.0, w_label: float = 0.0,
                                      stream=None) -> None:
        """``d_logits`` = ``row_grad`` (float32 per row; None: ones) times the loss's gradient, with the forward's
        ``lse``. ``d_logits`` may be ``logits``."""
        a, ins, l, g = self._distill_call(logits, teacher_ids, teacher_logits, labels, lse, row_grad, d_logits,
                                          temperature, w_teacher, w_label)
        self._check(_lib.slidedp_distill_loss_backward(self._h, a, *ins, l, g, d_logits.data_ptr(), _stream(stream, self.device)))

    def slidedp_distill_step(self, logits, teacher_ids, teacher_logits, labels, row_grad, loss, lse, d_logits,
                             temperature: float = 1.0, w_teacher: float = 1.0, w_label: float = 0.0,
                             stream=None) -> None:
        """``loss``, ``lse`` and ``d_logits`` in one pass over the logits."""
        a, ins, l, g = self._distill_call(logits, teacher_ids, teacher_logits, labels, lse, row_grad, d_logits,
                                          temperature, w_teacher, w_label)
        self._check(_lib.slidedp_distill_step(self._h, a, *ins, g, _flat(loss, "loss", torch.float32, logits.shape[:1]), l,
                                              d_logits.data_ptr(), _stream(stream, self.device)))

    @staticmethod
    def _embedding_args(tokens, table, table_dtype_of, grad_dtype, scale, accumulate):
        shape, dt = table.shape, table_dtype_of.dtype
        if len(shape) != 2 or dt not in _DTYPES or grad_dtype not in _DTYPES:
            raise TypeError("the table and its rows must be matrices of bfloat16 or float32")
        return _embedding_bytes(tokens, shape[0], shape[1], _DTYPES[dt], _DTYPES[grad_dtype], bool(accumulate), 0, scale)

    def slidedp_embedding(self, table, ids, out, scale: float = 1.0, stream=None) -> None:
        """``out`` [tokens, hidden] = ``scale`` times the rows of ``table`` [vocab, hidden] that the int32 ``ids`` [tokens] name;
        zeros for ids outside the table."""
        at, dt, shape, T = _block(self.device), table.dtype, table.shape, len(ids)
        a = self._embedding_args(T, table, table, dt, scale, False)
        _rows(at, dt, shape, table, "table")
        _rows(at + _R, dt, (T, shape[1]), out, "out")
        rc = _lib.slidedp_embedding(self._h, a, at, _flat(ids, "ids", torch.int32, (T,)), at + _R, _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_embedding_workspace(self, d_out, d_table) -> int:
        """Bytes of workspace that ``slidedp_embedding_backward`` needs."""
        return int(_lib.slidedp_embedding_workspace(self._embedding_args(len(d_out), d_table, d_out, d_table.dtype, 1.0, False)))

    def slidedp_embedding_backward(self, ids, d_out, d_table, workspace, scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
        """``d_table`` [vocab, hidden] (either type): the gradient of the table from that of the rows, ``d_out`` [tokens, hidden].
        ``accumulate`` adds to what it holds, and touches only the rows that have tokens."""
        at, shape, T = _block(self.device), d_table.shape, len(ids)
        a = self._embedding_args(T, d_table, d_out, d_table.dtype, scale, accumulate)
        _rows(at, d_out.dtype, (T, shape[1]), d_out, "d_out")
        _rows(at + _R, d_table.dtype, shape, d_table, "d_table")
        rc = _lib.slidedp_embedding_backward(self._h, a, _flat(ids, "ids", torch.int32, (T,)), at, at + _R,
                                             _workspace(workspace, _lib.slidedp_embedding_workspace(a)), _stream(stream, self.device))
        if rc:
            self._check(rc)

    @staticmethod
    def _block_norm_args(x, has_y, post_norm, pre_norm, gate, gate_sigmoid, residual_scale, eps):
        shape, dt = x.shape, x.dtype
        if dt not in _DTYPES or len(shape) != 2:
            raise TypeError("x must be [tokens, hidden] of bfloat16 or float32")
        return _block_norm_bytes(shape[0], shape[1], _DTYPES[dt], has_y, bool(post_norm), pre_norm,
                                 0 if gate is None else gate.dim(), bool(gate_sigmoid) and gate is not None, residual_scale, eps)

    @staticmethod
    def _block_norm_inputs(at, x, y, w_post, gate, w_pre):
        """The views of x, y and the gate at ``at``, and the weights' addresses."""
        dt, shape = x.dtype, x.shape
        H = (shape[1],)
        if gate is not None and gate.dim() == 1:
            _rows(at, dt, shape, x, "x", y, "y")
            _rows(at + 2 * _R, dt, (1, H[0]), gate[None], "gate")
        else:
            _rows(at, dt, shape, x, "x", y, "y", gate, "gate")
        return (None if w_post is None else _flat(w_post, "w_post", dt, H), None if w_pre is None else _flat(w_pre, "w_pre", dt, H))

    def slidedp_block_norm(self, x, y, w_post, gate, w_pre, x_out, h_out, residual_scale: float = 1.0, eps: float = 1e-6,
                           post_norm: bool = True, gate_sigmoid: bool = False, stream=None) -> None:
        """``x_out`` = ``x`` + ``residual_scale`` * gate * n with n the RMS norm of the block's output ``y`` times ``w_post``
        (``post_norm`` False: ``y`` itself), and the next block's input ``h_out`` = RMS norm of ``x_out`` times ``w_pre``
        (``h_out`` None: not wanted). All [tokens, hidden]; ``gate``: None, [hidden] or [tokens, hidden], through a sigmoid with
        ``gate_sigmoid``. ``y`` and ``x_out`` None: the first norm, of ``x`` alone."""
        at, has_y = _block(self.device), y is not None
        a = self._block_norm_args(x, has_y, post_norm and has_y, h_out is not None, gate, gate_sigmoid, residual_scale, eps)
        w_post, w_pre = self._block_norm_inputs(at, x, y, w_post, gate, w_pre)
        _rows(at + 3 * _R, x.dtype, x.shape, x_out, "x_out", h_out, "h_out")
        rc = _lib.slidedp_block_norm(self._h, a, at, at + _R, w_post, at + 2 * _R, w_pre, at + 3 * _R, at + 4 * _R, _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_block_norm_workspace(self, x) -> int:
        """Bytes of workspace that ``slidedp_block_norm_backward`` needs for rows like ``x``."""
        return int(_lib.slidedp_block_norm_workspace(self._block_norm_args(x, True, True, True, None, False, 1.0, 0.0)))

    def slidedp_block_norm_backward(self, x, y, w_post, gate, w_pre, dx_out, dh_out, dx, dy, dgate, dw_post, dw_pre, workspace,
                                    residual_scale: float = 1.0, eps: float = 1e-6, post_norm: bool = True, gate_sigmoid: bool = False,
                                    stream=None) -> None:
        """Gradients ``dx``, ``dy``, ``dgate`` (float32 [hidden] for a gate of that shape), ``dw_post`` and ``dw_pre`` (float32) from
        ``dx_out`` (None: zeros) and ``dh_out`` (None: the forward had no ``h_out``). The last three may be None."""
        at, dt, shape, f32, has_y = _block(self.device), x.dtype, x.shape, torch.float32, y is not None
        H = (shape[1],)
        a = self._block_norm_args(x, has_y, post_norm and has_y, dh_out is not None, gate, gate_sigmoid, residual_scale, eps)
        vector = gate is not None and gate.dim() == 1
        ws = None
        if dw_post is not None or dw_pre is not None or (vector and dgate is not None):
            ws = _workspace(workspace, _lib.slidedp_block_norm_workspace(a))
        w_post, w_pre = self._block_norm_inputs(at, x, y, w_post, gate, w_pre)
        _rows(at + 3 * _R, dt, shape, dx_out, "dx_out", dh_out, "dh_out", dx, "dx", dy, "dy")
        if vector and dgate is not None:
            _rows(at + 7 * _R, f32, (1, H[0]), dgate[None], "dgate")
        else:
            _rows(at + 7 * _R, dt, shape, dgate, "dgate")
        rc = _lib.slidedp_block_norm_backward(
            self._h, a, at, at + _R, w_post, at + 2 * _R, w_pre, *(at + i * _R for i in range(3, 8)),
            None if dw_post is None else _flat(dw_post, "dw_post", f32, H), None if dw_pre is None else _flat(dw_pre, "dw_pre", f32, H), ws,
            _stream(stream, self.device))
        if rc:
            self._check(rc)

    def _policy_call(self, logits, labels, old_logp, ref_logp, advantage, d_logits, temperature, clip_low, clip_high, kl_weight):
        """slidedp_policy_args and the inputs' addresses."""
        if logits.dtype not in _DTYPES or logits.dim() != 2:
            raise TypeError("logits must be [rows, vocab] of bfloat16 or float32")
        _block(self.device)
        dt, shape, f32 = logits.dtype, logits.shape, torch.float32
        rows, each = shape[0], shape[:1]
        a = _policy_bytes(rows, shape[1], _DTYPES[dt], 0, _matrix(logits, "logits", dt, shape),
                          0 if d_logits is None else _matrix(d_logits, "d_logits", dt, shape), temperature, clip_low, clip_high, kl_weight)
        return a, (logits.data_ptr(), _flat(labels, "labels", torch.int32, each),
                   None if old_logp is None else _flat(old_logp, "old_logp", f32, each),
                   None if ref_logp is None else _flat(ref_logp, "ref_logp", f32, each),
                   None if advantage is None else _flat(advantage, "advantage", f32, each))

    def slidedp_policy_loss(self, logits, labels, old_logp, ref_logp, advantage, loss, logp, temperature: float = 1.0, clip_low: float = 0.2,
                            clip_high: float = 0.2, kl_weight: float = 0.0, stream=None) -> None:
        """Per row the clipped policy ``loss`` and the log-probability ``logp`` of the int32 ``labels`` under ``logits`` [rows,
        vocab]; all other arguments float32 per row. With ``old_logp``, ``ref_logp``, ``advantage`` and ``loss`` None: the
        log-probabilities alone."""
        a, ins = self._policy_call(logits, labels, old_logp, ref_logp, advantage, None, temperature, clip_low, clip_high, kl_weight)
        f32, each = torch.float32, logits.shape[:1]
        rc = _lib.slidedp_policy_loss(self._h, a, *ins, None if loss is None else _flat(loss, "loss", f32, each), _flat(logp, "logp", f32, each),
                                      _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_policy_loss_backward(self, logits, labels, old_logp, ref_logp, advantage, logp, row_grad, d_logits, temperature: float = 1.0,
                                     clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0, stream=None) -> None:
        """``d_logits`` = ``row_grad`` (float32 per row; None: ones) times the loss's gradient, with the forward's ``logp``.
        ``d_logits`` may be ``logits``."""
        a, ins = self._policy_call(logits, labels, old_logp, ref_logp, advantage, d_logits, temperature, clip_low, clip_high, kl_weight)
        f32, each = torch.float32, logits.shape[:1]
        rc = _lib.slidedp_policy_loss_backward(self._h, a, *ins, _flat(logp, "logp", f32, each),
                                               None if row_grad is None else _flat(row_grad, "row_grad", f32, each), d_logits.data_ptr(),
                                               _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_policy_step(self, logits, labels, old_logp, ref_logp, advantage, row_grad, loss, logp, d_logits, temperature: float = 1.0,
                            clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0, stream=None) -> None:
        """``loss``, ``logp`` and ``d_logits`` in one pass over the logits."""
        a, ins = self._policy_call(logits, labels, old_logp, ref_logp, advantage, d_logits, temperature, clip_low, clip_high, kl_weight)
        f32, each = torch.float32, logits.shape[:1]
        rc = _lib.slidedp_policy_step(self._h, a, *ins, None if row_grad is None else _flat(row_grad, "row_grad", f32, each),
                                      None if loss is None else _flat(loss, "loss", f32, each), _flat(logp, "logp", f32, each),
                                      d_logits.data_ptr(), _stream(stream, self.device))
        if rc:
            self._check(rc)

    def slidedp_clip_grad_norm_workspace(self, grads) -> int:
        """Bytes of workspace that ``slidedp_clip_grad_norm`` needs for these tensors."""
        _block(self.device)
        return int(_lib.slidedp_clip_grad_norm_workspace(_tensors(grads, "grads"), len(grads)))

    def slidedp_clip_grad_norm(self, grads, outs, max_norm: float, result, workspace, scale: float = 1.0, stream=None) -> None:
        """``outs`` (may be ``grads``; None: the norm alone) = the tensors of ``grads`` times ``scale`` times the coefficient
        min(1, max_norm / (norm + 1e-6)), with the norm over all of them; bfloat16 or float32 each, contiguous. ``result``: four float64
        (sum of squares, norm, coefficient, 1.0 if the norm is not finite)."""
        _block(self.device)
        n, g = len(grads), _tensors(grads, "grads")
        o = None if outs is None else g if outs is grads else _tensors(outs, "outs")
        if outs is not None and len(outs) != n:
            raise ValueError("outs must hold as many tensors as grads")
        rc = _lib.slidedp_clip_grad_norm(self._h, g, o, n, scale, max_norm, _flat(result, "result", torch.float64, (4,)),
                                         _workspace(workspace, _lib.slidedp_clip_grad_norm_workspace(g, n)), _stream(stream, self.device))
        if rc:
            self._check(rc)


def slidedp_model_stream_step(n_total: int, R: int, chunk_elems: int, nbuf: int, h2d_gbs: float,
                              d2h_gbs: float, update_gparams_s: float, norm_gbs: float = 0.0,
                              per_copy_us: float = 0.0):
    """(lower_bound_ms, predicted_ms) of a host-resident step from measured rates."""
    r = _Rates(h2d_gbs, d2h_gbs, update_gparams_s, norm_gbs, per_copy_us)
    lo, pred = ctypes.c_double(), ctypes.c_double()
    rc = _lib.slidedp_model_stream_step(n_total, R, chunk_elems, nbuf, ctypes.byref(r),
                                        ctypes.byref(lo), ctypes.byref(pred))
    if rc != OK:
        raise SlideDPError(rc)
    return lo.value, pred.value


def shard_bounds(n: int, shards: int):
    """Contiguous shard bounds [(lo, hi), ...] of a flat space of n parameters over `shards`
    GPUs, every interior bound a multiple of NORM_TILE so that the shards' tile sums, gathered
    in shard order, are the tile sums of the unsharded step (argument arithmetic only)."""
    tiles = -(-n // NORM_TILE)
    bounds, lo_tile = [], 0
    for s in range(shards):
        hi_tile = lo_tile + tiles // shards + (1 if s < tiles % shards else 0)
        bounds.append((min(lo_tile * NORM_TILE, n), min(hi_tile * NORM_TILE, n)))
        lo_tile = hi_tile
    return bounds


def slidedp_create(device: int = 0, gpu_budget_bytes: int = 0) -> Context:
    return Context(device, gpu_budget_bytes)


def slidedp_grad_norm_noalloc(grads, n: int, inv_R: float, max_norm: float, out4, stream=None) -> None:
    """Global norm of one chunk for callers that must not allocate device memory (allocator
    callbacks, processes with a fully committed memory budget, plug-ins that only receive
    pointers): same result as ``slidedp_grad_norm`` + ``slidedp_grad_norm_finish``, but the
    tile sums live in a fixed 512 KiB array inside the library instead of a context.

    ``out4`` is a caller-owned device tensor of four float64 (sumsq, norm, coef, non-finite
    flag). ``n`` may not exceed ``NOALLOC_MAX_ELEMS``. Calls share the array, so only issue
    them ordered on one stream; make the first call on a device outside any stream capture.
    """
    rc = _lib.slidedp_grad_norm_noalloc(_grad_array(grads), len(grads), n, inv_R, max_norm,
                                        _ptr(out4), _stream(stream))
    if rc != OK:
        raise SlideDPError(rc)
