"""Global gradient norm, clipping and the update of many parameters (include/hybrid_attn_optim.h).

    grads, params = TensorList(grads), ParamList(masters, grads, m, v, copies)         # once, if the gradients are the same tensors in every step
    result = hybrid_attn_grad_norm(grads, max_norm)                                     # device (norm, factor)
    hybrid_attn_param_update_many(params, lr, kind=HA_OPT_ADAMW, step=step, clip=result)

Argument marshalling only, as in hybrid_attn; everything is public there.  Plain calls are marshalled by compiled code (csrc/ha_binding_calls.h).
"""
from __future__ import annotations

import ctypes

import torch

from . import hybrid_attn as _ha


class ha_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_uint64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ha_param(ctypes.Structure):
    _fields_ = [("master", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("param_io", ctypes.c_void_p),
                ("n", ctypes.c_uint64), ("grad_dtype", ctypes.c_int32), ("io_dtype", ctypes.c_int32)]


_T, _vp, _i = ctypes.POINTER(ha_tensor), ctypes.c_void_p, ctypes.c_int32
SIGNATURES = (
    ("hybrid_attn_grad_norm_workspace_bytes", [_i, _T], ctypes.c_size_t),
    ("hybrid_attn_grad_norm", [_i, _T, ctypes.c_float, _vp, _vp, ctypes.c_size_t, _vp], ctypes.c_int),
    ("hybrid_attn_grad_clip", [_i, _T, _T, _vp, _vp], ctypes.c_int),
    ("hybrid_attn_param_update_many", [ctypes.POINTER(_ha.ha_optimizer), _i, ctypes.POINTER(ha_param), _vp, _vp], ctypes.c_int),
)


def _one_device(tensors):
    for t in tensors:
        if t is not None:
            _ha._require_gpu(t)
            if not t.is_contiguous():
                raise ValueError("gradients and parameters must be contiguous")
    devices = {t.device for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError(f"gradients and parameters must be on one device, got {sorted(map(str, devices))}")
    return devices.pop() if devices else None


def _native(c, n, workspace_bytes, device):
    """What the compiled marshalling reads of a list."""
    return ctypes.addressof(c), n, workspace_bytes, -1 if device is None else device.index


class TensorList:
    """Contiguous bf16 or fp32 tensors on one GPU, with their descriptors for the C ABI.  It holds the tensors, and every call that takes it looks at the
    memory they have then (data, set_ and resize_ may give them another).  It does not see gradients that take a tensor's place: a program whose
    gradients are the same tensors in every step builds it once, one that sets them to None or makes new ones builds it every step."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.c = (ha_tensor * len(self.tensors))()
        self.device = self.sizes = None
        self.refresh()

    def refresh(self):
        """Describes the tensors as they are now."""
        native = _ha._CALLS or _ha._calls()
        if native and self.tensors and (done := native.describe_tensors(self.tensors, ctypes.addressof(self.c))) is not None:
            index, sizes = done
            device = self.device if self.device is not None and self.device.index == index else torch.device("cuda", index)
        else:
            device = _one_device(self.tensors)
            self.c[:] = [ha_tensor(t.data_ptr(), t.numel(), _ha._dtype_code(t), 0) for t in self.tensors]
            sizes = [t.numel() for t in self.tensors]
        if sizes != self.sizes or device != self.device:
            self.device, self.sizes = device, sizes
            self.workspace_bytes = _ha._lib().hybrid_attn_grad_norm_workspace_bytes(len(self.tensors), self.c)
            self.native = _native(self.c, len(self.tensors), self.workspace_bytes, self.device)

    def __len__(self):
        return len(self.tensors)


class ParamList:
    """Parameters for hybrid_attn_param_update_many: fp32 masters, their gradients (fp32 or bf16), AdamW's moments (None or lists of None: plain steps
    only) and the copies the forward reads (list, or None; single ones may be None).  It holds the tensors; what TensorList says of their memory, and of
    gradients that are new tensors, holds here too."""

    def __init__(self, masters, grads, m=None, v=None, param_io=None):
        masters, grads = list(masters), list(grads)
        n = len(masters)
        m, v, io = (list(x) if x is not None else [None] * n for x in (m, v, param_io))
        if not len(grads) == len(m) == len(v) == len(io) == n:
            raise ValueError("masters, grads, m, v and param_io must be lists of one length")
        self.tensors = (masters, grads, m, v, io)
        self.c = (ha_param * n)()
        self.device = self.native = None
        self.refresh()

    def refresh(self):
        """Describes the tensors as they are now."""
        native = _ha._CALLS or _ha._calls()
        if native and len(self) and (index := native.describe_params(self.tensors, ctypes.addressof(self.c))) is not None:
            device = self.device if self.device is not None and self.device.index == index else torch.device("cuda", index)
        else:
            device = self._describe()
        if device != self.device or self.native is None:
            self.device = device
            self.native = _native(self.c, len(self), 0, device)

    def _describe(self):
        device = _one_device([t for x in self.tensors for t in x])
        for p, g, a, b, c in zip(*self.tensors):
            if any(t is not None and t.dtype != torch.float32 for t in (p, a, b)):
                raise ValueError("masters, m and v must be fp32")
            if any(t is not None and t.numel() != p.numel() for t in (g, a, b, c)):
                raise ValueError("a master, its gradient, moments and copy must be of one size")

        def at(t):
            return None if t is None else t.data_ptr()
        self.c[:] = [ha_param(at(p), at(g), at(a), at(b), at(c), p.numel(), _ha._dtype_code(g), _ha.HA_BF16 if c is None else _ha._dtype_code(c))
                     for p, g, a, b, c in zip(*self.tensors)]
        return device

    def __len__(self):
        return len(self.tensors[0])


def _tensor_list(x) -> TensorList:
    return x if isinstance(x, TensorList) else TensorList(x)


def _result(t, device):
    if t.dtype != torch.float32 or tuple(t.shape) != (2,) or not t.is_contiguous() or device not in (None, t.device):
        raise ValueError(f"the result of hybrid_attn_grad_norm is a contiguous fp32 tensor [2] on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def hybrid_attn_grad_norm_workspace_bytes(grads) -> int:
    grads = _tensor_list(grads)
    grads.refresh()
    return grads.workspace_bytes


def hybrid_attn_grad_norm(grads, max_norm: float = float("inf"), result=None, workspace=None, stream=None):
    """Enqueue the global 2-norm of a TensorList (or a list of tensors) and the factor min(1, max_norm / norm) that brings it down to max_norm: returns
    a device fp32 tensor (norm, factor).  The factor is NaN where a gradient is not finite.  Does not synchronise."""
    grads = _tensor_list(grads)
    native = _ha._CALLS or _ha._calls()
    if native and (done := native.grad_norm(grads, max_norm, result, workspace, stream)) is not None:
        return done
    return _grad_norm(grads, max_norm, result, workspace, stream)


@_ha._allocations_follow_stream
def _grad_norm(grads, max_norm, result, workspace, stream):
    grads.refresh()
    device = grads.device if grads.device is not None else result.device if result is not None else torch.device("cuda", torch.cuda.current_device())
    with _ha._on_device(device):
        if result is None:
            result = torch.empty(2, dtype=torch.float32, device=device)
        _ha._require_gpu(result, workspace)
        _result(result, device)
        if workspace is None:
            workspace = torch.empty(grads.workspace_bytes, dtype=torch.uint8, device=device)
        elif workspace.device != device or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {device}")
        st = _ha._lib().hybrid_attn_grad_norm(len(grads), grads.c, max_norm, result.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                              _ha._stream_handle(stream, result))
    if st != _ha.HA_OK:
        raise _ha.HybridAttnError(st, "hybrid_attn_grad_norm")
    return result


def hybrid_attn_grad_clip(grads, result, out=None, stream=None):
    """Enqueue out = factor * grads for all tensors, with the factor of hybrid_attn_grad_norm's result; out None: in place.  A factor that is not finite
    leaves out as it was.  No tensor may stand in a list that is written twice.  Does not synchronise."""
    grads = _tensor_list(grads)
    out = grads if out is None else _tensor_list(out)
    native = _ha._CALLS or _ha._calls()
    if native and out.sizes == grads.sizes and native.grad_clip(grads, result, out, stream) is not None:
        return
    grads.refresh()
    out.refresh()
    if out.sizes != grads.sizes:
        raise ValueError("out must be a list of tensors of the gradients' sizes")
    _ha._require_gpu(result)
    if grads.device is not None and out.device != grads.device:
        raise ValueError(f"out must be on {grads.device}")
    _result(result, grads.device)
    with _ha._on_device_of(result):
        st = _ha._lib().hybrid_attn_grad_clip(len(grads), grads.c, out.c, result.data_ptr(), _ha._stream_handle(stream, result))
    if st != _ha.HA_OK:
        raise _ha.HybridAttnError(st, "hybrid_attn_grad_clip")


def hybrid_attn_param_update_many(params: ParamList, lr: float, kind: int = 0, step: int = 1, grad_scale: float = 1.0, beta1: float = 0.9,
                                  beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01, clip=None, stream=None):
    """One update of all parameters of a ParamList in place, as hybrid_attn_param_update makes it of one.  clip: hybrid_attn_grad_norm's result, whose factor
    multiplies the gradients besides grad_scale; where it is not finite, nothing changes.  No master, moment or copy may stand in the list twice.  Does not
    synchronise."""
    native = _ha._CALLS or _ha._calls()
    if native and native.update_many(params, lr, kind, step, grad_scale, beta1, beta2, eps, weight_decay, clip, stream) is not None:
        return
    params.refresh()
    if clip is not None:
        _ha._require_gpu(clip)
        _result(clip, params.device)
    if params.device is None:
        return
    _ha._fit_int32(kind=kind, step=step)
    opt = _ha.ha_optimizer(kind, step, lr, grad_scale, beta1, beta2, eps, weight_decay)
    with _ha._on_device(params.device):
        stream_handle = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(params.device.index)
        st = _ha._lib().hybrid_attn_param_update_many(opt, len(params), params.c, None if clip is None else clip.data_ptr(), stream_handle)
    if st != _ha.HA_OK:
        raise _ha.HybridAttnError(st, "hybrid_attn_param_update_many")
