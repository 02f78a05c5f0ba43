"""Rotary positions of queries and keys, alone and behind a norm of every head's row (include/hybrid_attn_rotary.h).

    rotary = hybrid_attn_rotary_grid(128)                      # or hybrid_attn_rotary_frequencies(128): a plain sequence
    places = hybrid_attn_grid_positions(21, 30, 52)            # int32 [N, 3]
    q, k = hybrid_attn_norm_rotate(q, k, w_q, w_k, rotary, places)
    dq, dk, dw_q, dw_k = hybrid_attn_norm_rotate_grad(grad_q, grad_k, q_in, k_in, w_q, w_k, rotary, places)
    x = hybrid_attn_rotate(x, rotary, places)                  # the rotation alone; hybrid_attn_rotate_grad: its gradient

q is a [B, H, N, d] view, k a [B, H_kv, N, d] view, each with strides of its own and a contiguous last dimension.  Argument marshalling only, as in
hybrid_attn; everything is public there.  Plain calls are marshalled by compiled code (csrc/ha_binding_rows.h), all others, and every error, here.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional

import torch

from . import block_sparse as _bs
from . import hybrid_attn as _ha


class ha_rotary(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_stride_b", ctypes.c_int64),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("magnitude", ctypes.c_float)]


class ha_rows_problem(ctypes.Structure):
    _fields_ = [*((n, ctypes.c_int32) for n in ("B", "H", "H_kv", "N", "d_head", "dtype")), ("eps", ctypes.c_float)]


_P, _R, _V, _vp, _sz = ctypes.POINTER(ha_rows_problem), ctypes.POINTER(ha_rotary), ctypes.POINTER(_bs.ha_view), ctypes.c_void_p, ctypes.c_size_t
SIGNATURES = (
    ("hybrid_attn_rotary_validate", [_P, _R], ctypes.c_int),
    ("hybrid_attn_rotate", [_P, _R, _V, _V, ctypes.c_int32, _vp], ctypes.c_int),
    ("hybrid_attn_norm_rotate", [_P, _R, _V, _V, _vp, _vp, _V, _V, _vp], ctypes.c_int),
    ("hybrid_attn_norm_rotate_grad_workspace_bytes", [_P], _sz),
    ("hybrid_attn_norm_rotate_grad", [_P, _R, *[_V] * 4, _vp, _vp, _V, _V, _vp, _vp, _vp, _sz, _vp], ctypes.c_int),
)


class Rotary(NamedTuple):
    """How positions rotate: radians per position of every pair (fp64 [rot_dim / 2] on the GPU), the axis of the position that each pair goes by (int32 [rot_dim / 2], or
    None: the first), whether a pair is two neighbouring channels or two that are rot_dim / 2 apart, and what rotated channels are multiplied with."""
    freq: torch.Tensor
    axis: Optional[torch.Tensor] = None
    interleaved: bool = True
    magnitude: float = 1.0


def hybrid_attn_rotary_frequencies(rot_dim: int, base: float = 10000.0, interleaved: bool = True, stretch: float = 1.0, original: Optional[int] = None,
                                   slow: float = 1.0, fast: float = 32.0, device="cuda") -> Rotary:
    """Rotary of a plain sequence: pair i turns by base^(-2 i / rot_dim) a position.  stretch s > 1 makes positions of s times the context fit: without `original` all
    frequencies are divided by s; with it (the tokens of the context that they were made for), those that make fewer than `slow` turns over it, the ones of
    more than `fast` turns stay, the share goes linearly with the turns in between, and rotated channels are multiplied with 1 + 0.1 log s."""
    if rot_dim < 0 or rot_dim % 2 or stretch < 1 or base <= 0:
        raise ValueError("rot_dim must be an even number, stretch at least 1 and base positive")
    if original is not None and (original < 1 or not fast > slow):
        raise ValueError("original must be a number of tokens, and fast more than slow")
    freq = base ** -(torch.arange(0, rot_dim, 2, dtype=torch.float64) / max(rot_dim, 1))
    magnitude = 1.0
    if original is None:
        freq /= stretch
    elif stretch > 1:
        divided = ((fast - original * freq / (2 * math.pi)) / (fast - slow)).clamp(0, 1)
        freq *= 1 - divided + divided / stretch
        magnitude = 1.0 + 0.1 * math.log(stretch)
    return Rotary(freq.to(device), None, interleaved, magnitude)


def hybrid_attn_rotary_grid(rot_dim: int, base: float = 10000.0, interleaved: bool = True, device="cuda") -> Rotary:
    """Rotary of tokens on a (frame, row, column) grid: rows and columns have a third of the pairs each, rounded down, frames the others; the pairs of an axis turn by
    base^(-i / its pairs)."""
    if rot_dim < 6 or rot_dim % 2 or base <= 0:
        raise ValueError("rot_dim must be an even number, at least 6, and base positive")
    third = rot_dim // 2 // 3
    shares = (rot_dim // 2 - 2 * third, third, third)
    freq = torch.cat([base ** -(torch.arange(n, dtype=torch.float64) / n) for n in shares])
    axis = torch.repeat_interleave(torch.arange(3, dtype=torch.int32), torch.tensor(shares))
    return Rotary(freq.to(device), axis.to(device), interleaved)


def hybrid_attn_grid_positions(frames: int, rows: int, cols: int, first_frame: int = 0, device="cuda") -> torch.Tensor:
    """Positions int32 [frames rows cols, 3] of the tokens of a clip in frame-major order."""
    at = torch.cartesian_prod(*(torch.arange(n, dtype=torch.int32) for n in (frames, rows, cols))).view(-1, 3)
    at[:, 0] += first_frame
    return at.to(device)


def _rotary_struct(rotary, positions, tokens, device, B=1) -> ha_rotary:
    """ha_rotary of a Rotary (or None: nothing is rotated) with positions int32 [tokens, axes] or, of B > 0 entries, [B, tokens, axes]."""
    if rotary is None:
        return ha_rotary(None, None, None, 0, 0, 1, 1, 1.0)
    freq, axis, interleaved, magnitude = rotary
    if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or freq.device != device:
        raise ValueError(f"freq must be a contiguous fp64 tensor [rot_dim / 2] on {device}")
    if axis is not None and (axis.dtype != torch.int32 or axis.shape != freq.shape or not axis.is_contiguous() or axis.device != device):
        raise ValueError(f"axis must be a contiguous int32 tensor {tuple(freq.shape)} on {device}")
    if positions is None or positions.dtype != torch.int32 or not positions.is_contiguous() or positions.device != device:
        raise ValueError(f"positions must be a contiguous int32 tensor on {device}")
    if positions.dim() not in (2, 3) or positions.shape[-2] != tokens or (positions.dim() == 3 and positions.shape[0] != B):
        raise ValueError(f"positions must be [{tokens}, axes]" + (f" or [{B}, {tokens}, axes]" if B else "") + f", got {tuple(positions.shape)}")
    _ha._fit_int32(rot_dim=2 * freq.numel(), n_axes=positions.shape[-1])
    stride = tokens * positions.shape[-1] if positions.dim() == 3 and B > 1 else 0
    return ha_rotary(freq.data_ptr(), None if axis is None else axis.data_ptr(), positions.data_ptr(), stride, 2 * freq.numel(), int(bool(interleaved)),
                     positions.shape[-1], magnitude)


def _rows_problem(q, k, eps=0.0) -> ha_rows_problem:
    if q.dim() != 4:
        raise ValueError(f"q must be a [B, H, N, d] view, got {tuple(q.shape)}")
    B, H, N, d = q.shape
    if k is not None and (k.dim() != 4 or (k.shape[0], k.shape[2], k.shape[3]) != (B, N, d)):
        raise ValueError(f"k must be [B={B}, H_kv, N={N}, d={d}], got {tuple(k.shape)}")
    Hkv = 0 if k is None else k.shape[1]
    _ha._fit_int32(B=B, H=H, H_kv=Hkv, N=N, d=d)
    return ha_rows_problem(B, H, Hkv, N, d, _ha._dtype_code(q), eps)


def _weight(name, w, d, device):
    if w is None:
        return None
    _bs._float32(name, w, (d,), device)
    return w.data_ptr()


def _output(name, given, like):
    """The tensor that is given for an output of like's shape, or a new one."""
    if given is None:
        return None if like is None else _bs._dense_like(like)
    if like is None:
        raise ValueError(f"{name} is given, but no keys are")
    _bs._same(like, ((name, given),))
    _bs._like_heads(name, given, like.shape)
    return given


def _view(t):
    return None if t is None else _bs._view(t)


def hybrid_attn_rotary_validate(problem: ha_rows_problem, rotary: ha_rotary) -> int:
    return _ha._lib().hybrid_attn_rotary_validate(problem, rotary)


def hybrid_attn_norm_rotate_grad_workspace_bytes(problem: ha_rows_problem) -> int:
    return _ha._lib().hybrid_attn_norm_rotate_grad_workspace_bytes(problem)


def hybrid_attn_rotate(x, rotary: Rotary, positions, out=None, stream=None):
    """Rotation of x [B, H, N, d] by positions, int32 [N, axes] or [B, N, axes]; out may be x itself.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.rotate(x, rotary, positions, False, out, stream)) is not None:
        return done
    return _rotate(x, rotary, positions, False, out, stream)


def hybrid_attn_rotate_grad(grad_out, rotary: Rotary, positions, out=None, stream=None):
    """Gradient of hybrid_attn_rotate's x from that of its result: the transposed rotation.  out may be grad_out itself.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.rotate(grad_out, rotary, positions, True, out, stream)) is not None:
        return done
    return _rotate(grad_out, rotary, positions, True, out, stream)


@_ha._allocations_follow_stream
def _rotate(x, rotary, positions, transposed, out, stream):
    _ha._require_gpu(x, out)
    with _ha._on_device_of(x):
        prob = _rows_problem(x, None)
        rot = _rotary_struct(rotary, positions, x.shape[2], x.device, x.shape[0])
        lib = _ha._lib()
        _bs._check(lib.hybrid_attn_rotary_validate(prob, rot), "hybrid_attn_rotary_validate")
        out = _output("out", out, x)
        _bs._check(lib.hybrid_attn_rotate(prob, rot, _view(x), _view(out), int(transposed), _ha._stream_handle(stream, x)), "hybrid_attn_rotate")
    return out


def hybrid_attn_norm_rotate(q, k, w_q=None, w_k=None, rotary: Optional[Rotary] = None, positions=None, eps: float = 1e-6, q_out=None, k_out=None, stream=None):
    """Queries and keys (k may be None) divided by the root of every row's mean square, times the weights (fp32 [d], or None), and rotated (rotary None: not): returns
    (q_out, k_out), which may be q and k themselves.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.norm_rotate(q, k, w_q, w_k, rotary, positions, eps, q_out, k_out, stream)) is not None:
        return done
    return _norm_rotate(q, k, w_q, w_k, rotary, positions, eps, q_out, k_out, stream)


@_ha._allocations_follow_stream
def _norm_rotate(q, k, w_q, w_k, rotary, positions, eps, q_out, k_out, stream):
    _ha._require_gpu(q, k, w_q, w_k, q_out, k_out)
    with _ha._on_device_of(q):
        prob = _rows_problem(q, k, eps)
        _bs._same(q, (("k", k),))
        rot = _rotary_struct(rotary, positions, q.shape[2], q.device, q.shape[0])
        lib = _ha._lib()
        _bs._check(lib.hybrid_attn_rotary_validate(prob, rot), "hybrid_attn_rotary_validate")
        w_q, w_k = _weight("w_q", w_q, q.shape[3], q.device), _weight("w_k", w_k, q.shape[3], q.device)
        q_out, k_out = _output("q_out", q_out, q), _output("k_out", k_out, k)
        _bs._check(lib.hybrid_attn_norm_rotate(prob, rot, _view(q), _view(k), w_q, w_k, _view(q_out), _view(k_out), _ha._stream_handle(stream, q)),
                   "hybrid_attn_norm_rotate")
    return q_out, k_out


def hybrid_attn_norm_rotate_grad(grad_q, grad_k, q, k, w_q=None, w_k=None, rotary: Optional[Rotary] = None, positions=None, eps: float = 1e-6, grad_in_q=None,
                                 grad_in_k=None, grad_w_q=None, grad_w_k=None, workspace=None, stream=None):
    """Gradients of q, k, w_q and w_k from those of hybrid_attn_norm_rotate's results; q, k and the rest as that took them.  Returns (grad_in_q, grad_in_k, grad_w_q,
    grad_w_k), the last two fp32 [d], each None where its tensor is.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.norm_rotate_grad(grad_q, grad_k, q, k, w_q, w_k, rotary, positions, eps, grad_in_q, grad_in_k, grad_w_q, grad_w_k, workspace, stream)) is not None:
        return done
    return _norm_rotate_grad(grad_q, grad_k, q, k, w_q, w_k, rotary, positions, eps, grad_in_q, grad_in_k, grad_w_q, grad_w_k, workspace, stream)


@_ha._allocations_follow_stream
def _norm_rotate_grad(grad_q, grad_k, q, k, w_q, w_k, rotary, positions, eps, grad_in_q, grad_in_k, grad_w_q, grad_w_k, workspace, stream):
    _ha._require_gpu(grad_q, grad_k, q, k, w_q, w_k, grad_in_q, grad_in_k, grad_w_q, grad_w_k, workspace)
    if (grad_k is None) != (k is None):
        raise ValueError("grad_k and k must both be given, or neither")
    with _ha._on_device_of(q):
        prob = _rows_problem(q, k, eps)
        _bs._same(q, (("k", k), ("grad_q", grad_q), ("grad_k", grad_k)))
        _bs._like_heads("grad_q", grad_q, q.shape)
        if k is not None:
            _bs._like_heads("grad_k", grad_k, k.shape)
        d = q.shape[3]
        rot = _rotary_struct(rotary, positions, q.shape[2], q.device, q.shape[0])
        lib = _ha._lib()
        _bs._check(lib.hybrid_attn_rotary_validate(prob, rot), "hybrid_attn_rotary_validate")
        sums = []
        for name, w, g, there in (("grad_w_q", w_q, grad_w_q, True), ("grad_w_k", w_k, grad_w_k, k is not None)):
            if w is None and g is not None:
                raise ValueError(f"{name} is given, but its weight is not")
            if w is not None and g is None and there:
                g = torch.empty(d, dtype=torch.float32, device=q.device)
            sums.append((g, _weight(name, g, d, q.device) if there else None))
        w_q, w_k = _weight("w_q", w_q, d, q.device), _weight("w_k", w_k, d, q.device)
        grad_in_q, grad_in_k = _output("grad_in_q", grad_in_q, q), _output("grad_in_k", grad_in_k, k)
        need = lib.hybrid_attn_norm_rotate_grad_workspace_bytes(prob) if sums[0][1] or sums[1][1] else 0
        workspace = _bs._workspace(need, workspace, q.device)
        _bs._check(lib.hybrid_attn_norm_rotate_grad(prob, rot, _view(grad_q), _view(grad_k), _view(q), _view(k), w_q, w_k, _view(grad_in_q), _view(grad_in_k), sums[0][1],
                                                    sums[1][1], workspace.data_ptr(), workspace.numel() * workspace.element_size(), _ha._stream_handle(stream, q)),
                   "hybrid_attn_norm_rotate_grad")
    return grad_in_q, grad_in_k, sums[0][0], sums[1][0] if k is not None else None
