"""Block-sparse attention (include/hybrid_attn_sparse.h): block means of the keys, choice of key blocks, forward and gradients.

    means = hybrid_attn_key_means(k)
    blocks = hybrid_attn_select_blocks(q, means, k.shape[2], n_select)
    out, lse = hybrid_attn_sparse_forward(q, k, v, blocks, with_lse=True)
    dq, dk, dv = hybrid_attn_sparse_grad(q, k, v, blocks, out, lse, grad_out)

q is a [B, H, N_q, d] view, k and v are [B, H_kv, N_k, d] views (H a multiple of H_kv), each with strides of its own and a contiguous last dimension.
Argument marshalling only, as in hybrid_attn; everything is public there.  Plain calls are marshalled by compiled code (csrc/ha_binding_calls.h), all others, and
every error, here.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import hybrid_attn as _ha


class ha_sparse_problem(ctypes.Structure):
    _fields_ = [*((n, ctypes.c_int32) for n in ("B", "H", "H_kv", "N_q", "N_k", "d_head", "dtype", "q_block", "k_block", "n_select", "causal", "keep_first",
                                                "near_tokens")),
                ("softmax_scale", ctypes.c_float), ("q_start", ctypes.c_void_p), ("key_len", ctypes.c_void_p)]


class ha_view(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


_P, _V, _vp, _sz = ctypes.POINTER(ha_sparse_problem), ctypes.POINTER(ha_view), ctypes.c_void_p, ctypes.c_size_t
SIGNATURES = (
    ("hybrid_attn_sparse_validate", [_P], ctypes.c_int),
    ("hybrid_attn_key_means", [_P, _V, ctypes.c_int32, _vp, _vp], ctypes.c_int),
    ("hybrid_attn_select_workspace_bytes", [_P], _sz),
    ("hybrid_attn_select_blocks", [_P, _V, _vp, _vp, _vp, _sz, _vp], ctypes.c_int),
    ("hybrid_attn_sparse_workspace_bytes", [_P], _sz),
    ("hybrid_attn_sparse_forward", [_P, _V, _V, _V, _vp, _V, _vp, _vp, _sz, _vp], ctypes.c_int),
    ("hybrid_attn_sparse_grad_workspace_bytes", [_P], _sz),
    ("hybrid_attn_sparse_grad", [_P, _V, _V, _V, _vp, _V, _vp, _V, _V, _V, _V, _vp, _sz, _vp], ctypes.c_int),
)


def _view(t: torch.Tensor) -> ha_view:
    sb, sh, sn, sd = t.stride()
    if sd != 1 and t.shape[3] > 1:
        raise ValueError("q, k, v and the gradients must have a contiguous last dimension")
    return ha_view(t.data_ptr(), sb, sh, sn)


def _per_entry(t: Optional[torch.Tensor], name: str, B: int, device) -> Optional[int]:
    """Address of an int32 tensor [B] (key_len, q_start), or None."""
    if t is None:
        return None
    if t.dtype != torch.int32 or tuple(t.shape) != (B,) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor [{B}] on {device}")
    return t.data_ptr()


def make_sparse_problem(q_shape, k_shape, dtype, device, q_block=128, k_block=64, n_select=1, causal=False, q_start=None, key_len=None, keep_first=0, near=-1,
                        softmax_scale=None) -> ha_sparse_problem:
    """ha_sparse_problem for q [B, H, N_q, d] and k [B, H_kv, N_k, d] of `dtype` on `device`."""
    if len(q_shape) != 4 or len(k_shape) != 4 or q_shape[0] != k_shape[0] or q_shape[3] != k_shape[3]:
        raise ValueError(f"q must be [B, H, N_q, d] and k [B, H_kv, N_k, d] with one B and d, got {tuple(q_shape)} and {tuple(k_shape)}")
    B, H, Nq, d = q_shape
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}: q, k, v must be bfloat16 or float32")
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    _ha._fit_int32(B=B, H=H, H_kv=k_shape[1], N_q=Nq, N_k=k_shape[2], d=d, q_block=q_block, k_block=k_block, n_select=n_select, keep_first=keep_first, near=near)
    return ha_sparse_problem(B, H, k_shape[1], Nq, k_shape[2], d, _ha.HA_BF16 if dtype == torch.bfloat16 else _ha.HA_F32, q_block, k_block, n_select,
                             int(bool(causal)), keep_first, near, softmax_scale, _per_entry(q_start, "q_start", B, device), _per_entry(key_len, "key_len", B, device))


def _check(status: int, where: str) -> None:
    if status != _ha.HA_OK:
        raise _ha.HybridAttnError(status, where)


def _same(q, named):
    for name, t in named:
        if t is not None and (t.device != q.device or t.dtype != q.dtype):
            raise ValueError(f"{name} must be {q.dtype} on {q.device}, got {t.dtype} on {t.device}")


def _like_heads(name, t, shape):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")


def _int32(name, t, shape, device):
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor {tuple(shape)} on {device}")


def _float32(name, t, shape, device):
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous fp32 tensor {tuple(shape)} on {device}")


def _workspace(need, workspace, device):
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace


def _cdiv(a, b):
    return -(-a // b)


def hybrid_attn_sparse_validate(problem: ha_sparse_problem) -> int:
    return _ha._lib().hybrid_attn_sparse_validate(problem)


def hybrid_attn_select_workspace_bytes(problem: ha_sparse_problem) -> int:
    return _ha._lib().hybrid_attn_select_workspace_bytes(problem)


def hybrid_attn_sparse_workspace_bytes(problem: ha_sparse_problem) -> int:
    return _ha._lib().hybrid_attn_sparse_workspace_bytes(problem)


def hybrid_attn_sparse_grad_workspace_bytes(problem: ha_sparse_problem) -> int:
    return _ha._lib().hybrid_attn_sparse_grad_workspace_bytes(problem)


def hybrid_attn_key_means(k, k_block: int = 64, key_len=None, only_last: int = 0, out=None, stream=None):
    """Mean of the keys of every block (those below key_len, int32 [B] or None: all): fp32 [B, H_kv, ceil(N_k / k_block), d].  only_last = m > 0 writes only
    the last m blocks of every batch entry that hold a key, into `out`, which then has to be given.  Does not synchronise."""
    native = _ha._CALLS or _ha._calls()
    if native and (means := native.key_means(k, k_block, key_len, only_last, out, stream)) is not None:
        return means
    return _key_means(k, k_block, key_len, only_last, out, stream)


@_ha._allocations_follow_stream
def _key_means(k, k_block, key_len, only_last, out, stream):
    _ha._require_gpu(k, out)
    if k.dim() != 4:
        raise ValueError("k must be a [B, H_kv, N_k, d] view")
    if only_last > 0 and out is None:
        raise ValueError("only_last needs out: the other blocks' means are left as they are")
    _ha._fit_int32(only_last=only_last)
    with _ha._on_device_of(k):
        B, H_kv, N_k, d = k.shape
        prob = make_sparse_problem((B, H_kv, 0, d), k.shape, k.dtype, k.device, k_block=k_block, key_len=key_len)      # (no queries: their limits are not the means')
        lib = _ha._lib()
        _check(lib.hybrid_attn_sparse_validate(prob), "hybrid_attn_sparse_validate")
        shape = (B, H_kv, _cdiv(N_k, k_block), d)
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=k.device)
        _float32("out", out, shape, k.device)
        _check(lib.hybrid_attn_key_means(prob, _view(k), only_last, out.data_ptr(), _ha._stream_handle(stream, k)), "hybrid_attn_key_means")
    return out


def hybrid_attn_select_blocks(q, means, n_keys: int, n_select: int, q_block: int = 128, k_block: int = 64, causal: bool = False, q_start=None, key_len=None,
                              keep_first: int = 0, near: int = -1, out=None, workspace=None, stream=None):
    """The n_select key blocks of highest score (sum of the tile's queries times the block's mean) for every tile of q_block queries: int32
    [B, H_kv, ceil(N_q / q_block), n_select] in rising order, -1 behind the last.  n_keys: N_k.  keep_first leading blocks and, with near >= 0, those
    within `near` tokens of the tile's positions are always among them.  Does not synchronise."""
    native = _ha._CALLS or _ha._calls()
    if native and (blocks := native.select_blocks(q, means, n_keys, n_select, q_block, k_block, causal, q_start, key_len, keep_first, near, out, workspace, stream)) is not None:
        return blocks
    return _select_blocks(q, means, n_keys, n_select, q_block, k_block, causal, q_start, key_len, keep_first, near, out, workspace, stream)


@_ha._allocations_follow_stream
def _select_blocks(q, means, n_keys, n_select, q_block, k_block, causal, q_start, key_len, keep_first, near, out, workspace, stream):
    _ha._require_gpu(q, means, out, workspace)
    if q.dim() != 4 or means.dim() != 4:
        raise ValueError("q must be a [B, H, N_q, d] view and means [B, H_kv, blocks, d]")
    with _ha._on_device_of(q):
        k_shape = (means.shape[0], means.shape[1], n_keys, means.shape[3])
        prob = make_sparse_problem(q.shape, k_shape, q.dtype, q.device, q_block, k_block, n_select, causal, q_start, key_len, keep_first, near)
        lib = _ha._lib()
        _check(lib.hybrid_attn_sparse_validate(prob), "hybrid_attn_sparse_validate")
        _float32("means", means, (*k_shape[:2], _cdiv(n_keys, k_block), k_shape[3]), q.device)
        shape = (q.shape[0], k_shape[1], _cdiv(q.shape[2], q_block), n_select)
        if out is None:
            out = torch.empty(shape, dtype=torch.int32, device=q.device)
        _int32("out", out, shape, q.device)
        workspace = _workspace(lib.hybrid_attn_select_workspace_bytes(prob), workspace, q.device)
        _check(lib.hybrid_attn_select_blocks(prob, _view(q), means.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                             _ha._stream_handle(stream, q)), "hybrid_attn_select_blocks")
    return out


def _attention_problem(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale):
    if q.dim() != 4 or k.dim() != 4 or blocks.dim() != 4:
        raise ValueError("q must be [B, H, N_q, d], k and v [B, H_kv, N_k, d] and blocks [B, H_kv, tiles, n_select]")
    _same(q, (("k", k), ("v", v)))
    _like_heads("v", v, k.shape)
    prob = make_sparse_problem(q.shape, k.shape, q.dtype, q.device, q_block, k_block, blocks.shape[3], causal, q_start, key_len, softmax_scale=softmax_scale)
    _check(_ha._lib().hybrid_attn_sparse_validate(prob), "hybrid_attn_sparse_validate")
    _int32("blocks", blocks, (q.shape[0], k.shape[1], _cdiv(q.shape[2], q_block), blocks.shape[3]), q.device)
    return prob


def hybrid_attn_sparse_forward(q, k, v, blocks, q_block: int = 128, k_block: int = 64, causal: bool = False, q_start=None, key_len=None,
                               softmax_scale: Optional[float] = None, with_lse: bool = False, out=None, lse=None, workspace=None, stream=None):
    """Softmax attention of every query over the keys of its tile's blocks; returns (out, lse): out like q, lse fp32 [B, H, N_q] (the logarithm of every
    row's sum of weights, what the gradients take) or None without with_lse.  causal: query i, at position q_start[b] + i (int32 [B], or None:
    N_k - N_q + i), sees the keys up to its own position; keys at and behind key_len (int32 [B], or None) are never seen.  Does not synchronise."""
    native = _ha._CALLS or _ha._calls()
    if native and (pair := native.sparse_forward(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale, with_lse, out, lse, workspace, stream)) is not None:
        return pair
    return _sparse_forward(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale, with_lse, out, lse, workspace, stream)


@_ha._allocations_follow_stream
def _sparse_forward(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale, with_lse, out, lse, workspace, stream):
    _ha._require_gpu(q, k, v, blocks, out, lse, workspace)
    with _ha._on_device_of(q):
        prob = _attention_problem(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale)
        lib = _ha._lib()
        if out is None:
            out = _dense_like(q)
        _same(q, (("out", out),))
        _like_heads("out", out, q.shape)
        if lse is None and with_lse:
            lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        if lse is not None:
            _float32("lse", lse, q.shape[:3], q.device)
        workspace = _workspace(lib.hybrid_attn_sparse_workspace_bytes(prob), workspace, q.device)
        _check(lib.hybrid_attn_sparse_forward(prob, _view(q), _view(k), _view(v), blocks.data_ptr(), _view(out), None if lse is None else lse.data_ptr(),
                                              workspace.data_ptr(), workspace.numel() * workspace.element_size(), _ha._stream_handle(stream, q)),
               "hybrid_attn_sparse_forward")
    return out, lse


def hybrid_attn_sparse_grad(q, k, v, blocks, out, lse, grad_out, q_block: int = 128, k_block: int = 64, causal: bool = False, q_start=None, key_len=None,
                            softmax_scale: Optional[float] = None, grad_q=None, grad_k=None, grad_v=None, workspace=None, stream=None):
    """Gradients of q, k and v (in their dtype) from that of `out`; out and lse as hybrid_attn_sparse_forward returned them for the same
    arguments.  Returns (grad_q, grad_k, grad_v).  Does not synchronise."""
    native = _ha._CALLS or _ha._calls()
    if native and (grads := native.sparse_grad(q, k, v, blocks, out, lse, grad_out, q_block, k_block, causal, q_start, key_len, softmax_scale, grad_q, grad_k, grad_v,
                                               workspace, stream)) is not None:
        return grads
    return _sparse_grad(q, k, v, blocks, out, lse, grad_out, q_block, k_block, causal, q_start, key_len, softmax_scale, grad_q, grad_k, grad_v, workspace, stream)


@_ha._allocations_follow_stream
def _sparse_grad(q, k, v, blocks, out, lse, grad_out, q_block, k_block, causal, q_start, key_len, softmax_scale, grad_q, grad_k, grad_v, workspace, stream):
    _ha._require_gpu(q, k, v, blocks, out, lse, grad_out, grad_q, grad_k, grad_v, workspace)
    with _ha._on_device_of(q):
        prob = _attention_problem(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale)
        lib = _ha._lib()
        _float32("lse", lse, q.shape[:3], q.device)
        grad_q = _dense_like(q) if grad_q is None else grad_q
        grad_k = _dense_like(k) if grad_k is None else grad_k
        grad_v = _dense_like(v) if grad_v is None else grad_v
        named = (("out", out, q), ("grad_out", grad_out, q), ("grad_q", grad_q, q), ("grad_k", grad_k, k), ("grad_v", grad_v, v))
        _same(q, [(n, t) for n, t, _ in named])
        for n, t, like in named:
            _like_heads(n, t, like.shape)
        workspace = _workspace(max(256, lib.hybrid_attn_sparse_grad_workspace_bytes(prob)), workspace, q.device)
        _check(lib.hybrid_attn_sparse_grad(prob, _view(q), _view(k), _view(v), blocks.data_ptr(), _view(out), lse.data_ptr(), _view(grad_out), _view(grad_q),
                                           _view(grad_k), _view(grad_v), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                           _ha._stream_handle(stream, q)), "hybrid_attn_sparse_grad")
    return grad_q, grad_k, grad_v


def _dense_like(t):
    """A new tensor in the order of t's dimensions in memory, without its gaps and broadcast dimensions."""
    order = sorted(range(3), key=lambda i: (-t.stride(i), i)) + [3]
    back = [order.index(i) for i in range(4)]
    return torch.empty([t.shape[i] for i in order], dtype=t.dtype, device=t.device).permute(back)
