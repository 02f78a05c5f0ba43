"""Caches of keys and values in pages (include/hybrid_attn_paged.h): storing new tokens, attention of new tokens over all that is stored, the weight that every stored
token gets in it, and eviction by that weight.

    where = dict(k_pages=k_pages, v_pages=v_pages, page_table=table, key_len=length, q_offset=offset)       # length counts the new tokens
    q = hybrid_attn_paged_append(q, k, v, **where, w_q=w_q, w_k=w_k, rotary=rotary, positions=positions, eps=1e-6)
    out, lse = hybrid_attn_paged_forward(q, **where, with_lse=True)
    hybrid_attn_paged_weights(q, k_pages, lse, weights, table, length, offset)
    length, weights, kept = hybrid_attn_paged_evict(k_pages, v_pages, weights, table, length, keep, new_table, keep_first=4, keep_last=256)

q is a [T, H, d] view of the new tokens of all sequences, one behind the other (those of sequence b from q_offset[b] on; q_offset None: the same number each), k and v are
[T, H_kv, d], and the pools k_pages and v_pages are [n_pages, H_kv, page, d] views, each with strides of its own and a contiguous last dimension.  page_table int32
[B, max_pages], key_len int32 [B], q_offset int32 [B + 1].  Argument marshalling only, as in hybrid_attn; everything is public there.  Plain calls are marshalled by compiled code
(csrc/ha_binding_rows.h), all others, and every error, here.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import block_sparse as _bs
from . import hybrid_attn as _ha
from . import rotary as _rot


class ha_paged_problem(ctypes.Structure):
    _fields_ = [*((n, ctypes.c_int32) for n in ("B", "H", "H_kv", "T", "d_head", "dtype", "n_pages", "page", "max_pages", "max_new", "causal")),
                ("softmax_scale", ctypes.c_float), ("page_table", ctypes.c_void_p), ("key_len", ctypes.c_void_p), ("q_offset", ctypes.c_void_p)]


_P, _R, _V, _vp, _sz, _i = (ctypes.POINTER(ha_paged_problem), ctypes.POINTER(_rot.ha_rotary), ctypes.POINTER(_bs.ha_view), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32)
SIGNATURES = (
    ("hybrid_attn_paged_validate", [_P], ctypes.c_int),
    ("hybrid_attn_paged_append", [_P, _R, _i, ctypes.c_float, _V, _V, _V, _vp, _vp, _V, _V, _V, _vp], ctypes.c_int),
    ("hybrid_attn_paged_workspace_bytes", [_P], _sz),
    ("hybrid_attn_paged_forward", [_P, _V, _V, _V, _V, _vp, _vp, _sz, _vp], ctypes.c_int),
    ("hybrid_attn_paged_weights_workspace_bytes", [_P], _sz),
    ("hybrid_attn_paged_weights", [_P, _V, _V, _vp, _vp, _vp, _vp, _sz, _vp], ctypes.c_int),
    ("hybrid_attn_paged_evict_workspace_bytes", [_P, _i], _sz),
    ("hybrid_attn_paged_evict", [_P, _i, _i, _i, _vp, _vp, _i, _V, _V, _vp, _vp, _vp, _vp, _sz, _vp], ctypes.c_int),
)


def make_paged_problem(q_shape, pages_shape, dtype, device, page_table, key_len, q_offset=None, max_new=None, causal=True, softmax_scale=None) -> ha_paged_problem:
    """ha_paged_problem for q [T, H, d] and pools [n_pages, H_kv, page, d] of `dtype` on `device`.  max_new None: T with q_offset, T / B without."""
    if len(q_shape) != 3 or len(pages_shape) != 4 or q_shape[2] != pages_shape[3]:
        raise ValueError(f"q must be [T, H, d] and the pools [n_pages, H_kv, page, d] with one d, got {tuple(q_shape)} and {tuple(pages_shape)}")
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}: q and the pools must be bfloat16 or float32")
    if page_table.dim() != 2:
        raise ValueError("page_table must be int32 [B, max_pages]")
    B, max_pages = page_table.shape
    T, H, d = q_shape
    _bs._int32("page_table", page_table, (B, max_pages), device)
    if max_new is None:
        if q_offset is None and (B == 0 or T % B):
            raise ValueError(f"without q_offset every sequence has the same number of new tokens: {T} rows are no multiple of {B}")
        max_new = T // B if q_offset is None else T
    if softmax_scale is None:
        softmax_scale = float(d) ** -0.5
    n_pages, H_kv, page, _ = pages_shape
    _ha._fit_int32(B=B, H=H, H_kv=H_kv, T=T, d=d, n_pages=n_pages, page=page, max_pages=max_pages, max_new=max_new)
    return ha_paged_problem(B, H, H_kv, T, d, _ha.HA_BF16 if dtype == torch.bfloat16 else _ha.HA_F32, n_pages, page, max_pages, max_new, int(bool(causal)), softmax_scale,
                            page_table.data_ptr(), _bs._per_entry(key_len, "key_len", B, device), _bs._per_entry(q_offset, "q_offset", B + 1, device))


def _packed(name, t):
    """View of [T, heads, d] rows."""
    if t is None:
        return None
    if t.dim() != 3:
        raise ValueError(f"{name} must be [T, heads, d], got {tuple(t.shape)}")
    st, sh, sd = t.stride()
    if sd != 1 and t.shape[2] > 1:
        raise ValueError(f"{name} must have a contiguous last dimension")
    return _bs.ha_view(t.data_ptr(), 0, sh, st)


def _packed_like(t):
    """A new tensor of t's shape in the order of its dimensions in memory, without its gaps and broadcast dimensions."""
    return torch.empty_like(t, memory_format=torch.contiguous_format) if t.stride(0) >= t.stride(1) else torch.empty_like(t.transpose(0, 1), memory_format=torch.contiguous_format).transpose(0, 1)


def _pools(q, k_pages, v_pages=None):
    _bs._same(q, (("k_pages", k_pages), ("v_pages", v_pages)))
    if k_pages.dim() != 4 or (v_pages is not None and v_pages.shape != k_pages.shape):
        raise ValueError("k_pages and v_pages must be [n_pages, H_kv, page, d] views of one shape")


def _slots(prob):
    return prob.B, prob.H_kv, prob.max_pages * prob.page


def hybrid_attn_paged_validate(problem: ha_paged_problem) -> int:
    return _ha._lib().hybrid_attn_paged_validate(problem)


def hybrid_attn_paged_workspace_bytes(problem: ha_paged_problem) -> int:
    return _ha._lib().hybrid_attn_paged_workspace_bytes(problem)


def hybrid_attn_paged_weights_workspace_bytes(problem: ha_paged_problem) -> int:
    return _ha._lib().hybrid_attn_paged_weights_workspace_bytes(problem)


def hybrid_attn_paged_evict_workspace_bytes(problem: ha_paged_problem, keep: int) -> int:
    _ha._fit_int32(keep=keep)
    return _ha._lib().hybrid_attn_paged_evict_workspace_bytes(problem, keep)


def _checked(*args, **kwargs):
    prob = make_paged_problem(*args, **kwargs)
    lib = _ha._lib()
    _bs._check(lib.hybrid_attn_paged_validate(prob), "hybrid_attn_paged_validate")
    return lib, prob


def hybrid_attn_paged_append(q, k, v, k_pages, v_pages, page_table, key_len, q_offset=None, max_new: Optional[int] = None, w_q=None, w_k=None,
                             rotary: Optional[_rot.Rotary] = None, positions=None, eps: Optional[float] = None, q_out=None, stream=None):
    """Store the new tokens' k and v [T, H_kv, d] in their slots (key_len counts them already) and return the queries that go with them; q may be None.  eps: queries and keys
    are normed for each head first, with the weights w_q and w_k (fp32 [d], or None); None: not.  rotary: they are rotated by positions, int32 [T, axes]; None: not.
    q_out may be q itself.  max_new: the most new tokens that a sequence has.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.paged_append(q, k, v, k_pages, v_pages, page_table, key_len, q_offset, max_new, w_q, w_k, rotary, positions, eps, q_out, stream)) is not None:
        return done[0]
    return _append(q, k, v, k_pages, v_pages, page_table, key_len, q_offset, max_new, w_q, w_k, rotary, positions, eps, q_out, stream)


@_ha._allocations_follow_stream
def _append(q, k, v, k_pages, v_pages, page_table, key_len, q_offset, max_new, w_q, w_k, rotary, positions, eps, q_out, stream):
    _ha._require_gpu(q, k, v, k_pages, v_pages, page_table, key_len, q_offset, w_q, w_k, positions, q_out)
    if eps is None and (w_q is not None or w_k is not None):
        raise ValueError("w_q and w_k are the norm's, which eps=None leaves out")
    if k.dim() != 3:
        raise ValueError(f"k must be [T, H_kv, d], got {tuple(k.shape)}")
    with _ha._on_device_of(k):
        _pools(k, k_pages, v_pages)
        _bs._same(k, (("q", q), ("v", v), ("q_out", q_out)))
        lib, prob = _checked(k.shape if q is None else q.shape, k_pages.shape, k.dtype, k.device, page_table, key_len, q_offset, max_new)
        T, d = prob.T, prob.d_head
        for name, t in (("k", k), ("v", v)):
            _bs._like_heads(name, t, (T, prob.H_kv, d))
        if q is None and q_out is not None:
            raise ValueError("q_out is given, but no queries are")
        if q is not None:
            q_out = _packed_like(q) if q_out is None else q_out
            _bs._like_heads("q_out", q_out, q.shape)
        rot = _rot._rotary_struct(rotary, positions, T, k.device, 0)
        w_q, w_k = _rot._weight("w_q", w_q, d, k.device), _rot._weight("w_k", w_k, d, k.device)
        _bs._check(lib.hybrid_attn_paged_append(prob, rot, int(eps is not None), 0.0 if eps is None else eps, _packed("q", q), _packed("k", k), _packed("v", v), w_q, w_k,
                                                _bs._view(k_pages), _bs._view(v_pages), _packed("q_out", q_out), _ha._stream_handle(stream, k)), "hybrid_attn_paged_append")
    return q_out


def hybrid_attn_paged_forward(q, k_pages, v_pages, page_table, key_len, q_offset=None, max_new: Optional[int] = None, causal: bool = True,
                              softmax_scale: Optional[float] = None, with_lse: bool = False, out=None, lse=None, workspace=None, stream=None):
    """Softmax attention of the new tokens q [T, H, d] over the slots of their sequences; returns (out, lse): out like q, lse fp32 [T, H] (the logarithm of every row's
    sum of weights) or None without with_lse.  causal: a new token sees the slots up to its own, otherwise all.  Rows of no sequence are left as they were.
    Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.paged_forward(q, k_pages, v_pages, page_table, key_len, q_offset, max_new, causal, softmax_scale, with_lse, out, lse, workspace, stream)) is not None:
        return done
    return _forward(q, k_pages, v_pages, page_table, key_len, q_offset, max_new, causal, softmax_scale, with_lse, out, lse, workspace, stream)


@_ha._allocations_follow_stream
def _forward(q, k_pages, v_pages, page_table, key_len, q_offset, max_new, causal, softmax_scale, with_lse, out, lse, workspace, stream):
    _ha._require_gpu(q, k_pages, v_pages, page_table, key_len, q_offset, out, lse, workspace)
    with _ha._on_device_of(q):
        _pools(q, k_pages, v_pages)
        lib, prob = _checked(q.shape, k_pages.shape, q.dtype, q.device, page_table, key_len, q_offset, max_new, causal, softmax_scale)
        if out is None:
            out = _packed_like(q)
        _bs._same(q, (("out", out),))
        _bs._like_heads("out", out, q.shape)
        if lse is None and with_lse:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        if lse is not None:
            _bs._float32("lse", lse, q.shape[:2], q.device)
        workspace = _bs._workspace(lib.hybrid_attn_paged_workspace_bytes(prob), workspace, q.device)
        _bs._check(lib.hybrid_attn_paged_forward(prob, _packed("q", q), _bs._view(k_pages), _bs._view(v_pages), _packed("out", out), None if lse is None else lse.data_ptr(),
                                                 workspace.data_ptr(), workspace.numel() * workspace.element_size(), _ha._stream_handle(stream, q)),
                   "hybrid_attn_paged_forward")
    return out, lse


def hybrid_attn_paged_weights(q, k_pages, lse, weights, page_table, key_len, q_offset=None, max_new: Optional[int] = None, causal: bool = True,
                              softmax_scale: Optional[float] = None, out=None, workspace=None, stream=None):
    """Add the weight that every slot got in hybrid_attn_paged_forward, from its queries and lse and the same arguments, to what it has had: weights fp32
    [B, H_kv, max_pages page], or None: nothing so far.  The sums go to out, or to weights itself; returned.  Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.paged_weights(q, k_pages, lse, weights, page_table, key_len, q_offset, max_new, causal, softmax_scale, out, workspace, stream)) is not None:
        return done
    return _weights(q, k_pages, lse, weights, page_table, key_len, q_offset, max_new, causal, softmax_scale, out, workspace, stream)


@_ha._allocations_follow_stream
def _weights(q, k_pages, lse, weights, page_table, key_len, q_offset, max_new, causal, softmax_scale, out, workspace, stream):
    _ha._require_gpu(q, k_pages, lse, weights, page_table, key_len, q_offset, out, workspace)
    with _ha._on_device_of(q):
        _pools(q, k_pages)
        lib, prob = _checked(q.shape, k_pages.shape, q.dtype, q.device, page_table, key_len, q_offset, max_new, causal, softmax_scale)
        _bs._float32("lse", lse, q.shape[:2], q.device)
        if out is None:
            out = torch.empty(_slots(prob), dtype=torch.float32, device=q.device) if weights is None else weights
        for name, t in (("weights", weights), ("out", out)):
            if t is not None:
                _bs._float32(name, t, _slots(prob), q.device)
        workspace = _bs._workspace(lib.hybrid_attn_paged_weights_workspace_bytes(prob), workspace, q.device)
        _bs._check(lib.hybrid_attn_paged_weights(prob, _packed("q", q), _bs._view(k_pages), lse.data_ptr(), None if weights is None else weights.data_ptr(), out.data_ptr(),
                                                 workspace.data_ptr(), workspace.numel() * workspace.element_size(), _ha._stream_handle(stream, q)),
                   "hybrid_attn_paged_weights")
    return out


def hybrid_attn_paged_evict(k_pages, v_pages, weights, page_table, key_len, keep: int, out_table, keep_first: int = 0, keep_last: int = 0, len_out=None, weights_out=None,
                            kept=None, workspace=None, stream=None):
    """Copy the `keep` slots of every sequence and key head that matter most to slots 0, 1, .. of the pages of out_table (int32 [B, out_pages]), in their order: the first
    keep_first, the last keep_last, and the others of the largest weights (fp32 [B, H_kv, max_pages page]), of equal ones the lower slot.  Returns (int32 [B] slots that
    stay, their weights with zeros behind them, int32 [B, H_kv, keep] which slots stayed with -1 behind them); len_out and weights_out may not lie on key_len and weights.
    Does not synchronise."""
    native = _ha._ROWS or _ha._rows()
    if native and (done := native.paged_evict(k_pages, v_pages, weights, page_table, key_len, keep, out_table, keep_first, keep_last, len_out, weights_out, kept, workspace, stream)) is not None:
        return done
    return _evict(k_pages, v_pages, weights, page_table, key_len, keep, out_table, keep_first, keep_last, len_out, weights_out, kept, workspace, stream)


@_ha._allocations_follow_stream
def _evict(k_pages, v_pages, weights, page_table, key_len, keep, out_table, keep_first, keep_last, len_out, weights_out, kept, workspace, stream):
    _ha._require_gpu(k_pages, v_pages, weights, page_table, key_len, out_table, len_out, weights_out, kept, workspace)
    with _ha._on_device_of(k_pages):
        _pools(k_pages, k_pages, v_pages)
        H_kv, d, device = k_pages.shape[1], k_pages.shape[3], k_pages.device
        lib, prob = _checked((0, H_kv, d), k_pages.shape, k_pages.dtype, device, page_table, key_len, max_new=0)
        if out_table.dim() != 2:
            raise ValueError("out_table must be int32 [B, out_pages]")
        _ha._fit_int32(keep=keep, keep_first=keep_first, keep_last=keep_last, out_pages=out_table.shape[1])
        _bs._int32("out_table", out_table, (prob.B, out_table.shape[1]), device)
        _bs._float32("weights", weights, _slots(prob), device)
        if keep < 1:
            raise ValueError(f"keep must be at least 1, got {keep}")
        len_out = torch.empty(prob.B, dtype=torch.int32, device=device) if len_out is None else len_out
        weights_out = torch.empty(_slots(prob), dtype=torch.float32, device=device) if weights_out is None else weights_out
        kept = torch.empty((prob.B, H_kv, keep), dtype=torch.int32, device=device) if kept is None else kept
        _bs._int32("len_out", len_out, (prob.B,), device)
        _bs._float32("weights_out", weights_out, _slots(prob), device)
        _bs._int32("kept", kept, (prob.B, H_kv, keep), device)
        workspace = _bs._workspace(lib.hybrid_attn_paged_evict_workspace_bytes(prob, keep), workspace, device)
        _bs._check(lib.hybrid_attn_paged_evict(prob, keep, keep_first, keep_last, weights.data_ptr(), out_table.data_ptr(), out_table.shape[1], _bs._view(k_pages), _bs._view(v_pages),
                                               len_out.data_ptr(), weights_out.data_ptr(), kept.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                               _ha._stream_handle(stream, k_pages)), "hybrid_attn_paged_evict")
    return len_out, weights_out, kept
