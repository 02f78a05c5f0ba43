"""Host checks of the calls of include/hybrid_attn_rotary.h and hybrid_attn_paged.h: every refusal comes ahead of the first HIP call, so they run without a GPU.  Addresses are
made up; no call here gets as far as using them."""
import ctypes
import math

import pytest
import torch

from paper_2509_24899_amd import block_sparse as bs
from paper_2509_24899_amd import hybrid_attn as ha

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = range(6)
AT = 1 << 20


def view(data=AT, b=0, h=128, n=512):
    return bs.ha_view(data, b, h, n)


def rows_problem(**more):
    return ha.ha_rows_problem(**{**dict(B=2, H=4, H_kv=2, N=10, d_head=128, dtype=ha.HA_BF16, eps=1e-6), **more})


def rotary(**more):
    return ha.ha_rotary(**{**dict(freq=AT, axis=AT, positions=AT, positions_stride_b=0, rot_dim=128, interleaved=1, n_axes=3, magnitude=1.0), **more})


@pytest.mark.parametrize("problem,rot,status", [
    ({}, {}, OK), (dict(N=0), dict(positions=None), OK), (dict(H_kv=0), {}, OK), ({}, dict(rot_dim=0, freq=None, positions=None), OK), ({}, dict(axis=None), OK),
    ({}, dict(interleaved=0, rot_dim=96), OK), ({}, dict(interleaved=1, rot_dim=6), OK), (dict(eps=0.0), {}, OK), ({}, dict(positions_stride_b=30), OK),
    (dict(B=0), {}, SHAPE), (dict(H=0), {}, SHAPE), (dict(H_kv=-1), {}, SHAPE), (dict(N=-1), {}, SHAPE), (dict(d_head=96), {}, UNSUPPORTED), (dict(dtype=2), {}, UNSUPPORTED),
    (dict(eps=-1e-6), {}, SHAPE), (dict(eps=math.nan), {}, SHAPE), (dict(eps=math.inf), {}, SHAPE), (dict(B=65536, H=1), {}, UNSUPPORTED), (dict(H_kv=40000), {}, UNSUPPORTED),
    (dict(B=16, N=1 << 24), {}, UNSUPPORTED), ({}, dict(rot_dim=130), SHAPE), ({}, dict(rot_dim=63), SHAPE), ({}, dict(rot_dim=-2), SHAPE),
    ({}, dict(interleaved=0, rot_dim=92), UNSUPPORTED), ({}, dict(interleaved=2), SHAPE), ({}, dict(n_axes=0), SHAPE), ({}, dict(n_axes=5), SHAPE),
    ({}, dict(magnitude=math.nan), SHAPE), ({}, dict(positions_stride_b=29), SHAPE), ({}, dict(positions_stride_b=-30), SHAPE), ({}, dict(freq=None), NULL),
    ({}, dict(positions=None), NULL), ({}, dict(freq=AT + 4), ALIGN), ({}, dict(axis=AT + 2), ALIGN), ({}, dict(positions=AT + 1), ALIGN)])
def test_rotary_problems(problem, rot, status):
    assert ha.hybrid_attn_rotary_validate(rows_problem(**problem), rotary(**rot)) == status


def test_rotary_views_weights_and_workspace():
    lib = ha._lib()
    p, r, good = rows_problem(), rotary(), view(b=5120)
    assert lib.hybrid_attn_rotary_validate(None, r) == NULL and lib.hybrid_attn_rotary_validate(p, None) == NULL
    assert lib.hybrid_attn_rotate(p, r, good, good, 0, None) == SHAPE                       # one tensor, and H_kv is not 0
    one = rows_problem(H_kv=0)
    assert lib.hybrid_attn_rotate(one, r, good, good, 2, None) == SHAPE
    for bad, status in ((None, NULL), (view(None, 5120), NULL), (view(AT + 8, 5120), ALIGN), (view(b=5120, n=516), ALIGN), (view(b=5120, h=-128), SHAPE), (view(b=1 << 45), SHAPE)):
        assert lib.hybrid_attn_rotate(one, r, bad, good, 0, None) == status and lib.hybrid_attn_rotate(one, r, good, bad, 0, None) == status
    for bad in (view(b=0), view(b=5120, h=64), view(b=5120, n=64)):                         # an output whose entries lie on one another
        assert lib.hybrid_attn_rotate(one, r, good, bad, 0, None) == SHAPE
    assert lib.hybrid_attn_norm_rotate(p, r, good, good, AT + 4, AT, good, good, None) == ALIGN
    assert lib.hybrid_attn_norm_rotate(p, r, good, None, AT, AT, good, good, None) == NULL
    grad = [p, r, good, good, good, good, AT, AT, good, good]
    need = ha.hybrid_attn_norm_rotate_grad_workspace_bytes(p)
    assert need > 0 and ha.hybrid_attn_norm_rotate_grad_workspace_bytes(rows_problem(B=0)) == 0
    for ws, n in ((None, need), (AT + 8, need), (AT, need - 1)):
        assert lib.hybrid_attn_norm_rotate_grad(*grad, AT, AT, ws, n, None) == WORKSPACE
    assert lib.hybrid_attn_norm_rotate_grad(*grad, AT + 2, AT, AT, need, None) == ALIGN


def paged(**more):
    return ha.ha_paged_problem(**{**dict(B=3, H=6, H_kv=2, T=7, d_head=128, dtype=ha.HA_BF16, n_pages=20, page=16, max_pages=5, max_new=4, causal=1, softmax_scale=0.1, page_table=AT,
                                         key_len=AT, q_offset=AT), **more})


@pytest.mark.parametrize("change,status", [
    ({}, OK), (dict(T=0, max_new=0), OK), (dict(q_offset=None, T=12), OK), (dict(max_pages=0, page_table=None), OK), (dict(n_pages=0), OK), (dict(page=256), OK),
    (dict(B=0), SHAPE), (dict(H=5), SHAPE), (dict(H_kv=0), SHAPE), (dict(T=-1), SHAPE), (dict(max_new=8), SHAPE), (dict(max_new=-1), SHAPE), (dict(q_offset=None), SHAPE),
    (dict(causal=2), SHAPE), (dict(softmax_scale=0.0), SHAPE), (dict(softmax_scale=math.nan), SHAPE), (dict(softmax_scale=1e31), SHAPE), (dict(n_pages=-1), SHAPE), (dict(max_pages=-1), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(d_head=80), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
    (dict(max_pages=(1 << 26) + 1), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(B=40000), UNSUPPORTED), (dict(T=(1 << 20) // 3 + 1), UNSUPPORTED),
    (dict(T=1 << 18, H=128, H_kv=128), UNSUPPORTED), (dict(page_table=None), NULL), (dict(key_len=None), NULL), (dict(page_table=AT + 2), ALIGN), (dict(key_len=AT + 1), ALIGN),
    (dict(q_offset=AT + 2), ALIGN)])
def test_paged_problems(change, status):
    assert ha.hybrid_attn_paged_validate(paged(**change)) == status
    assert status == OK or ha.hybrid_attn_paged_workspace_bytes(paged(**change)) == 0


def test_paged_views_and_workspaces():
    lib = ha._lib()
    p, rows, pool = paged(), view(n=768), view(b=4096, h=2048, n=128)
    assert lib.hybrid_attn_paged_validate(None) == NULL
    assert lib.hybrid_attn_paged_forward(paged(T=0, max_new=0), rows, pool, pool, rows, None, None, 0, None) == OK      # nothing to do
    for bad, status in ((None, NULL), (view(None), NULL), (view(AT + 4), ALIGN), (view(n=4), ALIGN), (view(h=-8), SHAPE)):
        assert lib.hybrid_attn_paged_forward(p, bad, pool, pool, rows, None, None, 0, None) == status
        assert lib.hybrid_attn_paged_forward(p, rows, bad, pool, rows, None, None, 0, None) == status
        assert lib.hybrid_attn_paged_forward(p, rows, pool, bad, rows, None, None, 0, None) == status
    assert lib.hybrid_attn_paged_forward(p, rows, view(b=1 << 30, h=128, n=1 << 27), pool, rows, None, None, 0, None) == SHAPE
    assert lib.hybrid_attn_paged_forward(p, rows, pool, pool, view(h=0, n=768), None, None, 0, None) == SHAPE
    assert lib.hybrid_attn_paged_forward(p, rows, pool, pool, rows, AT + 2, None, 0, None) == ALIGN
    long = paged(max_pages=4000, n_pages=4000)
    need = ha.hybrid_attn_paged_workspace_bytes(long)
    assert need > 0
    for ws, n in ((None, need), (AT + 16, need), (AT, need - 1)):
        assert lib.hybrid_attn_paged_forward(long, rows, pool, pool, rows, None, ws, n, None) == WORKSPACE
    append = dict(q=rows, k=rows, v=rows, w_q=None, w_k=None, kp=pool, vp=pool, out=rows)

    def store(norm=0, eps=0.0, r=None, **more):
        return lib.hybrid_attn_paged_append(p, r, norm, eps, *{**append, **more}.values(), None)
    assert store(norm=2) == SHAPE and store(norm=1, eps=-1.0) == SHAPE and store(norm=1, eps=math.nan) == SHAPE and store(q=None) == NULL and store(out=None) == NULL
    assert store(k=None) == NULL and store(kp=view(b=0, h=2048, n=128)) == SHAPE and store(norm=1, w_q=AT + 4) == ALIGN
    assert store(r=rotary(positions_stride_b=21)) == SHAPE and store(r=rotary(freq=None)) == NULL
    weigh = [p, rows, pool]
    assert lib.hybrid_attn_paged_weights(*weigh, None, AT, AT, None, 0, None) == NULL and lib.hybrid_attn_paged_weights(*weigh, AT, AT, None, None, 0, None) == NULL
    assert lib.hybrid_attn_paged_weights(*weigh, AT, AT + 1, AT, None, 0, None) == ALIGN

    def evict(keep=20, first=1, last=2, weights=AT, out_table=AT, out_pages=2, kp=pool, length=AT, out=AT + 4096, kept=AT):
        return lib.hybrid_attn_paged_evict(p, keep, first, last, weights, out_table, out_pages, kp, pool, length, out, kept, None, 0, None)
    assert evict(keep=0) == SHAPE and evict(first=-1) == SHAPE and evict(last=-1) == SHAPE and evict(first=10, last=11) == SHAPE and evict(out_pages=1) == SHAPE
    assert evict(first=2 ** 31 - 1, last=2 ** 31 - 1) == SHAPE and evict(out=AT) == SHAPE and evict(weights=None) == NULL and evict(out_table=None) == NULL and evict(kept=None) == NULL
    assert evict(length=None) == NULL and evict(kept=AT + 2) == ALIGN and evict(kp=view(AT + 8, 4096, 2048, 128)) == ALIGN and evict(kp=view(b=0, h=2048, n=128)) == SHAPE


def test_structures_are_the_headers():
    assert [ctypes.sizeof(s) for s in (ha.ha_rotary, ha.ha_rows_problem, ha.ha_paged_problem)] == [48, 28, 72]


def test_python_refusals_of_problems():
    table, length, dev = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.device("cpu")

    def make(q=(4, 2, 64), pages=(9, 2, 16, 64), dtype=torch.bfloat16, table=table, length=length, **more):
        return ha.make_paged_problem(q, pages, dtype, dev, table, length, **more)
    assert make().max_new == 2 and make(q_offset=torch.zeros(3, dtype=torch.int32)).max_new == 4
    for bad in (dict(q=(4, 2)), dict(q=(4, 2, 128)), dict(pages=(9, 2, 64)), dict(dtype=torch.float16), dict(table=table[0]), dict(table=table.long()), dict(length=length[:1]), dict(q=(3, 2, 64)),
                dict(max_new=2 ** 32), dict(pages=(2 ** 31, 2, 16, 64)), dict(q_offset=length), dict(table=table.t())):
        with pytest.raises(ValueError):
            make(**bad)


def test_frequencies():
    r = ha.hybrid_attn_rotary_frequencies(64, base=100.0, device="cpu")
    assert r.freq.dtype == torch.float64 and torch.allclose(r.freq, 100.0 ** -(torch.arange(32, dtype=torch.float64) / 32)) and r.magnitude == 1.0 and r.axis is None
    assert torch.allclose(ha.hybrid_attn_rotary_frequencies(64, 100.0, stretch=4.0, device="cpu").freq, r.freq / 4)
    s = ha.hybrid_attn_rotary_frequencies(128, stretch=8.0, original=4096, device="cpu")
    plain = ha.hybrid_attn_rotary_frequencies(128, device="cpu").freq
    turns = 4096 * plain / (2 * math.pi)
    assert torch.equal(s.freq[turns >= 32], plain[turns >= 32]) and torch.allclose(s.freq[turns <= 1], plain[turns <= 1] / 8) and s.magnitude == pytest.approx(1 + 0.1 * math.log(8))
    between = (turns > 1) & (turns < 32)
    assert between.any() and ((s.freq < plain) & (s.freq > plain / 8))[between].all()
    g = ha.hybrid_attn_rotary_grid(128, device="cpu")
    assert g.axis.bincount().tolist() == [22, 21, 21] and g.freq[g.axis == 2][0] == 1.0 and g.freq[g.axis == 1][3] == 10000.0 ** (-3 / 21)
    at = ha.hybrid_attn_grid_positions(2, 3, 4, first_frame=5, device="cpu")
    assert at.shape == (24, 3) and at[0].tolist() == [5, 0, 0] and at[23].tolist() == [6, 2, 3] and at[5].tolist() == [5, 1, 1] and at.is_contiguous()
    for bad in (dict(rot_dim=7), dict(rot_dim=64, stretch=0.5), dict(rot_dim=64, base=0), dict(rot_dim=64, stretch=2.0, original=0), dict(rot_dim=64, stretch=2.0, original=100, slow=4, fast=4)):
        with pytest.raises(ValueError):
            ha.hybrid_attn_rotary_frequencies(device="cpu", **bad)
    with pytest.raises(ValueError):
        ha.hybrid_attn_rotary_grid(4, device="cpu")
