"""The compiled marshalling of rotary positions and of paged caches (csrc/ha_binding_rows.h): plain calls give what the Python code gives, and everything else is left to that
code."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha


def test_is_built_and_leaves_host_tensors_alone():
    native = ha._rows()
    assert native
    x, p, i = torch.zeros(2, 1, 8, 64), torch.zeros(4, 2, 64), torch.zeros(2, 2, dtype=torch.int32)
    r = ha.hybrid_attn_rotary_frequencies(64, device="cpu")
    at = torch.zeros(8, 1, dtype=torch.int32)
    assert native.rotate(x, r, at, False, None, None) is None and native.rotate(x) is None and native.rotate(None, r, at, False, None, None) is None
    assert native.norm_rotate(x, x, None, None, r, at, 1e-6, None, None, None) is None
    assert native.norm_rotate_grad(x, x, x, x, None, None, r, at, 1e-6, None, None, None, None, None, None) is None
    assert native.paged_append(p, p, p, x, x, i, i[0], None, None, None, None, None, None, None, None, None) is None
    assert native.paged_append(None, None, p, x, x, i, i[0], None, None, None, None, None, None, None, None, None) is None
    assert native.paged_forward(p, x, x, i, i[0], None, None, True, None, False, None, None, None, None) is None
    assert native.paged_weights(p, x, p[..., 0], None, i, i[0], None, None, True, None, None, None, None) is None
    assert native.paged_evict(x, x, x, i, i[0], 1, i, 0, 0, None, None, None, None, None) is None
    with pytest.raises(ValueError, match="another number"):
        native.bind_rows((1, 2))


def test_a_module_of_other_structs_is_not_used(monkeypatch):
    from paper_2509_24899_amd import paged

    class longer(ha.ctypes.Structure):
        _fields_ = paged.ha_paged_problem._fields_ + [("more", ha.ctypes.c_int64)]
    monkeypatch.setattr(ha, "_ROWS", None)
    monkeypatch.setattr(paged, "ha_paged_problem", longer)
    assert ha._rows() is False and ha._calls()
    monkeypatch.setattr(ha, "_ROWS", None)


NAMES = ("rotate", "norm_rotate", "norm_rotate_grad", "paged_append", "paged_forward", "paged_weights", "paged_evict")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,layout", [(torch.bfloat16, "bhnd"), (torch.float32, "bnhd")])
def test_same_results_as_the_python_code(dtype, layout, monkeypatch):
    gen = torch.Generator().manual_seed(51)

    def tokens(*shape):
        x = torch.randn(shape, generator=gen).to(dtype).cuda()
        return x if layout == "bhnd" else x.transpose(1, 2).contiguous().transpose(1, 2)
    q, k, gq, gk = tokens(2, 4, 30, 64), tokens(2, 2, 30, 64), tokens(2, 4, 30, 64), tokens(2, 2, 30, 64)
    w = torch.rand(64, generator=gen).cuda() + 0.5
    r, at = ha.hybrid_attn_rotary_grid(48), torch.randint(0, 99, (2, 30, 3), generator=gen, dtype=torch.int32).cuda()
    plain, line = ha.hybrid_attn_rotary_frequencies(64, interleaved=False), torch.arange(30, dtype=torch.int32, device="cuda")[:, None].contiguous()
    pq, pk, pv = (torch.randn((5, h, 64), generator=gen).to(dtype).cuda() for h in (4, 2, 2))
    if layout == "bhnd":
        pq = pq.transpose(0, 1).contiguous().transpose(0, 1)
    pools = [tokens(12, 2, 16, 64) for _ in range(2)]
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    where = dict(page_table=table, key_len=torch.tensor([60, 33], dtype=torch.int32, device="cuda"), q_offset=torch.tensor([0, 1, 5], dtype=torch.int32, device="cuda"))
    weights = torch.rand(2, 2, 64, generator=gen).cuda()

    def run(native):
        took = []
        if native:
            class Watched:
                pass
            watched = Watched()
            for name in NAMES:
                def call(*a, f=getattr(native, name), name=name):
                    x = f(*a)
                    took.append((name, x is not None))
                    return x
                setattr(watched, name, call)
            native = watched
        monkeypatch.setattr(ha, "_ROWS", native)
        monkeypatch.setattr(ha, "_rows", lambda: native)
        k_pages, v_pages = (x.clone() for x in pools)
        all_ = [ha.hybrid_attn_rotate(q, r, at), ha.hybrid_attn_rotate(q, plain, line, out=torch.empty_like(q)), ha.hybrid_attn_rotate_grad(gq, r, at),
                *ha.hybrid_attn_norm_rotate(q, k, w, None, r, at, 1e-5), ha.hybrid_attn_norm_rotate(q, None, w)[0],
                *ha.hybrid_attn_norm_rotate_grad(gq, gk, q, k, w, w, r, at, grad_w_q=torch.empty_like(w)), *ha.hybrid_attn_norm_rotate_grad(gq, gk, q, k, None, w, r, at),
                *ha.hybrid_attn_norm_rotate_grad(gq, None, q, None)]
        q2 = ha.hybrid_attn_paged_append(pq, pk, pv, k_pages, v_pages, **where, max_new=4, w_q=w, w_k=w, rotary=plain, positions=line[:5], eps=1e-6)
        ha.hybrid_attn_paged_append(None, pk[:2], pv[:2], k_pages, v_pages, table, where["key_len"])
        out, lse = ha.hybrid_attn_paged_forward(q2, k_pages, v_pages, **where, with_lse=True)
        other, none = ha.hybrid_attn_paged_forward(q2, k_pages, v_pages, **where, max_new=4, causal=False, softmax_scale=0.25, out=torch.empty_like(q2))
        assert none is None
        sums = ha.hybrid_attn_paged_weights(q2, k_pages, lse, None, **where)
        given = weights.clone()
        assert ha.hybrid_attn_paged_weights(q2, k_pages, lse, given, **where, max_new=4).data_ptr() == given.data_ptr()
        left = ha.hybrid_attn_paged_evict(k_pages, v_pages, given, table, where["key_len"], 30, torch.arange(8, 12, dtype=torch.int32, device="cuda").view(2, 2), 1, 4)
        torch.cuda.synchronize()
        return [*all_, q2, out, lse, other, sums, given, *left, k_pages, v_pages], took
    with_native, took = run(ha._rows())
    assert took and all(t for _, t in took) and {name for name, _ in took} == set(NAMES)
    for i, (a, b) in enumerate(zip(with_native, run(False)[0])):
        assert (a is None) == (b is None) and (a is None or (torch.equal(a, b) and a.stride() == b.stride())), i
