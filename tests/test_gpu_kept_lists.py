"""A kept TensorList or ParamList works on the memory that its tensors have at the call, by the compiled marshalling and by the Python code."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["compiled", "python"])
def marshalling(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(ha, "_CALLS", False)
        monkeypatch.setattr(ha, "_calls", lambda: False)
    else:
        assert ha._calls()


def other_memory(t, how, values):
    """Gives t memory with `values`; returns what keeps the old one."""
    old, new = t.data, values.to(t.dtype).cuda()
    if how == "data":
        t.data = new
    elif how == "set_":
        t.set_(new)
    else:                                               # a larger tensor, whose memory is a new one
        t.resize_(values.numel())
        t.copy_(new)
    return old


@pytest.mark.parametrize("how", ["data", "set_", "resize_"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_and_clip_of_a_kept_list(marshalling, how, dtype):
    n = 50000 if how == "resize_" else 300
    t = [torch.full((300,), 2.0, dtype=dtype, device="cuda"), torch.zeros(7, device="cuda")]
    grads = ha.TensorList(t)
    norm, factor = ha.hybrid_attn_grad_norm(grads).tolist()
    assert abs(norm - 1200.0 ** 0.5) <= 1200.0 ** 0.5 * 2.0 ** -24 and factor == 1.0
    out = ha.TensorList([torch.empty_like(x) for x in t])
    kept = [other_memory(t[0], how, torch.full((n,), 4.0)), other_memory(out.tensors[0], how, torch.zeros(n))]
    assert ha.hybrid_attn_grad_norm_workspace_bytes(grads) == ha.hybrid_attn_grad_norm_workspace_bytes([x.clone() for x in t])
    result = ha.hybrid_attn_grad_norm(grads, 1.0)
    want = (16.0 * n) ** 0.5
    assert abs(float(result[0]) - want) <= want * 2.0 ** -23 and grads.sizes == [n, 7]
    ha.hybrid_attn_grad_clip(grads, result, out)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    assert ((out.tensors[0].double() - 4.0 / want).abs() <= 4.0 / want * (u + 2.0 ** -22)).all()
    ha.hybrid_attn_grad_clip(grads, result)
    assert torch.equal(t[0], out.tensors[0])
    if how != "resize_":                                # (there the old tensor moves along)
        assert (kept[0] == 2.0).all()


@pytest.mark.parametrize("how", ["data", "set_"])
@pytest.mark.parametrize("place", range(5))
def test_update_of_a_kept_list(marshalling, how, place):
    """One of the master, its gradient, its moments and its copy has other memory than at the call before."""
    def tensors():
        gen = torch.Generator().manual_seed(1)
        return [[(torch.rand(n, generator=gen) + 0.5).to(torch.bfloat16 if i == 4 else torch.float32).cuda() for n in (33, 4000)] for i in range(5)]
    kw = dict(lr=1e-2, kind=ha.HA_OPT_ADAMW, step=2, clip=torch.tensor([2.0, 0.5], device="cuda"))
    x, y = tensors(), tensors()
    params = ha.ParamList(*x)
    ha.hybrid_attn_param_update_many(params, **kw)
    ha.hybrid_attn_param_update_many(ha.ParamList(*y), **kw)
    kept = other_memory(x[place][1], how, x[place][1] * 1.5)
    before = kept.clone()
    y[place][1] = (y[place][1] * 1.5).clone()
    ha.hybrid_attn_param_update_many(params, **kw)
    ha.hybrid_attn_param_update_many(ha.ParamList(*y), **kw)
    assert all(torch.equal(a, b) for p, q in zip(x, y) for a, b in zip(p, q)) and torch.equal(kept, before)


def test_what_a_list_may_not_hold_is_refused_later_too(marshalling):
    f = [torch.ones(6, device="cuda"), torch.ones(4, device="cuda")]
    grads, params, result = ha.TensorList(f), ha.ParamList(f, [x.clone() for x in f]), torch.ones(2, device="cuda")
    f[1].data = torch.ones(4, 2, device="cuda")[:, 0]
    for call in (lambda: ha.hybrid_attn_grad_norm(grads), lambda: ha.hybrid_attn_grad_clip(grads, result), lambda: ha.hybrid_attn_param_update_many(params, 0.1),
                 lambda: ha.hybrid_attn_grad_clip(ha.TensorList([torch.ones(6, device="cuda"), torch.ones(4, device="cuda")]), result, grads)):
        with pytest.raises(ValueError, match="contiguous"):
            call()
    f[1].data = torch.ones(5, device="cuda")
    with pytest.raises(ValueError, match="one size"):
        ha.hybrid_attn_param_update_many(params, 0.1)
    with pytest.raises(ValueError, match="sizes"):
        ha.hybrid_attn_grad_clip(grads, result, [torch.ones(6, device="cuda"), torch.ones(4, device="cuda")])
    f[1].data = torch.ones(4, device="cuda")
    ha.hybrid_attn_param_update_many(params, 0.25)
    assert (f[1] == 0.75).all() and float(ha.hybrid_attn_grad_norm(grads)[1]) == 1.0
