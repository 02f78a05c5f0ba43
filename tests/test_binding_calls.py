"""The compiled marshalling of block-sparse attention and of the many-tensor optimiser (csrc/ha_binding_calls.h): plain calls give what the Python code gives,
and everything else is left to that code."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha


def test_is_built_and_leaves_host_tensors_alone():
    native = ha._calls()
    assert native
    t, i = torch.zeros(1, 1, 8, 64), torch.zeros(1, 1, 1, 1, dtype=torch.int32)
    assert native.key_means(t, 64, None, 0, None, None) is None and native.key_means(t) is None
    assert native.select_blocks(t, t, 8, 1, 128, 64, False, None, None, 0, -1, None, None, None) is None
    assert native.sparse_forward(t, t, t, i, 128, 64, False, None, None, None, False, None, None, None, None) is None
    assert native.sparse_grad(t, t, t, i, t, t[..., 0], t, 128, 64, False, None, None, None, None, None, None, None, None) is None
    assert native.grad_norm([t], 1.0, None, None, None) is None and native.grad_clip([t], t, [t], None) is None
    assert native.update_many([t], 1e-3, 0, 1, 1.0, 0.9, 0.999, 1e-8, 0.01, None, None) is None
    assert native.describe_tensors([t], 0) is None and native.describe_tensors((t,), 1) is None and native.describe_tensors([None], 1) is None
    assert native.describe_params(([t], [t], [None], [None], [None]), 0) is None and native.describe_params(([t], [], [None], [None], [None]), 1) is None
    with pytest.raises(ValueError, match="another number"):
        native.bind_calls((1, 2), None)


def test_a_module_of_other_structs_is_not_used(monkeypatch):
    from paper_2509_24899_amd import optim

    class longer(ha.ctypes.Structure):
        _fields_ = optim.ha_param._fields_ + [("more", ha.ctypes.c_int64)]
    monkeypatch.setattr(ha, "_CALLS", None)
    monkeypatch.setattr(optim, "ha_param", longer)
    assert ha._calls() is False
    monkeypatch.setattr(ha, "_CALLS", None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,layout,causal", [(torch.bfloat16, "bhnd", True), (torch.float32, "bnhd", False)])
def test_same_results_as_the_python_code(dtype, layout, causal, monkeypatch):
    gen = torch.Generator().manual_seed(50)

    def tokens(H, N):
        x = torch.randn((2, H, N, 64) if layout == "bhnd" else (2, N, H, 64), generator=gen).to(dtype).cuda()
        return x if layout == "bhnd" else x.transpose(1, 2)
    q, k, v, do = tokens(4, 300), tokens(2, 500), tokens(2, 500), tokens(4, 300)
    n, s = torch.tensor([500, 300], dtype=torch.int32, device="cuda"), torch.tensor([200, 10], dtype=torch.int32, device="cuda")
    mask = dict(causal=causal, q_start=s, key_len=n)
    grads = [torch.randn(m, generator=gen).cuda() for m in (1000, 7)]
    names = ("key_means", "select_blocks", "sparse_forward", "sparse_grad", "grad_norm", "grad_clip", "update_many", "describe_tensors", "describe_params")

    def run(native):
        took = []
        if native:
            class Watched:
                pass
            watched = Watched()
            for name in names:
                def call(*a, f=getattr(native, name), name=name):
                    r = f(*a)
                    took.append((name, r is not None))
                    return r
                setattr(watched, name, call)
            native = watched
        monkeypatch.setattr(ha, "_CALLS", native)
        monkeypatch.setattr(ha, "_calls", lambda: native)
        means = ha.hybrid_attn_key_means(k, key_len=n)
        ha.hybrid_attn_key_means(k, key_len=n, only_last=1, out=means)
        blocks = ha.hybrid_attn_select_blocks(q, means, 500, 4, near=0, **mask)
        out, lse = ha.hybrid_attn_sparse_forward(q, k, v, blocks, **mask, with_lse=True)
        plain, none = ha.hybrid_attn_sparse_forward(q, k, v, blocks, **mask, softmax_scale=0.1, out=torch.empty_like(q))
        assert none is None
        g = ha.hybrid_attn_sparse_grad(q, k, v, blocks, out, lse, do, **mask)
        lists, new = ha.TensorList(grads), [torch.zeros_like(x) for x in grads]
        result = ha.hybrid_attn_grad_norm(lists, 1.0)
        ha.hybrid_attn_grad_clip(lists, result, new)
        masters = [torch.ones_like(x) for x in grads]
        ha.hybrid_attn_param_update_many(ha.ParamList(masters, grads), 0.1, clip=result)
        torch.cuda.synchronize()
        return [means, blocks, out, lse, plain, *g, result, *new, *masters], took
    with_native, took = run(ha._calls())
    assert took and all(t for _, t in took) and {name for name, _ in took} == set(names)
    without, _ = run(False)
    for a, b in zip(with_native, without):
        assert torch.equal(a, b) and a.stride() == b.stride()


@pytest.mark.gpu
def test_lists_are_described_alike(monkeypatch):
    def field(x, name):
        return [getattr(e, name) for e in x.c]
    f = [torch.zeros(n, device="cuda") for n in (5, 0, 300)]
    half = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in (5, 0, 300)]
    made = []
    for native in (ha._calls(), False):
        monkeypatch.setattr(ha, "_CALLS", native)
        monkeypatch.setattr(ha, "_calls", lambda: native)
        made.append((ha.TensorList(f + half), ha.ParamList(f, half, f, f, [half[0], None, f[2]]), ha.ParamList(f, f)))
    from paper_2509_24899_amd import optim
    for a, b in zip(*made):
        struct = optim.ha_tensor if isinstance(a, ha.TensorList) else optim.ha_param
        assert len(a) == len(b) and a.device == b.device and a.native[1:] == b.native[1:]
        for name, _ in struct._fields_:
            assert field(a, name) == field(b, name), name
    assert made[0][0].sizes == made[1][0].sizes
    monkeypatch.undo()
    for wrong in ([f[2], half[2].cpu()], [f[2].view(30, 10).t()], [f[2].double()]):
        with pytest.raises((RuntimeError, ValueError, TypeError)):
            ha.TensorList(wrong)
    for masters, grads, m in ((half, f, None), (f, f[::-1], None), (f, f, half), (f, f[:2], None)):
        with pytest.raises(ValueError):
            ha.ParamList(masters, grads, m, m)


@pytest.mark.gpu
def test_what_is_not_plain_gets_the_python_codes_message():
    q = torch.zeros(1, 2, 100, 64, dtype=torch.bfloat16, device="cuda")
    blocks = torch.zeros(1, 2, 1, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="blocks must be"):
        ha.hybrid_attn_sparse_forward(q, q, q, blocks[:, :1])
    with pytest.raises(ValueError, match="blocks must be"):
        ha.hybrid_attn_sparse_forward(q, q, q, blocks.long())
    with pytest.raises(ValueError, match="k must be"):
        ha.hybrid_attn_sparse_forward(q, q.float(), q, blocks)
    with pytest.raises(ValueError, match="contiguous last dimension"):
        ha.hybrid_attn_sparse_forward(q.transpose(2, 3).contiguous().transpose(2, 3), q, q, blocks)
    with pytest.raises(ValueError, match="key_len must be"):
        ha.hybrid_attn_key_means(q, key_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="needs out"):
        ha.hybrid_attn_key_means(q, only_last=1)
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_key_means(q, k_block=32)
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_sparse_forward(q, q, q, blocks, softmax_scale=-1.0)
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_select_blocks(q, ha.hybrid_attn_key_means(q), 100, 1, causal=True)
    with pytest.raises(ha.HybridAttnError, match="workspace"):
        f = q.float()
        ha.hybrid_attn_sparse_forward(f, f, f, blocks, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ha.HybridAttnError):                                   # an output that is one memory for both heads
        ha.hybrid_attn_sparse_forward(q, q, q, blocks, out=q[:, :1].expand(1, 2, 100, 64))
    with pytest.raises(ValueError, match="unsupported dtype"):
        h = q.half()
        ha.hybrid_attn_key_means(h)
