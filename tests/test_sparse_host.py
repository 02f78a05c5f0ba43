"""Block-sparse attention and the many-tensor calls on the host: exported names, struct layouts, and every refusal, none of which reaches the GPU."""
import ctypes
import os
import re

import pytest
import torch

from oracle import block_sparse_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = range(6)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ha.LIB_PATH):
        from paper_2509_24899_amd.build import build_library
        build_library()
    return ha._lib()


@pytest.mark.parametrize("header,count", [("hybrid_attn_sparse.h", 8), ("hybrid_attn_optim.h", 4)])
def test_header_symbols_are_exported(lib, header, count):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    names = set(re.findall(r"\b(hybrid_attn_\w+)\s*\(", text))
    assert len(names) == count and all(hasattr(lib, n) for n in names)


def test_struct_layouts_match_the_headers(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "hybrid_attn_sparse.h"\n#include "hybrid_attn_optim.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu", '
                   'sizeof(ha_sparse_problem), offsetof(ha_sparse_problem, q_start), sizeof(ha_view), sizeof(ha_tensor), sizeof(ha_param), offsetof(ha_param, grad_dtype)); }')
    exe = tmp_path / "layout"
    assert os.system(f"gcc -I{ROOT}/include {src} -o {exe}") == 0
    got = tuple(map(int, os.popen(str(exe)).read().split()))
    assert got == (ctypes.sizeof(ha.ha_sparse_problem), ha.ha_sparse_problem.q_start.offset, ctypes.sizeof(ha.ha_view), ctypes.sizeof(ha.ha_tensor),
                   ctypes.sizeof(ha.ha_param), ha.ha_param.grad_dtype.offset)


def problem(**kw):
    base = dict(B=2, H=4, H_kv=2, N_q=300, N_k=500, d_head=128, dtype=ha.HA_BF16, q_block=128, k_block=64, n_select=4, causal=0, keep_first=0, near_tokens=-1,
                softmax_scale=0.1, q_start=None, key_len=None)
    return ha.ha_sparse_problem(*{**base, **kw}.values())


def view(heads=4, n=300, d=128, data=FAKE, **kw):
    return ha.ha_view(*{**dict(data=data, sb=heads * n * d, sh=n * d, sn=d), **kw}.values())


def test_valid_problems(lib):
    for kw in (dict(), dict(H=2), dict(d_head=64, dtype=ha.HA_F32), dict(q_block=64, k_block=128), dict(N_q=0), dict(N_k=0), dict(N_q=1, N_k=1), dict(n_select=1 << 20),
               dict(causal=1, near_tokens=0, keep_first=1)):
        assert lib.hybrid_attn_sparse_validate(problem(**kw)) == OK, kw


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(H=0), SHAPE), (dict(H_kv=0), SHAPE), (dict(H=3), SHAPE), (dict(N_q=-1), SHAPE), (dict(N_k=-1), SHAPE), (dict(d_head=0), SHAPE),
    (dict(d_head=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(q_block=32), UNSUPPORTED), (dict(k_block=256), UNSUPPORTED), (dict(n_select=0), SHAPE),
    (dict(n_select=(1 << 20) + 1), UNSUPPORTED), (dict(causal=2), SHAPE), (dict(keep_first=-1), SHAPE), (dict(near_tokens=-2), SHAPE), (dict(softmax_scale=0.0), SHAPE),
    (dict(softmax_scale=float("nan")), SHAPE), (dict(softmax_scale=float("inf")), SHAPE), (dict(softmax_scale=-1.0), SHAPE), (dict(softmax_scale=1e-31), SHAPE), (dict(softmax_scale=1e31), SHAPE), (dict(q_start=FAKE + 2), ALIGN),
    (dict(key_len=FAKE + 1), ALIGN), (dict(B=40000, H=2), UNSUPPORTED), (dict(N_q=(1 << 24) + 1), UNSUPPORTED), (dict(N_k=(1 << 29) + 1), UNSUPPORTED),
    (dict(N_q=1 << 24, n_select=1 << 14), UNSUPPORTED)])
def test_problem_errors(lib, kw, status):
    p = problem(**kw)
    assert lib.hybrid_attn_sparse_validate(p) == status
    assert lib.hybrid_attn_key_means(p, view(2, 500), 0, FAKE, None) == status
    assert lib.hybrid_attn_select_blocks(p, view(), FAKE, FAKE, FAKE, 1 << 40, None) == status
    assert lib.hybrid_attn_sparse_forward(p, view(), view(2, 500), view(2, 500), FAKE, view(), None, FAKE, 1 << 40, None) == status
    assert lib.hybrid_attn_sparse_grad(p, view(), view(2, 500), view(2, 500), FAKE, view(), FAKE, view(), view(), view(2, 500), view(2, 500), FAKE, 1 << 40, None) == status
    assert lib.hybrid_attn_sparse_workspace_bytes(p) == lib.hybrid_attn_sparse_grad_workspace_bytes(p) == lib.hybrid_attn_select_workspace_bytes(p) == 0
    assert lib.hybrid_attn_sparse_validate(None) == NULL


def forward(lib, p=None, q=None, k=None, v=None, blocks=FAKE, out=None, lse=FAKE, ws=FAKE - FAKE % 256, size=1 << 40):
    return lib.hybrid_attn_sparse_forward(p or problem(), q or view(), k or view(2, 500), v or view(2, 500), blocks, out or view(), lse, ws, size, None)


def grad(lib, p=None, blocks=FAKE, lse=FAKE, ws=FAKE - FAKE % 256, size=1 << 40, **kw):
    v = dict(q=view(), k=view(2, 500), v=view(2, 500), out=view(), dout=view(), dq=view(), dk=view(2, 500), dv=view(2, 500))
    v.update(kw)
    return lib.hybrid_attn_sparse_grad(p or problem(), v["q"], v["k"], v["v"], blocks, v["out"], lse, v["dout"], v["dq"], v["dk"], v["dv"], ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(data=None), NULL), (dict(data=FAKE + 8), ALIGN), (dict(sn=124), SHAPE), (dict(sn=132), ALIGN), (dict(sh=1 << 20 | 4), ALIGN), (dict(sb=1 << 21 | 12), ALIGN), (dict(sn=0), SHAPE),
    (dict(sh=-128), SHAPE), (dict(sb=-128), SHAPE), (dict(sn=1 << 24), SHAPE), (dict(sb=1 << 45), SHAPE)])
def test_view_errors(lib, bad, status):
    for name, heads, n in (("q", 4, 300), ("k", 2, 500), ("v", 2, 500), ("out", 4, 300)):
        assert forward(lib, **{name: view(heads, n, **bad)}) == status, name
    for name, heads, n in (("q", 4, 300), ("k", 2, 500), ("v", 2, 500), ("out", 4, 300), ("dout", 4, 300), ("dq", 4, 300), ("dk", 2, 500), ("dv", 2, 500)):
        assert grad(lib, **{name: view(heads, n, **bad)}) == status, name
    assert lib.hybrid_attn_key_means(problem(), view(2, 500, **bad), 0, FAKE, None) == status
    assert lib.hybrid_attn_select_blocks(problem(), view(**bad), FAKE, FAKE, FAKE, 1 << 40, None) == status


def test_outputs_are_not_broadcast(lib):
    for bad in (dict(sb=0), dict(sh=0)):
        assert forward(lib, out=view(**bad)) == SHAPE
        for name, heads, n in (("dq", 4, 300), ("dk", 2, 500), ("dv", 2, 500)):
            assert grad(lib, **{name: view(heads, n, **bad)}) == SHAPE, name


def test_pointers_and_workspaces(lib):
    f32 = problem(dtype=ha.HA_F32)
    assert forward(lib, blocks=None) == NULL and forward(lib, blocks=FAKE + 2) == ALIGN and forward(lib, lse=FAKE + 2) == ALIGN
    need = lib.hybrid_attn_sparse_workspace_bytes(f32)
    assert need >= 2 * 6 * (2 * 2 * 500) * 128                      # the pieces of k and v
    aligned = FAKE - FAKE % 256
    for ws, size in ((None, need), (aligned, need - 1), (aligned + 128, need)):
        assert forward(lib, p=f32, ws=ws, size=size) == WORKSPACE
    need = lib.hybrid_attn_sparse_grad_workspace_bytes(problem())
    for ws, size in ((None, need), (aligned, need - 1), (aligned + 128, need)):
        assert grad(lib, ws=ws, size=size) == WORKSPACE
    assert grad(lib, blocks=None) == NULL and grad(lib, lse=None) == NULL and grad(lib, lse=FAKE + 1) == ALIGN
    many = problem(N_q=128 * 300)                       # (few tiles need none)
    need = lib.hybrid_attn_select_workspace_bytes(many)
    assert need > 0

    def select(p=None, means=FAKE, out=FAKE, ws=aligned, size=need):
        return lib.hybrid_attn_select_blocks(p or many, view(n=128 * 100), means, out, ws, size, None)
    assert select(means=None) == NULL and select(out=None) == NULL and select(means=FAKE + 4) == ALIGN and select(out=FAKE + 1) == ALIGN
    assert select(ws=None) == WORKSPACE and select(size=need - 1) == WORKSPACE and select(ws=aligned + 64) == WORKSPACE
    # a causal choice without the tile's own blocks would look at later keys; kept blocks have to fit the list
    assert select(problem(causal=1)) == SHAPE and select(problem(keep_first=5)) == SHAPE and select(problem(near_tokens=200)) == SHAPE
    assert lib.hybrid_attn_key_means(problem(), view(2, 500), -1, FAKE, None) == SHAPE and lib.hybrid_attn_key_means(problem(), view(2, 500), 0, None, None) == NULL
    # nothing to do, nothing to look at
    assert forward(lib, p=problem(N_q=0), q=view(data=None), out=view(data=None), blocks=None, lse=None, ws=None, size=0) == OK
    assert lib.hybrid_attn_key_means(problem(N_k=0), view(data=None), 0, None, None) == OK and lib.hybrid_attn_select_blocks(problem(N_q=0), view(data=None), None, None, None, 0, None) == OK


def tensors(*items):
    return (ha.ha_tensor * len(items))(*[(*x, 0) for x in items])


def test_grad_norm_and_clip_errors(lib):
    f, b = ha.HA_F32, ha.HA_BF16
    good = tensors((FAKE, 1000, f), (FAKE + 2, 7, b), (None, 0, f))
    need = lib.hybrid_attn_grad_norm_workspace_bytes(3, good)
    assert need == 16 and lib.hybrid_attn_grad_norm_workspace_bytes(0, None) == 8

    def norm(n=3, t=good, max_norm=1.0, result=FAKE, ws=FAKE, size=need):
        return lib.hybrid_attn_grad_norm(n, t, max_norm, result, ws, size, None)

    def clip(n=3, t=good, out=good, result=FAKE):
        return lib.hybrid_attn_grad_clip(n, t, out, result, None)
    assert norm(n=-1) == SHAPE and norm(t=None) == NULL and norm(result=None) == NULL and norm(result=FAKE + 2) == ALIGN
    assert norm(ws=None) == WORKSPACE and norm(size=need - 1) == WORKSPACE and norm(ws=FAKE + 4) == ALIGN
    for m in (0.0, -1.0, float("nan")):
        assert norm(max_norm=m) == SHAPE
    assert clip(n=-1) == SHAPE and clip(t=None) == NULL and clip(out=None) == NULL and clip(result=None) == NULL and clip(result=FAKE + 1) == ALIGN
    for bad, status in (((None, 4, f), NULL), ((FAKE + 2, 4, f), ALIGN), ((FAKE + 1, 4, b), ALIGN), ((FAKE, 4, 7), UNSUPPORTED), ((FAKE, 1 << 41, f), SHAPE)):
        t = tensors(bad)
        assert norm(1, t) == status and clip(1, t, t) == status
        assert lib.hybrid_attn_grad_norm_workspace_bytes(1, t) == 0
    assert clip(1, tensors((FAKE, 4, f)), tensors((FAKE, 5, f))) == SHAPE and clip(1, tensors((FAKE, 4, f)), tensors((FAKE, 4, b))) == SHAPE


def test_param_update_many_errors(lib):
    def call(opt=None, count=1, result=None, **kw):
        o = ha.ha_optimizer(*{**dict(kind=ha.HA_OPT_ADAMW, step=1, lr=1e-3, grad_scale=1.0, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0), **(opt or {})}.values())
        p = ha.ha_param(*{**dict(master=FAKE, grad=FAKE, m=FAKE, v=FAKE, param_io=None, n=10, grad_dtype=ha.HA_F32, io_dtype=ha.HA_BF16), **kw}.values())
        return lib.hybrid_attn_param_update_many(o, count, ctypes.pointer(p), result, None)
    assert lib.hybrid_attn_param_update_many(None, 0, None, None, None) == NULL
    assert call(count=-1) == SHAPE and call(count=0) == OK and call(master=None) == NULL
    for kw, status in ((dict(grad=None), NULL), (dict(m=None), NULL), (dict(v=None), NULL), (dict(master=FAKE + 2), ALIGN), (dict(grad=FAKE + 2), ALIGN), (dict(m=FAKE + 1), ALIGN),
                       (dict(v=FAKE + 3), ALIGN), (dict(param_io=FAKE + 1), ALIGN), (dict(param_io=FAKE + 2, io_dtype=ha.HA_F32), ALIGN), (dict(param_io=FAKE), SHAPE),
                       (dict(param_io=FAKE + 64, io_dtype=3), UNSUPPORTED), (dict(grad_dtype=2), UNSUPPORTED), (dict(n=1 << 41), SHAPE), (dict(result=FAKE + 2), ALIGN)):
        result = kw.pop("result", None)
        assert call(result=result, **kw) == status, kw
    for opt, status in ((dict(kind=5), UNSUPPORTED), (dict(step=0), SHAPE), (dict(lr=-1.0), SHAPE), (dict(lr=float("nan")), SHAPE), (dict(beta1=1.0), SHAPE), (dict(beta2=-0.1), SHAPE),
                        (dict(eps=-1.0), SHAPE), (dict(weight_decay=float("inf")), SHAPE), (dict(grad_scale=float("inf")), SHAPE)):
        assert call(opt) == status, opt


def test_binding_refuses_cpu_tensors():
    q = torch.zeros(1, 2, 64, 64)
    with pytest.raises(RuntimeError, match="GPU only"):
        ha.hybrid_attn_key_means(q)
    with pytest.raises(RuntimeError, match="GPU only"):
        ha.hybrid_attn_sparse_forward(q, q, q, torch.zeros(1, 2, 1, 1, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="GPU only"):
        ha.TensorList([q])
    with pytest.raises(RuntimeError, match="GPU only"):
        ha.ParamList([q], [q])


def test_binding_checks_shapes_and_types():
    dev = torch.device("cuda", 0)
    with pytest.raises(ValueError, match="H_kv"):
        ha.make_sparse_problem((1, 2, 3), (1, 2, 3, 64), torch.bfloat16, dev)
    with pytest.raises(ValueError, match="one B and d"):
        ha.make_sparse_problem((1, 2, 3, 64), (2, 2, 3, 64), torch.bfloat16, dev)
    with pytest.raises(ValueError, match="unsupported dtype"):
        ha.make_sparse_problem((1, 2, 3, 64), (1, 2, 3, 64), torch.float16, dev)
    for bad in (torch.zeros(1, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)):
        with pytest.raises(ValueError, match="key_len must be"):
            ha.make_sparse_problem((1, 2, 3, 64), (1, 2, 3, 64), torch.bfloat16, dev, key_len=bad)


@pytest.mark.parametrize("first", ["block_sparse", "optim", "hybrid_attn"])
def test_modules_import_in_any_order(first):
    import subprocess
    import sys
    code = f"import paper_2509_24899_amd.{first}; from paper_2509_24899_amd import hybrid_attn as h; h.hybrid_attn_sparse_grad, h.ParamList"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT).returncode == 0


# ---- the oracle ------------------------------------------------------------------------------------------------------------------

def test_oracle_is_softmax_attention_where_every_block_is_listed():
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(2, 4, 70, 8, generator=gen, dtype=torch.float64) for _ in range(3))
    blocks = torch.arange(2, dtype=torch.int32).repeat(2, 4, 2, 1)
    for causal in (False, True):
        s = q @ k.transpose(2, 3) * 8 ** -0.5
        if causal:
            s = s.masked_fill(torch.triu(torch.ones(70, 70, dtype=torch.bool), 1), -torch.inf)
        x = [t.clone().requires_grad_() for t in (q, k, v)]
        s2 = x[0] @ x[1].transpose(2, 3) * 8 ** -0.5
        s2 = s2.masked_fill(torch.triu(torch.ones(70, 70, dtype=torch.bool), 1), -torch.inf) if causal else s2
        y = torch.softmax(s2, 3) @ x[2]
        do = torch.randn(y.shape, generator=gen, dtype=torch.float64)
        want = torch.autograd.grad((y * do).sum(), x)
        got = O.attention(q, k, v, blocks, 64, 64, causal, dout=do)
        assert torch.allclose(got["out"], y, rtol=1e-12, atol=1e-12) and torch.allclose(got["lse"], torch.logsumexp(s, 3), rtol=1e-12)
        for name, w in zip(("dq", "dk", "dv"), want):
            assert torch.allclose(got[name], w, rtol=1e-10, atol=1e-12), name


def test_oracle_sees_a_planted_mistake():
    """A key left out, or counted twice, is outside the bounds that the kernels are held to."""
    gen = torch.Generator().manual_seed(2)
    q, k, v, do = (torch.randn(1, 1, 128, 64, generator=gen).bfloat16().double() for _ in range(4))
    one = torch.tensor([0, 1, -1], dtype=torch.int32).view(1, 1, 1, 3)
    two = torch.tensor([0, 1, 1], dtype=torch.int32).view(1, 1, 1, 3)
    kw = dict(u=2.0 ** -8, u_logit=72 * 2.0 ** -24, u_out=2.0 ** -8)
    a, b = (O.attention(q, k, v, x, 128, 64, dout=do, **kw) for x in (one, two))
    c = O.attention(q, k, v, one, 128, 64, key_len=torch.tensor([120]), dout=do, **kw)
    for name in ("out", "lse", "dq", "dk", "dv"):
        for other in (b, c):
            assert ((a[name] - other[name]).abs() > a[name + "_tol"]).double().mean() > 0.05, name
