"""Global gradient norm, clipping and the update of many parameters against 64-bit formulas on the CPU.

Tolerances: squares and their sum are double, so the norm is one rounding to fp32 off (2^-24, and the sum's 2^-50), and the factor two, its own and
max_norm's, which is an fp32 argument; a clipped value is that factor's rounding, one
product and one rounding to its type off."""
import math

import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha
from paper_2509_24899_amd import workloads as W

pytestmark = pytest.mark.gpu
SIZES = [1, 2, 3, 5, 63, 64, 255, 1021, 4096, 8191, 8192, 8193, 40000, 0, 100003]


def grads_of(seed, sizes=SIZES, dtypes=(torch.float32, torch.bfloat16), odd=True):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        base = (torch.randn(n + 3, generator=gen) * 10 ** float(torch.rand(1, generator=gen) * 4 - 2)).to(dtypes[i % len(dtypes)]).cuda()
        out.append(base[i % 4 if odd else 0:][:n])              # starts at any element
    return out


def norm_of(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


@pytest.mark.parametrize("sizes", [SIZES, [7], [0], [], [3] * 300, [1 << 22, 1, (1 << 20) + 1]])
@pytest.mark.parametrize("max_norm", [1e-3, 1.0, 1e9, math.inf])
def test_norm_and_factor(sizes, max_norm):
    g = grads_of(1, sizes)
    norm, factor = ha.hybrid_attn_grad_norm(g, max_norm).tolist()
    want = norm_of(g)
    assert abs(norm - want) <= want * (2.0 ** -24 + 1e-12)
    f = min(1.0, max_norm / want) if want else 1.0
    assert abs(factor - f) <= f * (2.0 ** -23 + 1e-12) and (f < 1 or factor == 1.0)


@pytest.mark.parametrize("sizes", [[1], [1024 * 47, 1024], [1024 * 47 + 1, 1024], [1024 * 48, 1], [1] * 48, [1] * 49, [1000, 0, 1025, 5, 0, 7000, 33], [0] * 127 + [9], [0] * 128 + [9]])
def test_norm_of_few_values(sizes):
    """On both sides of the sizes that one workgroup takes, alone and with what an earlier call left in the workspace."""
    g = grads_of(7, sizes)
    ws = torch.full((ha.hybrid_attn_grad_norm_workspace_bytes(g) + 8,), 255, dtype=torch.uint8, device="cuda")
    want = norm_of(g)
    for workspace in (None, ws):
        norm, factor = ha.hybrid_attn_grad_norm(g, want / 3, workspace=workspace).tolist()
        assert abs(norm - want) <= want * (2.0 ** -24 + 1e-12) and abs(factor - 1 / 3) <= (2.0 ** -23 + 1e-12) / 3
    first = next(x for x in g if x.numel())
    first[-1] = math.nan
    assert all(math.isnan(x) for x in ha.hybrid_attn_grad_norm(g, 1.0).tolist())


def test_large_and_small_values():
    for x, n in ((3e38, 1000), (1e-38, 1000), (1e-45, 5)):
        g = [torch.full((n,), x, device="cuda")]
        norm = float(ha.hybrid_attn_grad_norm(g)[0])
        want = norm_of(g)
        assert norm == math.inf if want > 3.5e38 else abs(norm - want) <= want * 2.0 ** -23 + 1e-45
    # a norm beyond fp32 still clips
    g = [torch.full((1000,), 3e38, device="cuda")]
    out = [torch.empty_like(g[0])]
    ha.hybrid_attn_grad_clip(g, ha.hybrid_attn_grad_norm(g, 1.0), out)
    assert torch.allclose(out[0].double().norm().cpu(), torch.ones((), dtype=torch.float64), rtol=1e-5)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite(bad):
    g = grads_of(2)
    g[7][11] = bad
    result = ha.hybrid_attn_grad_norm(g, 1.0)
    norm, factor = result.tolist()
    assert math.isnan(norm) == math.isnan(bad) and math.isinf(norm) == math.isinf(bad) and math.isnan(factor)
    before = [x.clone() for x in g]
    ha.hybrid_attn_grad_clip(g, result)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, before))
    p = params_of(3, g)
    before = [[t.clone() if t is not None else None for t in x] for x in p]
    ha.hybrid_attn_param_update_many(ha.ParamList(p[0], g, *p[1:]), 1e-2, kind=ha.HA_OPT_ADAMW, clip=result)
    assert all(a is None or torch.equal(a, b) for x, y in zip(p, before) for a, b in zip(x, y))


@pytest.mark.parametrize("place", ["new", "in place", "other type"])
def test_clip(place):
    g = grads_of(4)
    want, norm = [x.double().cpu() for x in g], norm_of(g)
    for max_norm in (norm / 7, 2 * norm):
        result = ha.hybrid_attn_grad_norm(g, max_norm)
        other = {torch.float32: torch.bfloat16, torch.bfloat16: torch.float32}
        src = [x.clone() for x in g]
        room = [torch.full((x.numel() + 2,), 9.0, dtype=other[x.dtype] if place == "other type" else x.dtype, device="cuda") for x in g]
        out = src if place == "in place" else [r[1:-1] for r in room]
        ha.hybrid_attn_grad_clip(src, result, None if place == "in place" else out)
        f = min(1.0, max_norm / norm)
        for o, x, r in zip(out, want, room):
            u = 2.0 ** -8 if o.dtype == torch.bfloat16 else 2.0 ** -24
            assert ((o.double().cpu() - f * x).abs() <= (u + 2.0 ** -22) * f * x.abs()).all()
            assert float(r[0]) == float(r[-1]) == 9.0


def params_of(seed, grads):
    """masters, m, v, copies (bf16, fp32 or none in turn)."""
    gen = torch.Generator().manual_seed(seed)

    def some(f):
        return [f(torch.randn(g.numel(), generator=gen)).cuda() for g in grads]
    masters, m, v = some(lambda x: x), some(lambda x: 0.1 * x), some(lambda x: x * x * 1e-3 + 1e-6)
    io = [None if i % 3 == 2 else torch.zeros(g.numel(), dtype=(torch.bfloat16, torch.float32)[i % 3], device="cuda") for i, g in enumerate(grads)]
    return masters, m, v, io


@pytest.mark.parametrize("kind", [ha.HA_OPT_SGD, ha.HA_OPT_ADAMW])
@pytest.mark.parametrize("sizes", [SIZES, [5] * 130])
def test_update_of_many_is_that_of_each(kind, sizes):
    """Bit for bit what one call per tensor gives, in fp32 gradients and without a factor."""
    g = grads_of(5, sizes, (torch.float32,))
    one, many = params_of(6, g), params_of(6, g)
    kw = dict(lr=1e-2, kind=kind, step=3, grad_scale=0.37, weight_decay=0.02)
    for x, p, m, v, io in zip(g, *one):
        if x.numel():                                   # (the call of one takes no empty tensor)
            ha.hybrid_attn_param_update(p, x.clone(), m=m, v=v, param_io=io, **kw)
    ha.hybrid_attn_param_update_many(ha.ParamList(many[0], g, *many[1:]), **kw)
    assert all(a is None or torch.equal(a, b) for x, y in zip(one, many) for a, b in zip(x, y))


@pytest.mark.parametrize("kind", [ha.HA_OPT_SGD, ha.HA_OPT_ADAMW])
def test_clipped_update(kind):
    g = grads_of(7)
    p = params_of(8, g)
    start = [[None if t is None else t.double().cpu() for t in x] for x in p]
    norm = norm_of(g)
    result = ha.hybrid_attn_grad_norm(g, norm / 5)
    lr, b1, b2, eps, wd, step, gs = 1e-2, 0.9, 0.999, 1e-8, 0.02, 4, 2.0
    plist = ha.ParamList(p[0], g, None if kind == ha.HA_OPT_SGD else p[1], None if kind == ha.HA_OPT_SGD else p[2], p[3])
    ha.hybrid_attn_param_update_many(plist, lr, kind=kind, step=step, grad_scale=gs, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, clip=result)
    # betas are fp32 numbers to the call
    b1, b2 = (float(torch.tensor(b, dtype=torch.float32)) for b in (b1, b2))
    for i, x in enumerate(g):
        x = x.double().cpu() * gs / 5
        master, m, v = (start[j][i] for j in range(3))
        if kind == ha.HA_OPT_SGD:
            want = master - lr * x
            tol = 2.0 ** -22 * (master.abs() + lr * x.abs())
        else:
            m, v = b1 * m + (1 - b1) * x, b2 * v + (1 - b2) * x * x
            move = lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + eps)
            want = master * (1 - lr * wd) - move
            # half a dozen fp32 roundings behind one another; m's terms may cancel
            tol = 2.0 ** -22 * (master.abs() + 4 * move.abs()) + 2.0 ** -21 * lr * (x.abs() + start[1][i].abs()) / (v.sqrt() + eps)
            assert ((p[1][i].double().cpu() - m).abs() <= 2.0 ** -21 * (x.abs() + start[1][i].abs())).all()
            assert ((p[2][i].double().cpu() - v).abs() <= 2.0 ** -20 * v).all()
        assert ((p[0][i].double().cpu() - want).abs() <= tol).all()
        if p[3][i] is not None:
            assert torch.equal(p[3][i], p[0][i].to(p[3][i].dtype))


def test_norm_repeats_whatever_the_workspace_held():
    g = ha.TensorList(grads_of(9, [100000, 31, 4097]))
    got = [ha.hybrid_attn_grad_norm(g, 1.0, workspace=torch.full((g.workspace_bytes,), f, dtype=torch.uint8, device="cuda")) for f in (0, 255)]
    assert torch.equal(*got)


def test_captured_and_replayed():
    g = grads_of(10, [5000, 33, 20000])
    p, q = params_of(11, g), params_of(11, g)
    kw = dict(lr=1e-2, kind=ha.HA_OPT_ADAMW, step=2)
    plist, qlist, glist = ha.ParamList(p[0], g, *p[1:]), ha.ParamList(q[0], g, *q[1:]), ha.TensorList(g)
    ws, res = torch.empty(glist.workspace_bytes, dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ha.hybrid_attn_grad_norm(glist, 1.0, result=res, workspace=ws)
        ha.hybrid_attn_param_update_many(plist, **kw, clip=res)
    for turn in range(4):
        for x in g:
            x.mul_(1.0 + turn)
        torch.cuda.synchronize()
        graph.replay()
        ha.hybrid_attn_param_update_many(qlist, **kw, clip=ha.hybrid_attn_grad_norm(glist, 1.0))
        torch.cuda.synchronize()
        assert all(a is None or torch.equal(a, b) for x, y in zip(p, q) for a, b in zip(x, y)), turn


def test_another_stream():
    g = grads_of(12)
    want = ha.hybrid_attn_grad_norm(g, 1.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = [torch.empty_like(x) for x in g]
    res = ha.hybrid_attn_grad_norm(g, 1.0, stream=side)
    ha.hybrid_attn_grad_clip(g, res, out, stream=side)
    side.synchronize()
    assert torch.equal(res, want)


def test_refusals():
    g = grads_of(13)
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_grad_norm(g, 0.0)
    with pytest.raises(ValueError, match="result"):
        ha.hybrid_attn_grad_clip(g, torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError, match="sizes"):
        ha.hybrid_attn_grad_clip(g, torch.zeros(2, device="cuda"), [x[:-1] if x.numel() else x for x in g])
    with pytest.raises(ValueError, match="contiguous"):
        ha.TensorList([torch.zeros(4, 4, device="cuda").t()])
    with pytest.raises(ValueError, match="fp32"):
        ha.ParamList([torch.zeros(4, device="cuda", dtype=torch.bfloat16)], [torch.zeros(4, device="cuda")])
    with pytest.raises(ValueError, match="one size"):
        ha.ParamList([torch.zeros(4, device="cuda")], [torch.zeros(5, device="cuda")])
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_param_update_many(ha.ParamList([torch.zeros(4, device="cuda")], [torch.zeros(4, device="cuda")]), 1e-3, kind=ha.HA_OPT_ADAMW)


def test_a_layers_training_step():
    """The distillation step of the two feature maps on a teacher that block-sparse attention forms, with its gradients clipped: the calls of one
    training program behind one another."""
    w = W.Workload("step", 1, 2, 700, 128, "bf16", 128, 4, 128, 128, seed=41)
    q, k, v, fq, fk = ha.to_device(W.make_inputs(w))
    blocks = ha.hybrid_attn_select_blocks(q, ha.hybrid_attn_key_means(k), 700, 6)
    teacher, _ = ha.hybrid_attn_sparse_forward(q, k, v, blocks)
    loss, gq, gk, *_ = ha.hybrid_attn_value_distill_grad(q, k, v, fq, fk, w.R, y_teacher=teacher, teacher_is_cached=True)
    names = ("w1", "b1", "w2", "b2")
    leaves = [getattr(m, n) for m in (fq, fk) for n in names]
    grads = [m[n] for m in (gq, gk) for n in names]
    masters = [t.float().clone() for t in leaves]
    start = [t.clone() for t in masters]
    moments = [[torch.zeros_like(t) for t in masters] for _ in range(2)]
    copies = [t if t.dtype == torch.bfloat16 else None for t in leaves]
    result = ha.hybrid_attn_grad_norm(grads, norm_of(grads) / 2)
    assert abs(float(result[1]) - 0.5) < 1e-6 and float(loss[0]) > 0
    ha.hybrid_attn_param_update_many(ha.ParamList(masters, grads, *moments, copies), 1e-3, kind=ha.HA_OPT_ADAMW, weight_decay=0.0, clip=result)
    for p, s, g, c in zip(masters, start, grads, copies):
        # AdamW's first step moves every parameter by lr against its gradient's sign
        big = g.abs() > 1e-3 * g.abs().max()
        assert ((s - p)[big] * g[big].sign() > 0.9e-3).all() and ((s - p).abs() <= 1.01e-3).all()
        assert c is None or torch.equal(c, p.bfloat16())
