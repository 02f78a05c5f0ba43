"""Rotary positions, and the norm with them, against their definitions in 64 bits (oracle/rotary_oracle.py, which derives how far fp32 may be off).  The result is rounded to
the tensors' type: half a step, 2^-8 of bf16 and 2^-24 of fp32."""
import math

import pytest
import torch

from oracle import rotary_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def tokens(gen, B, H, N, d, dtype, layout="bhnd", gain=1.0):
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    x = (torch.randn(shape, generator=gen) * gain).to(dtype).cuda()
    return x if layout == "bhnd" else x.transpose(1, 2)


def close(got, want, off, what=""):
    assert torch.isfinite(got).all(), what
    over = (got.double().cpu() - want).abs() - off - want.abs() * STEP.get(got.dtype, 0.0)
    assert (over <= 0).all(), (what, float(over.max()), float(off.max()))


def rotary_of(rot, axes, interleaved, stretch=1.0, magnitude=None):
    r = ha.hybrid_attn_rotary_grid(rot, interleaved=interleaved) if axes == 3 else ha.hybrid_attn_rotary_frequencies(rot, interleaved=interleaved, stretch=stretch, original=4096)
    return r if magnitude is None else r._replace(magnitude=magnitude)


def places(gen, B, N, axes, far, own):
    shape = (B, N, axes) if own else (N, axes)
    return torch.randint(-far, far + 1, shape, generator=gen, dtype=torch.int32).cuda()


CASES = [
    # B, H, Hkv, N, d, dtype, layout, rot, interleaved, axes, far, positions for each entry
    (1, 1, 1, 1, 64, torch.bfloat16, "bhnd", 64, True, 1, 10, False),
    (1, 2, 2, 1024, 64, torch.float32, "bhnd", 64, True, 3, 16, False),
    (2, 3, 1, 333, 128, torch.bfloat16, "bnhd", 128, True, 3, 50, False),
    (2, 12, 4, 67, 128, torch.bfloat16, "bnhd", 128, False, 1, 1000, True),
    (2, 6, 2, 501, 64, torch.float32, "bnhd", 32, False, 1, 2 ** 31 - 2, True),
    (3, 5, 5, 17, 128, torch.float32, "bhnd", 96, False, 1, 1000000, False),
    (1, 7, 1, 45, 128, torch.float32, "bhnd", 90, True, 3, 200, False),
    (1, 2, 2, 31, 64, torch.bfloat16, "bhnd", 6, True, 3, 40, False),
    (2, 9, 3, 16, 64, torch.bfloat16, "bnhd", 8, False, 1, 40, True),
    (1, 24, 24, 15, 128, torch.bfloat16, "bhnd", 128, True, 1, 5, False),
    (1, 2, 2, 40000, 64, torch.bfloat16, "bhnd", 64, True, 1, 40000, False),
]


@pytest.mark.parametrize("B,H,Hkv,N,d,dtype,layout,rot,interleaved,axes,far,own", CASES)
def test_rotate(B, H, Hkv, N, d, dtype, layout, rot, interleaved, axes, far, own):
    gen = torch.Generator().manual_seed(N + d)
    x, at, r = tokens(gen, B, H, N, d, dtype, layout), places(gen, B, N, axes, far, own), rotary_of(rot, axes, interleaved, 4.0)
    for f, back in ((ha.hybrid_attn_rotate, False), (ha.hybrid_attn_rotate_grad, True)):
        close(f(x, r, at), *O.turn(x, r.freq, r.axis, at, interleaved, r.magnitude, back))
        y = x.clone()
        assert f(y, r, at, out=y) is y and torch.equal(y, f(x, r, at))


@pytest.mark.parametrize("B,H,Hkv,N,d,dtype,layout,rot,interleaved,axes,far,own", CASES)
def test_norm_rotate_and_gradients(B, H, Hkv, N, d, dtype, layout, rot, interleaved, axes, far, own):
    gen = torch.Generator().manual_seed(N + d + 1)
    q, k = tokens(gen, B, H, N, d, dtype, layout, 3.0), tokens(gen, B, Hkv, N, d, dtype, layout, 0.01)
    gq, gk = tokens(gen, B, H, N, d, dtype, layout), tokens(gen, B, Hkv, N, d, dtype, layout)
    w_q, w_k = ((torch.randn(d, generator=gen) + 1).cuda() for _ in range(2))
    at, r, eps = places(gen, B, N, axes, far, own), rotary_of(rot, axes, interleaved), 1e-5
    q2, k2 = ha.hybrid_attn_norm_rotate(q, k, w_q, w_k, r, at, eps)
    dq, dk, dw_q, dw_k = ha.hybrid_attn_norm_rotate_grad(gq, gk, q, k, w_q, w_k, r, at, eps)
    groups = B * -(-N // (2048 // d))
    terms = (H + Hkv) * -(-groups // min(groups, 1024))
    for x, y, w, g, dx, dw, name in ((q, q2, w_q, gq, dq, dw_q, "q"), (k, k2, w_k, gk, dk, dw_k, "k")):
        close(y, *O.norm_rotate(x, w, eps, r, at), name)
        want = O.norm_rotate_grad(g, x, w, eps, r, at, terms)
        close(dx, *want[:2], "d" + name)
        close(dw, *want[2:], "dw_" + name)
    again = ha.hybrid_attn_norm_rotate_grad(gq, gk, q, k, w_q, w_k, r, at, eps)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dw_q, dw_k)))
    # in place, without keys, without weights, without rotation
    a, b = q.clone(), k.clone()
    ha.hybrid_attn_norm_rotate(a, b, w_q, w_k, r, at, eps, q_out=a, k_out=b)
    assert torch.equal(a, q2) and torch.equal(b, k2)
    assert torch.equal(ha.hybrid_attn_norm_rotate(q, None, w_q, None, r, at, eps)[0], q2)
    close(ha.hybrid_attn_norm_rotate(q, k, eps=eps)[1], *O.norm_rotate(k, None, eps, None, None))
    want = O.norm_rotate_grad(gq, q, None, eps, r, at, terms)[:2]
    alone = ha.hybrid_attn_norm_rotate_grad(gq, None, q, None, None, None, r, at, eps, grad_in_q=gq)
    assert alone[0] is gq and alone[1:] == (None, None, None)
    close(gq, *want)


def test_gradients_against_differences():
    """Central differences of sum(g . out) in fp32: the third derivative's part is h^2 / 6 times some units, the rounding's 2^-24 / h of the sum of magnitudes."""
    gen = torch.Generator().manual_seed(3)
    B, H, Hkv, N, d = 1, 2, 1, 5, 64
    q, k, gq, gk = (tokens(gen, B, h, N, d, torch.float32) for h in (H, Hkv, H, Hkv))
    w_q, w_k = ((torch.randn(d, generator=gen) * 0.2 + 1).cuda() for _ in range(2))
    at, r = places(gen, B, N, 1, 100, False), rotary_of(64, 1, False)
    dq, dk, dw_q, dw_k = ha.hybrid_attn_norm_rotate_grad(gq, gk, q, k, w_q, w_k, r, at)

    def value(*t):
        a, b = ha.hybrid_attn_norm_rotate(*t, r, at)
        return float((a.double() * gq.double()).sum() + (b.double() * gk.double()).sum())
    args, h = [q, k, w_q, w_k], 2.0 ** -5
    size = float((gq.abs().sum() + gk.abs().sum()) * 3)
    for i, grad in enumerate((dq, dk, dw_q, dw_k)):
        for at_ in (0, 63, grad.numel() // 2, grad.numel() - 1):
            moved = []
            for sign in (1, -1):
                t = [x.clone() for x in args]
                t[i].view(-1)[at_] += sign * h
                moved.append((value(*t), float(t[i].view(-1)[at_])))
            slope = (moved[0][0] - moved[1][0]) / (moved[0][1] - moved[1][1])
            assert abs(slope - float(grad.reshape(-1)[at_])) <= h * h * 4 + size * 2.0 ** -22 / h, (i, at_)


def test_channels_that_pass_through_keep_infinities_to_themselves():
    for interleaved in (True, False):
        x = torch.ones(1, 1, 3, 64, device="cuda")
        x[..., 40], x[..., 47] = math.inf, math.nan
        at = torch.arange(3, dtype=torch.int32, device="cuda")[:, None].contiguous()
        y = ha.hybrid_attn_rotate(x, rotary_of(16, 1, interleaved), at)
        assert torch.equal(y[..., 16:].nan_to_num(7, 8), x[..., 16:].nan_to_num(7, 8)) and torch.isfinite(y[..., :16]).all()


def test_no_tokens():
    q = torch.zeros(2, 3, 0, 64, device="cuda")
    w, at = torch.ones(64, device="cuda"), torch.zeros(0, 1, dtype=torch.int32, device="cuda")
    r = rotary_of(64, 1, True)
    assert ha.hybrid_attn_rotate(q, r, at).shape == q.shape
    assert ha.hybrid_attn_norm_rotate(q, q, w, w, r, at)[1].shape == q.shape
    dw = torch.full((64,), 5.0, device="cuda")
    got = ha.hybrid_attn_norm_rotate_grad(q, q, q, q, w, w, r, at, grad_w_q=dw)
    assert got[2] is dw and not dw.any() and not got[3].any()


def test_captured_with_an_eager_run_between_the_replays():
    gen = torch.Generator().manual_seed(9)
    q, k, g = (tokens(gen, 1, 4, 200, 128, torch.bfloat16) for _ in range(3))
    w = torch.ones(128, device="cuda")
    at, r = places(gen, 1, 200, 1, 100, False), rotary_of(128, 1, True)

    def step():
        return (*ha.hybrid_attn_norm_rotate(q, k, w, w, r, at), *ha.hybrid_attn_norm_rotate_grad(g, g, q, k, w, w, r, at), ha.hybrid_attn_rotate(q, r, at))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(3):
        q.copy_(tokens(torch.Generator().manual_seed(seed), 1, 4, 200, 128, torch.bfloat16))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream_and_with_refusals():
    x = torch.randn(1, 2, 50, 64, device="cuda")
    at, r = torch.arange(50, dtype=torch.int32, device="cuda")[:, None].contiguous(), rotary_of(64, 1, True)
    want = ha.hybrid_attn_rotate(x, r, at)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ha.hybrid_attn_rotate(x, r, at, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    for bad in (at[:40].contiguous(), at.long(), at.cpu(), None):
        with pytest.raises((ValueError, RuntimeError)):
            ha.hybrid_attn_rotate(x, r, bad)
    for bad in (r._replace(freq=r.freq.float()), r._replace(axis=torch.zeros(5, dtype=torch.int32, device="cuda")), r._replace(magnitude=math.inf), r._replace(freq=torch.zeros(40, dtype=torch.float64, device="cuda"))):
        with pytest.raises((ValueError, ha.HybridAttnError)):
            ha.hybrid_attn_rotate(x, bad, at)
    with pytest.raises(ValueError):
        ha.hybrid_attn_norm_rotate(x, x.half().float()[:, :, :20], rotary=r, positions=at)
    with pytest.raises(ValueError):
        ha.hybrid_attn_norm_rotate(x, x.bfloat16(), rotary=r, positions=at)
    with pytest.raises(ValueError):
        ha.hybrid_attn_norm_rotate(x, x, torch.ones(32, device="cuda"))
    with pytest.raises(RuntimeError):
        ha.hybrid_attn_rotate(x.cpu(), r, at)
