"""fp32 tensors with finite values above bf16's largest, 3.3895e38, whose first piece must not round to infinity.  One key holds such values, so that sums do not
overflow, and logits and dP are products with values small enough to bring them down (2^-125, a normal number of one piece)."""
import pytest
import torch

from oracle import block_sparse_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.float32).max
UNITS = dict(u=5 * 2.0 ** -24, u_out=2.0 ** -24)


def randn(gen, N, d):
    return torch.randn(1, 1, N, d, generator=gen)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 70])
def test_values(N, d):
    gen = torch.Generator().manual_seed(1)
    q, k, v, do = (randn(gen, N, d) for _ in range(4))
    big = (3.402e38, -3.402e38, 3.396e38, -3.3962e38, 3.39e38)      # (a weight may be 1 + 1e-6 before it is divided by the sum of weights)
    for i, value in enumerate(big):
        v[:, :, 0, 5 * i + 1] = value
        do[..., 5 * i + 1] *= 2.0 ** -125
    q, k, v, do = (x.cuda() for x in (q, k, v, do))
    blocks = torch.zeros(1, 1, -(-N // 64), 1, dtype=torch.int32, device="cuda")
    if N > 64:
        blocks = torch.tensor([[0, -1], [0, 1]], dtype=torch.int32, device="cuda").view(1, 1, 2, 2)
    out, lse = ha.hybrid_attn_sparse_forward(q, k, v, blocks, 64, 64, True, with_lse=True)
    grads = ha.hybrid_attn_sparse_grad(q, k, v, blocks, out, lse, do, 64, 64, True)
    want = O.attention(q, k, v, blocks, 64, 64, True, dout=do, u_logit=(5 + d + 8) * 2.0 ** -24, **UNITS)
    assert torch.isfinite(want["out"]).all() and want["out"].abs().max() > 3.39e38
    # A piece is a multiple of 2^-133 (bf16's smallest number), so the third one of a dO near 2^-125 is off by up to 2^-134, whatever dO's own precision: dP_ij by
    # 2^-134 sum_c |v_jc|, which delta, formed of dO itself, does not share.
    qd, kd, vd = (x.double().cpu()[0, 0] for x in (q, k, v))
    weights = torch.softmax((qd @ kd.t() * d ** -0.5).masked_fill(torch.ones(N, N, dtype=torch.bool).triu(1), -torch.inf), 1)
    off = weights * (2.0 ** -134 * vd.abs().sum(1)) * d ** -0.5
    want["dq_tol"] += off @ kd.abs()
    want["dk_tol"] += off.t() @ qd.abs()
    want["dv_tol"] += (weights.sum(0) * 2.0 ** -134)[:, None]
    for name, got in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads)):
        assert ((got.double().cpu() - want[name]).abs() <= want[name + "_tol"]).all(), name


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 70])
@pytest.mark.parametrize("where", ["k", "q"])
def test_logits(where, N, d):
    gen = torch.Generator().manual_seed(3)
    small, big, v, do = (randn(gen, N, d) for _ in range(4))
    for i, value in enumerate((LARGEST, -LARGEST, 3.396e38, -3.3962e38, 3.39e38)):
        small[..., 5 * i + 1], big[:, :, N // 2, 5 * i + 1] = 2.0 ** -125, value
    q, k = (x.cuda() for x in ((small, big) if where == "k" else (big, small)))
    v = v.cuda()
    blocks = torch.tensor([0, 1], dtype=torch.int32, device="cuda").repeat(1, 1, -(-N // 64), 1)
    out, lse = ha.hybrid_attn_sparse_forward(q, k, v, blocks, 64, 64, with_lse=True)
    want = O.attention(q, k, v, blocks, 64, 64, u_logit=(5 + d + 8) * 2.0 ** -24, **UNITS)
    for name, got in (("out", out), ("lse", lse)):
        assert ((got.double().cpu() - want[name]).abs() <= want[name + "_tol"]).all(), name
