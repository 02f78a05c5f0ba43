"""What the elementwise bounds of bf16 results leave room for: that dS add up to nothing in every row, and how far results are off on the average.

Rows of dS.  sum_j dS_ij = 0.  A column of K that holds one value c for all keys makes column 0 of dQ_i equal to scale c sum_j dS_ij, and dK summed over the keys is
scale sum_i q_i sum_j dS_ij; with V far from zero the output's rounding alone puts delta off by more than dS_ij are.  Tiles of up to 512 keys take what is
left over out of dQ again, and put delta right for dK.  Bounds (u = 2^-8, half a step of bf16; f = fp32 sums, (d + 8) 2^-24 of the terms' absolute values, and 2^-20
for what the exponentials and the recomputed weights are off):
  left over in dQ     t = u sum |dS| + e, with e what delta is off: sum_c |dO_c| 2 u sum_j p_j |v_jc| (weights rounded, output rounded)
  dQ_i0               scale c (u t [t P rounded] + f sum |dS| + sum_j p_j f sum_c |dO_c v_jc|)
  sum_j dK_jc         sum_i scale |q_ic| (u sum |dS| [dS rounded] + sum_j p_j f sum_c |dO_c v_jc|) + u sum_j |dK_jc| [stored]
Without the correction dQ_i0 is scale c t for a t of random sign, some times its bound; test_bounds_see_rows_that_are_left_as_they_are has that on the CPU.

On the average.  Rounding to bf16 is off by 2^-8 / sqrt(3) of the power of two below a value, which is 2^-8 * 0.39 = 0.153 % of it on the average (root mean square, mantissas spread
over their logarithm; up to 0.17 % for other spreads).  Results that are sums of terms rounded independently (weights or dS), rounded again when stored, are off
by sqrt(2) times that: 0.22 - 0.24 %.  The limit is 0.3 %: a second rounding of the same terms, or one of four of them left out, does not pass."""
import math

import pytest
import torch

from oracle import block_sparse_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

U = 2.0 ** -8


def rounded(x):
    return x.to(torch.bfloat16).double()


def far_values(seed, Nq, Nk, d, only_row=None):
    """q [.., 0] = 0, k [.., 0] = c, v around a value of each column's own between 64 and 128: one head, all bf16 values."""
    gen = torch.Generator().manual_seed(seed)
    q, k, v, do = (torch.randn(1, 1, n, d, generator=gen) for n in (Nq, Nk, Nk, Nq))
    q[..., 0], k[..., 0], v = 0, 4.0, v + 64 + 64 * torch.rand(d, generator=gen)
    if only_row is not None:
        q[:, :, [i for i in range(Nq) if i != only_row]] = 0
    return [x.bfloat16() for x in (q, k, v, do)]


def terms(q, k, v, do):
    """Weights and dS in 64 bits, what delta may be off, and the fp32 sums of dP."""
    q, k, v, do = (x.double()[0, 0] for x in (q, k, v, do))
    d = q.shape[1]
    p = torch.softmax(q @ k.t() * d ** -0.5, 1)
    out, dp = p @ v, do @ v.t()
    ds = p * (dp - (do * out).sum(1, keepdim=True))
    f = (d + 8) * 2.0 ** -24 + 2.0 ** -20
    e = (do.abs() * 2 * U * (p @ v.abs())).sum(1)
    f_dp = f * (p * (do.abs() @ v.abs().t())).sum(1)
    return dict(p=p, dp=dp, ds=ds, out=out, e=e, f_dp=f_dp, f=f, sum_ds=ds.abs().sum(1), q=q, k=k, v=v, do=do, scale=d ** -0.5)


def dq_bound(t):
    left = U * t["sum_ds"] + t["e"]
    return t["scale"] * 4.0 * (U * left + t["f"] * t["sum_ds"] + t["f_dp"])


def dk_sum_bound(t):
    dk = t["scale"] * t["ds"].t() @ t["q"]
    return t["scale"] * (t["q"].abs() * (U * t["sum_ds"] + t["f_dp"])[:, None]).sum(0) + U * dk.abs().sum(0)


SHAPES = [(130, 64, 64), (130, 448, 64), (130, 512, 128), (64, 512, 64), (1, 130, 64), (33, 16, 128)]


@pytest.mark.parametrize("Nq,Nk,d", SHAPES)
def test_bounds_see_rows_that_are_left_as_they_are(Nq, Nk, d):
    """The same roundings in 64 bits: with the correction within the bounds, without it, or with its sign turned, outside."""
    t = terms(*far_values(1, Nq, Nk, d, Nq - 1))
    e = rounded(t["p"] * 128)                            # weights rounded at some power of two
    out = rounded(e @ t["v"] / (t["p"] * 128).sum(1, keepdim=True))
    delta = (t["do"] * out).sum(1, keepdim=True)
    raw = t["p"] * (t["dp"] - delta)
    total = rounded(raw).sum(1, keepdim=True)

    def dq0(correction):
        return t["scale"] * 4.0 * (rounded(raw).sum(1) + rounded(-correction * total * t["p"]).sum(1))

    def dk_sum(correction):
        ds = t["p"] * (t["dp"] - delta - correction * raw.sum(1, keepdim=True))
        return rounded(t["scale"] * rounded(ds).t() @ t["q"]).sum(0)
    assert (dq0(1.0).abs() <= dq_bound(t)).all()
    assert (dk_sum(1.0).abs() <= dk_sum_bound(t)).all()
    for wrong in (0.0, -1.0):
        assert (dq0(wrong).abs() > dq_bound(t)).double().mean() > 0.5
        assert (dk_sum(wrong).abs() > dk_sum_bound(t)).any(), wrong


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk,d", SHAPES)
@pytest.mark.parametrize("qb,kb", [(64, 64), (128, 64), (128, 128)])
@pytest.mark.parametrize("row", [None, "middle", "last"])
def test_dS_of_a_row_add_up_to_nothing(Nq, Nk, d, qb, kb, row):
    x = far_values(1, Nq, Nk, d, {None: None, "middle": Nq // 2, "last": Nq - 1}[row])
    t = terms(*x)
    q, k, v, do = (a.cuda() for a in x)
    blocks = torch.arange(-(-Nk // kb), dtype=torch.int32, device="cuda").repeat(1, 1, -(-Nq // qb), 1)
    out, lse = ha.hybrid_attn_sparse_forward(q, k, v, blocks, qb, kb, with_lse=True)
    dq, dk, _ = ha.hybrid_attn_sparse_grad(q, k, v, blocks, out, lse, do, qb, kb)
    assert (dq[0, 0, :, 0].double().cpu().abs() <= dq_bound(t)).all()
    assert (dk[0, 0].double().cpu().sum(0).abs() <= dk_sum_bound(t)).all()


def relative(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("qb,kb,sel", [(64, 64, 1), (64, 64, 8), (128, 64, 8), (128, 128, 3), (64, 128, 12), (128, 64, 20)])
@pytest.mark.parametrize("causal", [False, True])
def test_results_on_the_average(d, qb, kb, sel, causal):
    gen = torch.Generator().manual_seed(2)
    N = 1500
    q, k, v, do = (torch.randn(1, h, N, d, generator=gen).bfloat16().cuda() for h in (2, 1, 1, 2))
    tiles, blocks = -(-N // qb), -(-N // kb)
    lists = torch.stack([torch.randperm(blocks, generator=gen)[:sel].sort().values for _ in range(tiles)]).to(torch.int32)
    if causal:                                          # a tile's own blocks among them
        lists[:, 0] = torch.arange(tiles) * qb // kb
    lists = lists.view(1, 1, tiles, sel).cuda()
    out, lse = ha.hybrid_attn_sparse_forward(q, k, v, lists, qb, kb, causal, with_lse=True)
    got = (out, *ha.hybrid_attn_sparse_grad(q, k, v, lists, out, lse, do, qb, kb, causal))
    want = O.attention(q, k, v, lists, qb, kb, causal, dout=do)
    off = {n: relative(g, want[n]) for n, g in zip(("out", "dq", "dk", "dv"), got)}
    assert all(x < 0.003 for x in off.values()), off
    seen = torch.isfinite(want["lse"])
    assert (lse.double().cpu() - want["lse"])[seen].abs().max() < 1e-5 * math.log(N)
