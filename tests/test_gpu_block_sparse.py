"""Block-sparse attention against the definition in 64 bits (oracle/block_sparse_oracle.py), at the sizes, masks and layouts where it can go wrong.

Tolerances.  bf16: products of bf16 values are exact in fp32, so a logit is off by the fp32 sum alone (d terms, d 2^-24 of the sum of absolute terms); a
weight or a term of the gradients is rounded to bf16 (2^-8 of its value) before it is multiplied, and the result is (2^-8).  fp32: an operand in three
pieces of 8 bits is off by 2^-24 of its value, and the three products left out are 2^-24, 2^-24 and 2^-32 of theirs: 5 2^-24 a product; weights and terms in the
gradients are split likewise.
The oracle adds these up over the terms of every single result."""
import numpy as np
import pytest
import torch

from oracle import block_sparse_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu


def units(dtype, d):
    return dict(u=2.0 ** -8, u_logit=(d + 8) * 2.0 ** -24, u_out=2.0 ** -8) if dtype == torch.bfloat16 else \
        dict(u=5 * 2.0 ** -24, u_logit=(5 + d + 8) * 2.0 ** -24, u_out=2.0 ** -24)


def tokens(gen, B, H, N, d, dtype, layout="bhnd", gain=1.0):
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    x = (torch.randn(shape, generator=gen) * gain).to(dtype).cuda()
    return x if layout == "bhnd" else x.transpose(1, 2)


def problem(seed, B=1, H=2, Hkv=2, Nq=200, Nk=None, d=128, dtype=torch.bfloat16, qb=128, kb=64, sel=3, causal=False, ragged=None, starts=None, layout="bhnd", gain=1.0):
    gen = torch.Generator().manual_seed(seed)
    Nk = Nq if Nk is None else Nk
    q, k, v, do = tokens(gen, B, H, Nq, d, dtype, layout, gain), tokens(gen, B, Hkv, Nk, d, dtype, layout, gain), tokens(gen, B, Hkv, Nk, d, dtype, layout), tokens(gen, B, H, Nq, d, dtype, layout)
    T, Tk = -(-Nq // qb), -(-Nk // kb)
    rows = [torch.randperm(max(Tk, 1), generator=gen)[:min(sel, Tk)].sort().values for _ in range(B * Hkv * T)]
    blocks = torch.full((B, Hkv, T, sel), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        blocks.view(-1, sel)[i, :len(r)] = r.to(torch.int32)
    def per_entry(x):
        return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    return dict(q=q, k=k, v=v, dout=do, blocks=blocks.cuda(), args=dict(q_block=qb, k_block=kb, causal=causal, q_start=per_entry(starts), key_len=per_entry(ragged)))


def reference(p, scale=None):
    a, d = p["args"], p["q"].shape[3]
    return O.attention(p["q"], p["k"], p["v"], p["blocks"], a["q_block"], a["k_block"], a["causal"], a["q_start"], a["key_len"], scale, p["dout"], **units(p["q"].dtype, d))


def close(name, got, ref, what=""):
    got, want, tol = got.double().cpu(), ref[name], ref[name + "_tol"]
    assert torch.equal(torch.isneginf(got), torch.isneginf(want)), (name, what)
    fine = torch.isfinite(want)
    off = ((got - want).abs() - tol)[fine]
    assert torch.isfinite(got[fine]).all() and (off <= 0).all(), (name, what, float(off.max()), float(tol.max()))


def check(p, scale=None, grad=True):
    out, lse = ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], p["blocks"], **p["args"], softmax_scale=scale, with_lse=True)
    ref = reference(p, scale)
    close("out", out, ref)
    close("lse", lse, ref)
    if grad:
        grads = ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], p["blocks"], out, lse, p["dout"], **p["args"], softmax_scale=scale)
        for name, g in zip(("dq", "dk", "dv"), grads):
            close(name, g, ref)
    return out, lse, ref


BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("qb,kb", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_forward_and_gradients(d, dtype, qb, kb, causal):
    check(problem(1, Nq=333, d=d, dtype=dtype, qb=qb, kb=kb, sel=2, causal=causal))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Nq,Nk", [(1, 1), (1, 700), (2, 63), (31, 64), (33, 65), (64, 129), (129, 31), (257, 130)])
def test_lengths(dtype, Nq, Nk):
    check(problem(2, Nq=Nq, Nk=Nk, dtype=dtype, sel=4))
    check(problem(3, Nq=Nq, Nk=Nk, dtype=dtype, d=64, sel=2, causal=True, starts=[0]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G", [2, 3, 8])
def test_heads_that_share_keys(dtype, G):
    check(problem(4, B=2, H=2 * G, Hkv=2, Nq=150, dtype=dtype, d=64, qb=64, causal=True))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_projection_layout_and_strides(dtype):
    check(problem(5, B=2, H=3, Hkv=3, Nq=190, dtype=dtype, layout="bnhd"))
    p = problem(6, B=2, H=3, Hkv=3, Nq=190, dtype=dtype)
    wide = torch.zeros(2, 3, 2 * 190, 256, dtype=dtype, device="cuda")
    wide[:, :, ::2, 128:] = p["k"]
    p["k"] = wide[:, :, ::2, 128:]                      # every other row of a wider tensor
    p["v"] = p["v"][:, :1].expand(2, 3, 190, 128)       # one head's values for all
    p["q"] = p["q"][:1].expand(2, 3, 190, 128)          # one batch entry's queries for both
    check(p)


def test_broadcast_gradients_are_whole_tensors():
    p = problem(7, B=2, H=2, Hkv=2, Nq=70)
    p["k"] = p["k"][:1].expand(2, 2, 70, 128)
    out, lse = ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], p["blocks"], **p["args"], with_lse=True)
    _, dk, _ = ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], p["blocks"], out, lse, p["dout"], **p["args"])
    assert dk.shape == p["k"].shape and dk.stride(0) > 0
    close("dk", dk, reference(p))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing(dtype):
    # causal rows ahead of their tile's only block, entries without keys, lists without blocks
    p = problem(8, B=3, Nq=140, dtype=dtype, d=64, qb=64, sel=1, causal=True, ragged=[0, 70, 140])
    p["blocks"][0] = 0
    p["blocks"][1, 0] = -1
    p["blocks"][2, :, :, 0] = torch.tensor([1, 1, 2], device="cuda", dtype=torch.int32)
    out, lse, ref = check(p)
    assert torch.isneginf(ref["lse"]).sum() > 100 and not out[torch.isneginf(lse)].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ragged,starts", [([200, 131, 1], None), ([64, 0, 199], [0, 0, 60]), ([200, 100, 300], [-50, 199, 3])])
def test_ragged_batches_and_places(dtype, ragged, starts):
    check(problem(9, B=3, Nq=90, Nk=200, dtype=dtype, qb=64, causal=True, ragged=ragged, starts=starts))
    check(problem(10, B=3, Nq=90, Nk=200, dtype=dtype, qb=64, ragged=ragged))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.0e38])
def test_nothing_behind_the_last_key_is_used(dtype, bad):
    p = problem(11, B=2, Nq=100, Nk=300, dtype=dtype, kb=128, sel=3, ragged=[170, 129], causal=True, starts=[69, 28])
    for b, n in enumerate((170, 129)):
        p["k"][b, :, n:], p["v"][b, :, n:] = bad, bad
    check(p)
    # a causal tile never reads behind its own last position
    p = problem(12, Nq=1, Nk=300, dtype=dtype, causal=True, starts=[140], sel=5)
    p["k"][:, :, 141:], p["v"][:, :, 141:] = bad, bad
    check(p)


def test_indices_outside_and_repeated():
    p = problem(13, Nq=130, Nk=200, sel=6)
    p["blocks"][:] = torch.tensor([3, -7, 1, 1, 4, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    check(p)                                            # block 1 counts twice, 4 does not exist
    p["blocks"][:] = torch.tensor([-1, -1, -2 ** 31, 9, 0, 0], dtype=torch.int32, device="cuda")
    check(p)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_lists(dtype):
    check(problem(14, H=1, Hkv=1, Nq=70, Nk=9000, dtype=dtype, d=64, qb=64, kb=64, sel=140))


def test_gradients_over_more_blocks_than_are_counted_at_once():
    check(problem(51, H=1, Hkv=1, Nq=700, Nk=64 * 4100 + 5, d=64, qb=64, kb=64, sel=6))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sel", [1, 2, 3, 4, 7])
def test_more_short_tiles_than_two_to_a_cu(d, sel):
    """Tiles of 64 queries with less of LDS each, lists that end at every place of the unrolled loop."""
    check(problem(60 + sel, B=1, H=26, Hkv=2, Nq=1270, Nk=64 * 9 - 40, d=d, qb=64, kb=64, sel=sel))
    check(problem(70 + sel, B=2, H=13, Hkv=1, Nq=1270, d=d, qb=64, kb=128, sel=sel, causal=True, ragged=[1270, 700], starts=[0, -300]))


def test_lists_around_the_length_that_is_walked_twice():
    """448, 512 and 576 keys to a row, in tiles of one launch (causal) and of one length."""
    check(problem(52, H=2, Hkv=1, Nq=900, d=64, qb=64, kb=64, sel=16, causal=True))
    for sel in (7, 8, 9):
        check(problem(53 + sel, H=1, Hkv=1, Nq=130, Nk=1000, qb=128, kb=64, sel=sel))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,Nq", [(1, 1), (3, 1), (8, 4), (32, 1), (5, 6), (1, 32), (33, 1), (11, 3)])
def test_few_queries(dtype, d, G, Nq):
    # one list for all queries of a group: up to 32 of them, and one more
    for sel, kb in ((1, 64), (7, 128), (40, 64)):
        check(problem(23, B=2, H=2 * G, Hkv=2, Nq=Nq, Nk=2777, d=d, dtype=dtype, kb=kb, sel=sel, causal=True, ragged=[2777, 1500], starts=[2777 - Nq, 1500 - Nq]), grad=False)
    check(problem(24, H=G, Hkv=1, Nq=Nq, Nk=200, d=d, dtype=dtype, sel=3, layout="bnhd"))


def test_many_heads_of_few_queries():
    check(problem(25, B=70, H=4, Hkv=4, Nq=1, Nk=300, d=64, sel=4), grad=False)            # lists that are not cut
    check(problem(26, B=3, H=2, Hkv=1, Nq=9, Nk=20000, d=64, sel=200, kb=64), grad=False)   # and ones that are, into many ranges


def test_popular_blocks_are_joined_from_parts():
    p = problem(15, H=2, Hkv=1, Nq=64 * 150 + 3, Nk=200, d=64, qb=64, kb=64, sel=2)       # 151 tiles on four blocks: parts of 64
    check(p)


@pytest.mark.parametrize("gain,scale", [(4.0, None), (1.0, 1.0), (0.01, 30.0)])
def test_peaked_logits(gain, scale):
    check(problem(16, Nq=180, d=64, gain=gain), scale)


def test_rising_maxima():
    p = problem(17, Nq=64, Nk=640, qb=64, sel=10, d=64)
    p["k"] *= torch.linspace(0.05, 6.0, 640, device="cuda")[None, None, :, None]
    check(p)


def test_results_repeat_bit_for_bit_whatever_the_workspace_held():
    p = problem(18, B=2, H=4, Hkv=2, Nq=400, causal=True, sel=3)
    prob = ha.make_sparse_problem(p["q"].shape, p["k"].shape, BF16, p["q"].device, n_select=3, causal=True)
    got = []
    for fill in (0, 255):
        ws = torch.full((max(1, ha.hybrid_attn_sparse_workspace_bytes(prob)),), fill, dtype=torch.uint8, device="cuda")
        out, lse = ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], p["blocks"], **p["args"], with_lse=True, workspace=ws)
        ws = torch.full((ha.hybrid_attn_sparse_grad_workspace_bytes(prob),), fill, dtype=torch.uint8, device="cuda")
        got.append((out, lse, *ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], p["blocks"], out, lse, p["dout"], **p["args"], workspace=ws)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_outputs_are_written_in_full_and_nothing_beside_them():
    p = problem(19, Nq=77, Nk=131, d=64, sel=2, causal=True, starts=[54])
    out, lse, ref = check(p)
    room = {n: torch.full((1, 2, N + 2, 96), 7.0, dtype=BF16, device="cuda") for n, N in (("out", 77), ("dq", 77), ("dk", 131), ("dv", 131))}
    view = {n: t[:, :, 1:-1, 16:80] for n, t in room.items()}
    ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], p["blocks"], **p["args"], out=view["out"])
    ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], p["blocks"], out, lse, p["dout"], **p["args"], grad_q=view["dq"], grad_k=view["dk"], grad_v=view["dv"])
    for n, t in view.items():
        close(n, t, ref)
        t.fill_(7.0)
        assert (room[n] == 7.0).all(), n


def test_gradient_against_differences():
    """The derivative along random directions, from central differences of the 64-bit forward."""
    p = problem(20, B=1, H=4, Hkv=2, Nq=70, Nk=130, d=64, dtype=F32, qb=64, sel=2, causal=True, starts=[60])
    a = p["args"]
    out, lse, ref = check(p)
    grads = ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], p["blocks"], out, lse, p["dout"], **a)

    def loss(x):
        y = O.attention(x["q"], x["k"], x["v"], p["blocks"], 64, a["k_block"], True, a["q_start"])["out"]
        return float((y * p["dout"].double().cpu()).sum())
    gen = torch.Generator().manual_seed(21)
    for name, g, tol in zip(("q", "k", "v"), grads, ("dq_tol", "dk_tol", "dv_tol")):
        way, h = torch.randn(g.shape, generator=gen, dtype=torch.float64), 1e-4
        x = {n: p[n].double().cpu() for n in ("q", "k", "v")}
        up, down = dict(x, **{name: x[name] + h * way}), dict(x, **{name: x[name] - h * way})
        slope = (loss(up) - loss(down)) / (2 * h)
        # h^2 terms: below 1e-6 of the sum of |g way| for logits of this size
        assert abs(slope - float((g.double().cpu() * way).sum())) <= float((ref[tol] * way.abs()).sum()) + 1e-6 * float((g.double().cpu() * way).abs().sum())


def test_long_offsets():
    """Rows that lie beyond 2^32 bytes of a tensor's start."""
    N, d = 1100, 64
    base = torch.zeros((N - 1) * (1 << 21) + 2 * d, dtype=BF16, device="cuda")
    k = base.as_strided((1, 1, N, d), (base.numel(), base.numel(), 1 << 21, 1))
    v = base.as_strided((1, 1, N, d), (base.numel(), base.numel(), 1 << 21, 1), d)
    p = problem(22, H=1, Hkv=1, Nq=40, Nk=N, d=d, qb=64, sel=3)
    k.copy_(p["k"])
    v.copy_(p["v"])
    p["blocks"][:] = torch.tensor([0, 9, 17], dtype=torch.int32, device="cuda")
    p["k"], p["v"] = k, v
    out, lse = ha.hybrid_attn_sparse_forward(p["q"], k, v, p["blocks"], **p["args"], with_lse=True)
    ref = reference(p)
    close("out", out, ref)
    means = ha.hybrid_attn_key_means(k, 64)
    assert torch.equal(means.cpu(), O.key_means(k, 64).float())
    dq, dk, dv = ha.hybrid_attn_sparse_grad(p["q"], k, v, p["blocks"], out, lse, p["dout"], **p["args"], grad_k=torch.empty(1, 1, N, d, dtype=BF16, device="cuda"),
                                            grad_v=torch.empty(1, 1, N, d, dtype=BF16, device="cuda"))
    close("dq", dq, ref)
    close("dk", dk, ref)


# ---- the choice ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,kb", [(64, 64), (128, 128)])
@pytest.mark.parametrize("ragged", [None, [0, 1, 64, 200, 333, 500]])
def test_key_means(dtype, d, kb, ragged):
    gen = torch.Generator().manual_seed(30)
    k = tokens(gen, 6, 3, 333, d, dtype, "bnhd")
    n = None if ragged is None else torch.tensor(ragged, dtype=torch.int32, device="cuda")
    if ragged:
        for b, m in enumerate(ragged):
            k[b, :, m:] = float("nan")
    got, want = ha.hybrid_attn_key_means(k, kb, key_len=n).cpu(), O.key_means(k, kb, n)
    # one rounding to fp32, and of fp32 keys the double sum's
    assert ((got.double() - want).abs() <= 2.0 ** -24 * want.abs() * (1 + 1e-6) + 1e-16).all()


@pytest.mark.parametrize("m", [1, 2, 9])
def test_last_means_only(m):
    gen = torch.Generator().manual_seed(31)
    k = tokens(gen, 4, 2, 500, 64, BF16)
    n = torch.tensor([0, 64, 257, 500], dtype=torch.int32, device="cuda")
    got = ha.hybrid_attn_key_means(k, 64, key_len=n, only_last=m, out=torch.full((4, 2, 8, 64), 5.0, device="cuda")).cpu()
    want = O.key_means(k, 64, n).float()
    for b, held in enumerate((0, 64, 257, 500)):
        last = -(-held // 64)
        for j in range(8):
            if max(0, last - m) <= j < last:
                assert torch.equal(got[b, :, j], want[b, :, j])
            else:
                assert (got[b, :, j] == 5.0).all()


def chosen(q, k, sel, qb, kb, **mask):
    means = ha.hybrid_attn_key_means(k, kb, key_len=mask.get("key_len"))
    return ha.hybrid_attn_select_blocks(q, means, k.shape[2], sel, qb, kb, **mask).cpu(), O.select(q, means, k.shape[2], sel, qb, kb, **mask)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(), dict(keep_first=1), dict(near=0), dict(near=70), dict(causal=True, near=0), dict(causal=True, near=64, keep_first=2)])
@pytest.mark.parametrize("qb,kb", [(64, 64), (128, 64), (64, 128)])
def test_choice(dtype, d, kw, qb, kb):
    gen = torch.Generator().manual_seed(32)
    q, k = tokens(gen, 2, 4, 707, d, dtype, "bnhd"), tokens(gen, 2, 2, 707, d, dtype)
    got, want = chosen(q, k, 7, qb, kb, **kw)
    assert torch.equal(got, want)


@pytest.mark.parametrize("Nk,sel", [(1, 1), (64, 3), (65, 2), (16 * 64, 16), (300 * 64, 5), (700 * 64 - 3, 33), (1500 * 64, 64), (2100 * 64 + 1, 300)])
def test_choice_of_many_blocks_for_one_query(Nk, sel):
    gen = torch.Generator().manual_seed(33)
    q, k = tokens(gen, 2, 2, 1, 64, BF16), tokens(gen, 2, 1, Nk, 64, BF16)
    got, want = chosen(q, k, sel, 128, 64, causal=True, near=0)
    assert torch.equal(got, want)


@pytest.mark.parametrize("N,Nk,H,sel,kb", [(64 * 300, 64 * 200, 1, 5, 64), (64 * 130, 64 * 600, 2, 16, 64), (64 * 100, 64 * 1000, 3, 9, 64), (64 * 260, 128 * 1100, 1, 64, 128), (64 * 1030, 64 * 256, 1, 7, 64),
                                           (64 * 1025, 64 * 257, 1, 20, 64), (64 * 140, 64 * 2100, 1, 40, 64)])
def test_choice_of_many_tiles(N, Nk, H, sel, kb):
    gen = torch.Generator().manual_seed(36)
    q, k = tokens(gen, 1, H, N - 7, 64, BF16), tokens(gen, 1, H, Nk - 1, 64, BF16)
    means = ha.hybrid_attn_key_means(k, kb)
    got = ha.hybrid_attn_select_blocks(q, means, Nk - 1, sel, 64, kb)
    rows = torch.nn.functional.pad(q.double(), (0, 0, 0, 7)).view(1, H, N // 64, 64, 64).sum(3)
    best = torch.sort(rows @ means.double().transpose(2, 3).contiguous(), dim=3, descending=True, stable=True).indices[..., :sel]
    assert torch.equal(got, best.sort(dim=3).values.to(torch.int32))


def test_choice_of_ragged_batches():
    gen = torch.Generator().manual_seed(34)
    q, k = tokens(gen, 4, 2, 100, 64, BF16), tokens(gen, 4, 2, 900, 64, BF16)
    n = torch.tensor([0, 30, 500, 900], dtype=torch.int32, device="cuda")
    s = torch.tensor([0, -20, 400, 800], dtype=torch.int32, device="cuda")
    for kw in (dict(), dict(q_start=s, causal=True, near=0), dict(q_start=s, near=40, keep_first=1)):        # (100 tokens would not fit a list of six)
        got, want = chosen(q, k, 6, 64, 64, key_len=n, **kw)
        assert torch.equal(got, want), kw
    assert (got[0] == -1).all()


def test_equal_scores_go_to_the_lowest_index():
    gen = torch.Generator().manual_seed(35)
    q = tokens(gen, 1, 1, 200, 64, BF16)
    k = tokens(gen, 1, 1, 64, 64, BF16).repeat(1, 1, 40, 1)                 # forty equal blocks
    got, want = chosen(q, k, 6, 64, 64)
    assert torch.equal(got, want) and got[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5]
    k[:, :, 64 * 7:64 * 9] *= 2
    k[:, :, 64 * 20:64 * 21] = 0
    got, want = chosen(q, k, 6, 64, 64)
    assert torch.equal(got, want)
    got, want = chosen(torch.zeros_like(q), -k, 5, 64, 64, near=0)          # zeros of both signs are equal
    assert torch.equal(got, want)


# ---- streams, graphs, one run of all ---------------------------------------------------------------------------------------------

def all_calls(p, **kw):
    a = p["args"]
    means = ha.hybrid_attn_key_means(p["k"], a["k_block"], key_len=a["key_len"], **kw)
    blocks = ha.hybrid_attn_select_blocks(p["q"], means, p["k"].shape[2], 4, near=0 if a["causal"] else -1, **a, **kw)
    out, lse = ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], blocks, **a, with_lse=True, **kw)
    return (means, blocks, out, lse, *ha.hybrid_attn_sparse_grad(p["q"], p["k"], p["v"], blocks, out, lse, p["dout"], **a, **kw))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_choice_and_attention_together(dtype):
    p = problem(40, B=2, H=4, Hkv=2, Nq=500, dtype=dtype, d=64, qb=64, causal=True, ragged=[500, 333])
    got = all_calls(p)
    p["blocks"] = got[1]
    ref = reference(p)
    for name, x in zip(("out", "lse", "dq", "dk", "dv"), got[2:]):
        close(name, x, ref)
    # with every block chosen, and no mask, it is the framework's plain softmax attention (which rounds fp32 inputs to bf16)
    if dtype == BF16:
        p = problem(41, Nq=512)
        every = torch.arange(8, dtype=torch.int32, device="cuda").repeat(1, 2, 4, 1)
        out, _ = ha.hybrid_attn_sparse_forward(p["q"], p["k"], p["v"], every)
        plain = ha.hybrid_attn_forward(p["q"], p["k"], p["v"], None, None, 1)
        mag = O.attention(p["q"], p["k"], p["v"], every, 128, 64, **units(BF16, 128))["out_tol"]
        assert ((out.double() - plain.double()).abs().cpu() <= 2 * mag).all()


def test_another_stream():
    p = problem(42, B=2, Nq=300, causal=True)
    want = all_calls(p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_calls(p, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed():
    p = problem(43, B=2, H=4, Hkv=2, Nq=300, causal=True, ragged=[300, 200])
    q = problem(44, B=2, H=4, Hkv=2, Nq=300, causal=True, ragged=[111, 290])
    want = [all_calls(x) for x in (p, q)]
    held = {n: p[n].clone() for n in ("q", "k", "v", "dout")}
    live = dict(p, **held, args=dict(p["args"], key_len=p["args"]["key_len"].clone()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_calls(live)
    for turn in range(4):
        src, ref = ((p, want[0]), (q, want[1]))[turn % 2]
        for n in held:
            live[n].copy_(src[n])
        live["args"]["key_len"].copy_(src["args"]["key_len"])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = all_calls(src)
        for a, b, c in zip(got, ref, again):
            assert torch.equal(a, b) and torch.equal(c, b), turn
