"""Single tokens over bf16 caches keep every weight in two bf16 pieces.  The first is cut off to 8 bits and leaves less than 2^-7 of the weight, of which the second is the rounding, off by
2^-8 of that at most (and no less than 2^-20 of the weight): 2^-15 + 2^-20 together, where one rounded piece is off by up to 2^-8.  Values that cancel make that visible next to the output's own rounding."""
import pytest
import torch

from oracle import paged_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha

BF, PAGE = torch.bfloat16, 16


def cancelling(seed, lengths, d, H, Hkv):
    """(cache, whose values weigh up to nothing but a rounding of the heaviest slot's for the first query head of every key head; weights [B, H, slots] and the size of the logits in 64 bits)"""
    gen = torch.Generator().manual_seed(seed)
    B, G = len(lengths), H // Hkv
    q = torch.randn(B, H, d, generator=gen).to(BF)
    k, v = (torch.randn(B, Hkv, PAGE, d, generator=gen).to(BF) for _ in range(2))
    s = torch.einsum("bhgd,bhjd->bhgj", q.double().view(B, Hkv, G, d), k.double()) * d ** -0.5
    there = torch.arange(PAGE) < torch.tensor(lengths)[:, None]
    p = torch.softmax(s.masked_fill(~there[:, None, None], -torch.inf), -1)
    size = torch.einsum("bhgd,bhjd->bhgj", q.double().abs().view(B, Hkv, G, d), k.double().abs()) * d ** -0.5
    top = p[:, :, 0].argmax(-1)
    for b in range(B):
        for h in range(Hkv):
            j = int(top[b, h])
            v[b, h, j] = 0
            v[b, h, j] = (-(p[b, h, 0] @ v[b, h].double()) / p[b, h, 0, j]).to(BF)
    return q, k, v, p, (size * there[:, None, None]).amax(-1)


def bound(p, v, size, d, piece):
    """(definition's outputs, how far they may be off) with weights that are off by `piece` of themselves."""
    out, spread = torch.einsum("bhgj,bhjd->bhgd", p, v.double()), torch.einsum("bhgj,bhjd->bhgd", p, v.double().abs())
    e = size * (d + 21) * O.U + 8 * O.U               # of a weight, as the oracle of paged attention has it
    return out, spread * (2 * e[..., None] + piece + 2 * (PAGE / 8 + 64) * O.U) + out.abs() * 2.0 ** -8


TWO = 2.0 ** -15 + 2.0 ** -20
CASES = [(1, [5, 9, 16, 3], 128, 2, 2), (2, [7, 2, 13, 4, 6], 64, 6, 2), (3, [16] * 8, 128, 8, 1)]


@pytest.mark.parametrize("case", CASES)
def test_one_piece_would_show(case):
    """Weights relative to the largest, rounded to bf16 once, leave the bound that two pieces hold to."""
    q, k, v, p, size = cancelling(*case)
    out, off = bound(p, v, size, case[2], TWO)
    top = p.amax(-1, keepdim=True)
    one = torch.einsum("bhgj,bhjd->bhgd", (p / top).to(BF).double() * top, v.double()).to(BF).double()
    assert ((one - out).abs() > off).any()
    assert ((one - out).abs() <= bound(p, v, size, case[2], 2.0 ** -8)[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_two_pieces(case):
    _, lengths, d, H, Hkv = case
    q, k, v, p, size = cancelling(*case)
    B = len(lengths)
    table = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    got, _ = ha.hybrid_attn_paged_forward(q.cuda(), k.cuda(), v.cuda(), table, torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    out, off = bound(p, v, size, d, TWO)
    over = (got.double().cpu().view(out.shape) - out).abs() - off
    assert (over <= 0).all(), float(over.max())
