"""Sums over very many slots or rows whose weights are nearly equal.  Added up one behind the other in fp32 they lose a part that grows with their number (524288 terms: 0.6 %), so that the
tolerances here do not depend on it.  u = 2^-24 is half a step of fp32."""
import math

import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
KINDS = [(128, BF), (64, BF), (128, F32), (64, F32)]


def one_page_many_times(d, dtype, slots, B, page=256):
    """Keys and values of one key head whose slots all lie on page 0, but for the last page, which is page 1; (key pool, value pool, where)."""
    gen = torch.Generator().manual_seed(d)
    k, v = torch.randn(2, 1, page, d, generator=gen) * 0.01, torch.randn(2, 1, page, d, generator=gen)
    table = torch.zeros(B, slots // page, dtype=torch.int32)
    table[:, -1] = 1
    return k.to(dtype).cuda(), v.to(dtype).cuda(), dict(page_table=table.cuda(), key_len=torch.full((B,), slots, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("d,dtype", KINDS)
@pytest.mark.parametrize("rows", [1 << 16, 1 << 20])
def test_weights_of_very_many_rows(rows, d, dtype):
    """Queries of zeros: a row gives every slot exp(-lse), which the caller's lse makes 0.74 or so.  A weight is off by the exponent's rounding, |lse log2 e| u, and the exponential's, 2 u; a sum
    by 16 u of a step of 32 rows, and by 4 u for its halves, what has been left over and what was there before."""
    G, slots = 8, 1 << 16
    k, v, where = one_page_many_times(d, dtype, slots, 1)
    lse = 0.3 + 1e-3 * torch.randn(rows // G, G, generator=torch.Generator().manual_seed(1)).cuda()
    q = torch.zeros(1, 1, d, dtype=dtype, device="cuda").expand(rows // G, G, d)
    got = ha.hybrid_attn_paged_weights(q, k, lse, None, **where, causal=False).double()
    want = torch.exp(-lse.double()).sum()
    assert ((got - want).abs() <= (1 + 2 + 16 + 4) * U * want).all(), float(((got - want) / want).abs().max())


def totals(q, k, slots, scale):
    """Logarithms of the sums of weights, in 64 bits, of queries [n, d] over the slots of one_page_many_times."""
    s = q.double() @ k.double().flatten(0, 2).t() * scale
    page = k.shape[2]
    many = torch.full((2 * page,), 0.0, dtype=torch.float64, device="cuda")
    many[:page] = math.log(slots // page - 1)
    return torch.logsumexp(s + many, 1), (q.double().abs() @ k.double().abs().flatten(0, 2).t()).amax(1) * scale


@pytest.mark.parametrize("d,dtype", KINDS)
@pytest.mark.parametrize("B,G,new", [(1, 128, 1040), (600, 1, 1)])
def test_totals_of_very_many_slots(B, G, new, d, dtype):
    """Chunks and single tokens, both more than are cut into ranges.  One key stands out, so that the other weights are 0.74 or so of the largest.  Logits are off by (d + 16) u of their
    products' sizes (fp32: six products for one, 5 u more), a weight by its exponent's rounding and the exponential's, 4 u, sums by 64 u of up to four steps of 32 slots and by 8 u for halves,
    waves and what has been left over, the logarithm by 4 u of itself."""
    slots = 1 << 18
    k, v, where = one_page_many_times(d, dtype, slots, B)
    q = torch.randn(B * new, 1, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    q[..., 0] = 1.0
    k[1, 0, 7, 0] = 0.3 * math.sqrt(d)
    k[0, 0, :, 0], k[1, 0, :7, 0], k[1, 0, 8:, 0] = 0, 0, 0
    q = q.cuda().expand(B * new, G, d)
    _, lse = ha.hybrid_attn_paged_forward(q, k, v, **where, causal=False, with_lse=True)
    want, size = totals(q[:, 0], k, slots, d ** -0.5)
    off = (size * (d + 21) + 4 + 64 + 8 + 4 * want.abs()) * U
    over = (lse.double() - want[:, None]).abs()
    assert (over <= off[:, None]).all(), (float(over.max()), float(off.min()))
