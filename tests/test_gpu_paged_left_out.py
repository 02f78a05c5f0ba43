"""Tokens that the caller takes out of the weights of slots (lse = -infinity): whatever their queries hold, NaN and infinities among it, shows nowhere."""
import math

import pytest
import torch

from oracle import paged_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha
from tests.test_gpu_paged import BF, F32, cache, close, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
@pytest.mark.parametrize("new", [[1, 2, 1], [90, 1, 33], [40, 70, 200]])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_tokens_without_weight(what, new, d, dtype, causal):
    """The definition's sums less what those tokens would have had; as far off as the sums with them may be, and by lse's rounding to fp32."""
    lengths, H, Hkv = [900, 300, 417], 8, 2
    c = cache(60, lengths, new, H=H, Hkv=Hkv, d=d, dtype=dtype, page=32)
    row = torch.arange(c["T"])
    left_out = (row == 0) | (row == new[0] + new[1] - 1) | (row % 37 == 5)
    want = reference(c, causal)
    sums, row = want["weights"].clone(), 0
    for b, n in enumerate(lengths):
        for i in range(new[b]):
            see = n - new[b] + i + 1 if causal else n
            for h in range(H if left_out[row] else 0):
                keys, _ = O.stored(c["k"].cpu(), c["where"]["page_table"][b].cpu(), see, h // (H // Hkv), c["k"].shape[0])
                sums[b, h // (H // Hkv), :see] -= torch.exp(keys @ c["q"][row, h].double().cpu() * d ** -0.5 - want["lse"][row, h])
            row += 1
    lse = want["lse"].float().cuda()
    lse[left_out.cuda()] = -math.inf
    c["q"][left_out.cuda()] = what
    got = ha.hybrid_attn_paged_weights(c["q"], c["k"], lse, None, **c["where"], causal=causal)
    close(got, sums, want["weights_off"] + want["weights"] * want["lse"].abs().max() * O.U, "weights")
