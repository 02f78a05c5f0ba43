"""The choice of many tiles on both sides of every number of blocks at which its keys take more registers."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("blocks", [255, 256, 257, 511, 512, 513, 640, 641, 767, 768, 769, 1023, 1024, 1025])
@pytest.mark.parametrize("sel", [1, 64, 65])
def test_both_sides_of_every_step(blocks, sel, d):
    gen = torch.Generator().manual_seed(37)
    tiles = 1030 if blocks <= 256 else 130                                       # more than are chosen for on their own
    q = torch.randn(1, 1, tiles * 64, d, generator=gen).bfloat16().cuda()
    means = torch.randn(1, 1, blocks, d, generator=gen).cuda()
    got = ha.hybrid_attn_select_blocks(q, means, blocks * 64, sel, 64, 64)
    scores = q.double().view(1, 1, tiles, 64, d).sum(3) @ means.double().transpose(2, 3).contiguous()
    best = torch.sort(scores, dim=3, descending=True, stable=True).indices[..., :sel]
    assert torch.equal(got, best.sort(dim=3).values.to(torch.int32))
