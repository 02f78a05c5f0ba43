"""Clipping on a stream of its own: what it writes, behind work of that stream."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("place", ["new", "in place"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_clip_on_another_stream(place, dtype):
    gen = torch.Generator().manual_seed(12)
    g = [torch.randn(n, generator=gen).to(dtype).cuda() for n in (1 << 22, 1, 5003, 0, 700)]
    result = ha.hybrid_attn_grad_norm(g, 1.0)
    want = [torch.full_like(x, 3.0) for x in g]
    ha.hybrid_attn_grad_clip(g, result, want)
    late, out = [torch.zeros_like(x) for x in g], [torch.zeros_like(x) for x in g]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                       # the gradients come on that stream, just before the calls
        for x, y in zip(late, g):
            x.copy_(y)
    res = ha.hybrid_attn_grad_norm(late, 1.0, stream=side)
    ha.hybrid_attn_grad_clip(late, res, None if place == "in place" else out, stream=side)
    side.synchronize()
    assert torch.equal(res, result) and float(result[1]) < 1.0
    got = late if place == "in place" else out
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if place == "new":
        assert all(torch.equal(a, b) for a, b in zip(late, g))
