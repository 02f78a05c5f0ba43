"""Where the calls of rotary positions and paged caches write: every buffer they write is carved out of a larger allocation between two bands of a sentinel, workspaces are filled
with the bits of NaN, and the bands must be left as they were, over the degenerate sizes and those around the ends of tiles and pages.  And fp32 values up to the largest."""
import math

import pytest
import torch

from oracle import paged_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha
from tests.test_gpu_paged import BF, F32, cache, check, packed

pytestmark = pytest.mark.gpu
BAND = 1 << 16


class Bands:
    def __init__(self):
        self.kept = []

    def like(self, shape, dtype, fill=None):
        n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
        whole = torch.full((BAND + n + BAND + 256,), 0x5A, dtype=torch.uint8, device="cuda")
        self.kept.append((whole, n))
        t = whole[BAND:BAND + n].view(dtype).view(shape)
        if fill is not None:
            t.copy_(fill)
        return t

    def workspace(self, n):
        t = self.like((max(n, 256),), torch.uint8)
        return t.fill_(255)

    def check(self):
        torch.cuda.synchronize()
        for whole, n in self.kept:
            assert (whole[:BAND] == 0x5A).all() and (whole[BAND + n:] == 0x5A).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,H,Hkv", [(1, 1, 1), (15, 3, 1), (16, 2, 2), (17, 5, 5), (33, 1, 1), (1025, 12, 4)])
def test_rows(N, H, Hkv, d, dtype):
    b, gen = Bands(), torch.Generator().manual_seed(N)
    q, k = (torch.randn((2, h, N, d), generator=gen).to(dtype).cuda() for h in (H, Hkv))
    w = torch.ones(d, device="cuda")
    r, at = ha.hybrid_attn_rotary_frequencies(d, interleaved=N % 2 == 0), torch.arange(N, dtype=torch.int32, device="cuda")[:, None].contiguous()
    got = ha.hybrid_attn_norm_rotate(q, k, w, w, r, at, q_out=b.like(q.shape, dtype), k_out=b.like(k.shape, dtype))
    assert all(torch.equal(x, y) for x, y in zip(got, ha.hybrid_attn_norm_rotate(q, k, w, w, r, at)))
    ha.hybrid_attn_rotate(q, r, at, out=b.like(q.shape, dtype))
    need = ha.hybrid_attn_norm_rotate_grad_workspace_bytes(ha.ha_rows_problem(2, H, Hkv, N, d, ha.HA_BF16 if dtype == BF else ha.HA_F32, 1e-6))
    outs = dict(grad_in_q=b.like(q.shape, dtype), grad_in_k=b.like(k.shape, dtype), grad_w_q=b.like((d,), torch.float32), grad_w_k=b.like((d,), torch.float32))
    got = ha.hybrid_attn_norm_rotate_grad(q, k, q, k, w, w, r, at, **outs, workspace=b.workspace(need))
    assert all(torch.equal(x, y) for x, y in zip(got, ha.hybrid_attn_norm_rotate_grad(q, k, q, k, w, w, r, at)))
    b.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (128, 64), (64, 256)])
@pytest.mark.parametrize("lengths,new,H,Hkv,max_pages", [([1], [1], 1, 1, None), ([33, 0, 64], [1, 1, 1], 6, 2, None), ([70, 5], [40, 5], 3, 1, None), ([2500, 1300], [1, 1], 4, 4, None),
                                                         ([1500, 90], [90, 2], 8, 2, None), ([20, 40], [3, 1], 2, 1, 0), ([40] * 70, [1, 2] * 35, 2, 1, None)])
def test_pages(lengths, new, H, Hkv, max_pages, d, page, dtype):
    b = Bands()
    c = cache(len(lengths) + d, lengths, new, H=H, Hkv=Hkv, d=d, dtype=dtype, page=page, before=1, behind=1, max_pages=max_pages)
    where, T = c["where"], c["T"]
    k_pages, v_pages = (b.like(x.shape, dtype, x) for x in (c["k"], c["v"]))
    rows = [packed(c["gen"], T, h, d, dtype, "bnhd") for h in (Hkv, Hkv)]
    r, at = ha.hybrid_attn_rotary_frequencies(d), torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
    q = ha.hybrid_attn_paged_append(c["q"], *rows, k_pages, v_pages, **where, rotary=r, positions=at, eps=1e-6, q_out=b.like((T, H, d), dtype, torch.zeros(T, H, d)))
    prob = ha.make_paged_problem(q.shape, k_pages.shape, dtype, q.device, **where)
    out, lse = b.like(q.shape, dtype), b.like(q.shape[:2], torch.float32, torch.zeros(T, H))
    ha.hybrid_attn_paged_forward(q, k_pages, v_pages, **where, out=out, lse=lse, workspace=b.workspace(ha.hybrid_attn_paged_workspace_bytes(prob)))
    slots = (len(lengths), Hkv, where["page_table"].shape[1] * page)
    sums = ha.hybrid_attn_paged_weights(q, k_pages, lse, None, **where, out=b.like(slots, torch.float32), workspace=b.workspace(ha.hybrid_attn_paged_weights_workspace_bytes(prob)))
    assert torch.isfinite(out[1:-1]).all() and torch.isfinite(sums).all()
    keep = 17
    width = -(-keep // page)
    spare = b.like((k_pages.shape[0] + len(lengths) * width, Hkv, page, d), dtype), b.like((k_pages.shape[0] + len(lengths) * width, Hkv, page, d), dtype)
    for pool, x in zip(spare, (k_pages, v_pages)):
        pool[:len(x)] = x
    free = torch.arange(k_pages.shape[0], len(spare[0]), dtype=torch.int32, device="cuda").view(len(lengths), width)
    prob.n_pages = len(spare[0])
    got = ha.hybrid_attn_paged_evict(*spare, sums, where["page_table"], where["key_len"], keep, free, 1, 3, len_out=b.like((len(lengths),), torch.int32), weights_out=b.like(slots, torch.float32),
                                     kept=b.like((*slots[:2], keep), torch.int32), workspace=b.workspace(ha.hybrid_attn_paged_evict_workspace_bytes(prob, keep)))
    want = O.evict(spare[0].cpu(), spare[1].cpu(), sums.cpu(), where["page_table"].cpu(), where["key_len"].cpu(), keep, free.cpu(), 1, 3)
    assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want[2:]))
    b.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_largest_fp32_values(new, d):
    """Values between bf16's largest and fp32's, whose first piece must not become infinite: one slot's values, so that sums do not overflow, and keys of a column whose queries
    are 0 or bring them down (2^-125)."""
    c = cache(30, [200, 70], new, d=d, dtype=F32, page=32)
    for i, value in enumerate((3.402e38, -3.402e38, 3.396e38, -3.3962e38, 3.39e38)):      # (a weight may be 1 + 1e-6 before it is divided by the sum of weights)
        c["v"][c["where"]["page_table"][0, 0], :, 0, 5 * i + 1] = value
        c["k"][c["where"]["page_table"][0, 0], :, 7, 5 * i + 1] = value
        c["q"][..., 5 * i + 1] = 2.0 ** -125 if i else 0.0
    check(c)


def test_sums_of_large_values():
    """What is summed before it is divided by the sum of the weights must fit: all slots at 2^-10 of the largest value, 200 of them with weights of 1 at most, are 2^-2 of it."""
    c = cache(33, [200, 70], [40, 3], dtype=F32, page=32)
    v = c["v"]
    v[:] = torch.sign(v) * torch.finfo(torch.float32).max / 1024
    check(c)


def test_check_is_the_other_files():
    """The runs of the other file hold here too, with a row of the largest size of group."""
    check(cache(31, [65, 64], [1, 1], H=32, Hkv=1, d=64, page=16))
    check(cache(32, [65, 64], [2, 1], H=33, Hkv=1, d=64, page=16))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pools_of_more_than_four_gib(dtype):
    """Pages at the far end of pools that 32 bits do not address give what the same pages in small pools give, bit for bit."""
    page, d, Hkv = 256, 128, 1
    used, n = 12, (5 << 30) // (page * d * Hkv * (2 if dtype == BF else 4))
    far = [torch.empty((n, Hkv, page, d), dtype=dtype, device="cuda") for _ in range(2)]
    gen = torch.Generator().manual_seed(34)
    near = [torch.randn((used, Hkv, page, d), generator=gen).to(dtype).cuda() for _ in range(2)]
    for x, y in zip(far, near):
        x[n - used:] = y
    table = torch.randperm(8, generator=gen).to(torch.int32).view(2, 4).cuda()
    q, k, v = (packed(gen, 41, h, d, dtype, "bnhd") for h in (2, 1, 1))
    got = []
    for (kp, vp), shift in ((far, n - used), (near, 0)):
        for offset, length, new in (([0, 1, 2], [1000, 700], 1), ([0, 40, 41], [900, 64], 40)):
            where = dict(page_table=table + shift, key_len=torch.tensor(length, dtype=torch.int32, device="cuda"), q_offset=torch.tensor(offset, dtype=torch.int32, device="cuda"), max_new=new)
            T = offset[-1]
            ha.hybrid_attn_paged_append(None, k[:T], v[:T], kp, vp, **where)
            out, lse = ha.hybrid_attn_paged_forward(q[:T], kp, vp, **where, with_lse=True)
            weights = ha.hybrid_attn_paged_weights(q[:T], kp, lse, None, **where)
            got.append([out, lse, weights])
        left = ha.hybrid_attn_paged_evict(kp, vp, weights, where["page_table"], where["key_len"], 500, torch.arange(8, 12, dtype=torch.int32, device="cuda").view(2, 2) + shift, 2, 3)
        got.append([*left, kp[len(kp) - used:], vp[len(vp) - used:]])
    for a, b in zip(got[:3], got[3:]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,interleaved", [(BF, True), (BF, False), (F32, True)])
def test_streams_that_go_past_the_cache(dtype, interleaved):
    """A call of so many rows that they are read and written past the memory-side cache gives what calls of parts of them give."""
    N, d, H = 36000 if dtype == BF else 18000, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(35)
    q, k, g = (torch.randn((1, h, N, d), generator=gen, device="cuda").to(dtype) for h in (H, 2, H))
    w, r = torch.rand(d, generator=gen, device="cuda"), ha.hybrid_attn_rotary_frequencies(d, interleaved=interleaved)
    at = torch.arange(N, dtype=torch.int32, device="cuda")[:, None].contiguous()
    whole = [ha.hybrid_attn_rotate(q, r, at), *ha.hybrid_attn_norm_rotate(q, k, w, w, r, at), *ha.hybrid_attn_norm_rotate_grad(g, k, q, k, w, w, r, at)]
    for lo in range(0, N, 9000):
        part = [x[:, :, lo:lo + 9000] for x in (q, k, g)]
        here = at[lo:lo + 9000].contiguous()
        some = [ha.hybrid_attn_rotate(part[0], r, here), *ha.hybrid_attn_norm_rotate(*part[:2], w, w, r, here), *ha.hybrid_attn_norm_rotate_grad(part[2], part[1], *part[:2], w, w, r, here)]
        for x, y in zip(whole[:5], some[:5]):
            assert torch.equal(x[:, :, lo:lo + 9000], y)


def test_eviction_past_the_cache():
    n, page, d, keep = 60000, 128, 128, 50000
    width, gen = -(-n // page), torch.Generator(device="cuda").manual_seed(36)
    pools = [torch.randn((2 * width, 3, page, d), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    table = torch.randperm(2 * width, generator=gen, device="cuda").to(torch.int32).view(2, 1, width)
    weights = torch.rand((1, 3, width * page), generator=gen, device="cuda")
    before = [x[table[0, 0].long()].transpose(0, 1).flatten(1, 2) for x in pools]
    _, _, kept = ha.hybrid_attn_paged_evict(*pools, weights, table[0], torch.tensor([n], dtype=torch.int32, device="cuda"), keep, table[1])
    for x, y in zip(pools, before):
        after = x[table[1, 0].long()].transpose(0, 1).flatten(1, 2)[:, :keep]
        assert torch.equal(after, y.gather(1, kept[0].long()[..., None].expand(-1, -1, d)))
