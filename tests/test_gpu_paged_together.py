"""Paged caches as programs run them: batches of chunks and single tokens whose slots are cut into ranges, captured steps over a cache that grows, graphs that share a workspace, calls on
two streams at once."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha
from tests.test_gpu_paged import BF, F32, cache, check, packed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,dtype,page", [(128, BF, 16), (128, BF, 64), (64, BF, 16), (64, BF, 256), (128, F32, 32), (64, F32, 16)])
def test_chunks_beside_single_tokens_in_ranges(d, dtype, page, causal):
    check(cache(31, [2900, 2500, 1200, 0, 33], [130, 1, 40, 0, 2], H=6, Hkv=2, d=d, dtype=dtype, page=page, before=1, behind=2), causal)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
def test_like_chunks_of_several_tiles(d, dtype):
    check(cache(32, [700, 75, 1999], [75] * 3, H=10, Hkv=2, d=d, dtype=dtype, page=32, uniform=True), True)       # 375 rows to a sequence and key head


def test_a_captured_step_over_a_cache_that_grows():
    c = cache(33, [1500, 700, 40], [1, 1, 1], H=12, Hkv=4, page=64, max_pages=40, uniform=True)
    w, B = c["where"], 3
    table = torch.arange(B * 40, dtype=torch.int32, device="cuda").view(B, 40)
    pools = [torch.randn(B * 40, 4, 64, 128, generator=c["gen"]).to(BF).cuda() for _ in range(2)]
    length, at = w["key_len"].clone(), torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    where = dict(page_table=table, key_len=length, max_new=1)
    r = ha.hybrid_attn_rotary_frequencies(128)
    new = [packed(c["gen"], B, h, 128, BF, "bnhd") for h in (12, 4, 4)]
    weights = torch.zeros(B, 4, 40 * 64, device="cuda")

    def step(pools, weights):
        q = ha.hybrid_attn_paged_append(*new, *pools, **where, rotary=r, positions=at, eps=1e-6)
        out, lse = ha.hybrid_attn_paged_forward(q, *pools, **where, with_lse=True)
        return out, lse, ha.hybrid_attn_paged_weights(q, pools[0], lse, weights, **where)
    eager, eager_weights = [x.clone() for x in pools], weights.clone()
    step([x.clone() for x in pools], weights.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(pools, weights)
    for i in range(4):
        length += 1 + 300 * i                         # (slots that nothing has been stored in are the pools' own noise)
        at.copy_((length - 1)[:, None])
        for j, x in enumerate(new):
            x.copy_(packed(torch.Generator().manual_seed(10 * i + j), B, x.shape[1], 128, BF, "bnhd"))
        graph.replay()
        want = step(eager, eager_weights)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(pools, eager))


def test_two_graphs_that_share_a_workspace():
    cases = [cache(34, [2900, 2500], [130, 1], H=6, Hkv=2, page=16), cache(35, [3000, 64, 700], [1, 1, 60], H=8, Hkv=2, page=64, d=64)]
    shared = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(255)
    graphs, got, want = [], [], []
    for c in cases:
        want.append(ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], with_lse=True))
        lse = want[-1][1]
        want[-1] += (ha.hybrid_attn_paged_weights(c["q"], c["k"], lse, None, **c["where"]),)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            out, lse = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], with_lse=True, workspace=shared)
            got.append((out, lse, ha.hybrid_attn_paged_weights(c["q"], c["k"], lse, None, **c["where"], workspace=shared)))
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for i in order:
            for x in got[i]:
                x.fill_(7.0)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i])), (order, i)


def test_a_captured_eviction_of_a_long_cache():
    page, held, keep = 64, [9000, 100], 4000
    max_pages, spare = 150, 2 * -(-keep // page)
    gen = torch.Generator().manual_seed(36)
    pools = [torch.randn(2 * max_pages + spare, 2, page, 64, generator=gen).to(BF).cuda() for _ in range(2)]
    table = torch.arange(2 * max_pages, dtype=torch.int32, device="cuda").view(2, max_pages)
    to = (torch.arange(spare, dtype=torch.int32, device="cuda") + 2 * max_pages).view(2, -1)
    weights, length = torch.rand(2, 2, max_pages * page, generator=gen).cuda(), torch.tensor(held, dtype=torch.int32, device="cuda")

    def run(pools):
        return ha.hybrid_attn_paged_evict(*pools, weights, table, length, keep, to, keep_first=3, keep_last=20)
    eager = [x.clone() for x in pools]
    run([x.clone() for x in pools])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(pools)
    for i in range(3):
        weights.copy_(torch.rand(weights.shape, generator=gen))
        length[1] = 100 + 4500 * i
        graph.replay()
        want = run(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(pools, eager))


def test_two_streams_at_once():
    cases = [cache(37, [2900, 2500], [130, 1], H=6, Hkv=2, page=16), cache(38, [3000, 2000], [1, 1], H=8, Hkv=2, page=64, d=64, dtype=F32)]
    want = [ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"])[0] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], stream=s)[0] for c, s in zip(cases, streams)] for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 40]])
@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_sequence(new, dtype, d, what):
    c = cache(39, [300, 1500, 77], new, H=4, Hkv=2, d=d, dtype=dtype, page=32)
    want = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], with_lse=True)
    page = c["where"]["page_table"][1, 3].item()      # slots 96 .. 127 of the sequence in the middle
    rows = slice(new[0], new[0] + new[1])
    c["k"][page, 1, 5, 3] = what
    c["v"][page, 0, 5, 3] = what
    got = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], with_lse=True)
    assert not torch.isfinite(got[0][rows, :2, 3]).any()          # the key head whose value it is
    for a, b in zip(got, want):
        a[rows] = b[rows]
        assert torch.equal(a, b)


@pytest.mark.parametrize("d,dtype,page", [(64, BF, 16), (128, BF, 64), (64, F32, 32)])
def test_many_sequences_of_both_kinds_in_ranges(d, dtype, page):
    check(cache(40, [1500, 40] + [90, 33] * 34 + [0, 2000], [33, 1] * 35 + [0, 3], H=2, Hkv=1, d=d, dtype=dtype, page=page))
