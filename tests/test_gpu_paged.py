"""Paged caches against their definitions in 64 bits (oracle/paged_oracle.py, which derives how far the kernels may be off), at the lengths, pages and masks where they can go
wrong."""
import math

import pytest
import torch

from oracle import paged_oracle as O
from oracle import rotary_oracle as R
from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def packed(gen, T, heads, d, dtype, layout, gain=1.0):
    x = (torch.randn((T, heads, d) if layout == "bnhd" else (heads, T, d), generator=gen) * gain).to(dtype).cuda()
    return x if layout == "bnhd" else x.transpose(0, 1)


def cache(seed, lengths, new, H=4, Hkv=2, d=128, dtype=BF, page=16, layout="bhnd", spare=2, max_pages=None, uniform=False, gain=1.0, before=0, behind=0):
    """A cache whose pages stand in any order, whose unused slots hold NaN, and the new rows of all sequences (`before` and `behind` rows belong to none)."""
    gen = torch.Generator().manual_seed(seed)
    B, most = len(lengths), max(1, max(lengths))
    max_pages = -(-most // page) if max_pages is None else max_pages
    n_pages = B * max_pages + spare
    table = torch.randperm(n_pages, generator=gen)[:B * max_pages].view(B, max_pages).to(torch.int32)
    pools = []
    for _ in range(2):
        pool = torch.full((n_pages, Hkv, page, d), math.nan, dtype=dtype)
        for b, n in enumerate(lengths):
            for i in range(min(-(-n // page), max_pages)):
                rows = min(page, n - i * page)
                pool[table[b, i], :, :rows] = (torch.randn((Hkv, rows, d), generator=gen) * gain).to(dtype)
        pools.append(pool.cuda() if layout == "bhnd" else pool.transpose(1, 2).contiguous().cuda().transpose(1, 2))
    offset = torch.tensor([before + sum(new[:i]) for i in range(B + 1)], dtype=torch.int32)
    T = before + sum(new) + behind
    where = dict(page_table=table.cuda(), key_len=torch.tensor(lengths, dtype=torch.int32).cuda(), q_offset=None if uniform else offset.cuda(),
                 max_new=new[0] if uniform else max(new))
    return dict(gen=gen, q=packed(gen, T, H, d, dtype, layout, gain), k=pools[0], v=pools[1], where=where, T=T)


def reference(c, causal=True, scale=None, q=None):
    q, w = c["q"] if q is None else q, c["where"]
    return O.attention(q, c["k"], c["v"], w["page_table"], w["key_len"], w["q_offset"], w["max_new"], causal, q.shape[2] ** -0.5 if scale is None else scale, q.dtype == BF)


def close(got, want, off, what=""):
    got = got.double().cpu()
    rows = ~torch.isnan(want)                         # rows of no sequence
    assert torch.equal(torch.isneginf(got)[rows], torch.isneginf(want)[rows]), what
    rows &= torch.isfinite(want)
    over = ((got - want).abs() - off)[rows]
    assert torch.isfinite(got[rows]).all() and (over <= 0).all(), (what, float(over.max()), float(off[rows].max()))


def check(c, causal=True, scale=None):
    q = c["q"]
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    got = ha.hybrid_attn_paged_forward(q, c["k"], c["v"], **c["where"], causal=causal, softmax_scale=scale, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    want = reference(c, causal, scale)
    close(out, want["out"], want["out_off"], "out")
    close(lse, want["lse"], want["lse_off"], "lse")
    left = torch.isnan(want["lse"]).cuda()            # rows of no sequence are left as they were
    assert (out[left] == 7).all() and (lse[left] == 7).all()
    again = ha.hybrid_attn_paged_forward(q, c["k"], c["v"], **c["where"], causal=causal, softmax_scale=scale, with_lse=True)
    there = ~left
    assert torch.equal(again[0][there], out[there]) and torch.equal(again[1][there], lse[there])
    if left.any():
        lse = torch.where(left, 0.0, lse)
    B, Hkv, slots = want["weights"].shape
    before = torch.rand((B, Hkv, slots), generator=c["gen"]).cuda()
    sums = ha.hybrid_attn_paged_weights(q, c["k"], lse, before, **c["where"], causal=causal, softmax_scale=scale, out=torch.empty_like(before))
    total = want["weights"] + before.double().cpu()
    close(sums, total, want["weights_off"] + total * O.U, "weights")
    new = ha.hybrid_attn_paged_weights(q, c["k"], lse, None, **c["where"], causal=causal, softmax_scale=scale)
    close(new, want["weights"], want["weights_off"], "new weights")
    assert ha.hybrid_attn_paged_weights(q, c["k"], lse, before, **c["where"], causal=causal, softmax_scale=scale) is before and torch.equal(before, sums)


# sequences of no, one and many slots, at and around the ends of pages and steps; single tokens and chunks, more new tokens than slots, none
SINGLE = [
    dict(lengths=[1], new=[1]),
    dict(lengths=[1, 2, 15, 16, 17, 31, 32, 33], new=[1] * 8, uniform=True),
    dict(lengths=[500, 0, 129, 128], new=[1, 1, 1, 1], H=12, Hkv=4),
    dict(lengths=[700], new=[1], H=12, Hkv=12, page=64, uniform=True),
    dict(lengths=[333, 1000], new=[4, 4], H=8, Hkv=1, page=32, uniform=True),
    dict(lengths=[333, 1000, 77], new=[3, 1, 2], H=8, Hkv=1, page=256, before=2, behind=3),
    dict(lengths=[5, 3], new=[8, 2], H=2, Hkv=2, page=16),
    dict(lengths=[2100, 64], new=[1, 1], H=32, Hkv=1, page=128, max_pages=40),
]
CHUNKS = [
    dict(lengths=[40], new=[40], H=2, Hkv=2),
    dict(lengths=[300, 64, 129], new=[65, 64, 33], H=3, Hkv=3, page=64),
    dict(lengths=[513, 1, 260, 90, 0, 31], new=[100, 1, 0, 90, 5, 31], H=6, Hkv=2, page=16, before=1, behind=2),
    dict(lengths=[257, 400], new=[50, 50], H=10, Hkv=2, page=32, uniform=True),
    dict(lengths=[1300], new=[129], H=2, Hkv=1, page=128, max_pages=12),
    dict(lengths=[20, 700], new=[40, 300], H=1, Hkv=1, page=256),
    dict(lengths=[150] * 70, new=[33, 1] * 35, H=2, Hkv=1, page=32),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
@pytest.mark.parametrize("i", range(len(SINGLE)))
def test_single_tokens(i, d, dtype, layout, causal):
    check(cache(i, d=d, dtype=dtype, layout=layout, **SINGLE[i]), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_chunks(i, d, dtype, causal):
    check(cache(100 + i, d=d, dtype=dtype, layout="bnhd" if i % 2 else "bhnd", **CHUNKS[i]), causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[1, 1], [70, 2]])
def test_large_logits_and_another_scale(dtype, new):
    check(cache(7, [300, 90], new, dtype=dtype, gain=4.0, page=32), scale=0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 70]])
def test_pages_that_are_not_there_and_lengths_out_of_range(dtype, new):
    """Slots on them do not take part; a length counts as the nearer end."""
    c = cache(8, [300, 200, 200], new, dtype=dtype, H=6, Hkv=2)
    table = c["where"]["page_table"]
    table[0, 3], table[0, 18], table[1, 0], table[1, 12] = -1, 2 ** 31 - 1, c["k"].shape[0], -2 ** 31
    table[2, :] = -5
    check(c)
    check(c, causal=False)
    c["where"]["key_len"][:] = torch.tensor([2 ** 31 - 1, -3, 10 ** 6], dtype=torch.int32)
    for pool in (c["k"], c["v"]):
        pool[torch.isnan(pool)] = 0.5
    check(c)


def test_rows_behind_max_new_are_left():
    c = cache(9, [50, 60], [10, 3])
    c["where"]["max_new"] = 7
    check(c)


def test_shared_pages_and_broadcast_queries():
    c = cache(10, [64, 80], [1, 1], page=16)
    c["where"]["page_table"][1, :4] = c["where"]["page_table"][0, :4]
    c["q"] = c["q"][:1].expand(2, 4, 128)
    check(c)


def test_many_sequences_and_a_split_long_one():
    check(cache(11, [9000, 3], [1, 1], H=2, Hkv=1, page=128))
    check(cache(12, [5000], [140], H=3, Hkv=1, page=64))


@pytest.mark.parametrize("dtype,d,page", [(BF, 64, 16), (F32, 64, 32)])
@pytest.mark.parametrize("B", [65, 1100])
def test_more_sequences_than_a_wave_has_lanes(B, dtype, d, page):
    """One long sequence among short and empty ones, single tokens and chunks; B = 1100 is more than the sums over sequences take at once."""
    gen = torch.Generator().manual_seed(B)
    lengths, new = torch.randint(0, 60, (B,), generator=gen).tolist(), torch.randint(0, 3, (B,), generator=gen).tolist()
    lengths[B // 2], new[B // 2], lengths[-1], new[-1] = 3000, 1, 1500, 1
    check(cache(B, lengths, new, H=2, Hkv=1, d=d, dtype=dtype, page=page))
    if B == 65:
        new[3], lengths[3] = 70, 90
        check(cache(B, lengths, new, H=2, Hkv=1, d=d, dtype=dtype, page=page))


def test_values_that_are_not_finite_stay_in_their_slots():
    """An infinite value under a weight shows in the rows that see it, and no row of another sequence."""
    c = cache(13, [100, 100], [1, 1], page=32)
    c["v"][c["where"]["page_table"][0, 1], :, 5, 7] = math.inf
    out, _ = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"])
    assert torch.isposinf(out[0, :, 7]).all() and torch.isfinite(out[1]).all() and torch.isfinite(out[0, :, :7]).all()


@pytest.mark.parametrize("d,dtype,layout", [(128, BF, "bhnd"), (64, BF, "bnhd"), (128, F32, "bnhd"), (64, F32, "bhnd")])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("norm", [True, False])
def test_append(d, dtype, layout, interleaved, norm):
    c = cache(14, [70, 0, 33, 20, 16, 3], [5, 1, 0, 20, 1, 6], H=6, Hkv=2, d=d, dtype=dtype, layout=layout, before=1, behind=2)
    c["where"]["page_table"][0, 4] = -1               # the last six slots of the first sequence
    gen, T = c["gen"], c["T"]
    k, v = packed(gen, T, 2, d, dtype, layout, 2.0), packed(gen, T, 2, d, dtype, layout)
    w_q, w_k = ((torch.randn(d, generator=gen) + 1).cuda() for _ in range(2))
    if not norm:
        w_q = w_k = None
    r = ha.hybrid_attn_rotary_grid(d // 2 - 16, interleaved=interleaved)
    at = torch.randint(-500, 500, (T, 3), generator=gen, dtype=torch.int32).cuda()
    k_was, v_was = c["k"].clone(), c["v"].clone()
    q_out = torch.full_like(c["q"], 7.0)
    where = c["where"]
    got = ha.hybrid_attn_paged_append(c["q"], k, v, c["k"], c["v"], **where, w_q=w_q, w_k=w_k, rotary=r, positions=at, eps=1e-6 if norm else None, q_out=q_out)
    assert got is q_out
    step = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    turned = []
    for x, w in ((c["q"], w_q), (k, w_k)):
        x = x.transpose(0, 1)[None]
        y, off = R.norm_rotate(x, w, 1e-6, r, at) if norm else R.turn(x, r.freq, r.axis, at, interleaved, r.magnitude)
        turned.append((y[0].transpose(0, 1), (off + step * y.abs())[0].transpose(0, 1)))
    k_want, k_off, v_want = k_was.double().cpu(), torch.zeros(k_was.shape, dtype=torch.float64), v_was.cpu()
    written = torch.zeros(T, dtype=torch.bool)
    for b in range(6):
        lo, hi = O.rows_of(b, where["q_offset"].cpu(), None, T)
        written[lo:hi] = True
        for i in range(lo, hi):
            slot = int(where["key_len"][b]) - (hi - i)
            page = int(where["page_table"][b, slot // 16]) if slot >= 0 else -1
            if page >= 0:
                k_want[page, :, slot % 16], k_off[page, :, slot % 16], v_want[page, :, slot % 16] = turned[1][0][i], turned[1][1][i], v[i].cpu()
    assert torch.equal(c["v"].cpu().nan_to_num(9.0), v_want.nan_to_num(9.0))
    k_got = c["k"].double().cpu()
    assert torch.equal(torch.isnan(k_got), torch.isnan(k_want)) and ((k_got - k_want).abs() <= k_off)[~torch.isnan(k_want)].all()
    assert ((q_out.double().cpu() - turned[0][0]).abs() <= turned[0][1])[written].all() and (q_out[~written.cuda()] == 7).all()
    # in place, and without queries
    k_pages, v_pages, q = k_was.clone(), v_was.clone(), c["q"].clone()
    more = dict(w_k=w_k, rotary=r, positions=at, eps=1e-6 if norm else None)
    ha.hybrid_attn_paged_append(q, k, v, k_pages, v_pages, **where, w_q=w_q, **more, q_out=q)
    assert torch.equal(q[written.cuda()], q_out[written.cuda()]) and torch.equal(k_pages.nan_to_num(9.0), c["k"].nan_to_num(9.0))
    k_pages.copy_(k_was)
    assert ha.hybrid_attn_paged_append(None, k, v, k_pages, v_pages, **where, **more) is None and torch.equal(k_pages.nan_to_num(9.0), c["k"].nan_to_num(9.0))


def test_append_as_it_is():
    """Without norm and rotation keys and values are copied bit for bit."""
    c = cache(15, [40, 17], [2, 2], uniform=True)
    k, v = (packed(c["gen"], 4, 2, 128, BF, "bnhd") for _ in range(2))
    assert torch.equal(ha.hybrid_attn_paged_append(c["q"], k, v, c["k"], c["v"], **c["where"]), c["q"])
    table = c["where"]["page_table"]
    for pool, x in ((c["k"], k), (c["v"], v)):
        assert torch.equal(pool[table[0, 2], :, 6:8], x[:2].transpose(0, 1)) and torch.equal(pool[table[1, 0], :, 15], x[2]) and torch.equal(pool[table[1, 1], :, 0], x[3])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 1, 0), (40, 4, 8), (100, 0, 100), (64, 64, 0), (130, 1, 2), (1000, 3, 3)])
@pytest.mark.parametrize("kind,max_pages", [("many", None), ("few", None), ("few", 600)])
def test_evict(keep, first, last, dtype, d, kind, max_pages):
    """Weights of many values, and of few with NaN, infinities and both zeros among them: ties go to the lower slot.  Tables of more than 8192 slots are chosen from in another way."""
    c = cache(16, [300, 0, 39, 1, 129, 300], [0] * 6, Hkv=3, d=d, dtype=dtype, spare=6 * 65, layout="bnhd" if d == 64 else "bhnd", max_pages=max_pages)
    w = c["where"]
    slots = w["page_table"].shape[1] * 16
    x = torch.randn((6, 3, slots), generator=c["gen"])
    if kind == "few":
        x = torch.tensor([0.0, -0.0, 1.0, math.nan, math.inf, -math.inf, -1.0])[torch.randint(0, 7, x.shape, generator=c["gen"])]
    used = set(w["page_table"].flatten().tolist())
    free = [i for i in range(c["k"].shape[0]) if i not in used]
    width = -(-keep // 16) + (keep % 16 == 1)
    out_table = torch.tensor(free[:6 * width], dtype=torch.int32).view(6, width).cuda()
    w["page_table"][0, 2], out_table[4, 0] = -1, 2 ** 30      # a page that is not there, and one that nothing can go to
    for pool in (c["k"], c["v"]):
        pool.nan_to_num_(3.0)
    want = O.evict(c["k"].cpu(), c["v"].cpu(), x, w["page_table"].cpu(), w["key_len"].cpu(), keep, out_table.cpu(), first, last)
    got = ha.hybrid_attn_paged_evict(c["k"], c["v"], x.cuda(), w["page_table"], w["key_len"], keep, out_table, first, last)
    for a, b, name in zip((c["k"], c["v"], *got), want, ("k", "v", "length", "weights", "kept")):
        assert torch.equal(a.cpu().nan_to_num(9.0, 8.0, 7.0), b.nan_to_num(9.0, 8.0, 7.0)), name


@pytest.mark.parametrize("n,keep,values", [(20011, 15003, 1000), (70001, 123, 10 ** 9), (9000, 8999, 1), (8192, 5000, 3)])
def test_evict_a_long_sequence(n, keep, values):
    gen, page = torch.Generator().manual_seed(17), 128
    pages, width = -(-n // page), -(-keep // page)
    k = torch.randn(pages + width, 1, page, 64, generator=gen).bfloat16().cuda()
    v, table = k.flip(0).contiguous(), torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    weights = torch.rand(1, 1, pages * page, generator=gen).mul(values).floor().cuda()      # ties, and nothing but ties
    length, out, kept = ha.hybrid_attn_paged_evict(k, v, weights, table, torch.tensor([n], dtype=torch.int32, device="cuda"), keep,
                                                   torch.arange(pages, pages + width, dtype=torch.int32, device="cuda")[None], 10, 100)
    score = weights[0, 0, :n].clone()
    score[:10] = score[n - 100:] = math.inf
    want = torch.sort(score, descending=True, stable=True).indices[:keep].sort().values
    assert int(length) == keep and torch.equal(kept[0, 0].long(), want) and torch.equal(out[0, 0, :keep], weights[0, 0, want]) and not out[0, 0, keep:].any()
    for pool in (k, v):
        assert torch.equal(pool[pages:, 0].flatten(0, 1)[:keep], pool[:pages, 0].flatten(0, 1)[want])


def test_a_run_of_them_as_a_program_makes_it():
    """Prompt, single tokens, eviction, single tokens again: caches and outputs as plain attention over the tokens that are left gives them."""
    gen = torch.Generator().manual_seed(18)
    H, Hkv, d, page, keep, steps = 4, 2, 64, 16, 48, 3
    n_pages, width = 40, 8
    k_pages, v_pages = (torch.zeros(n_pages, Hkv, page, d, device="cuda") for _ in range(2))
    tables = torch.randperm(n_pages, generator=gen).to(torch.int32).cuda()
    table, spare = tables[:2 * width].view(2, width), tables[2 * width:4 * width].view(2, width)
    weights = torch.zeros(2, Hkv, width * page, device="cuda")
    length, r, w = torch.zeros(2, dtype=torch.int32, device="cuda"), ha.hybrid_attn_rotary_frequencies(d), torch.ones(d, device="cuda")
    held = [[[] for _ in range(Hkv)] for _ in range(2)]      # (key, value, weight so far) of every slot that is left, in 64 bits
    seen = 0
    for step, new in enumerate([[70, 41]] + [[1, 1]] * steps + ["evict"] + [[1, 1]] * steps + [[5, 1]]):
        if new == "evict":
            length, weights, kept = ha.hybrid_attn_paged_evict(k_pages, v_pages, weights, table, length, keep, spare, keep_first=2, keep_last=8)
            table, spare = spare, table
            for b in range(2):
                for h in range(Hkv):
                    held[b][h] = [held[b][h][j] for j in kept[b, h].tolist() if j >= 0]
                    assert len(held[b][h]) == min(keep, seen - (29 if b else 0))
            continue
        T = sum(new)
        q, k, v = (torch.randn(T, h, d, generator=gen).cuda() for h in (H, Hkv, Hkv))
        at = torch.cat([torch.arange(n) + seen for n in new]).to(torch.int32)[:, None].contiguous().cuda()
        seen += new[0]
        length += torch.tensor(new, dtype=torch.int32, device="cuda")
        where = dict(page_table=table, key_len=length, q_offset=torch.tensor([0, new[0], T], dtype=torch.int32, device="cuda"), max_new=max(new))
        q2 = ha.hybrid_attn_paged_append(q, k, v, k_pages, v_pages, **where, w_q=w, w_k=w, rotary=r, positions=at, eps=1e-6)
        out, lse = ha.hybrid_attn_paged_forward(q2, k_pages, v_pages, **where, with_lse=True)
        ha.hybrid_attn_paged_weights(q2, k_pages, lse, weights, **where)
        k2 = R.norm_rotate(k.transpose(0, 1)[None], w, 1e-6, r, at)[0][0].transpose(0, 1)
        row = 0
        for b, n in enumerate(new):
            for h in range(Hkv):
                old = len(held[b][h])
                held[b][h] += [[k2[row + i, h], v[row + i, h].double().cpu(), 0.0] for i in range(n)]
                keys, values = (torch.stack([x[j] for x in held[b][h]]) for j in (0, 1))
                for i in range(n):
                    for g in (2 * h, 2 * h + 1):
                        p = torch.softmax(keys[:old + i + 1] @ q2[row + i, g].double().cpu() * d ** -0.5, 0)
                        assert torch.allclose(out[row + i, g].double().cpu(), p @ values[:old + i + 1], atol=2e-5)
                        for j, x in enumerate(p.tolist()):
                            held[b][h][j][2] += x
                assert torch.allclose(weights[b, h, :old + n].double().cpu(), torch.tensor([x[2] for x in held[b][h]], dtype=torch.float64), atol=1e-4)
            row += n


def test_captured_with_an_eager_run_between_the_replays():
    c = cache(19, [300, 90], [1, 1], H=12, Hkv=4, uniform=True)
    k, v = (packed(c["gen"], 2, 4, 128, BF, "bnhd") for _ in range(2))
    r = ha.hybrid_attn_rotary_frequencies(128)
    at = torch.tensor([[299], [89]], dtype=torch.int32, device="cuda")
    weights = torch.zeros(2, 4, c["where"]["page_table"].shape[1] * 16, device="cuda")

    def step():
        q = ha.hybrid_attn_paged_append(c["q"], k, v, c["k"], c["v"], **c["where"], rotary=r, positions=at, eps=1e-6)
        out, lse = ha.hybrid_attn_paged_forward(q, c["k"], c["v"], **c["where"], with_lse=True)
        return q, out, lse, ha.hybrid_attn_paged_weights(q, c["k"], lse, weights, **c["where"], out=torch.empty_like(weights))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(3):
        c["q"].copy_(packed(torch.Generator().manual_seed(seed), 2, 12, 128, BF, "bnhd"))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream_with_a_given_workspace():
    c = cache(20, [2000, 90], [1, 1], page=64)
    want = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"])[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    w = c["where"]
    prob = ha.make_paged_problem(c["q"].shape, c["k"].shape, BF, c["q"].device, **w)
    workspace = torch.empty(ha.hybrid_attn_paged_workspace_bytes(prob), dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    got = ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **w, workspace=workspace, stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(ha.HybridAttnError):
        ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **w, workspace=workspace[:256])


def test_calls_that_are_refused():
    c = cache(21, [40, 17], [2, 1])
    q, k, v, w = c["q"], c["k"], c["v"], c["where"]
    new = packed(c["gen"], 3, 2, 128, BF, "bnhd")
    weights = torch.zeros(2, 2, w["page_table"].shape[1] * 16, device="cuda")
    lse = torch.zeros(3, 4, device="cuda")
    free = torch.zeros(2, 1, dtype=torch.int32, device="cuda")

    def forward(q=q, k=k, v=v, **more):
        return lambda: ha.hybrid_attn_paged_forward(q, k, v, **{**w, **more})
    bad = [forward(q=q.float()), forward(k=k[..., :64]), forward(v=v[:, :1]), forward(page_table=w["page_table"].long()), forward(page_table=w["page_table"][0]),
           forward(key_len=w["key_len"][:1]), forward(q_offset=w["q_offset"][:2].contiguous()), forward(q_offset=None), forward(max_new=4), forward(max_new=-1), forward(max_new=2 ** 32),
           forward(out=q[:1]), forward(lse=lse[:2]), forward(softmax_scale=0.0), forward(q=q.cpu()), forward(k=k[:, :, :15], v=v[:, :, :15]), forward(q=q[..., ::2]),
           lambda: ha.hybrid_attn_paged_append(q, new, new[:2], k, v, **w), lambda: ha.hybrid_attn_paged_append(q, new, new, k, v, **w, w_q=torch.ones(128, device="cuda")),
           lambda: ha.hybrid_attn_paged_append(None, new, new, k, v, **w, q_out=q), lambda: ha.hybrid_attn_paged_append(q, new, new, k, v, **w, eps=-1.0),
           lambda: ha.hybrid_attn_paged_append(q, new, new, k, v, **w, rotary=ha.hybrid_attn_rotary_frequencies(128), positions=torch.zeros(2, 1, dtype=torch.int32, device="cuda")),
           lambda: ha.hybrid_attn_paged_append(q, new, new, k, v, **w, rotary=ha.hybrid_attn_rotary_frequencies(128), positions=torch.zeros(2, 3, 1, dtype=torch.int32, device="cuda")),
           lambda: ha.hybrid_attn_paged_weights(q, k, lse, weights[:1], **w), lambda: ha.hybrid_attn_paged_weights(q, k, lse.double(), weights, **w),
           lambda: ha.hybrid_attn_paged_evict(k, v, weights, w["page_table"], w["key_len"], 17, free), lambda: ha.hybrid_attn_paged_evict(k, v, weights, w["page_table"], w["key_len"], 0, free),
           lambda: ha.hybrid_attn_paged_evict(k, v, weights, w["page_table"], w["key_len"], 8, free, 5, 4), lambda: ha.hybrid_attn_paged_evict(k, v, weights, w["page_table"], w["key_len"], 8, free, weights_out=weights)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, RuntimeError, ha.HybridAttnError)):
            call()
            print(i)
