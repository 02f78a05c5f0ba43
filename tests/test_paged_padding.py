"""New tokens of paged caches in the rows of a larger buffer: rows that belong to no sequence cost neither workspace nor results (CPU: the plan; GPU: the calls)."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

AT = 1 << 20


def paged(**more):
    return ha.ha_paged_problem(**{**dict(B=1, H=32, H_kv=8, T=64, d_head=128, dtype=ha.HA_BF16, n_pages=512, page=64, max_pages=512, max_new=64, causal=1, softmax_scale=0.1, page_table=AT,
                                         key_len=AT, q_offset=AT), **more})


@pytest.mark.parametrize("dtype,d", [(ha.HA_BF16, 128), (ha.HA_BF16, 64), (ha.HA_F32, 128), (ha.HA_F32, 64)])
@pytest.mark.parametrize("B,max_new", [(1, 64), (1, 9), (3, 40), (200, 33)])
def test_the_workspace_does_not_grow_with_rows_of_no_sequence(B, max_new, dtype, d):
    """It is at most that of B sequences with max_new rows each."""
    most = ha.hybrid_attn_paged_workspace_bytes(paged(B=B, max_new=max_new, T=B * max_new, q_offset=None, dtype=dtype, d_head=d))
    few = ha.hybrid_attn_paged_workspace_bytes(paged(B=B, max_new=1, T=B, dtype=dtype, d_head=d))      # (what single tokens among them take)
    for T in (B * max_new, 8192, 65536):
        assert ha.hybrid_attn_paged_workspace_bytes(paged(B=B, max_new=max_new, T=T, dtype=dtype, d_head=d)) <= most + few


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("new,max_new", [([70, 1, 0, 33], 70), ([40, 40], 40), ([50, 3, 90], 60)])
def test_rows_of_no_sequence_change_nothing(new, max_new, d, dtype):
    """The sequences' rows come out right among many times as many of none, which are left as they were; sequences with more than max_new among them."""
    from tests.test_gpu_paged import BF, F32, cache, check
    c = cache(50, [2000, 700, 90, 33][:len(new)], new, H=6, Hkv=2, d=d, dtype=BF if dtype == "bf16" else F32, page=32, before=700, behind=3000)
    c["where"]["max_new"] = max_new
    check(c)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,new,H,Hkv,before", [([377, 578, 168, 889, 216, 549, 574, 448, 705], [0, 4, 0, 1, 1, 0, 2, 1, 0], 128, 2, 5), ([900] * 8, [130, 1, 1, 0, 2, 1, 1, 1], 6, 2, 100),
                                                      ([2000, 1500, 300], [129, 64, 1], 1, 1, 200)])
def test_rows_ahead_of_the_first_sequence_where_tiles_go_by_the_offsets(lengths, new, H, Hkv, before, dtype):
    """The tiles of rows ahead of the first sequence hold nothing, also for the kernel that joins ranges, and what lies around the outputs stays as it is."""
    from tests.test_gpu_paged import BF, F32, cache, check
    from tests.test_gpu_paged_memory import Bands
    c = cache(51, lengths, new, H=H, Hkv=Hkv, dtype=BF if dtype == "bf16" else F32, page=32, before=before)
    check(c)
    b = Bands()
    prob = ha.make_paged_problem(c["q"].shape, c["k"].shape, c["q"].dtype, c["q"].device, **c["where"])
    out, lse = b.like(c["q"].shape, c["q"].dtype), b.like(c["q"].shape[:2], torch.float32)
    ha.hybrid_attn_paged_forward(c["q"], c["k"], c["v"], **c["where"], out=out, lse=lse, workspace=b.workspace(ha.hybrid_attn_paged_workspace_bytes(prob)))
    b.check()
    assert (out[:before].contiguous().view(torch.uint8) == 0x5A).all() and (lse[:before].contiguous().view(torch.uint8) == 0x5A).all()
