"""New tokens of paged caches in the rows of a larger buffer: rows that belong to no sequence cost neither workspace nor results (CPU: the plan; GPU: the calls)."""
import pytest

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
