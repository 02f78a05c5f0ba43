"""Eviction refuses outputs that lie on what it still reads: the new lengths on the old ones, the new weights on the old ones, in whole or in part.  Host checks, ahead of the first
HIP call; addresses are made up."""
import pytest

from paper_2509_24899_amd import block_sparse as bs
from paper_2509_24899_amd import hybrid_attn as ha

SHAPE, WORKSPACE = 2, 5
LENGTHS, WEIGHTS, ELSEWHERE = 1 << 20, 2 << 20, 4 << 20
B, H_KV, PAGE, PAGES = 3, 2, 16, 1000          # 16000 slots: the choice needs a workspace, without which a call that is not refused for its outputs goes no further


def evict(len_out, weights_out):
    p = ha.ha_paged_problem(B=B, H=6, H_kv=H_KV, T=7, d_head=128, dtype=ha.HA_BF16, n_pages=20, page=PAGE, max_pages=PAGES, max_new=4, causal=1, softmax_scale=0.1, page_table=ELSEWHERE,
                            key_len=LENGTHS, q_offset=ELSEWHERE)
    pool = bs.ha_view(ELSEWHERE, 4096, 2048, 128)
    return ha._lib().hybrid_attn_paged_evict(p, 20, 1, 2, WEIGHTS, ELSEWHERE, 2, pool, pool, len_out, weights_out, ELSEWHERE, None, 0, None)


SIZE = 4 * B * H_KV * PAGE * PAGES


@pytest.mark.parametrize("len_out,weights_out,status", [
    (ELSEWHERE, ELSEWHERE, WORKSPACE), (LENGTHS + 4 * B, ELSEWHERE, WORKSPACE), (LENGTHS - 4 * B, ELSEWHERE, WORKSPACE), (ELSEWHERE, WEIGHTS + SIZE, WORKSPACE),
    (ELSEWHERE, WEIGHTS - SIZE, WORKSPACE), (LENGTHS, ELSEWHERE, SHAPE), (LENGTHS + 4, ELSEWHERE, SHAPE), (LENGTHS - 4 * B + 4, ELSEWHERE, SHAPE), (ELSEWHERE, WEIGHTS, SHAPE),
    (ELSEWHERE, WEIGHTS + SIZE - 4, SHAPE), (ELSEWHERE, WEIGHTS - SIZE + 4, SHAPE)])
def test_outputs_on_inputs(len_out, weights_out, status):
    assert evict(len_out, weights_out) == status
