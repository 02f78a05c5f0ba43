"""Whole numbers that do not fit the C ABI's 32 bits are refused by the Python code, which would cut them off otherwise (near=2**32 would count as 0)."""
import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha

Q, K, DEV = (1, 2, 3, 64), (1, 2, 9, 64), torch.device("cuda", 0)


@pytest.mark.parametrize("name", ["q_block", "k_block", "n_select", "keep_first", "near"])
@pytest.mark.parametrize("x", [2 ** 31, 2 ** 32 + 64, -2 ** 31 - 1, -2 ** 32])
def test_numbers_of_a_problem(name, x):
    with pytest.raises(ValueError, match=name):
        ha.make_sparse_problem(Q, K, torch.bfloat16, DEV, **{name: x})


@pytest.mark.parametrize("shape,other", [((1, 2, 2 ** 32 + 3, 64), (1, 2, 9, 64)), ((1, 2, 3, 64), (1, 2, 2 ** 32, 64)), ((2 ** 32 + 1, 2, 3, 64), (2 ** 32 + 1, 2, 3, 64))])
def test_sizes_of_a_problem(shape, other):
    with pytest.raises(ValueError, match="32 bits"):
        ha.make_sparse_problem(shape, other, torch.bfloat16, DEV)


def test_the_ends_of_the_range_are_taken():
    p = ha.make_sparse_problem(Q, K, torch.bfloat16, DEV, n_select=2 ** 31 - 1, near=-2 ** 31)
    assert p.n_select == 2 ** 31 - 1 and p.near_tokens == -2 ** 31 and ha.hybrid_attn_sparse_validate(p) != ha.HA_OK


@pytest.mark.gpu
def test_numbers_of_calls():
    q = torch.zeros(1, 2, 100, 64, dtype=torch.bfloat16, device="cuda")
    means = ha.hybrid_attn_key_means(q)
    for kw in (dict(near=2 ** 32), dict(keep_first=2 ** 32), dict(n_keys=100 + 2 ** 32), dict(n_select=1 + 2 ** 32)):
        with pytest.raises(ValueError):
            ha.hybrid_attn_select_blocks(q, means, **{**dict(n_keys=100, n_select=1), **kw})
    with pytest.raises(ValueError, match="only_last"):
        ha.hybrid_attn_key_means(q, only_last=2 ** 32 + 1, out=means)
    f = [torch.ones(4, device="cuda")]
    before = f[0].clone()
    for kw in (dict(step=2 ** 32 + 1), dict(kind=2 ** 32)):
        with pytest.raises(ValueError, match="32 bits"):
            ha.hybrid_attn_param_update_many(ha.ParamList(f, f), 0.1, **kw)
    assert torch.equal(f[0], before)
