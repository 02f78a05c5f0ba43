"""Block means of caches that hold more tokens than a call takes queries: the means have no queries, and no limit of theirs applies."""
import contextlib

import pytest
import torch

from paper_2509_24899_amd import hybrid_attn as ha


@pytest.mark.parametrize("B,H,N,kb", [(1, 1, (1 << 24) + 1, 64), (1, 1, 1 << 29, 128), (64, 8, 64 * 16384, 64), (2, 2048, 64 * 2048, 64)])
def test_means_of_as_many_blocks_as_the_problem_admits(B, H, N, kb, monkeypatch):
    """The Python code hands the library a problem that it admits (checked by the library; nothing is started)."""
    lib, seen = ha._lib(), []
    monkeypatch.setattr(ha, "_CALLS", False)
    monkeypatch.setattr(ha, "_calls", lambda: False)

    def means(p, view, only_last, out, stream):
        assert lib.hybrid_attn_sparse_validate(p) == ha.HA_OK
        seen.append((p.B, p.H_kv, p.N_k, p.d_head, p.k_block, view.stride_n))
        return ha.HA_OK
    monkeypatch.setattr(lib, "hybrid_attn_key_means", means)
    for name in ("_require_gpu", "_stream_handle"):
        monkeypatch.setattr(ha, name, lambda *_: None)
    monkeypatch.setattr(ha, "_on_device_of", lambda _: contextlib.nullcontext())
    ha.hybrid_attn_key_means(torch.empty(B, H, N, 64, dtype=torch.bfloat16, device="meta"), kb)
    assert seen == [(B, H, N, 64, kb, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_means_of_a_long_cache(native, monkeypatch):
    if not native:
        monkeypatch.setattr(ha, "_CALLS", False)
        monkeypatch.setattr(ha, "_calls", lambda: False)
    N = (1 << 24) + 70
    k = torch.randint(-100, 100, (1, 1, N, 64), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    means = ha.hybrid_attn_key_means(k, 64)
    sums = k[0, 0, :1 << 24].view(-1, 64, 64).sum(1, dtype=torch.float32)
    assert torch.equal(means[0, 0, :1 << 18], sums / 64) and torch.equal(means[0, 0, 1 << 18], k[0, 0, 1 << 24:-6].sum(0, dtype=torch.float32) / 64)
    last = k[0, 0, -6:].sum(0, dtype=torch.float64) / 6
    assert ((means[0, 0, -1] - last).abs() <= last.abs() * 2.0 ** -24 * (1 + 1e-9)).all()
    ha.hybrid_attn_key_means(k, 64, only_last=1, out=means)
    assert ((means[0, 0, -1] - last).abs() <= last.abs() * 2.0 ** -24 * (1 + 1e-9)).all()
