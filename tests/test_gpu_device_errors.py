"""A device error ends a call of block-sparse attention or of the many-tensor optimiser: it may follow launches that are on their way, so that the call is
made once, by the compiled marshalling or by the Python code, and raises.  A refusal, which has enqueued nothing, is left to the Python code's message.
The library's functions are replaced by ones that count and start nothing."""
import ctypes

import pytest
import torch

from paper_2509_24899_amd import block_sparse, optim
from paper_2509_24899_amd import hybrid_attn as ha

pytestmark = pytest.mark.gpu
REPLACED = ("hybrid_attn_key_means", "hybrid_attn_select_blocks", "hybrid_attn_sparse_forward", "hybrid_attn_sparse_grad", "hybrid_attn_grad_norm", "hybrid_attn_grad_clip",
            "hybrid_attn_param_update_many")


@pytest.fixture
def library(monkeypatch):
    """calls, status: names of the functions called, and what they give."""
    lib, state = ha._lib(), dict(calls=[], status=ha.HA_ERR_DEVICE)
    keep = []
    for name, arguments, result in (*block_sparse.SIGNATURES, *optim.SIGNATURES):
        if name in REPLACED:
            def stand_in(*_, name=name):
                state["calls"].append(name)
                return state["status"]
            keep.append(ctypes.CFUNCTYPE(result, *arguments)(stand_in))
            monkeypatch.setattr(lib, name, keep[-1])
    monkeypatch.setattr(ha, "_CALLS", None)
    assert ha._calls()                                  # bound to the replaced functions
    yield state
    monkeypatch.undo()
    ha._CALLS = None
    assert ha._calls()                                  # and to the library's again
    g = torch.ones(4, device="cuda")
    assert ha.hybrid_attn_grad_norm([g])[0] == 2.0


def calls_of_all():
    q = torch.zeros(1, 2, 100, 64, dtype=torch.bfloat16, device="cuda")
    means, blocks = torch.zeros(1, 2, 2, 64, device="cuda"), torch.zeros(1, 2, 1, 2, dtype=torch.int32, device="cuda")
    lse, g, result = torch.zeros(1, 2, 100, device="cuda"), [torch.ones(5, device="cuda"), torch.ones(7, device="cuda")], torch.ones(2, device="cuda")
    return dict(hybrid_attn_key_means=lambda: ha.hybrid_attn_key_means(q),
                hybrid_attn_select_blocks=lambda: ha.hybrid_attn_select_blocks(q, means, 100, 2),
                hybrid_attn_sparse_forward=lambda: ha.hybrid_attn_sparse_forward(q, q, q, blocks),
                hybrid_attn_sparse_grad=lambda: ha.hybrid_attn_sparse_grad(q, q, q, blocks, q, lse, q),
                hybrid_attn_grad_norm=lambda: ha.hybrid_attn_grad_norm(g),
                hybrid_attn_grad_clip=lambda: ha.hybrid_attn_grad_clip(g, result),
                hybrid_attn_param_update_many=lambda: ha.hybrid_attn_param_update_many(ha.ParamList(g, g), 0.1, clip=result))


@pytest.mark.parametrize("name", REPLACED)
@pytest.mark.parametrize("native", [True, False])
def test_a_device_error_is_raised_by_the_first_call(library, native, name, monkeypatch):
    call = calls_of_all()[name]
    if not native:
        monkeypatch.setattr(ha, "_CALLS", False)
        monkeypatch.setattr(ha, "_calls", lambda: False)
    with pytest.raises(ha.HybridAttnError, match=name) as e:
        call()
    assert e.value.status == ha.HA_ERR_DEVICE and library["calls"] == [name]


@pytest.mark.parametrize("name", REPLACED)
def test_a_refusal_is_raised_once_by_the_python_code(library, name):
    call = calls_of_all()[name]
    library["status"] = ha.HA_ERR_SHAPE
    with pytest.raises(ha.HybridAttnError, match=name) as e:
        call()
    assert e.value.status == ha.HA_ERR_SHAPE and library["calls"] == [name, name]
