"""Which lists hold the blocks that are always kept: the refusal of hybrid_attn_select_blocks against a count over all tiles and blocks, behind the stand-in for
the runtime's launch functions (nothing is started), and the shortest lists that hold them on the GPU."""
import os
import subprocess
import sys
import textwrap

import pytest
import torch

from oracle import block_sparse_oracle as O
from paper_2509_24899_amd import hybrid_attn as ha
from test_launch_limits import ROOT, STAND_IN

CHILD = r"""
import ctypes, random, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)       # ahead of the runtime that torch loads
from paper_2509_24899_amd import hybrid_attn as ha, block_sparse as bs
lib, FAKE = ha._lib(), 0x7F0000001000
ref, rng = ctypes.byref, random.Random(5)

def most_kept(Nq, Nk, qb, kb, causal, first, near, start):
    most = 0
    for t in range(-(-Nq // qb)):
        lo, hi = start + t * qb, start + min((t + 1) * qb, Nq) - 1
        most = max(most, sum((j < first or (near >= 0 and j * kb + kb - 1 >= lo - near and j * kb <= hi + (0 if causal else near))) and not (causal and j * kb > hi)
                             for j in range(-(-Nk // kb))))
    return most

def choose(Nq, Nk, qb, kb, causal, first, near, sel, q_start):
    p = bs.ha_sparse_problem(1, 1, 1, Nq, Nk, 64, ha.HA_BF16, qb, kb, sel, causal, first, near, 0.1, q_start, None)
    q = bs.ha_view(FAKE, Nq * 64, Nq * 64, 64)
    st = lib.hybrid_attn_select_blocks(ref(p), ref(q), FAKE, FAKE, FAKE + 0xF00, ctypes.c_size_t(1 << 60), None)
    log = ctypes.POINTER(ctypes.c_uint32 * 4)()
    assert (stand_in.recorded(ref(log)) > 0) == (st == ha.HA_OK)
    assert st in (ha.HA_OK, ha.HA_ERR_SHAPE)
    return st == ha.HA_OK

held = refused = 0
for _ in range(3000):
    qb, kb, causal = rng.choice((64, 128)), rng.choice((64, 128)), rng.choice((0, 1))
    Nq = rng.choice((1, 5, 63, 64, 65, 128, 192, 256, 320, rng.randint(1, 700)))
    Nk = rng.choice((Nq, Nq, 64, 128, 640, rng.randint(1, 900)))
    first, near = rng.choice((0, 0, 1, 2, 9)), rng.choice((0, 0, 1, 63, 64, 65, 128, 200)) if causal else rng.choice((-1, 0, 1, 63, 64, 65, 128, 200))
    Tk = -(-Nk // kb)
    kept = most_kept(Nq, Nk, qb, kb, causal, first, near, Nk - Nq)
    what = (Nq, Nk, qb, kb, causal, first, near, kept)
    for sel in {max(1, kept - 1), max(1, kept), kept + 1}:
        fits = sel >= min(kept, Tk)
        assert choose(Nq, Nk, qb, kb, causal, first, near, sel, None) == fits, (what, sel)
        held, refused = held + fits, refused + (not fits)
    # with places that only the device has, no list that may be too short is taken
    worst = max(most_kept(Nq, Nk, qb, kb, causal, first, near, s) for s in range(-Nq - 8, Nk + 8, 7))
    for sel in range(1, worst):
        assert not choose(Nq, Nk, qb, kb, causal, first, near, sel, FAKE), (what, sel)
assert held > 2000 and refused > 1000, (held, refused)
"""


def test_refused_exactly_where_a_list_does_not_hold_them(tmp_path):
    source, so, child = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so", tmp_path / "child.py"
    source.write_text(STAND_IN)
    child.write_text(textwrap.dedent(CHILD))
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(source), "-o", str(so)], check=True)
    run = subprocess.run([sys.executable, str(child), str(so)], cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-6000:]


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,qb,kb,near,first,sel", [(320, 64, 64, 0, 0, 1), (320, 64, 64, 64, 0, 2), (256, 128, 64, 0, 0, 2), (256, 64, 128, 0, 0, 1), (300, 64, 64, 0, 1, 2),
                                                     (100, 128, 128, 0, 1, 1), (64 * 40, 64, 64, 0, 0, 1)])
def test_the_shortest_lists_that_hold_them(Nq, qb, kb, near, first, sel):
    gen = torch.Generator().manual_seed(1)
    q, k = (torch.randn(2, 2, Nq, 64, generator=gen).bfloat16().cuda() for _ in range(2))
    means = ha.hybrid_attn_key_means(k, kb)
    got = ha.hybrid_attn_select_blocks(q, means, Nq, sel, qb, kb, causal=True, near=near, keep_first=first).cpu()
    assert torch.equal(got, O.select(q, means, Nq, sel, qb, kb, causal=True, near=near, keep_first=first))
    assert (got[:, :, -1, -1] == (Nq - 1) // kb).all()
    if sel > 1:
        with pytest.raises(ha.HybridAttnError):
            ha.hybrid_attn_select_blocks(q, means, Nq, sel - 1, qb, kb, causal=True, near=near, keep_first=first)
