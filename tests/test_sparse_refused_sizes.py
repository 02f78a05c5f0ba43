"""Problems without queries whose key blocks are more than the gradients take: refused ahead of any launch, whatever the workspace, as those with queries are.
Behind the stand-in for the runtime's launch functions, which starts nothing."""
import os
import subprocess
import sys
import textwrap

from test_launch_limits import ROOT, STAND_IN

CHILD = r"""
import ctypes, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)       # ahead of the runtime that torch loads
from paper_2509_24899_amd import hybrid_attn as ha, block_sparse as bs
lib, FAKE = ha._lib(), 0x7F0000001000
ref = ctypes.byref

def grad(B, H, Hkv, Nq, Nk, d, f32, kb, size):
    p = bs.ha_sparse_problem(B, H, Hkv, Nq, Nk, d, ha.HA_F32 if f32 else ha.HA_BF16, 64, kb, 1, 0, 0, -1, 0.1, None, None)
    assert lib.hybrid_attn_sparse_validate(ref(p)) == ha.HA_OK
    q, k = bs.ha_view(FAKE, H * Nq * d, Nq * d, d), bs.ha_view(FAKE, Hkv * Nk * d, Nk * d, d)
    need = lib.hybrid_attn_sparse_grad_workspace_bytes(ref(p))
    st = lib.hybrid_attn_sparse_grad(ref(p), ref(q), ref(k), ref(k), FAKE, ref(q), FAKE, ref(q), ref(q), ref(k), ref(k), FAKE + 0xF00,
                                     ctypes.c_size_t(need if size is None else size), None)
    log = ctypes.POINTER(ctypes.c_uint32 * 4)()
    return need, st, stand_in.recorded(ref(log))

for d in (64, 128):
    for f32 in (False, True):
        # 2^22 blocks of keys, and one more: of one head, of many, with blocks of 128 keys
        for B, H, Nk, kb in ((1, 1, 1 << 28, 64), (64, 8, 1 << 19, 64), (2, 1, 1 << 28, 128)):
            need, st, n = grad(B, H, H, 0, Nk, d, f32, kb, None)
            assert need > 0 and st == ha.HA_OK and n > 0, (B, H, Nk, kb, need, st, n)
            need, st, n = grad(B, H, H, 0, Nk, d, f32, kb, need - 1)
            assert st == 5 and n == 0                   # HA_ERR_WORKSPACE
            for Nq in (0, 1):
                for size in (0, 256, 1 << 60):
                    need, st, n = grad(B, H, H, Nq, Nk + 1, d, f32, kb, size)
                    assert need == 0 and st == ha.HA_ERR_UNSUPPORTED and n == 0, (B, H, Nq, Nk, kb, size, need, st, n)
"""


def test_key_blocks_beyond_the_gradients_are_refused_without_queries_too(tmp_path):
    source, so, child = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so", tmp_path / "child.py"
    source.write_text(STAND_IN)
    child.write_text(textwrap.dedent(CHILD))
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(source), "-o", str(so)], check=True)
    run = subprocess.run([sys.executable, str(child), str(so)], cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-6000:]
