"""Launch geometry of block-sparse attention and of the many-tensor optimiser at the largest problems that their checks admit: no launch may exceed what the
device takes (a grid of 2^31 - 1 x 65535 x 65535 blocks, 1024 work-items to a block, 2^32 - 1 work-items along a dimension).  Nothing is started."""
import subprocess
import os
import sys
import textwrap

from test_launch_limits import ROOT, STAND_IN

CHILD = r"""
import ctypes, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)       # ahead of the runtime that torch loads
from paper_2509_24899_amd import hybrid_attn as ha, block_sparse as bs, optim
lib, FAKE, BIG = ha._lib(), 0x7F0000001000, ctypes.c_size_t(1 << 60)
ref = ctypes.byref
bad, refused, counts = [], 0, {}

def check(what, status, may_refuse=False):
    global refused
    log = ctypes.POINTER(ctypes.c_uint32 * 4)()
    n = stand_in.recorded(ref(log))
    if may_refuse and status == ha.HA_ERR_UNSUPPORTED:
        refused += 1
        assert n == 0, what
        return
    assert status == ha.HA_OK, (what, status)
    assert n > 0, what
    counts[what[0]] = counts.get(what[0], 0) + 1
    for i in range(n):
        x, y, z, block = log[i]
        if not (0 < x < 2 ** 31 and 0 < y <= 65535 and 0 < z <= 65535 and 0 < block <= 1024 and x * block < 2 ** 32):
            bad.append((what, f"launch {i} of {n}", (x, y, z), block))

def view(heads, n, d):
    return bs.ha_view(FAKE, heads * n * d, n * d, d)

for B, H, Hkv, Nq, Nk, sel in ((1, 1, 1, 1 << 24, 1 << 16, 4), (1, 1, 1, 1 << 24, 1 << 16, 4096), (1, 65535, 65535, 1024, 4096, 64), (65535, 1, 1, 1024, 8192, 128),
                              (1, 1, 1, 1, 1 << 29, 64), (1, 65535, 1, 64, 1 << 28, 1 << 20), (255, 257, 257, 1000, 8000, 300), (15, 4096, 64, 1024, 1 << 19, 64),
                              (64, 1023, 1, 1, 1 << 20, 100), (1, 16, 16, 1 << 22, 1 << 25, 64), (4, 4, 4, 1 << 20, 1 << 20, 2000), (1, 1, 1, 0, 1 << 20, 4), (3, 2, 1, 70, 0, 4)):
    for d in (64, 128):
        for f32 in (False, True):
            for qb, kb in ((64, 64), (128, 64), (64, 128), (128, 128)):
                p = bs.ha_sparse_problem(B, H, Hkv, Nq, Nk, d, ha.HA_F32 if f32 else ha.HA_BF16, qb, kb, sel, 0, 0, -1, 0.1, None, None)
                what = (B, H, Hkv, Nq, Nk, sel, d, f32, qb, kb)
                if lib.hybrid_attn_sparse_validate(ref(p)) != ha.HA_OK:
                    assert B * H * -(-Nq // qb) > 1 << 20 or B * Hkv * -(-Nk // kb) > 1 << 23 or -(-Nq // qb) * sel > 1 << 30, what
                    continue
                q, k = view(H, Nq, d), view(Hkv, Nk, d)
                if Nk:
                    check(("means",) + what, lib.hybrid_attn_key_means(ref(p), ref(k), 0, FAKE, None))
                    check(("last means",) + what, lib.hybrid_attn_key_means(ref(p), ref(k), 7, FAKE, None))
                if Nq:
                    check(("choice",) + what, lib.hybrid_attn_select_blocks(ref(p), ref(q), FAKE, FAKE, FAKE + 0xF00, BIG, None))
                    check(("forward",) + what, lib.hybrid_attn_sparse_forward(ref(p), ref(q), ref(k), ref(k), FAKE, ref(q), FAKE, FAKE + 0xF00, BIG, None))
                check(("gradients",) + what, lib.hybrid_attn_sparse_grad(ref(p), ref(q), ref(k), ref(k), FAKE, ref(q), FAKE, ref(q), ref(q), ref(k), ref(k), FAKE + 0xF00,
                                                                         BIG, None), may_refuse=True)
for count, n in ((1, 1 << 40), (3, 1 << 38), (500, 1), (300, 1 << 30), (200000, 5)):
    t = (optim.ha_tensor * count)(*[(FAKE, n, ha.HA_BF16, 0)] * count)
    check(("norm", count, n), lib.hybrid_attn_grad_norm(count, t, 1.0, FAKE, FAKE, BIG, None))
    check(("clip", count, n), lib.hybrid_attn_grad_clip(count, t, t, FAKE, None))
    ps = (optim.ha_param * count)(*[(FAKE, FAKE, None, None, None, n, ha.HA_F32, ha.HA_BF16)] * count)
    o = ha.ha_optimizer(ha.HA_OPT_SGD, 1, 1e-3, 1.0, 0.9, 0.999, 1e-8, 0.0)
    check(("update", count, n), lib.hybrid_attn_param_update_many(ref(o), count, ps, FAKE, None))
print(counts, "refused", refused)
for b in bad[:40]:
    print(*b, flush=True)
sys.exit(1 if bad else 0)
"""


def test_no_launch_exceeds_the_device(tmp_path):
    source, so, child = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so", tmp_path / "child.py"
    source.write_text(STAND_IN)
    child.write_text(textwrap.dedent(CHILD))
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(source), "-o", str(so)], check=True)
    run = subprocess.run([sys.executable, str(child), str(so)], cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True, timeout=300)
    print(run.stdout[-3000:])
    assert run.returncode == 0, (run.stdout + run.stderr)[-6000:]
