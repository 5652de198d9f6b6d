"""The KSA_DEBUG build of the paged calls: every place in the pools, the outputs and the workspace is checked before it is
accessed, and none is outside."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import sys
sys.path.insert(0, %(root)r)
import torch
from paper_2604_24432_b200 import binding as ksa
from tests.paged_check import Strict
from tests.test_gpu_paged import BY_RULE, DEV, FEW, MANY, SHAPES
assert ksa.LIB_PATH.endswith("_debug.so")
ctx = ksa.Context(0)
long_runs = [(8, 1, 9, 16, 4, 128, 64, 0, [(2003, 700)], 0), (8, 1, 9, 8, 1, 64, 16, 0, [(77, 800), (0, 0), (1500, 300)], 3),
             (64, 8, 2, 16, 2, 64, 128, 0, [(66, 330), (70, 300)], 0), (8, 1, 5, 16, 2, 128, 32, 0, [(900, 1), (13, 1400), (0, 0), (300, 2), (44, 17)], 2),
             (8, 1, 3, 4, 1, 64, 16, 0, [(i %% 60, 1 + i %% 2) for i in range(90)], 2)]
for k, m, C, Hq, Hkv, D, ps, flags, spans, pad in SHAPES + long_runs:
    for fmt in ("bf16", "e4m3"):
        for kernel in (BY_RULE, FEW, MANY):
            s = Strict(ctx, k, m, C, Hq, Hkv, D, ps, fmt, [max(1, a + n) for a, n in spans], flags | kernel, seed=29)
            s.fill(spans)
            assert ctx.device_status() == 0, ("append", ctx.device_status())
            back = [torch.empty((sum(n for _, n in spans) + pad, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            s.cache.gather(s.batch(spans), *back)
            assert ctx.device_status() == 0, ("gather", ctx.device_status())
            out, lse = s.attn(spans, pad)                  # (asserts the status)
            s.check(out, lse, spans, sample=3)
print("debug paged ok")
"""


@pytest.mark.gpu
def test_debug_build_of_the_paged_calls():
    from paper_2604_24432_b200 import build as ksa_build
    ksa_build.build(variant="debug")
    env = dict(os.environ, KSA_B200_LIB_VARIANT="debug")
    r = subprocess.run([sys.executable, "-c", SCRIPT % dict(root=ROOT)], capture_output=True, text=True, env=env, timeout=600, cwd=ROOT)
    assert r.returncode == 0, (r.stdout[-1500:], r.stderr[-3000:])
    assert "debug paged ok" in r.stdout
