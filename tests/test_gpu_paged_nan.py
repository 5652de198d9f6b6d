"""NaN in paged attention: pools that start as NaN must leave no trace in any output (the checks of test_gpu_paged.py let NaN
pass, those here look for it), and rows that stand for NaN reach those that see them."""
import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from tests.paged_check import Strict
from tests.test_gpu_paged import DEV, FEW, MANY, SHAPES, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", [MANY, FEW])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("k,m,C,Hq,Hkv,D,ps,flags,spans,pad", SHAPES)
def test_what_nobody_sees_leaves_no_trace(ctx, kernel, fmt, k, m, C, Hq, Hkv, D, ps, flags, spans, pad):
    s = Strict(ctx, k, m, C, Hq, Hkv, D, ps, fmt, [max(1, a + n) for a, n in spans], flags | kernel, seed=11)
    s.fill(spans)
    out, lse = s.attn(spans, pad)
    s.check(out, lse, spans, sample=8)


@pytest.mark.parametrize("kernel,n,ws", [(FEW, 1, None), (FEW, 5, None), (MANY, 5, None), (MANY, 300, None), (MANY, 700, 256), (MANY, 700, None)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("ps", [16, 128])
def test_released_pages_and_workspaces_of_nan(ctx, kernel, n, ws, fmt, ps):
    """Text before every window given back, rows behind the sequence and the workspace NaN."""
    k, m, C, a = 8, 1, 9, 2003
    s = Strict(ctx, k, m, C, 8, 2, 128, ps, fmt, [a + n + 40, 33], seed=5, flags=kernel)
    spans = [(a, n), (20, 3)]
    s.fill(spans)
    first = max(0, a // 9 - C) * k // ps
    gone = torch.from_numpy(s.text[0, :first].copy()).to(DEV)
    s.text[0, :first] = -1
    for t in (s.cache.kpages, s.cache.vpages):
        t[gone] = float("nan")
    for t in (s.cache.kscale, s.cache.vscale):
        if t is not None:
            t[gone] = 255
    room = torch.full(((ws or 32 << 20) // 2,), float("nan"), dtype=torch.bfloat16, device=DEV)
    out, lse = s.attn(spans, workspace=room)
    s.check(out, lse, spans, sample=8)


@pytest.mark.parametrize("kernel,n,ws", [(FEW, 6, False), (MANY, 70, False), (MANY, 700, True)])
@pytest.mark.parametrize("what", ["key", "val"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_rows_of_nan_reach_those_that_see_them(ctx, kernel, n, ws, what, bad):
    """Row 3 of chunk 20 of the first sequence, as a row that is not finite (scale byte 255): the text of its window and its chunk's
    summary see it.  The other sequence does not change."""
    k, m, C = 8, 1, 4
    s = Strict(ctx, k, m, C, 8, 2, 128, 16, "e4m3", [900, 900], seed=5, flags=kernel)
    row = 20 * 9 + 3
    (s.key if what == "key" else s.val)[0][row, 1, 17] = bad
    spans = [(row + 2, n), (row, n)]
    s.fill(spans)
    out, lse = s.attn(spans, **({} if ws else dict(workspace=torch.empty(256, dtype=torch.uint8, device=DEV))))
    a = torch.arange(row + 2, row + 2 + n)
    chunk, r = a // 9, a % 9
    sees = torch.where(r < 8, chunk - C <= 20, chunk == 20).to(DEV)
    assert torch.isnan(out[:n][sees][:, 4:]).all()                    # the query heads of KV head 1
    if what == "key":
        assert torch.isnan(lse[4:, :n][:, sees]).all()
    s.q, s.key, s.val = s.q[1:], s.key[1:], s.val[1:]
    s.check(out[n:], lse[:, n:], spans[1:], sample=8)
