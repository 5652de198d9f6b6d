"""Paged attention of values at the ends of their range, against the definitions in 64 bits, by each of the two kernels: value rows
from zeros to the largest scale, beside one another and out of one another's sight, queries of zeros, one key that outweighs
thousands.  The bounds are those of paged_ref.check."""
import math

import numpy as np
import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from tests.paged_check import Strict
from tests.test_gpu_paged import DEV, FEW, MANY, _i32, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def _no_workspace(s, spans):
    """The call over the e4m3 pages themselves."""
    return s.attn(spans, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))


def _size(rows, byte, seed=0):
    """Rows whose e4m3 scale byte is `byte`: largest value 237 times the scale."""
    g = torch.Generator().manual_seed(seed)
    x = torch.rand(rows, generator=g, dtype=torch.float64) * 2 - 1
    x[..., 0] = 1.0
    return (x * 237.0 * 2.0 ** (byte - 127)).bfloat16()


# ---- value rows of any size ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel,before,n", [(FEW, 300, 1), (FEW, 300, 5), (FEW, 2500, 5), (MANY, 300, 40), (MANY, 2500, 40)])
@pytest.mark.parametrize("byte", [30, 186, 234, 235, 240, 247])
@pytest.mark.parametrize("where", ["alone", "beside", "zeros beside"])
def test_value_rows_of_any_scale(ctx, kernel, before, n, byte, where):
    s = Strict(ctx, 8, 1, 1 << 10, 8, 2, 128, 32, "e4m3", [before + n], seed=byte, flags=kernel)
    v = s.val[0]
    if where == "zeros beside":
        v.zero_()
    pick = slice(None) if where == "alone" else slice(None, None, 7)
    v[pick] = _size(v[pick].shape, byte)
    spans = [(before, n)]
    s.fill(spans)
    out, lse = _no_workspace(s, spans)
    s.check(out, lse, spans, sample=6)


@pytest.mark.parametrize("kernel,before,n", [(FEW, 300, 5), (FEW, 2500, 1), (MANY, 300, 40), (MANY, 2500, 40), (MANY, 2500, 300)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("byte", [45, 186, 220, 247])
@pytest.mark.parametrize("where", ["alone", "beside", "unseen beside"])
def test_value_rows_of_any_size_in_bf16(ctx, kernel, before, n, fmt, byte, where):
    """The same values in bf16 pages, and in the bf16 copy of e4m3 pages (300 rows of 4 query heads)."""
    s = Strict(ctx, 8, 1, 1 << 10, 8, 2, 128, 32, fmt, [before + n], seed=byte, flags=kernel)
    v = s.val[0]
    pick = slice(None) if where == "alone" else slice(None, None, 7) if where == "beside" else slice(before + n // 2, None)
    v[pick] = _size(v[pick].shape, byte)
    spans = [(before, n)]
    s.fill(spans)
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=6)


# ---- rows out of one another's sight -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel,before,n", [(FEW, 300, 5), (FEW, 2500, 5), (MANY, 300, 40), (MANY, 2500, 40)])
@pytest.mark.parametrize("what", ["key", "val"])
@pytest.mark.parametrize("byte", [155, 186, 247])
def test_rows_beside_large_ones_that_they_do_not_see(ctx, kernel, before, n, what, byte):
    """The later half of the new rows is large; the earlier half comes before them, in the same query tile."""
    s = Strict(ctx, 8, 1, 1 << 10, 8, 2, 128, 32, "e4m3", [before + n], seed=byte, flags=kernel)
    rows = (s.key if what == "key" else s.val)[0]
    rows[before + n // 2:] = _size(rows[before + n // 2:].shape, byte)
    spans = [(before, n)]
    s.fill(spans)
    out, lse = _no_workspace(s, spans)
    half = n // 2
    if what == "key":                                      # (scores of the others are beyond fp32 at the largest scale)
        spans = [(before, half)]
        out, lse = out[:half], lse[:, :half]
    s.check(out, lse, spans, sample=10)


# ---- queries of zeros -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel,before,n", [(FEW, 300, 5), (MANY, 300, 40), (MANY, 2500, 40)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("keys", [0.0, 1e-3, 1.0])
@pytest.mark.parametrize("q", [0.0, 1e-30])
def test_small_queries_and_keys(ctx, kernel, before, n, fmt, keys, q):
    """Every second query of zeros or next to nothing, over keys of zeros, small and ordinary ones."""
    s = Strict(ctx, 8, 1, 1 << 10, 8, 2, 128, 32, fmt, [before + n], seed=2, flags=kernel)
    s.q[0][::2] = (s.q[0][::2].double() * q).bfloat16()
    s.key[0] = (s.key[0].double() * keys).bfloat16()
    spans = [(before, n)]
    s.fill(spans)
    out, lse = _no_workspace(s, spans)
    s.check(out, lse, spans, sample=10)


# ---- one key that outweighs thousands --------------------------------------------------------------------------------------
@pytest.mark.parametrize("kernel,n,ws", [(FEW, 1, False), (FEW, 4, False), (MANY, 70, False), (MANY, 70, True)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("gap,sink", [(8, 0.0), (16, 0.0), (16, 2.0 ** -6), (18, 0.0), (18, 2.0 ** -6), (24, 0.0), (40, 0.0)])
def test_one_key_that_outweighs_the_others(ctx, kernel, n, ws, fmt, gap, sink):
    """An attention sink: a first key whose score stands `gap` above those of 3,000 others, with a value row of zeros or a small one.
    ws: with the workspace, where the call takes one."""
    before = 3000
    s = Strict(ctx, 8, 0, 1 << 20, 16, 1, 128, 64, fmt, [before + n], seed=7, flags=kernel)
    s.q[0].fill_(1.0)
    s.key[0].zero_()
    s.key[0][0] = gap / math.sqrt(128.0)
    s.val[0].abs_()
    s.val[0][0] *= sink
    spans = [(before, n)]
    s.fill(spans)
    out, lse = s.attn(spans) if ws else _no_workspace(s, spans)
    s.check(out, lse, spans, sample=3)
