"""What the paged calls promise of their arguments on the device: lengths, padding rows, pools without scales."""
import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from tests.paged_check import Strict
from tests.test_gpu_paged import BY_RULE, DEV, FEW, MANY, _i32, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", [BY_RULE, MANY, FEW])
@pytest.mark.parametrize("n", [1, 130, 700])
@pytest.mark.parametrize("others", [1, 70])                    # (more than 64 sequences are looked for in another way)
def test_packed_rows_start_at_0(ctx, kernel, n, others):
    """cu_rows[0] other than 0: reported, and of the first sequence nothing is written."""
    s = Strict(ctx, 8, 1, 4, 16, 2, 64, 16, "e4m3", [900, 900] + [20] * (others - 1), seed=6, flags=kernel)
    spans = [(60, n), (60, n)] + [(10, 1)] * (others - 1)
    s.fill(spans)
    b = s.batch(spans)
    cu = b.cu_rows.clone()
    cu[0] = 1
    b = ksa.PagedBatch(b.cached, cu, b.text_table, b.summ_table)
    q = s.rows(s.q, spans)
    out, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.full((16, q.shape[0]), -1.0, device=DEV)
    back = [torch.full((q.shape[0], 2, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    rows = [s.rows(x, spans) for x in (s.key, s.val)]
    for call in (lambda: s.cache.attn(b, q, out, lse), lambda: s.cache.gather(b, *back), lambda: s.cache.append(b, *rows)):
        ctx.clear_device_status()
        call()
        torch.cuda.synchronize()
        assert ctx.device_status() == ksa.KSA_PAGED_STATUS_BAD_ROWS
    ctx.clear_device_status()
    assert (out[:n] == 7.0).all() and (lse[:, :n] == -1.0).all() and all((t[:n] == 7.0).all() for t in back)
    s.check(out[n:], lse[:, n:], [(0, 0)] + spans[1:], sample=2)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("seqs", [2, 40])
def test_what_stands_in_padding_rows_does_not_matter(ctx, fmt, seqs):
    """Rows behind the last sequence may be read, as memory of the tensors, and are used for nothing."""
    s = Strict(ctx, 8, 1, 4, 8, 8, 128, 16, fmt, [40] * seqs, seed=6)
    spans, have = [(3, 30)] * seqs, 30 * seqs
    pools = []
    for fill in (0.0, float("nan")):
        s.poison()
        kk, vv = (torch.full((have + 50, 8, 128), fill, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        kk[:have], vv[:have] = s.rows(s.key, spans), s.rows(s.val, spans)
        s.cache.append(s.batch(spans), kk, vv)
        pools.append([t.view(torch.uint8).clone() for t in (s.cache.kpages, s.cache.vpages, s.cache.kscale, s.cache.vscale) if t is not None])
    assert all(torch.equal(x, y) for x, y in zip(*pools))


def test_pools_without_their_scales_hold_nothing(ctx):
    """Scales of zeros would read them as 2^-127 times what they hold."""
    s = Strict(ctx, 8, 0, 100, 4, 2, 64, 16, "e4m3", [40], seed=6)
    s.append([(0, 40)])
    again = ksa.PagedCache(ctx, s.cache.spec, s.cache.kpages, s.cache.vpages)
    got = [torch.zeros((40, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    again.gather(s.batch([(0, 40)]), *got)
    assert all(torch.isnan(g).all() for g in got)
    b = s.batch([(0, 40)])
    again.append(b, s.rows(s.key, [(0, 40)]), s.rows(s.val, [(0, 40)]))
    again.gather(b, *got)
    for g, x in zip(got, (s.key, s.val)):
        assert (g.double().cpu().numpy() == s.cached_values(x[0])).all()
