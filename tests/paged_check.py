"""A server whose results are looked at for NaN too: `paged_ref.check` compares with `>`, which is false for one."""
import numpy as np

from tests import paged_ref as ref
from tests.test_gpu_paged import Server


def cached_values(x):
    """What e4m3 pages hold of rows [.., D], in 64 bits: paged_ref.values(*paged_ref.quantise_row(row)) of all rows at once."""
    top = np.abs(x).max(-1)
    fine = np.isfinite(top)
    e = np.full(top.shape, -110)
    for _ in range(230):
        e += fine & (top > 448.0 * np.exp2(e.astype(float)))
    scale = np.exp2(e.astype(float))[..., None]
    y = np.where(fine[..., None], np.abs(x), 0.0) / scale
    last = np.where(e == 120, 119, 126)[..., None]
    i = np.minimum(np.searchsorted(ref.E4M3, y, side="right") - 1, last)
    j = np.minimum(i + 1, last)
    up = (y - ref.E4M3[i] > ref.E4M3[j] - y) | ((y - ref.E4M3[i] == ref.E4M3[j] - y) & (i % 2 == 1))
    return np.where(fine[..., None], np.copysign(ref.E4M3[np.where(up, j, i)] * scale, x), np.nan)


def check(got_out, got_lse, want, D):
    """paged_ref.check, of results that are numbers."""
    assert np.isfinite(got_out).all() and np.isfinite(got_lse).all(), (int((~np.isfinite(got_out)).sum()), int((~np.isfinite(got_lse)).sum()))
    ref.check(got_out, got_lse, want, D)


class Strict(Server):
    def cached_values(self, rows):
        return rows.double().numpy() if self.fmt == "bf16" else cached_values(rows.double().numpy())

    def check(self, out, lse, spans, sample=None):
        rows = sum(n for _, n in spans)
        assert bool(np.isfinite(out[:rows].float().cpu().numpy()).all()) and bool(np.isfinite(lse[:, :rows].cpu().numpy()).all())
        super().check(out, lse, spans, sample)
