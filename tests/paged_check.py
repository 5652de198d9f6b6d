"""A server whose results are looked at for NaN too: `paged_ref.check` compares with `>`, which is false for one."""
import numpy as np

from tests import paged_ref as ref
from tests.test_gpu_paged import Server


def check(got_out, got_lse, want, D):
    """paged_ref.check, of results that are numbers."""
    assert np.isfinite(got_out).all() and np.isfinite(got_lse).all(), (int((~np.isfinite(got_out)).sum()), int((~np.isfinite(got_lse)).sum()))
    ref.check(got_out, got_lse, want, D)


class Strict(Server):
    def check(self, out, lse, spans, sample=None):
        rows = sum(n for _, n in spans)
        assert bool(np.isfinite(out[:rows].float().cpu().numpy()).all()) and bool(np.isfinite(lse[:, :rows].cpu().numpy()).all())
        super().check(out, lse, spans, sample)
