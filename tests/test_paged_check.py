"""The checks that the paged cache's GPU tests lean on, by themselves."""
import numpy as np
import pytest
import torch

from tests import paged_check, paged_ref as ref


def _case():
    rng = np.random.default_rng(0)
    q, key, val = rng.normal(size=(2, 4, 64)), rng.normal(size=(20, 2, 64)), rng.normal(size=(20, 2, 64))
    return ref.attention(q, key, val, 8, 1, 1, 18, 0.125)


def test_check_takes_the_reference_itself():
    want = _case()
    paged_check.check(want[0], want[1], want, 64)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_check_refuses_what_is_no_number(which, value):
    want = _case()
    got = [want[0].copy(), want[1].copy()]
    got[which].flat[3] = value
    with pytest.raises(AssertionError):
        paged_check.check(*got, want, 64)


def test_values_of_all_rows_at_once():
    rng = np.random.default_rng(1)
    rows = rng.normal(size=(400, 64)) * np.exp2(rng.uniform(-126, 127, (400, 1)))
    rows[:3] = 0.0
    rows[3, 5], rows[4, 5], rows[5] = np.inf, np.nan, 3.38e38
    rows[6:20, 0] = 448.0 * 2.0 ** np.arange(-7, 7)
    x = torch.tensor(rows).bfloat16().double().numpy()
    want = np.stack([ref.values(*ref.quantise_row(r)) for r in x])
    np.testing.assert_array_equal(paged_check.cached_values(x), want)
