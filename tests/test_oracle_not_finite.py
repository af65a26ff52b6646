"""The oracle's folds of states whose lse is NaN: the row becomes NaN, unlike one that is empty (CPU)."""
import numpy as np

from oracle import attention as oa


def _states(n):
    rng = np.random.default_rng(n)
    o, lse = rng.standard_normal((n, 1, 3, 2, 4)), rng.standard_normal((n, 1, 2, 3))
    lse[:, 0, 0, 0] = -np.inf
    lse[n - 1, 0, 0, 0] = np.nan                     # NaN in one state, empty in the others
    lse[:, 0, 1, 2] = -np.inf
    return list(o), list(lse)


def _check(o, lse):
    assert np.isnan(o[0, 0, 0]).all() and np.isnan(lse[0, 0, 0])
    assert (o[0, 2, 1] == 0).all() and lse[0, 1, 2] == -np.inf
    o[0, 0, 0], lse[0, 0, 0] = 0, 0
    assert not np.isnan(o).any() and not np.isnan(lse).any()


def test_combine_keeps_nan():
    for n in (1, 2, 5):
        _check(*oa.combine(*_states(n)))
