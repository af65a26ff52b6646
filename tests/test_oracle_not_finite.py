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


def test_merge_keeps_nan():
    for order in ((0, 1, 2, 3), (3, 0, 1, 2)):
        parts_o, parts_l = _states(4)
        o, lse = oa.empty_state(1, 3, 2, 4)
        for x in order:
            o, lse = oa.merge(o, lse, parts_o[x], parts_l[x])
        _check(o, lse)
