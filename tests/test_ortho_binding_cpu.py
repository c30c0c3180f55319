"""Numbers that the C structures of an orthogonalisation plan cannot hold are refused by the binding, without a GPU."""
import pytest

import paper_1905_05957_amd as P


@pytest.mark.parametrize("call", [
    dict(d=2 ** 64 + 100), dict(d=-2 ** 64 + 100), dict(mats=[(2 ** 64, 2, 2)]), dict(mats=[(2 ** 64 + 5, 2, 2, 3)]),
    dict(mats=[(0, 2, 2, 2 ** 64 + 2)]), dict(mats=[(0, 2 ** 32 + 2, 2)]), dict(mats=[(0, 2, 2 ** 32 + 2)]), dict(steps=2 ** 32 + 5),
    dict(steps=2 ** 32 + 5, coef=(1.5, -0.5, 0.0)), dict(scale=2 ** 32), dict(mats=[(0, 2, 2), (2 ** 64 + 4, 2, 2)]),
], ids=str)
def test_numbers_that_would_be_cut_are_refused(call):
    with pytest.raises(ValueError, match="no (32|64)-bit number"):
        P.OrthoPlan(**{**dict(d=100, mats=[(0, 2, 2)]), **call})


@pytest.mark.parametrize("steps", [0, -1, 33, 2 ** 31 - 1])
@pytest.mark.parametrize("coef", [None, (1.5, -0.5, 0.0)])
def test_numbers_of_steps_out_of_range(steps, coef):
    # one triple for every step: no list of so many is made
    with pytest.raises(P.DsError, match="shape"):
        P.OrthoPlan(100, [(0, 2, 2)], steps=steps, coef=coef)
