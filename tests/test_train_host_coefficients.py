"""Which coefficients an orthogonalised update takes, no GPU: the limits that the header gives, just inside and just
outside.  (A step with b = c = 0 multiplies by a; what roundings add is reckoned as 2 % and 0.001.)"""
import pytest

import paper_2109_08751_b200 as sp


def takes(*triples):
    try:
        sp.OrthoPlan(1, 8, 8, steps=len(triples), coefficients=triples).destroy()
        return True
    except sp.SparbitError as e:
        assert e.code == sp.ERR_ARG
        return False


@pytest.mark.parametrize("sign", [1, -1])
def test_values_before_a_step_and_after_the_last(sign):
    assert takes((sign * 6.7, 0, 0), (1, 0, 0)) and not takes((sign * 6.9, 0, 0), (1, 0, 0))
    assert takes((sign * 62.7, 0, 0)) and not takes((sign * 62.8, 0, 0))
    assert takes((6, 0, 0), (sign * 10, 0, 0)) and not takes((6, 0, 0), (sign * 10.5, 0, 0))


@pytest.mark.parametrize("sign", [1, -1])
def test_the_polynomial(sign):
    assert takes((0, sign * 48, 0)) and not takes((0, sign * 48.1, 0))
    assert takes((0, 0, sign * 48)) and not takes((0, 0, sign * 48.1))
    # 60 (t - t^2) is at most 15, 200 (t - t^2) 50
    assert takes((0, sign * 60, -sign * 60)) and not takes((0, sign * 200, -sign * 200))
