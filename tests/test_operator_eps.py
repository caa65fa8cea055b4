"""eps of norm_fwd above a float's range is refused (host; of no rows, so that nothing is
launched whatever the answer)."""
import pytest

from paper_2607_05804_amd import turnkl as T
from test_operator_abi import norm_fwd


@pytest.mark.parametrize("eps", [3.5e38, 1e39, 1e308])
def test_eps_above_the_largest_float_is_refused(eps):
    assert norm_fwd(n=0, x=0, y=0, eps=eps) == T.ERR_INVALID_ARG


def test_eps_of_a_float_is_not():
    for eps in (0.0, 1e-300, 1e-45, 1e-6, 3.4e38):
        assert norm_fwd(n=0, x=0, y=0, eps=eps) == T.OK
