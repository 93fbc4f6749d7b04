"""The angles of an unstretched form are those of the calls without a form, bit for bit: theta_i = 2^(i c), c = -2 log2(base) / rotary_dim."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2602_07529_b200 import binding as B
from test_step_refusals import INVALID, OK


def wanted(base, rd):
    c = -2.0 * math.log2(base) / float(rd)
    return np.asarray([math.exp2(float(i) * c) for i in range(rd // 2)])


@pytest.mark.parametrize("rd", [16, 48, 64, 128])
@pytest.mark.parametrize("base", [1.0, 2.0, 1e4, 5e5, 1e6, 1e300])
def test_plain_angles_are_those_of_the_calls_without_a_form(base, rd):
    theta = B.RopeForm(B.ROPE_HALVES, rd, base=base).theta
    assert np.array_equal(theta, wanted(base, rd)) and theta[0] == 1.0
    # stretched by nothing: the same angles
    for scaling in ("linear", "base"):
        assert np.array_equal(B.RopeForm(B.ROPE_PAIRS, rd, base=base, scaling=scaling, factor=1.0).theta, theta)
    assert np.array_equal(B.RopeForm(B.ROPE_HALVES, rd, base=base, scaling="linear", factor=8.0).theta, theta / 8.0)


def test_a_base_that_overflows_is_refused():
    """1e300 stretched by 1e300 is no number; unstretched it is one."""
    f = B._RopeForm()
    init = lambda scaling, factor: B.lib.mv_rope_form_init(C.byref(f), 0, 0, 64, 1e300, scaling, factor, 1.0, 0.0, 1.0, 1.0)
    assert init(0, 1.0) == OK and init(2, 1e300) == INVALID
    assert init(1, 1e300) == OK and np.isfinite(f.theta[:32]).all()
