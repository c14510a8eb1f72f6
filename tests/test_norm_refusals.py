"""Planes that the gradient of group norm would overwrite before it has read them, refused before anything reaches the device."""
import pytest

import paper_2603_27156_amd as gsr
from test_norm_host import BAD, P, grad


@pytest.mark.parametrize("change", [dict(), dict(lddx=9, ldx=9), dict(lddx=9), dict(layout=1, ldx=4, lddx=4, lddy=4), dict(dtype=1), dict(ptr=None, graphs=1)])
def test_a_gradient_over_its_input_is_refused(change):
    """Every graph's rows are read again while others' are written: dx_out may be dy, but not x."""
    assert grad(dx=2 * P, **change) == BAD
    assert "dx_out is x" in gsr.gsr_last_error()
