"""Outputs of the serving entry points that would overwrite rows other workgroups
still read are refused before anything is launched (no GPU needed)."""
import os

import pytest

from paper_2308_13137_amd import oq
from tests.test_abi_serve import BF, F32, FAKE, INVALID, norm

pytestmark = pytest.mark.skipif(not os.path.exists(oq.LIB_PATH), reason="liboq.so not built")

FAR = FAKE + (1 << 30)
T, D = 4, 256                   # test_abi_serve's norm: 4 rows of 256


@pytest.mark.parametrize("x_dt,r_dt", [(BF, F32), (F32, BF)])
def test_norm_sum_over_a_residual_of_another_type(x_dt, r_dt):
    """Row t of H lies in other rows of R than t: a workgroup of another row may still read them."""
    xs, rs = ((2, 4) if x_dt == BF else (4, 2))
    for at in (0, T * D * rs - 16, 16 - T * D * xs):         # the same address; R's last bytes; its first
        assert norm(X=FAR, x_dt=x_dt, R=FAKE, r_dt=r_dt, H=FAKE + at) == INVALID


@pytest.mark.parametrize("dt", [BF, F32])
def test_norm_sum_that_overlaps_an_input_in_part(dt):
    size = T * D * (2 if dt == BF else 4)
    for at in (16, -16, size - 16, 16 - size):
        assert norm(X=FAKE, x_dt=dt, R=FAR, r_dt=dt, H=FAKE + at) == INVALID
        assert norm(X=FAR, x_dt=dt, R=FAKE, r_dt=dt, H=FAKE + at) == INVALID
