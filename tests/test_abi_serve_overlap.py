"""Outputs of the serving entry points that would overwrite rows other workgroups
still read are refused before anything is launched (no GPU needed: calls that are
not refused for it stop at a workspace that is too small)."""
import os

import pytest

from paper_2308_13137_amd import oq
from tests.test_abi_serve import BF, F32, FAKE, INVALID, WORKSPACE, append, attend, batch, norm

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


def test_append_queries_over_rows_still_to_be_read():
    """5 rows of 4 query and 2 key heads of 128 (test_abi_serve's batch): Q [5, 512], K and V [5, 256]."""
    w, kw, rows = 512, 256, 5
    apart = dict(Q=FAKE, K=FAKE + (1 << 28), V=FAKE + (1 << 29), lq=w, lk=kw, lv=kw, out=FAR)
    # another type, columns of a wider tensor, shifted rows
    for kw_ in (dict(dt=F32, out=FAKE), dict(dt=F32, out=FAKE + (rows * w * 2 - 1) // 16 * 16), dict(lq=1024, out=FAKE),
                dict(out=FAKE + 16), dict(out=FAKE - 16), dict(out=FAKE + (rows * w - 8) * 2),
                dict(lq=8192, out=FAKE + 3 * 8192 * 2 + 1008), dict(lq=8192, out=FAKE + 4 * 8192 * 2 - 16)):
        assert append(**{**apart, **kw_}) == INVALID, kw_
    # keys and values, also between their rows
    for name in ("K", "V"):
        for at in (0, 16, -16, (rows * kw - 8) * 2):
            assert append(**{**apart, "out": apart[name] + at}) == INVALID, (name, at)
        ld = "l" + name.lower()
        assert append(**{**apart, ld: 2048, "out": apart[name] + 2048 * 2 * 2 + 496}) == INVALID


def test_attend_output_over_queries_still_to_be_read():
    long = batch(n_seq=1, max_pages=512, max_q=3, tokens=3)      # 3 rows of 512, split: needs a workspace
    for lq, O in ((1024, FAKE), (512, FAKE + 16), (512, FAKE - 16), (512, FAKE + 2 * 1024 + 1008),
                  (4096, FAKE + 8192 + 1008), (4096, FAKE + 2 * 8192 - 16)):
        assert attend(None, long, lq=lq, Q=FAKE, O=O, ws=None) == INVALID, (lq, O)
    # the queries themselves; the gap between two rows; before and behind them
    for lq, O in ((512, FAKE), (4096, FAKE + 1024), (4096, FAKE + 8192 - 3 * 1024), (4096, FAKE + 2 * 8192 + 1024),
                  (512, FAKE - 3 * 1024), (512, FAKE + 3 * 1024)):
        assert attend(None, long, lq=lq, Q=FAKE, O=O, ws=None) == WORKSPACE, (lq, O)
    one = batch(n_seq=1, max_pages=512, max_q=1, tokens=1)       # a single row has no stride
    assert attend(None, one, lq=4096, Q=FAKE, O=FAKE, ws=None) == WORKSPACE
