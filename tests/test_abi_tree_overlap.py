"""Host-only: which overlaps of rows side by side are refused (every call here is)."""
import os

import pytest

from paper_2308_13137_amd import oq
from tests.test_abi_serve import BF, F32, FAKE, INVALID
from tests.test_abi_tree import probs, verify

pytestmark = pytest.mark.skipif(not os.path.exists(oq.LIB_PATH), reason="liboq.so not built")


@pytest.mark.parametrize("dt,ld,at", [*((F32, 300, at) for at in (0, 1, 99, 201, 299, -99, -1, -201 + 300, 605, 999, -999, -801)),
                                      *((BF, 600, at) for at in (0, 1, 49, 201, 299, -99, -1, -300, 605, 949, -999))])
def test_probs_over_logits_of_the_same_pitch(dt, ld, at):
    """Four rows of 100 values 1,200 bytes apart, P's likewise `at` floats behind them."""
    size = 100 if dt == F32 else 50
    assert any(abs(at + 300 * k + 50 - size / 2) < 50 + size / 2 for k in range(-3, 4))
    assert probs(dt=dt, ld=ld, ldp=300, P=FAKE + 4 * at) == INVALID
    assert b"overlap" in oq.lib().oq_last_error()


@pytest.mark.parametrize("at", [0, 100, 248, 250, 500, 600, 899, 250 * 5 + 9])
def test_probs_over_logits_of_another_pitch(at):
    """P counts as one piece from its first row to its last."""
    assert probs(dt=F32, ld=300, ldp=250, P=FAKE + 4 * (at - 250 * 3 - 99 if at > 900 else at)) == INVALID
    assert b"overlap" in oq.lib().oq_last_error()


@pytest.mark.parametrize("at", [99, 0, 198, 199, 200 * 4 + 99, -1, -2])
def test_verify_outputs_over_rows(at):
    """P: five rows of 100, 200 apart; count has three values."""
    assert verify(n=3, max_q=1, max_path=1, ldp=200, P=FAKE + (1 << 20), count=FAKE + (1 << 20) + 4 * at) == INVALID
    assert b"overlap the inputs" in oq.lib().oq_last_error()


def test_verify_outputs_over_inputs_of_no_tokens():
    """Without tokens the ranges and numbers of each tree are inputs still."""
    kw = dict(n=2, max_q=0, max_path=0, T=0, parent=None, token=None, P=None, u=None)
    for bad in (dict(count=FAKE + 8), dict(next=FAKE + 4096 - 4)):
        assert verify(**{**kw, "qs": FAKE, "un": FAKE + 4096, **bad}) == INVALID
        assert b"overlap the inputs" in oq.lib().oq_last_error()
