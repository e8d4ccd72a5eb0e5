"""Host-only checks of the entry points for drafted tokens: arguments are refused before
anything is launched (no GPU needed: every call here fails validation or is a no-op)."""
import ctypes as C
import os

import pytest
import torch

from paper_2308_13137_amd import oq
from tests import tree_ref
from tests.test_abi_serve import BF, F32, FAKE, INVALID, ODD, OK, UNSUPPORTED, WORKSPACE, batch, cache

pytestmark = pytest.mark.skipif(not os.path.exists(oq.LIB_PATH), reason="liboq.so not built")
FAR = FAKE + (1 << 30)
HALF = FAKE + 2                 # not aligned to 4 bytes


def append(c=None, b=None, **kw):
    a = dict(parent=FAKE, Q=FAKE, lq=512, K=FAKE + (1 << 28), lk=512, V=FAKE + (1 << 29), lv=512, dt=BF, heads=4,
             rope=None, n_rope=0, s_a=None, out=FAR, st=None)
    a.update(kw)
    return oq.lib().oq_kv_append_tree(C.byref(c or cache()), C.byref(b or batch()), *a.values())


def attend(c=None, b=None, **kw):
    a = dict(parent=FAKE, Q=FAKE, lq=512, heads=4, O=FAKE, LSE=None, ws=FAKE, n=1 << 40, st=None)
    a.update(kw)
    return oq.lib().oq_kv_attend_tree(C.byref(c or cache()), C.byref(b or batch()), *a.values())


def commit(c=None, b=None, **kw):
    a = dict(path=FAKE, max_path=3, count=FAKE, st=None)
    a.update(kw)
    return oq.lib().oq_kv_commit(C.byref(c or cache()), C.byref(b or batch()), *a.values())


def probs(**kw):
    a = dict(X=FAKE, dt=BF, ld=100, T=4, V=100, temp=None, P=FAR, ldp=100, st=None)
    a.update(kw)
    return oq.lib().oq_token_probs(*a.values())


def verify(**kw):
    a = dict(n=2, max_q=3, T=5, qs=FAKE, parent=FAKE, token=FAKE, P=FAKE, ldp=100, Q=None, ldq=0, V=100, replace=1,
             u=FAKE, un=FAKE, path=FAR, max_path=3, count=FAR + 64, next=FAR + 128, st=None)
    a.update(kw)
    return oq.lib().oq_tree_verify(*a.values())


@pytest.mark.parametrize("call", [append, attend, commit])
def test_cache_and_batch_rejects(call):
    for kw in (dict(head_dim=96), dict(page=16), dict(page=96), dict(page=256)):
        assert call(cache(**kw)) == UNSUPPORTED
    for kw in (dict(n_pages=0), dict(n_slots=0), dict(kv_heads=0), dict(k_codes=None), dict(v_codes=ODD),
               dict(k_scale=None), dict(v_scale=ODD), dict(k_window=None), dict(v_window=ODD)):
        assert call(cache(**kw)) == INVALID
    for kw in (dict(n_seq=-1), dict(n_seq=65536), dict(max_pages=0), dict(max_q=-1), dict(tokens=-1), dict(max_q=6),
               dict(max_pages=2 ** 26), dict(table=None), dict(length=None), dict(q_start=None), dict(table=0x10002),
               dict(slot=0x10001)):
        assert call(None, batch(**kw)) == INVALID
    # a tree has at most a page's tokens
    for page in (32, 64, 128):
        assert call(cache(page=page), batch(max_q=page + 1, tokens=1000)) == UNSUPPORTED
    assert call(None, batch(n_seq=0, table=None, length=None, q_start=None)) == OK
    assert call(None, batch(max_q=0)) == OK


def test_append_and_attend_reject():
    for kw in (dict(parent=None), dict(parent=HALF), dict(Q=None), dict(K=ODD), dict(V=None), dict(out=None), dict(out=ODD),
               dict(dt=9), dict(heads=3), dict(heads=0), dict(lq=256), dict(lk=128), dict(lv=260),
               dict(rope=FAKE, n_rope=0), dict(rope=ODD, n_rope=8), dict(s_a=ODD), dict(dt=F32, out=FAKE),
               dict(lq=1024, out=FAKE), dict(out=FAKE + 16), dict(out=FAKE + (1 << 28)), dict(out=FAKE + (1 << 29) + 64)):
        assert append(**kw) == INVALID, kw
    for kw in (dict(parent=None), dict(parent=HALF), dict(Q=None), dict(Q=ODD), dict(O=None), dict(O=ODD), dict(LSE=ODD),
               dict(ws=ODD), dict(heads=3), dict(lq=508), dict(lq=256), dict(O=FAKE + 16), dict(lq=1024)):
        assert attend(**kw) == INVALID, kw
    L, n = oq.lib(), C.c_size_t(0)
    b = batch(n_seq=1, max_pages=512, max_q=5, tokens=5)         # a few rows over 32,768 tokens: split
    assert L.oq_kv_attend_tree_workspace_size(C.byref(cache()), C.byref(b), 4, C.byref(n)) == OK and n.value > 0
    assert attend(None, b, ws=None) == WORKSPACE and attend(None, b, n=n.value - 1) == WORKSPACE
    assert L.oq_kv_attend_tree_workspace_size(C.byref(cache()), C.byref(b), 3, C.byref(n)) == INVALID
    assert L.oq_kv_attend_tree_workspace_size(C.byref(cache()), C.byref(b), 4, None) == INVALID


def test_too_many_tiles():
    for b, heads in ((batch(n_seq=65535, max_q=64, tokens=2 ** 22, max_pages=8), 2 ** 17),
                     (batch(n_seq=65535, max_q=64, tokens=65535 * 64, max_pages=8), 256)):
        assert attend(None, b, heads=heads, lq=heads * 128) == UNSUPPORTED


def test_commit_rejects():
    for kw in (dict(path=None), dict(path=HALF), dict(count=None), dict(count=HALF), dict(max_path=-1)):
        assert commit(**kw) == INVALID, kw
    assert commit(max_path=0, path=None) == OK


def test_probs_rejects():
    for kw in (dict(X=None), dict(P=None), dict(X=FAKE + 1), dict(X=HALF, dt=F32), dict(P=HALF), dict(temp=HALF), dict(dt=7),
               dict(T=-1), dict(V=0), dict(ld=99), dict(ldp=99), dict(P=FAKE), dict(P=FAKE + 796), dict(P=FAKE - 1596),
               dict(dt=F32, P=FAKE)):
        assert probs(**kw) == INVALID, kw
    assert probs(V=2 ** 20 + 1, ld=2 ** 21, ldp=2 ** 21) == UNSUPPORTED
    assert probs(T=0, X=None, P=None) == OK


def test_probs_over_their_temperature():
    """A row's workgroups each read its temperature: no row of P lies over one."""
    for kw in (dict(temp=FAR), dict(temp=FAR + 1596), dict(temp=FAR - 12), dict(temp=FAR + 396, ldp=110),
               dict(temp=FAR + 436, ldp=110), dict(temp=FAR, T=1)):
        assert probs(**kw) == INVALID and b"temperature" in oq.lib().oq_last_error(), kw
    assert probs(T=0, temp=FAR) == OK


def test_verify_rejects():
    for kw in (dict(n=-1), dict(max_q=-1), dict(T=-1), dict(max_q=6, max_path=6), dict(max_path=2), dict(V=0), dict(ldp=99),
               dict(Q=FAKE, ldq=99), dict(qs=None), dict(parent=None), dict(token=None), dict(P=None), dict(u=None),
               dict(un=None), dict(path=None), dict(count=None), dict(next=None), dict(T=2 ** 31),
               *(dict(**{k: HALF}) for k in ("qs", "parent", "token", "P", "Q", "u", "un", "path", "count", "next")
                 if k != "Q"), dict(Q=HALF, ldq=100)):
        assert verify(**kw) == INVALID, kw
    # outputs over inputs, or over each other: the last byte of P (5 rows of 100), the first of u, inside path
    far = dict(qs=FAKE, parent=FAKE + 4096, token=FAKE + 8192, u=FAKE + 12288, un=FAKE + 16384, P=FAKE + (1 << 20))
    for kw in (dict(path=FAKE + 8), dict(count=FAKE + 4096 + 16), dict(next=FAKE + 8192 - 4), dict(path=FAKE + 12288 - 20),
               dict(count=FAKE + 16384 + 4), dict(next=FAKE + (1 << 20) + 1996), dict(Q=FAR + (1 << 20), ldq=100, path=FAR + (1 << 20)),
               dict(count=FAR + 20), dict(next=FAR + 68), dict(path=FAR + 128)):
        assert verify(**{**far, **kw}) == INVALID, kw
    assert verify(max_q=129, T=500, max_path=129) == UNSUPPORTED
    assert verify(V=2 ** 20 + 1, ldp=2 ** 21) == UNSUPPORTED
    assert verify(n=0, qs=None, path=None, count=None, next=None, u=None, un=None, P=None) == OK


def test_binding_refuses_host_tensors():
    i, f = torch.zeros(2, dtype=torch.int32), torch.ones(2, 8)
    for call in (lambda: oq.token_probs(f), lambda: oq.tree_verify(i, i, i, 1, f, f[0], f[0])):
        with pytest.raises(oq.OQError, match="GPU"):
            call()


def test_reference_by_hand():
    """Two siblings, worked out: p = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4)."""
    P = torch.tensor([[0.5, 0.25, 0.25], [0.25, 0.25, 0.5], [1.0, 0.0, 0.0]])
    Q = torch.tensor([[0.25, 0.5, 0.25]]).repeat(3, 1)
    tree = [-1, 0, 0]
    # token 1 is kept with probability 1/2; then r = (1/4, 0, 0) / (1/4): token 0 is kept for certain
    assert tree_ref.verify64([9, 1, 0], tree, P, Q, [0, 0.49, 0.9], 0.3, True) == ([0, 1], 1)
    assert tree_ref.verify64([9, 1, 0], tree, P, Q, [0, 0.5, 0.9], 0.3, True) == ([0, 2], 0)
    # token 2 is not in r after that
    assert tree_ref.verify64([9, 1, 2], tree, P, Q, [0, 0.5, 0.0], 0.99, True) == ([0], 0)
    # without a draft's probabilities: kept with probability p(x), then with p(x) / (1 - p(1))
    assert tree_ref.verify64([9, 1, 2], tree, P, None, [0, 0.25, 0.32], 0.5, True) == ([0, 2], 0)
    assert tree_ref.verify64([9, 1, 2], tree, P, None, [0, 0.25, 0.34], 0.5, True) == ([0], 0)
    # 1/3 of q is left to token 0 without replacement: r = 1 there, so it is kept in any case
    assert tree_ref.verify64([9, 1, 0], tree, P, Q, [0, 0.5, 0.99], 0.3, False) == ([0, 2], 0)
