"""Host-only checks of the serving entry points: arguments are refused before
anything is launched (no GPU needed: every call here fails validation, is a
no-op or only sizes a workspace)."""
import ctypes as C
import os

import pytest
import torch

from paper_2308_13137_amd import oq

pytestmark = pytest.mark.skipif(not os.path.exists(oq.LIB_PATH), reason="liboq.so not built")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x10000                  # aligned, never dereferenced: validation fails first
ODD = 0x10004
BF, F32 = oq.OQ_BF16, oq.OQ_F32


def norm(**kw):
    a = dict(X=FAKE, x_dt=BF, R=FAKE, r_dt=BF, T=4, D=256, gain=FAKE, bias=None, eps=1e-6, bits=8, H=FAKE,
             X_dq=None, dq_dt=BF, codes=FAKE, h=FAKE, z=FAKE, st=None)
    a.update(kw)
    return oq.lib().oq_rmsnorm_quant(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INVALID), (dict(gain=None), INVALID), (dict(D=252), INVALID), (dict(D=0), INVALID),
    (dict(T=-1), INVALID), (dict(x_dt=7), INVALID), (dict(r_dt=7), INVALID), (dict(X_dq=FAKE, dq_dt=7), INVALID),
    (dict(D=32776), UNSUPPORTED), (dict(bits=1), UNSUPPORTED), (dict(bits=9), UNSUPPORTED),
    (dict(bits=1 | oq.ACT_SYM), UNSUPPORTED), (dict(bits=16 | oq.ACT_SYM), INVALID), (dict(bits=16), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(R=None), INVALID),
    (dict(X=ODD), INVALID), (dict(R=ODD), INVALID), (dict(gain=ODD), INVALID), (dict(bias=ODD), INVALID),
    (dict(H=ODD), INVALID), (dict(codes=ODD), INVALID), (dict(h=ODD), INVALID), (dict(z=ODD), INVALID),
    (dict(T=0, X=None, gain=None), OK),
])
def test_norm_rejects(kw, status):
    assert norm(**kw) == status


def pack(**kw):
    a = dict(codes=FAKE, c_out=32, c_in=64, packed=FAKE, wsum=FAKE, st=None)
    a.update(kw)
    return oq.lib().oq_int8_pack(*a.values())


def lin(**kw):
    a = dict(x=FAKE, h=FAKE, z=FAKE, n=4, c_in=64, w=FAKE, ws=FAKE, hw=FAKE, zw=FAKE, B=None, c_out=32, Y=FAKE,
             y_dt=BF, st=None)
    a.update(kw)
    return oq.lib().oq_int8_linear(*a.values())


def test_linear_rejects():
    for f, out in ((pack, "c_out"), (lin, "c_out")):
        assert f(c_in=72) == INVALID and f(c_in=0) == INVALID and f(**{out: -1}) == INVALID
        assert f(c_in=65552) == UNSUPPORTED and f(**{out: 2 ** 31 - 1}) == UNSUPPORTED
    for name in ("codes", "packed", "wsum"):
        assert pack(**{name: None}) == INVALID and pack(**{name: ODD}) == INVALID
    for name in ("x", "h", "z", "w", "ws", "hw", "zw", "Y"):
        assert lin(**{name: None}) == INVALID and lin(**{name: ODD}) == INVALID
    assert lin(B=ODD) == INVALID and lin(y_dt=5) == INVALID and lin(n=-1) == INVALID
    assert lin(n=2 ** 22 + 1) == UNSUPPORTED and lin(n=2 ** 22, c_out=2 ** 16 + 1) == UNSUPPORTED
    assert pack(c_out=0, codes=None) == OK
    assert lin(n=0, x=None) == OK and lin(c_out=0, w=None) == OK


def cache(**kw):
    a = dict(n_pages=8, n_slots=2, page=64, kv_heads=2, head_dim=128, k_codes=FAKE, v_codes=FAKE, k_scale=FAKE,
             v_scale=FAKE, k_window=FAKE, v_window=FAKE)
    a.update(kw)
    return oq.KVCacheDesc(*a.values())


def batch(**kw):
    a = dict(n_seq=2, max_pages=4, max_q=3, tokens=5, table=FAKE, slot=None, length=FAKE, q_start=FAKE)
    a.update(kw)
    return oq.KVBatch(*a.values())


def append(c=None, b=None, **kw):
    a = dict(Q=FAKE, lq=512, K=FAKE, lk=512, V=FAKE, lv=512, dt=BF, heads=4, rope=None, n_rope=0, s_a=None,
             out=FAKE, st=None)
    a.update(kw)
    return oq.lib().oq_kv_append(C.byref(c or cache()), C.byref(b or batch()), *a.values())


def attend(c=None, b=None, **kw):
    a = dict(Q=FAKE, lq=512, heads=4, O=FAKE, LSE=None, ws=FAKE, n=1 << 40, st=None)
    a.update(kw)
    return oq.lib().oq_kv_attend(C.byref(c or cache()), C.byref(b or batch()), *a.values())


def read(c=None, b=None, **kw):
    a = dict(begin=FAKE, rs=FAKE, rows=4, max_rows=4, K=FAKE, V=FAKE, dt=BF, st=None)
    a.update(kw)
    return oq.lib().oq_kv_read(C.byref(c or cache()), C.byref(b or batch()), *a.values())


@pytest.mark.parametrize("call", [append, attend, read])
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
    assert call(None, batch(n_seq=0, table=None, length=None, q_start=None)) == OK


def test_append_rejects():
    for kw in (dict(Q=None), dict(K=ODD), dict(V=None), dict(out=None), dict(out=ODD), dict(dt=9), dict(heads=3),
               dict(heads=0), dict(lq=256), dict(lk=128), dict(lv=260), dict(rope=FAKE, n_rope=0),
               dict(rope=ODD, n_rope=8), dict(s_a=ODD)):
        assert append(**kw) == INVALID
    assert append(None, batch(max_q=0), Q=None) == OK


def test_attend_rejects_and_sizes():
    for kw in (dict(Q=None), dict(Q=ODD), dict(O=None), dict(O=ODD), dict(LSE=ODD), dict(ws=ODD), dict(heads=3),
               dict(lq=508), dict(lq=256)):
        assert attend(**kw) == INVALID
    L, n = oq.lib(), C.c_size_t(0)
    b = batch(n_seq=1, max_pages=512, max_q=1, tokens=1)         # one row over 32,768 tokens: split
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(b), 4, C.byref(n)) == OK and n.value > 0
    assert attend(None, b, ws=None) == WORKSPACE and attend(None, b, n=n.value - 1) == WORKSPACE
    # rows behind the sequences do not make it larger
    more = batch(n_seq=1, max_pages=512, max_q=1, tokens=1 << 20)
    m = C.c_size_t(0)
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(more), 4, C.byref(m)) == OK and m.value == n.value
    # neither do batch and length: whole splits are bounded by what fills the GPU
    big = batch(n_seq=4096, max_pages=4096, max_q=1, tokens=4096)
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(big), 64, C.byref(m)) == OK and m.value < 1 << 30
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(b), 3, C.byref(n)) == INVALID
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(b), 1 << 18, C.byref(n)) == INVALID
    assert L.oq_kv_attend_workspace_size(C.byref(cache()), C.byref(b), 4, None) == INVALID
    huge = batch(n_seq=65535, max_q=2 ** 20, tokens=2 ** 30)
    assert attend(None, huge, heads=64, lq=8192) == UNSUPPORTED
    huge = batch(n_seq=65535, max_q=2 ** 30, tokens=2 ** 31 - 1, max_pages=2 ** 24)
    assert attend(None, huge, heads=1 << 17, lq=1 << 24) == UNSUPPORTED


def test_read_and_table_reject():
    for kw in (dict(begin=None), dict(rs=None), dict(rs=0x10002), dict(rows=-1), dict(max_rows=-1), dict(K=ODD),
               dict(V=ODD), dict(dt=4)):
        assert read(**kw) == INVALID
    assert read(K=None, V=None) == OK and read(rows=0) == OK
    L = oq.lib()
    for a in ((-1, 128, 1e4, FAKE), (8, 127, 1e4, FAKE), (8, 128, 0.0, FAKE), (8, 128, float("inf"), FAKE),
              (8, 128, 1e4, None), (8, 128, 1e4, ODD), ((1 << 24) + 1, 128, 1e4, FAKE)):
        assert L.oq_rope_table(*a, None) == INVALID
    assert L.oq_rope_table(0, 128, 1e4, None, None) == OK


def test_binding_refuses_host_tensors():
    x, g = torch.zeros(2, 64), torch.ones(64)
    for call in (lambda: oq.rmsnorm_quant(x, g, 8), lambda: oq.int8_pack(x.to(torch.uint8)),
                 lambda: oq.int8_linear(x.to(torch.uint8), g, g, x, x, g, g),
                 lambda: oq.KVCache(2, 32, 1, 64, 1, device="cpu"), lambda: oq.rope_table(4, 64, device="cpu")):
        with pytest.raises(oq.OQError, match="GPU"):
            call()
