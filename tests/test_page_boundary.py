"""CPU tests of the paged cache's C entry points: invalid arguments are refused before a device is touched."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def F():
    from paper_2607_07144_amd import fkv
    return fkv


P = ctypes.c_void_p
g, odd, half = P(0x10000), P(0x10001), P(0x10008)   # never dereferenced
ref = ctypes.byref


def test_plan_arguments(F):
    E = F.FKV_ERR_INVALID_ARG

    def plan(page=16, n=4, kv=g, new=g, free=g, nf=9, head=None, tab=g, width=3, nt=5, slots=g, pos=None, qs=g, end=P(0x20000),
             ho=g, nh=None, st=None, bad=None):
        return F.lib.fkv_page_plan(page, n, kv, new, free, nf, head, tab, width, nt, slots, pos, qs, end, ho, nh, st, bad, None)

    for page in (0, 8, 24, 272, -16):
        assert plan(page=page) == E
    for kw in (dict(n=-1), dict(n=1 << 31), dict(nf=-1), dict(nt=-1), dict(nt=1 << 31), dict(width=0), dict(width=1 << 27),
               dict(kv=None), dict(new=None), dict(tab=None), dict(end=None), dict(qs=None), dict(ho=None), dict(slots=None),
               dict(free=None), dict(kv=odd), dict(slots=P(0x10004)), dict(head=g), dict(end=g), dict(nh=g, head=g), dict(pos=odd),
               dict(bad=odd), dict(head=odd), dict(tab=odd), dict(qs=odd), dict(nh=odd)):
        assert plan(**kw) == E, kw


def test_store_and_load_arguments(F):
    E = F.FKV_ERR_INVALID_ARG
    D, R = F.fkv_page_desc, F.fkv_row_desc
    desc, rows = D(8, 16, 2, 64, 0), R(4, 0, 128, 64, 0)

    def store(d=desc, rk=rows, rv=rows, k=g, v=g, n=4, slots=g, kc=g, vc=g, sc=g, bad=None):
        return F.lib.fkv_page_store(None if d is None else ref(d), None if rk is None else ref(rk),
                                    None if rv is None else ref(rv), k, v, n, slots, kc, vc, sc, bad, None)

    def load(d=desc, rk=rows, rv=rows, k=g, v=g, n=4, slots=g, kc=g, vc=g, sc=g):
        return F.lib.fkv_page_load(None if d is None else ref(d), kc, vc, sc, n, slots, None if rk is None else ref(rk),
                                   None if rv is None else ref(rv), k, v, None)

    for bad in (None, D(0, 16, 2, 64, 0), D(8, 24, 2, 64, 0), D(8, 272, 2, 64, 0), D(8, 16, 0, 64, 0), D(8, 16, 2, 72, 0),
                D(8, 16, 2, 272, 0), D(8, 16, 2, 0, 0), D(8, 16, 2, 64, 2), D(1 << 31, 16, 2, 64, 0)):
        assert store(d=bad) == E and load(d=bad) == E
    for bad in (None, R(0, 0, 128, 64, 0), R(4, 0, 127, 64, 0), R(4, 0, 128, -64, 0), R(4, 4, 128, 64, 0), R(4, 0, 128, 64, 2)):
        assert store(rk=bad) == E and store(rv=bad) == E and load(rk=bad) == E and load(rv=bad) == E
    assert store(rv=R(4, 0, 128, 64, 1)) == E and load(rk=R(4, 0, 128, 64, 1)) == E
    for kw in (dict(k=half), dict(v=half), dict(kc=half), dict(vc=half), dict(sc=P(0x10004)), dict(kc=None), dict(vc=None),
               dict(sc=None), dict(slots=None), dict(slots=P(0x10004)), dict(n=-1)):
        assert store(**kw) == E and load(**kw) == E, kw
    assert store(k=None) == E and store(v=None) == E and store(bad=odd) == E
    assert store(n=0, k=None, v=None, slots=None) == 0 and load(n=0, slots=None) == 0
    assert load(k=None, v=None, rk=None, rv=None) == 0


def attend_desc(F, **kw):
    base = dict(n_req=2, n_tokens=4, max_new=2, max_kv=64, max_pages=4, q_stride_token=256, q_stride_head=64, o_stride_token=256,
                o_stride_head=64, q_heads=4, type=0, scale=0.125, softcap=0.0, causal=1, window=0, sinks=0)
    return F.fkv_attend_desc(**{**base, **kw})


def test_attend_arguments(F):
    E = F.FKV_ERR_INVALID_ARG
    desc = F.fkv_page_desc(8, 16, 2, 64, 0)

    def attend(d=desc, kc=g, vc=g, sc=g, q=g, tab=g, kv=g, qs=g, slopes=None, prefix=None, first=None, out=g, lse=None, ws=None,
               nws=0, **kw):
        t = attend_desc(F, **kw)
        return F.lib.fkv_page_attend(None if d is None else ref(d), ref(t), kc, vc, sc, q, tab, kv, qs, slopes, prefix, first, out,
                                     lse, ws, nws, None)

    for kw in (dict(d=None), dict(kc=None), dict(vc=half), dict(sc=P(0x10004)), dict(q=None), dict(q=half), dict(out=None),
               dict(out=half), dict(tab=None), dict(kv=None), dict(qs=odd), dict(slopes=odd), dict(prefix=odd), dict(first=odd),
               dict(lse=odd), dict(q_heads=3), dict(q_heads=0), dict(type=2), dict(scale=math.nan), dict(scale=math.inf),
               dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf), dict(causal=2), dict(window=-1), dict(sinks=-1),
               dict(max_new=0), dict(max_kv=-1), dict(max_pages=0), dict(n_req=-1), dict(n_tokens=-1), dict(q_stride_token=4),
               dict(o_stride_head=-8)):
        assert attend(**kw) == E, kw
    assert attend(n_req=0, q=None, out=None) == 0 and attend(n_tokens=0, q=None) == 0


def test_attend_scratch(F):
    """A call that splits the keys says how much scratch it takes and refuses less."""
    desc = F.fkv_page_desc(4096, 16, 2, 64, 0)
    t = attend_desc(F, n_req=1, n_tokens=1, max_new=1, max_kv=32768, max_pages=2048)
    need = F.lib.fkv_page_attend_workspace(ref(desc), ref(t))
    assert need > 0
    args = (ref(desc), ref(t), g, g, g, g, g, g, g, None, None, None, g, None)
    assert F.lib.fkv_page_attend(*args, None, 0, None) == F.FKV_ERR_SCRATCH_TOO_SMALL
    assert F.lib.fkv_page_attend(*args, g, need - 1, None) == F.FKV_ERR_SCRATCH_TOO_SMALL
    assert F.lib.fkv_page_attend(*args, half, need, None) == F.FKV_ERR_INVALID_ARG
    one = attend_desc(F, max_kv=64)
    assert F.lib.fkv_page_attend_workspace(ref(desc), ref(one)) == 0
    assert F.lib.fkv_page_attend_workspace(None, ref(one)) == 0
    assert F.lib.fkv_page_attend_workspace(ref(desc), ref(attend_desc(F, q_heads=3))) == 0


def test_reference_plan_by_hand():
    """The plan that the GPU's is checked against, on a case worked out by hand."""
    import numpy as np
    import pages_reference
    t = np.array([[7, -1, -1], [3, 4, -1], [-1, -1, -1]], np.int32)
    p = pages_reference.plan(16, np.array([10, 32, 0]), np.array([7, 1, 40]), np.array([20, 21, 22, 23]), 0, t, 48)
    assert p["tables"].tolist() == [[7, 20, -1], [3, 4, 21], [-1, -1, -1]]
    assert p["status"].tolist() == [0, 0, 1] and p["kv_end"].tolist() == [17, 33, 0] and p["q_start"].tolist() == [0, 7, 8, 48]
    assert p["slots"][:8].tolist() == [122, 123, 124, 125, 126, 127, 320, 336] and (p["slots"][8:] == -1).all()
    assert p["head"] == 2 and p["next_head"] == 2
