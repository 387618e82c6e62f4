"""CPU tests of the C entry points for long contexts on the paged cache: invalid arguments are refused before a device is
touched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def F():
    from paper_2607_07144_amd import fkv
    return fkv


P = ctypes.c_void_p
g, odd, half = P(0x10000), P(0x10001), P(0x10008)   # never dereferenced


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_append_arguments(F):
    E = F.FKV_ERR_INVALID_ARG
    D, R, T = F.fkv_page_desc, F.fkv_row_desc, F.fkv_rotate_desc
    desc, rows, rotate = D(8, 16, 2, 64, 0), R(4, 0, 128, 64, 0), T(100, 64, 0, 4)

    def append(d=desc, t=rotate, rq=rows, ro=rows, rk=rows, rv=rows, q=g, out=g, k=g, v=g, n=4, slots=g, pos=g, tab=g, kc=g, vc=g,
               sc=g, boxes=None, bad=None):
        return F.lib.fkv_page_append(ref(d), ref(t), ref(rq), ref(ro), ref(rk), ref(rv), q, out, k, v, n, slots, pos, tab, kc, vc, sc,
                                     boxes, bad, None)

    for d in (None, D(0, 16, 2, 64, 0), D(8, 24, 2, 64, 0), D(8, 16, 0, 64, 0), D(8, 16, 2, 72, 0), D(8, 16, 2, 64, 2)):
        assert append(d=d) == E
    for bad in (None, R(0, 0, 128, 64, 0), R(4, 0, 127, 64, 0), R(4, 0, 128, -64, 0), R(4, 4, 128, 64, 0), R(4, 0, 128, 64, 2),
                R(4, 0, 128, 64, 1)):
        for name in ("rq", "ro", "rk", "rv"):
            assert append(**{name: bad}) == E, name
    for t in (None, T(100, 8, 0, 4), T(100, 80, 0, 4), T(100, -16, 0, 4), T(0, 64, 0, 4), T(-1, 64, 0, 4), T((1 << 31) + 1, 64, 0, 4),
              T(100, 64, 2, 4), T(100, 64, -1, 4), T(100, 64, 0, 0), T(100, 64, 0, 65536)):
        assert append(t=t) == E
    for kw in (dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(slots=None), dict(pos=None), dict(tab=None), dict(kc=None),
               dict(vc=None), dict(sc=None), dict(q=half), dict(out=half), dict(k=half), dict(v=half), dict(slots=P(0x10004)),
               dict(pos=odd), dict(tab=half), dict(kc=half), dict(vc=half), dict(sc=P(0x10004)), dict(boxes=half), dict(bad=odd),
               dict(n=-1), dict(n=1 << 62)):
        assert append(**kw) == E, kw
    assert append(n=0, k=None, v=None, slots=None, pos=None) == 0
    assert append(n=0, t=None, q=None, out=None, rq=None, ro=None, tab=None, pos=None) == 0
    assert append(n=1 << 40) == F.FKV_ERR_UNSUPPORTED
    assert append(n=1 << 40, t=T(100, 64, 0, 65535)) == F.FKV_ERR_UNSUPPORTED
