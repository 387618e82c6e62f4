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


def select_desc(F, **kw):
    base = dict(n_req=2, n_tokens=4, max_new=2, max_kv=64, max_pages=4, q_stride_token=256, q_stride_head=64, q_heads=4, type=0,
                causal=1, n_select=2, keep_first=1, keep_last=1)
    return F.fkv_select_desc(**{**base, **kw})


def test_select_arguments(F):
    E = F.FKV_ERR_INVALID_ARG
    desc = F.fkv_page_desc(8, 16, 2, 64, 0)

    def select(d=desc, box=g, sc=g, q=g, tab=g, kv=g, qs=g, sel=g, ws=g, nws=1 << 20, **kw):
        t = select_desc(F, **kw)
        return F.lib.fkv_page_select(ref(d), ref(t), box, sc, q, tab, kv, qs, sel, ws, nws, None)

    for kw in (dict(d=None), dict(d=F.fkv_page_desc(8, 24, 2, 64, 0)), dict(box=None), dict(box=half), dict(sc=None), dict(sc=P(0x10004)),
               dict(q=None), dict(q=half), dict(tab=None), dict(tab=odd), dict(kv=None), dict(kv=odd), dict(qs=None), dict(qs=odd),
               dict(sel=None), dict(sel=odd), dict(ws=half), dict(q_heads=3), dict(q_heads=0), dict(type=2), dict(causal=2), dict(max_new=0),
               dict(max_kv=-1), dict(max_pages=0), dict(n_req=-1), dict(n_tokens=-1), dict(q_stride_token=4), dict(q_stride_head=-8),
               dict(n_select=0), dict(n_select=(1 << 20) + 1), dict(keep_first=-1), dict(keep_last=-1), dict(keep_first=2)):
        assert select(**kw) == E, kw
    assert select(n_req=0, q=None, sel=None) == 0 and select(n_tokens=0, q=None) == 0
    assert F.lib.fkv_page_select(ref(desc), None, g, g, g, g, g, g, g, g, 1 << 20, None) == E
    many = dict(n_tokens=200, max_new=100)      # (few rows need no scratch)
    assert select(ws=None, **many) == select(nws=2 * 200 * 16 * 4 - 1, **many) == F.FKV_ERR_SCRATCH_TOO_SMALL


def test_select_scratch(F):
    """A score a row, KV head and page, rows of 16 pages; none where all pages are selected, nor for few rows."""
    desc = F.fkv_page_desc(8, 16, 2, 64, 0)
    need = lambda **kw: F.lib.fkv_page_select_workspace(ref(desc), ref(select_desc(F, **{**dict(n_tokens=200, max_new=100), **kw})))     # noqa: E731
    assert need() == 2 * 200 * 16 * 4
    assert need(max_kv=300, max_pages=40) == 2 * 200 * 32 * 4
    assert need(n_select=4) == 0 and need(max_kv=32) == 0 and need(max_pages=2) == 0
    assert need(n_select=0) == 0 and F.lib.fkv_page_select_workspace(None, ref(select_desc(F))) == 0
    assert need(max_new=2) == 0 and need(max_new=32) == 0 and need(max_new=33) > 0
    assert need(max_new=1, max_kv=16 * 512, max_pages=512) == 0 and need(max_new=1, max_kv=16 * 513, max_pages=513) > 0
    assert need(max_new=1, n_req=128) == 0 and need(max_new=1, n_req=129) > 0
    wide = F.fkv_page_desc(8, 16, 65535, 64, 0)
    assert F.lib.fkv_page_select_workspace(ref(wide), ref(select_desc(F, q_heads=65535, n_tokens=1 << 30, max_kv=1 << 30,
                                                                      max_pages=1 << 26))) == (1 << 64) - 1


def test_select_of_too_many_rows(F):
    desc = F.fkv_page_desc(8, 16, 2, 64, 0)
    for kw in (dict(n_req=1 << 30), dict(n_req=1 << 20, max_new=1 << 20), dict(max_new=1 << 30)):
        t = select_desc(F, **{**dict(n_tokens=1 << 30), **kw})
        assert F.lib.fkv_page_select(ref(desc), ref(t), g, g, g, g, g, g, g, g, 1 << 40, None) == F.FKV_ERR_UNSUPPORTED, kw


def attend_desc(F, **kw):
    base = dict(n_req=2, n_tokens=4, max_new=2, max_kv=64, max_pages=4, q_stride_token=256, q_stride_head=64, o_stride_token=256,
                o_stride_head=64, q_heads=4, type=0, scale=0.125, softcap=0.0, causal=1, window=0, sinks=0)
    return F.fkv_attend_desc(**{**base, **kw})


def test_attend_selected_arguments(F):
    E = F.FKV_ERR_INVALID_ARG
    desc = F.fkv_page_desc(8, 16, 2, 64, 0)

    def attend(d=desc, ns=4, sel=g, kc=g, vc=g, sc=g, q=g, tab=g, kv=g, qs=g, slopes=None, prefix=None, first=None, out=g, lse=None,
               ws=g, nws=1 << 30, **kw):
        t = attend_desc(F, **kw)
        return F.lib.fkv_page_attend_selected(ref(d), ref(t), ns, sel, kc, vc, sc, q, tab, kv, qs, slopes, prefix, first, out, lse, ws,
                                              nws, None)

    for kw in (dict(d=None), dict(ns=0), dict(ns=-1), dict(ns=(1 << 20) + 1), dict(sel=None), dict(sel=odd), dict(kc=None), dict(vc=half),
               dict(sc=P(0x10004)), dict(q=None), dict(q=half), dict(out=None), dict(out=half), dict(tab=None), dict(kv=None), dict(qs=odd),
               dict(slopes=odd), dict(prefix=odd), dict(first=odd), dict(lse=odd), dict(ws=half), dict(q_heads=3), dict(q_heads=0),
               dict(type=2), dict(scale=float("nan")), dict(softcap=-1.0), dict(causal=2), dict(window=-1), dict(sinks=-1), dict(max_new=0),
               dict(max_kv=-1), dict(max_pages=0), dict(n_req=-1), dict(n_tokens=-1), dict(q_stride_token=4), dict(o_stride_head=-8)):
        assert attend(**kw) == E, kw
    assert attend(n_req=0, q=None, out=None) == 0 and attend(n_tokens=0, q=None) == 0
    for kw in (dict(n_req=1 << 30, max_new=1 << 30, q_heads=65534), dict(max_new=1 << 30, q_heads=65534), dict(n_req=1 << 30, q_heads=65534)):
        kw = {**dict(n_tokens=1 << 30), **kw}
        assert attend(**kw) == F.FKV_ERR_UNSUPPORTED, kw


def test_attend_selected_scratch(F):
    """A call that splits the lists says how much scratch it takes and refuses less."""
    desc = F.fkv_page_desc(4096, 64, 2, 64, 0)
    t = attend_desc(F, n_req=1, n_tokens=1, max_new=1, max_kv=32768, max_pages=512)
    need = F.lib.fkv_page_attend_selected_workspace(ref(desc), ref(t), 128)
    assert need > 0
    args = (ref(desc), ref(t), 128, g, g, g, g, g, g, g, g, None, None, None, g, None)
    assert F.lib.fkv_page_attend_selected(*args, None, 0, None) == F.FKV_ERR_SCRATCH_TOO_SMALL
    assert F.lib.fkv_page_attend_selected(*args, g, need - 1, None) == F.FKV_ERR_SCRATCH_TOO_SMALL
    assert F.lib.fkv_page_attend_selected_workspace(ref(desc), ref(t), 1) == 0
    assert F.lib.fkv_page_attend_selected_workspace(None, ref(t), 128) == 0
    assert F.lib.fkv_page_attend_selected_workspace(ref(desc), ref(t), 0) == 0


def test_tensors_of_another_device(F, monkeypatch):
    """A call runs on the current device's stream: tensors of another device are refused before it."""
    from types import SimpleNamespace
    monkeypatch.setattr(F, "_TORCH", SimpleNamespace(_C=SimpleNamespace(_cuda_getDevice=lambda: 1), cuda=SimpleNamespace(current_device=None)))
    t = [SimpleNamespace(get_device=lambda i=i: i) for i in range(2)]
    F._here(t[1], None, t[1])
    for bad in ((t[0],), (t[1], t[0]), (t[1], None, t[0])):
        with pytest.raises(ValueError):
            F._here(*bad)
