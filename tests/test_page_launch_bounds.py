"""CPU tests of the paged calls' launch shapes at the ends of their arguments' ranges: each call returns, with an error
where the sizes are beyond what can be, before a device is touched."""
import ctypes
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# in a process of its own: a division by zero in the library would end the one it is in
ATTEND = """
import ctypes, sys
sys.path.insert(0, %r)
from paper_2607_07144_amd import fkv as F
ref = ctypes.byref
desc = F.fkv_page_desc(8, 16, 1, 64, 0)
for n_req, n_tokens, max_new, q_heads, max_kv in ((1 << 30, 1 << 30, 1 << 30, 32768, 64), (1 << 26, 4, 1 << 30, 32768, 1 << 30),
                                                  (1, 4, 1 << 30, 65535, 1 << 30), (1 << 30, 1, 1, 1, 1 << 30), (7, 1, 1 << 30, 1, 64)):
    t = F.fkv_attend_desc(n_req, n_tokens, max_new, max_kv, 1 << 26, 64, 64, 64, 64, q_heads, 0, 0.125, 0.0, 1, 0, 0)
    print(F.lib.fkv_page_attend_workspace(ref(desc), ref(t)), flush=True)
""" % ROOT


def test_attend_shapes_of_any_sizes():
    p = subprocess.run([sys.executable, "-c", ATTEND], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, (p.returncode, p.stdout, p.stderr[-500:])
    assert len(p.stdout.split()) == 5


def test_attend_join_of_too_many_rows_is_refused_at_once():
    from paper_2607_07144_amd import fkv as F
    ref, g = ctypes.byref, ctypes.c_void_p(0x10000)
    desc = F.fkv_page_desc(8, 16, 1, 64, 0)
    t = F.fkv_attend_desc(1 << 30, 4, 16, 1 << 20, 1 << 26, 64, 64, 64, 64, 1, 0, 0.125, 0.0, 1, 0, 0)
    need = F.lib.fkv_page_attend_workspace(ref(desc), ref(t))
    assert F.lib.fkv_page_attend(ref(desc), ref(t), g, g, g, g, g, g, g, None, None, None, g, None, g, need,
                                 None) == F.FKV_ERR_UNSUPPORTED


def test_store_and_load_of_too_many_rows():
    from paper_2607_07144_amd import fkv as F
    ref, g = ctypes.byref, ctypes.c_void_p(0x10000)
    rows = F.fkv_row_desc(1 << 62, 0, 128, 64, 0)
    for heads in (4, 16, 3):
        desc = F.fkv_page_desc(8, 16, heads, 64, 0)
        for n in (1 << 62, 1 << 60, (1 << 63) - 1, (1 << 40) + 1):
            assert F.lib.fkv_page_store(ref(desc), ref(rows), ref(rows), g, g, n, g, g, g, g, None, None) == F.FKV_ERR_INVALID_ARG
            assert F.lib.fkv_page_load(ref(desc), g, g, g, n, g, ref(rows), ref(rows), g, g, None) == F.FKV_ERR_INVALID_ARG
