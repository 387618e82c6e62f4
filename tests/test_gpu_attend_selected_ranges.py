"""Attention to lists at the ends of the rows' and scales' ranges, of few items and of so many that a wave has one: against
64 bits, with the bounds of select_reference.py."""
import pytest
import torch

import select_reference as ref
from test_gpu_select import lists, requests, up

pytestmark = pytest.mark.gpu

INT8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def inputs(page, heads, group, d, codes, kind, lengths, n_selected, seed):
    n_pages = sum(-(-kv // page) for kv, _ in lengths) + 3
    pool = ref.pool(n_pages, heads, page, d, codes, seed + 1)
    tables, kv, starts = requests(lengths, page, n_pages, seed)
    n = int(starts[-1])
    q = torch.randn((n, heads * group, d), generator=torch.Generator().manual_seed(seed + 2)).to(kind)
    selected = lists(lengths, page, heads, n_selected, True, seed + 3, "picked").reshape(n, heads, n_selected)
    return pool, tables, kv, starts, q, selected


def call(fkv, pool, tables, kv, starts, q, selected, lengths, **how):
    out, lse = fkv.fkv_page_attend_selected(up(pool), q.cuda(), tables.cuda(), kv.cuda(), starts.cuda(), selected.cuda(),
                                            max(n for _, n in lengths), max(t for t, _ in lengths), want_lse=True, **how)
    torch.cuda.synchronize()
    return out.cpu().double(), lse.cpu().double()


FEW, MANY = [(200, 3), (130, 1)], [(330, 128), (70, 3)]


@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("page,group,d", [(64, 3, 128), (64, 8, 64), (16, 4, 80), (48, 5, 256)])
@pytest.mark.parametrize("lengths", [FEW, MANY])
@pytest.mark.parametrize("power", [-120, 104, 120, 125])
def test_bfloat16_rows_near_the_types_ends(fkv, codes, page, group, d, lengths, power):
    """Rows of 2^power and keys of 2^-power: scores are those of rows of 1."""
    heads, n = 16, 4
    pool, tables, kv, starts, q, selected = inputs(page, heads, group, d, codes, BF16, lengths, n, d + page)
    q = (q.clamp(-3.5, 3.5).float() * 2.0 ** power).to(BF16)
    pool[2][:, :, 0] *= 2.0 ** -power
    assert torch.isfinite(q).all() and (pool[2] > 0).all()
    got, lse = call(fkv, pool, tables, kv, starts, q, selected, lengths)
    tiles = -(-n * (page // 16) // 4)
    items = len(q) * heads if len(lengths) * max(m for _, m in lengths) >= 2 * len(q) else len(lengths) * max(m for _, m in lengths) * heads
    shifted = tiles if codes == INT8 and (items >= 2048 or tiles == 1) else 0
    want, wlse, off, loff = ref.attend_selected(*pool, q, tables, kv, starts, selected, d ** -0.5, shifted=shifted)
    half = torch.finfo(BF16).eps / 2
    assert ((lse - wlse).abs() <= loff).all()
    assert ((got - want).abs() <= off + half * (want.abs() + off) + 2.0 ** -25).all()
