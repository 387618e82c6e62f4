"""The paged 8-bit cache at the sizes where its calls take another form: many rows, many requests, long and wide rows."""
import numpy as np
import pytest
import torch

import pages_reference as ref
from test_gpu_pages import E4M3, INT8, dev

pytestmark = pytest.mark.gpu


def random_pages(n_pages, page, heads, d, codes, seed):
    g = torch.Generator().manual_seed(seed)
    k = ref.to_codes(torch.randn((n_pages, heads, page, d), generator=g) * 40, codes)
    v = ref.to_codes(torch.randn((n_pages, heads, page // 16, d, 16), generator=g) * 40, codes)
    scales = torch.rand((n_pages, heads, 2), generator=g) * 2.0 ** -4 + 2.0 ** -9
    return k, v, scales


def check_load(fkv, pool, slots, rows):
    """fkv_page_load of a CPU pool against code * scale in 64 bits: one rounding to the row type, one to fp32 before it."""
    k, v, scales = pool
    n_pages, heads, page, d = k.shape
    gk, gv = fkv.fkv_page_load(fkv.Pages(k.cuda(), v.cuda(), scales.cuda()), dev(slots, torch.int64), rows)
    ok = torch.from_numpy((slots >= 0) & (slots < n_pages * page))
    at = np.clip(slots, 0, n_pages * page - 1)
    p, o = torch.from_numpy(at // page), torch.from_numpy(at % page)
    u = 2.0 ** -11 if rows == torch.float16 else 2.0 ** -8
    for got, every in zip((gk, gv), ref.values(k, v, scales)):
        want = torch.where(ok[:, None, None], every[p, :, o], 0.0)
        assert ((got.cpu().double() - want).abs() <= want.abs() * (u + 2.0 ** -23) + 2.0 ** -25).all()


@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16)])
def test_load_of_many_rows_in_no_order(fkv, codes, rows):
    """More than 32,768 rows x heads, so that a wave has 64 rows, each a segment of its own or nearly."""
    pool = random_pages(135, 16, 16, 32, codes, 1)
    slots = np.random.default_rng(2).permutation(135 * 16)[:2101]
    slots[[5, 64, 1000]] = -1, 135 * 16, -7
    assert 2101 * 16 > 32768
    check_load(fkv, pool, slots, rows)


@pytest.mark.parametrize("codes", [INT8, E4M3])
def test_the_largest_bfloat16_rows_come_back(fkv, codes):
    """Pages whose largest element is the largest bfloat16 number, its negative or the one below it: code * scale is
    finite for every code, and so is what is read back, beside zeros and small elements too."""
    top = torch.finfo(torch.bfloat16).max
    below = torch.tensor([0x7f7e], dtype=torch.int16).view(torch.bfloat16).float().item()
    x = torch.zeros((64, 2, 16), dtype=torch.bfloat16)
    x[0, :, 0], x[1, :, 1], x[2, :, 2:9], x[3, 0] = top, -top, 1.0, torch.linspace(-top, top, 16).bfloat16()
    x[16, :, 3], x[17] = below, 7.0e37
    x[32, :, 3], x[33] = -top, -1.7e38
    x[48:] = top
    for n in (64, 1):      # the second with a row a page
        pages = fkv.fkv_pages(4, 16, 2, 16, codes)
        slots = torch.arange(64) if n == 64 else torch.arange(4) * 16
        rows = x[slots]
        fkv.fkv_page_store(pages, rows.cuda(), rows.flip(2).contiguous().cuda(), slots.cuda())
        for got, every in zip(fkv.fkv_page_load(pages, slots.cuda(), torch.bfloat16), ref.values(*(t.cpu() for t in pages))):
            want = every[slots // 16, :, slots % 16]
            assert got.isfinite().all()
            assert ((got.cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -23)).all()
