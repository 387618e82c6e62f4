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
