"""The paged 8-bit cache at the sizes where its calls take another form: many rows, many requests, long and wide rows."""
import math

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


def check_pool(fkv, pool, q, tables, kv, q_start, max_new, max_kv, bound=None, **opt):
    """fkv_page_attend of a CPU pool against 64 bits, within the reference's bounds."""
    k, v, scales = pool
    want, lse, off, loff = ref.attend(k, v, scales, q, tables, kv, q_start, q.shape[2] ** -0.5, **opt)
    dopt = {name: (x.cuda() if isinstance(x, torch.Tensor) else x) for name, x in opt.items()}
    got, glse = fkv.fkv_page_attend(fkv.Pages(k.cuda(), v.cuda(), scales.cuda()), q.cuda(), tables.cuda(), kv.cuda(),
                                    q_start.cuda(), max_new, max_kv, want_lse=True, **dopt)
    got, glse = got.cpu().double(), glse.cpu().double()
    u = 2.0 ** -11 if q.dtype == torch.float16 else 2.0 ** -8
    empty = lse == -math.inf
    assert torch.equal(glse == -math.inf, empty) and not got[empty].any()
    worst = ((got - want).abs() / (off + u * (want.abs() + off) + 2.0 ** -24)).max()
    assert worst <= 1, float(worst)
    assert ((glse - lse).abs()[~empty] <= loff[~empty]).all()


@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("kv,new", [(200, 1), (1000, 1), (3000, 2), (9000, 1), (200, 40), (9000, 40)])
def test_attend_values_near_the_end_of_bfloat16(fkv, codes, page, kv, new):
    """Values of 1e38: a sum of a few of them is beyond fp32, their weighted mean is not, however the keys are split."""
    n_pages = -(-kv // page)
    k, v, scales = random_pages(n_pages, page, 2, 64, codes, 3)
    v = (v.float().abs() + (20 if codes == INT8 else 16)).clamp(max=ref.LARGEST[codes]).to(codes)
    scales[:, :, 1] = 2.6e38 / ref.LARGEST[codes] * (0.3 + 0.7 * torch.rand((n_pages, 2)))
    q = torch.randn((new, 4, 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16) * 0.02
    tables = torch.randperm(n_pages, generator=torch.Generator().manual_seed(5)).int()[None]
    check_pool(fkv, (k, v, scales), q, tables, torch.tensor([kv], dtype=torch.int32), torch.tensor([0, new], dtype=torch.int32),
               new, kv)


@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("opt", [{}, dict(softcap=30.0), dict(slopes=True)])
@pytest.mark.parametrize("new", [1, 4, 300])
def test_attend_large_values_behind_a_mask(fkv, codes, rows, page, opt, new):
    """A row's result has the same bits of accuracy whatever the values that its mask hides: documents of values 2^25 times
    those of the next or more, and a last one, which the rows before it do not see yet."""
    kv, n_pages = 448, 448 // page
    k, v, scales = random_pages(n_pages, page, 2, 64, codes, 6)
    # (binary16 results of both kinds of documents have to stay within its range)
    large, small = (2.0 ** 11, 2.0 ** -14) if new == 300 and rows == torch.float16 else (2.0 ** 40, 2.0 ** -9)
    size = torch.full((448,), small)
    cut = 208 if page == 16 else 192                  # (inside a tile of 64 keys where a page may end there)
    size[:cut], size[384:] = large, large     # tokens of the first document, and of the last
    scales[:, :, 1] *= size[::page, None]
    tables = torch.arange(n_pages, dtype=torch.int32)[None]
    last = kv if new == 300 else 384 - 9              # (few rows: none of the last document's)
    pos = torch.arange(last - new, last)
    first = torch.where(pos < cut, 0, torch.where(pos < 384, cut, 384)).int()
    q = torch.randn((new, 4, 64), generator=torch.Generator().manual_seed(7)).to(rows) * 0.1
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = torch.tensor([0.001, 0.01, 0.02, 0.1])
    check_pool(fkv, (k, v, scales), q, tables, torch.tensor([last], dtype=torch.int32), torch.tensor([0, new], dtype=torch.int32),
               new, last, first=first, **opt)
    check_pool(fkv, (k, v, scales), q, tables, torch.tensor([last], dtype=torch.int32), torch.tensor([0, new], dtype=torch.int32),
               new, last, window=100, **opt)


@pytest.mark.parametrize("cap", [30.0, 128.0, 129.0, 1e3, 1e4, 1e6, 1e30])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("kv,new", [(200, 1), (3000, 1), (700, 40), (700, 130)])
def test_attend_large_caps(fkv, cap, slopes, kv, new):
    """cap * tanh(x / cap) for caps far above the scores, where tanh is nearly its argument.  The scores are bound to
    2^-21 of a cap of at most 128, and to 2^-20 of their own size for a larger one, beside the dot product's
    (d + 8) 2^-24 sum |q k|."""
    page, heads, group, d = 16, 2, 2, 64
    n_pages = -(-kv // page)
    k, v, scales = random_pages(n_pages, page, heads, d, INT8, 8)
    scales[:, :, 0] = 2.0 ** -5
    tables = torch.randperm(n_pages, generator=torch.Generator().manual_seed(9)).int()
    q = torch.randn((new, heads * group, d), generator=torch.Generator().manual_seed(10)).to(torch.float16)
    kk, vv = (t[tables.long()].transpose(0, 1).reshape(heads, -1, d)[:, :kv].repeat_interleave(group, 0) for t in ref.values(k, v, scales))
    x = torch.stack([q[:, h].double() @ kk[h].t() for h in range(4)]) * d ** -0.5          # [head][row][key]
    size = torch.stack([q[:, h].double().abs() @ kk[h].abs().t() for h in range(4)]) * d ** -0.5
    z = cap * torch.tanh(x / cap)
    off = size * (d + 8) * 2.0 ** -24 + z.abs() * 2.0 ** -20 + (cap * 2.0 ** -21 if cap <= 128 else 0.0)
    slope = torch.tensor([0.5, 0.1, 0.03, 0.002])
    pos, j = torch.arange(kv - new, kv), torch.arange(kv)
    far = (pos[:, None] - j).abs()
    if slopes:
        z = z - slope.double()[:, None, None] * far
        off = off + slope.double()[:, None, None] * far * 2.0 ** -21 + z.abs() * 2.0 ** -21
    z = torch.where(j <= pos[:, None], z, -math.inf)
    lse = z.logsumexp(2)
    w = torch.exp(z - lse[:, :, None])
    big = torch.where(w > 2.0 ** -30, off, 0.0).amax(2)
    assert big.max() < 0.02
    got, glse = fkv.fkv_page_attend(fkv.Pages(k.cuda(), v.cuda(), scales.cuda()), q.cuda(), tables[None].cuda(),
                                    dev([kv], torch.int32), dev([0, new], torch.int32), new, kv, softcap=cap,
                                    slopes=slope.cuda() if slopes else None, want_lse=True)
    err = (glse.cpu().double().t() - lse).abs()
    assert (err <= 2 * big + lse.abs() * 2.0 ** -20 + 2.0 ** -18).all(), float(err.max())
    out = (w @ vv).transpose(0, 1)
    most = (2.0 ** -11 + 4 * big.t()[:, :, None] + 2.0 ** -18) * (w @ vv.abs()).transpose(0, 1)
    assert ((got.cpu().double() - out).abs() <= most + 2.0 ** -11 * (out.abs() + most) + 2.0 ** -24).all()
