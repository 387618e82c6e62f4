"""The paged 8-bit cache at the sizes where its calls take another form: many rows, many requests, long and wide rows."""
import math

import numpy as np
import pytest
import torch

import pages_reference as ref
from test_gpu_pages import E4M3, INT8, _slopes, bits, check_attend, dev, make_pool, make_rows, slot_map

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


def check_pool(fkv, pool, q, tables, kv, q_start, max_new, max_kv, **opt):
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


# ---------------------------------------------------------------- forms that the sizes of a call choose

MANY = [
    # page, heads, d, code type, row type, (before, new) of each request: more than 32,768 rows x heads
    (16, 16, 32, INT8, torch.float16, [(0, 1000), (5, 333), (15, 1), (3, 9), (0, 16), (16, 747)]),
    (48, 16, 48, E4M3, torch.bfloat16, [(47, 2), (1, 46), (0, 48), (13, 1999)] + [(7, 3)] * 20),
    (64, 24, 80, INT8, torch.bfloat16, [(0, 1301), (63, 1), (20, 60), (0, 5)]),
    (256, 24, 16, INT8, torch.float16, [(0, 700), (100, 90), (255, 2), (3, 600), (30, 70)]),
    (128, 24, 128, E4M3, torch.float16, [(9, 120), (0, 128), (127, 3), (0, 1150)]),
    (16, 40, 16, E4M3, torch.float16, [(k % 16, 1) for k in range(823)]),
    (32, 12, 64, INT8, torch.bfloat16, [(30, 5)] * 560),
]


@pytest.mark.parametrize("page,heads,d,codes,rows,lengths", MANY)
@pytest.mark.parametrize("special", [False, True])
def test_store_of_many_rows(fkv, page, heads, d, codes, rows, lengths, special):
    """A wave looks at a page's worth of rows: several runs in it, runs that begin before and end after it, and rows
    of no page between them."""
    n_pages = sum(-(-(kv + new) // page) for kv, new in lengths) + 2
    slots, _ = slot_map(lengths, page, n_pages, d)
    n = len(slots)
    gaps = np.flatnonzero(np.diff(slots) != 1) + 1                         # between requests, and pages apart
    sent = np.insert(slots, [gaps[0], gaps[0], gaps[-1], n], [-1, n_pages * page + 3, -2 ** 40, n_pages * page])
    assert len(sent) * heads > 32768 and len(sent) % min(page, 64)
    k, v, scales = random_pages(n_pages, page, heads, d, codes, 11)
    rk, rv = make_rows(len(sent), heads, d, rows, 12, special), make_rows(len(sent), heads, d, rows, 13, special)
    pages = fkv.Pages(k.cuda(), v.cuda(), scales.cuda())
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    fkv.fkv_page_store(pages, rk.cuda(), rv.cuda(), dev(sent), n_bad=bad)
    torch.cuda.synchronize()
    assert int(bad) == 2
    was = k.clone()
    ref.store(k, v, scales, rk, rv, sent)
    seen = torch.zeros((n_pages, page), dtype=torch.bool)
    for i, m in ref.runs(slots, page):
        p, o = divmod(int(slots[i]), page)
        seen[p, :o + m] = True
    assert torch.equal(bits(pages.scales), bits(scales))
    valid = seen[:, None, :, None]
    for got, want in ((pages.k.cpu(), k), (pages.v.cpu(), v)):
        got, want = (x.view(torch.uint8) if x.dim() == 4 else x.view(torch.uint8).transpose(-1, -2).reshape(k.shape) for x in (got, want))
        assert torch.equal(torch.where(valid, got, 0), torch.where(valid, want, 0))
    untouched = ~seen.any(1)
    assert untouched.any() and torch.equal(bits(pages.k)[untouched], bits(was)[untouched])


@pytest.mark.parametrize("page,heads,d,codes", [(16, 16, 64, INT8), (48, 24, 80, E4M3), (64, 16, 128, INT8), (256, 40, 16, E4M3),
                                               (32, 17, 256, INT8)])
@pytest.mark.parametrize("rows", [torch.float16, torch.bfloat16])
def test_load_of_many_rows(fkv, page, heads, d, codes, rows):
    """64 rows a wave: contexts in order from any offset, and rows in no order with some of no page."""
    n_pages = -(-2200 // page)
    pool = random_pages(n_pages, page, heads, d, codes, 14)
    rng = np.random.default_rng(15)
    whole = (rng.permutation(n_pages)[:, None] * page + np.arange(page)).reshape(-1)
    mixed = rng.integers(-2, n_pages * page + 2, 2103)
    for slots in (whole[7:2190], mixed):
        assert len(slots) * heads > 32768 and len(slots) % 64
        check_load(fkv, pool, slots, rows)
    # and head-major streams, the second of K only
    pages = fkv.Pages(*(t.cuda() for t in pool))
    slots = dev(whole[3:3 + 3 * 711].reshape(3, 711))
    x = torch.empty((2, 3, heads, 711, d), dtype=rows, device="cuda")
    fkv.fkv_page_load(pages, slots, k=x[0], v=x[1])
    k, v = fkv.fkv_page_load(pages, slots.view(-1), rows)
    assert torch.equal(x[0].transpose(1, 2).reshape(k.shape), k) and torch.equal(x[1].transpose(1, 2).reshape(v.shape), v)
    only = torch.zeros_like(x[0])
    fkv.fkv_page_load(pages, slots, k=only)
    assert torch.equal(only, x[0])


def check_sample(fkv, lengths, new, page, heads, group, d, codes, rows, seed, most=40, **opt):
    """A causal call checked at some of its rows, each taken as a request of one row that ends at its position."""
    k, v, scales, tables = make_pool(lengths, page, heads, d, codes, seed)
    n = sum(new)
    q = torch.randn((n, heads * group, d), generator=torch.Generator().manual_seed(seed + 1)).to(rows)
    start = np.concatenate(([0], np.cumsum(new)))
    got, glse = fkv.fkv_page_attend(fkv.Pages(k.cuda(), v.cuda(), scales.cuda()), q.cuda(), tables.cuda(), dev(lengths, torch.int32),
                                    dev(start, torch.int32), max(new), max(lengths), want_lse=True,
                                    **{name: (x.cuda() if isinstance(x, torch.Tensor) else x) for name, x in opt.items()})
    got, glse = got.cpu().double(), glse.cpu().double()
    assert got.isfinite().all()
    rng = np.random.default_rng(seed)
    pick = np.unique(np.concatenate((start[:-1], start[1:] - 1, rng.integers(0, n, most))))      # first and last ones too
    r = np.searchsorted(start, pick, side="right") - 1
    kv = np.maximum(np.array(lengths)[r] - np.array(new)[r] + pick - start[r] + 1, 0)
    if codes == E4M3:      # a product with a NaN code that no row sees would be one
        for c in (k, v):
            b = c.view(torch.uint8)
            b[b == 0x7f] = 0
    want, lse, off, loff = ref.attend(k, v, torch.nan_to_num(scales), q[pick], tables[r], torch.from_numpy(kv),
                                      np.arange(len(pick) + 1), d ** -0.5, **opt)
    u = 2.0 ** -11 if rows == torch.float16 else 2.0 ** -8
    empty = lse == -math.inf
    assert torch.equal(glse[pick] == -math.inf, empty) and not got[pick][empty].any()
    worst = ((got[pick] - want).abs() / (off + u * (want.abs() + off) + 2.0 ** -24)).max()
    assert worst <= 1, float(worst)
    assert ((glse[pick] - lse).abs()[~empty] <= loff[~empty]).all()


@pytest.mark.parametrize("opt", [{}, dict(softcap=30.0), dict(slopes=True), dict(softcap=500.0, slopes=True), dict(window=150, sinks=5)])
@pytest.mark.parametrize("page", [48, 64])
@pytest.mark.parametrize("d", [80, 96, 112, 128])
@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16)])
def test_attend_blocks_of_256_rows(fkv, codes, rows, d, page, opt):
    """At least 4096 rows of a KV head, even requests, 64 < d <= 128: eight waves a block, the last block part full; the
    keys in one piece, and (fewer rows of more keys) in two or more that are joined."""
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = _slopes(32)
    for lengths, new in (([300, 131], [130, 131]), ([1100], [131])):
        assert max(new) * 32 >= 4096 and 4 * sum(new) >= 3 * len(new) * max(new) and (max(new) * 32) % 256
        check_sample(fkv, lengths, new, page, 1, 32, d, codes, rows, d + page, most=8, **opt)


@pytest.mark.parametrize("opt", [{}, dict(softcap=30.0, slopes=True), dict(softcap=500.0), dict(window=70, sinks=3)])
@pytest.mark.parametrize("d,page", [(144, 16), (256, 64), (192, 256)])
@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16)])
def test_attend_few_rows_of_more_than_128_channels(fkv, codes, rows, d, page, opt):
    """At most 1024 keys: a block a head; more: the line of tiles, joined by a block a row; many rows: 64-key tiles."""
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = _slopes(8)
    check_attend(fkv, [1000, 17, 0, 260], [1, 1, 1, 1], page, 2, 4, d, codes, rows, seed=d, **opt)
    check_attend(fkv, [700, 64], [2, 2], page, 1, 8, d, codes, rows, seed=d + 1, **opt)
    check_attend(fkv, [9000, 40], [1, 1], page, 1, 8, d, codes, rows, seed=d + 2, **opt)
    check_sample(fkv, [5000], [40], page, 1, 8, d, codes, rows, d + 3, most=4, **opt)


@pytest.mark.parametrize("codes,rows", [(INT8, torch.bfloat16), (E4M3, torch.float16)])
def test_attend_of_more_requests_than_a_block_has_threads(fkv, codes, rows):
    """The line of tiles of 257 and 700 requests, long ones first, among and last, some empty and some without rows."""
    for n in (257, 700):
        rng = np.random.default_rng(n)
        lengths = rng.integers(0, 200, n)
        lengths[[0, n // 2, n - 1]] = 1500, 2100, 1100
        new = (rng.random(n) < 0.8).astype(int)
        new[[0, n // 2, n - 1]] = 1
        check_attend(fkv, lengths.tolist(), new.tolist(), 16, 2, 4, 32, codes, rows, seed=n)


@pytest.mark.parametrize("n", [64, 65, 90])
def test_attend_prompts_of_more_than_64_requests(fkv, n):
    """Up to 64 requests go out by length, more in order; both with lengths alike, empty ones and none of the rows."""
    rng = np.random.default_rng(n)
    lengths = rng.integers(0, 150, n)
    lengths[5:12] = 77
    new = np.minimum(rng.integers(0, 31, n), lengths)
    new[3], lengths[3] = 30, 400
    check_attend(fkv, lengths.tolist(), new.tolist(), 32, 1, 2, 32, INT8, torch.float16, seed=n)


@pytest.mark.parametrize("codes", [INT8, E4M3])
def test_attend_one_head_of_many_tiles(fkv, codes):
    """A head of 1600 tiles in more pieces than any other test's, the join taking several rounds of its splits."""
    check_sample(fkv, [102_400 - 7], [3], 256, 1, 2, 64, codes, torch.float16, 21, most=1)
