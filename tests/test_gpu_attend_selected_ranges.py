"""Attention to lists at the ends of the rows' and scales' ranges, of few items and of so many that a wave has one: against
64 bits, with the bounds of select_reference.py."""
import math

import pytest
import torch

import pages_reference as pages
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


@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("page,group,d", [(64, 3, 128), (64, 8, 64), (16, 4, 80)])
@pytest.mark.parametrize("lengths", [FEW, MANY])
@pytest.mark.parametrize("how", [{}, dict(slopes=0.01), dict(softcap=1e36)])
def test_keys_near_the_types_ends(fkv, codes, page, group, d, lengths, how):
    """Keys of up to 2^117 and binary16 rows: scores are finite and so far apart that a row's best key has all the weight."""
    heads, n = 16, 4
    pool, tables, kv, starts, q, selected = inputs(page, heads, group, d, codes, F16, lengths, n, d + page)
    pool[2][:, :, 0] *= 2.0 ** 111
    q = torch.where(q.abs() < 2.0 ** -5, 2.0 ** -5, q).to(F16)
    got, lse = call(fkv, pool, tables, kv, starts, q, selected, lengths, scale=2.0 ** -3,
                    **{k: torch.full((heads * group,), x, device="cuda") if k == "slopes" else x for k, x in how.items()})
    assert torch.isfinite(got).all()
    want, top, err, sure = best(pool, tables, kv, starts, q, selected, 2.0 ** -3)
    # the best key is taken where the next is further off than both scores' errors, (d + 8) 2^-24 of the sum of 255 units of a
    # scale; a cap keeps their order and takes t^2 / 3 of them, less than 2^-13 of scores of up to 0.019 of it
    assert sure.float().mean() > 0.9
    half = torch.finfo(F16).eps / 2
    # (a weight of 1 times its value scale is rounded to 11 bits)
    assert ((got - want).abs() <= (half + 2.0 ** -11 + 2.0 ** -18) * want.abs() + 383 * 2.0 ** -19 * pool[2][:, :, 1].max() + 2.0 ** -25)[sure].all()
    assert top.max() < 1.9e34 and ((lse - top).abs() <= err + top.abs() * 2.0 ** -13)[sure].all()


def best(pool, tables, kv, starts, q, selected, scale, gap=2.0 ** 20):
    """The value row of each row's best key, its score and that one's error, and whether the next one is far enough below."""
    n_pages, heads, page, d = pool[0].shape
    kk, vv = pages.values(*pool)
    n, q_heads, _ = q.shape
    group = q_heads // heads
    want, sure = torch.zeros((n, q_heads, d), dtype=torch.float64), torch.zeros((n, q_heads), dtype=torch.bool)
    top, off = torch.zeros((2, n, q_heads), dtype=torch.float64)
    for r in range(len(kv)):
        b, e = int(starts[r]), int(starts[r + 1])
        for i in range(b, e):
            pos = int(kv[r]) - (e - b) + (i - b)
            for h in range(heads):
                column = selected[i, h].long()
                column = column[column >= 0]
                ids, j = tables[r, column].long(), (column[:, None] * page + torch.arange(page)).flatten()
                see = j <= pos
                ks, vs, sc = kk[ids, h].reshape(-1, d)[see], vv[ids, h].reshape(-1, d)[see], pool[2][ids, h, 0].double().repeat_interleave(page)[see]
                for hq in range(h * group, (h + 1) * group):
                    x = q[i, hq].double()
                    z = ks @ x * scale
                    err = sc * 255 * x.abs().sum() * scale * (d + 8) * 2.0 ** -24 + z.abs() * 2.0 ** -20
                    o = z.argsort(descending=True)
                    want[i, hq], top[i, hq], off[i, hq] = vs[o[0]], z[o[0]], err[o[0]]
                    sure[i, hq] = len(o) == 1 or bool((z[o[0]] - z[o[1:]] > err[o[0]] + err[o[1:]] + gap).all())
    return want, top, off, sure


@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("page,group,d,tiles", [(64, 1, 16, 16384), (64, 5, 80, 700), (32, 2, 128, 3000)])
def test_long_lists_of_many_items(fkv, codes, page, group, d, tiles):
    """A wave over thousands of tiles, the same pages again and again: what int8 codes are shifted by leaves no errors that grow
    with the list.  Most value codes are 0, so that the weights' own rounding takes little."""
    heads, kv, n = 16, 64, 128
    g = torch.Generator().manual_seed(d)
    k, v, scales = ref.pool(kv // page, heads, page, d, codes, 1)
    v = (torch.rand(v.shape, generator=g) < 1 / 32).float().to(codes)
    scales[:, :, 1] = torch.linspace(1.5, 1.0, kv // page)[:, None]
    tables = torch.arange(kv // page, dtype=torch.int32)[None]
    q = torch.randn((n, heads * group, d), generator=g).half()
    entries = tiles * 64 // page
    selected = (torch.arange(entries, dtype=torch.int32) % (kv // page)).expand(n, heads, entries).contiguous()
    got, lse = call(fkv, (k, v, scales), tables, torch.tensor([kv], dtype=torch.int32), torch.tensor([0, n], dtype=torch.int32), q,
                    selected, [(kv, n)], causal=False)
    kk, vv = (t.transpose(0, 1).reshape(heads, kv, d) for t in pages.values(k, v, scales))
    rows = q.double().reshape(n, heads, group, d).transpose(0, 1).reshape(heads, n * group, d)
    as_rows = lambda t: t.reshape(heads, n, group, -1).transpose(0, 1).reshape(n, heads * group, -1)     # noqa: E731
    z = torch.stack([a @ b.T for a, b in zip(rows, kk)]) * d ** -0.5
    w = torch.softmax(z, -1)
    of_key = scales.double().repeat_interleave(page, 0).transpose(0, 1)       # [heads][kv][2]
    want, unit = as_rows(w @ vv), as_rows(w @ of_key[..., 1:])
    # A score: d + 8 roundings of sums of 255 units of a scale, and its exponential's.  A weight: 11 bits.  The values' sums: 64
    # roundings a tile of the sums so far, and of what one tile adds and its 128 take off, 383 units of its weights at most.
    big = as_rows(rows.abs().sum(-1, keepdim=True) * of_key[:, :, :1].amax(1, keepdim=True) * 255 * d ** -0.5 * (d + 8) * 2.0 ** -24
                  + z.abs().amax(-1, keepdim=True) * 2.0 ** -21)
    assert big.max() < 0.05
    room = (2.0 ** -11 + 4 * big + tiles * 64 * 2.0 ** -24) * want + (64 + 16) * 2.0 ** -24 * 383 * unit
    assert ((got - want).abs() <= room + torch.finfo(F16).eps / 2 * (want + room) + 2.0 ** -25).all(), float(((got - want).abs() / room).max())
    exact = as_rows(torch.logsumexp(z, -1)[..., None] + math.log(tiles * 64 / kv))
    assert ((lse[..., None] - exact).abs() <= 2 * big + (tiles * 64 + 64) * 2.0 ** -24 + exact.abs() * 2.0 ** -20).all()


@pytest.mark.parametrize("entries", [70, 512, 4096])
@pytest.mark.parametrize("n_req,max_new", [(1 << 20, 4096), (512, 2048), (4, 1)])
def test_split_lists_of_few_rows_in_many_places(fkv, entries, n_req, max_new):
    """Long lists of four rows of four requests, among many requests without rows and with a loose bound on a request's rows: the
    same as of those four alone."""
    page, heads, group, d, width = 64, 2, 2, 64, 8
    pool = up(ref.pool(40, heads, page, d, INT8, 1))
    g = torch.Generator().manual_seed(entries)
    q = torch.randn((4, heads * group, d), generator=g).half().cuda()
    tables = torch.randint(0, 40, (n_req, width), generator=g, dtype=torch.int32)
    kv, new = torch.full((n_req,), 17, dtype=torch.int32), torch.zeros(n_req, dtype=torch.int64)
    at = [n_req * i // 4 for i in range(4)]
    kv[at], new[at] = torch.tensor([512, 300, 77, 1], dtype=torch.int32), 1
    starts = torch.cat((torch.zeros(1, dtype=torch.int64), new.cumsum(0))).int()
    selected = torch.randint(-1, width, (4, heads, entries), generator=g, dtype=torch.int32).cuda()
    got = fkv.fkv_page_attend_selected(pool, q, tables.cuda(), kv.cuda(), starts.cuda(), selected, max_new, 512, want_lse=True)
    alone = fkv.fkv_page_attend_selected(pool, q, tables[at].cuda(), kv[at].cuda(), torch.arange(5, dtype=torch.int32, device="cuda"), selected,
                                         1, 512, want_lse=True)
    assert all(torch.equal(a, b) for a, b in zip(got, alone))
    want, wlse, off, loff = ref.attend_selected(*(t.cpu() for t in pool), q.cpu(), tables[at], kv[at], torch.arange(5), selected.cpu(), d ** -0.5)
    assert ((got[0].cpu().double() - want).abs() <= off + torch.finfo(F16).eps / 2 * (want.abs() + off) + 2.0 ** -25).all()
    assert ((got[1].cpu().double() - wlse).abs() <= loff).all()
