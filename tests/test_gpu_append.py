"""Rows rotated and written into the paged cache on the GPU: codes, scales, boxes and query rows against the fp32
operations that define them, bit for bit."""
import math

import numpy as np
import pytest
import torch

import pages_reference as pages
import select_reference as ref

pytestmark = pytest.mark.gpu

INT8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def bits(t):
    return t.detach().cpu().contiguous().view(torch.uint8)


def up(pool):
    return tuple(t.cuda() for t in pool)


def rows(n, heads, d, dtype, seed, special=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g)
    x[:, :, :2] *= 10
    if special and n:
        x[0, 0, 3], x[-1, -1, 5], x[n // 2, 0, 0] = math.inf, -math.inf, math.nan
    return x.to(dtype)


def state(page, heads, d, codes, lengths, seed):
    """(CPU pool, boxes as fp32, slots, positions, tables, n_pages): the pages hold the tokens before the call."""
    n_pages = sum(-(-(kv + new) // page) for kv, new in lengths) + 3
    slots, positions, tables = ref.slot_map(lengths, page, n_pages, seed)
    pool = ref.pool(n_pages, heads, page, d, codes, seed + 1)
    boxes = torch.zeros((n_pages, heads, 2, d))
    for (kv, _), t in zip(lengths, tables):
        for j in range(-(-kv // page)):
            boxes[t[j]] = ref.box_of(pool[0][t[j]], min(page, kv - j * page))
    return pool, boxes, slots, positions, tables, n_pages


def same(got, want, slots, page):
    """Codes of every token up to the last one written, and all scales: bit for bit."""
    k, v, scales = (t.cpu() for t in got)
    assert torch.equal(bits(scales), bits(want[2]))
    end = {}
    for i, n in pages.runs(slots, page):
        p, o = divmod(int(slots[i]), page)
        if 0 <= p < k.shape[0]:
            end[p] = o + n
    for p in range(k.shape[0]):
        n = end.get(p, page)
        assert torch.equal(bits(k[p][:, :n]), bits(want[0][p][:, :n])), p
        gv, wv = (t[p].view(torch.uint8).transpose(-1, -2).reshape(k.shape[1], page, -1) for t in (v, want[1]))
        assert torch.equal(gv[:, :n], wv[:, :n]), p


CASES = [
    # page, heads, q_heads, d, rot, pairs, codes, rows, (before, new) of each request
    (16, 1, 1, 16, 16, False, INT8, F16, [(0, 1)]),
    (16, 2, 6, 64, 64, False, INT8, F16, [(0, 16), (3, 1), (15, 1), (16, 2), (7, 40), (0, 5)]),
    (16, 3, 3, 80, 80, False, E4M3, BF16, [(1, 1), (2, 14), (0, 33), (5, 30)]),
    (48, 2, 14, 96, 32, True, INT8, BF16, [(0, 47), (47, 2), (13, 100), (1, 1)]),
    (64, 8, 9, 128, 128, False, E4M3, F16, [(0, 64), (63, 1), (10, 7), (0, 130), (61, 5)]),
    (64, 2, 5, 128, 64, False, INT8, BF16, [(0, 200), (0, 1), (30, 3)]),
    (256, 2, 2, 256, 256, True, INT8, F16, [(0, 300), (100, 90), (2, 1)]),
    (128, 1, 4, 48, 16, False, E4M3, F16, [(9, 120), (0, 128), (127, 3)]),
    (256, 1, 1, 112, 112, True, E4M3, BF16, [(9, 300), (0, 1)]),
    (64, 1, 17, 144, 96, False, INT8, F16, [(60, 70), (0, 1)]),
    (16, 4, 8, 64, 64, False, INT8, F16, [(5, 3)] * 400),
    (32, 2, 2, 32, 32, True, E4M3, BF16, [(31, 1)] * 1100),
    (64, 8, 8, 32, 32, False, INT8, F16, [(0, 5000), (70, 130)]),     # whole pages' worth a wave
    (256, 16, 1, 16, 16, True, INT8, BF16, [(250, 2500)]),
]


@pytest.mark.parametrize("page,heads,q_heads,d,rot,pairs,codes,kind,lengths", CASES)
@pytest.mark.parametrize("special", [False, True])
def test_append_matches_its_definition(fkv, page, heads, q_heads, d, rot, pairs, codes, kind, lengths, special):
    pool, boxes, slots, positions, _, n_pages = state(page, heads, d, codes, lengths, d + page)
    n = len(slots)
    k, v, q = rows(n, heads, d, kind, 1, special), rows(n, heads, d, kind, 2, special), rows(n, q_heads, d, kind, 3, special)
    tab = ref.table(int(positions.max()) + 1, rot)
    got, gbox = up(pool), boxes.to(codes).cuda()
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = fkv.fkv_page_append(got, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(positions).cuda(),
                              tab.cuda(), q=q.cuda(), pairs=pairs, boxes=gbox, n_bad=bad)
    torch.cuda.synchronize()
    ref.append(*pool, k, v, slots, positions, tab, pairs, boxes)
    same(got, pool, slots, page)
    assert torch.equal(gbox.cpu().float(), boxes)
    want = ref.turned(q, positions, tab, pairs).to(kind)
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=7.0), torch.nan_to_num(want, nan=7.0))
    assert int(bad) == 0


@pytest.mark.parametrize("codes,kind", [(INT8, F16), (E4M3, BF16)])
def test_append_without_rotation_is_store(fkv, codes, kind):
    page, heads, d, lengths = 32, 3, 96, [(0, 70), (31, 2), (5, 9)]
    pool, boxes, slots, positions, _, n_pages = state(page, heads, d, codes, lengths, 5)
    k, v, q = (rows(len(slots), heads, d, kind, s).cuda() for s in (1, 2, 3))
    one, two, gbox = up(pool), up(pool), boxes.to(codes).cuda()
    sl = torch.from_numpy(slots).cuda()
    fkv.fkv_page_store(one, k, v, sl)
    copied = fkv.fkv_page_append(two, k, v, sl, q=q, boxes=gbox)
    torch.cuda.synchronize()
    for a, b in zip(one, two):
        assert torch.equal(bits(a), bits(b))
    assert torch.equal(copied, q)
    ref.append(*pool, k.cpu(), v.cpu(), slots, boxes=boxes)
    assert torch.equal(gbox.cpu().float(), boxes)
    assert fkv.fkv_page_append(two, k, v, sl) is None


def test_append_of_streams_in_place_and_strided(fkv):
    """Rows [b][heads][t][d], slices of wider rows; query rows turned where they lie."""
    page, heads, group, d, lengths = 16, 2, 3, 64, [(0, 21), (30, 21)]
    pool, boxes, slots, positions, _, n_pages = state(page, heads, d, INT8, lengths, 9)
    wide = torch.randn((2, 30, heads * (group + 2), d + 8), generator=torch.Generator().manual_seed(4)).to(F16).cuda()
    part = wide[:, 3:24, :, :d].transpose(1, 2)
    q, k, v = part[:, :heads * group], part[:, heads * group:heads * (group + 1)], part[:, heads * (group + 1):]
    before = wide.clone()
    flat = lambda t: t.transpose(1, 2).reshape(-1, t.shape[1], d).cpu()   # noqa: E731
    fq, fk, fv = flat(q), flat(k), flat(v)
    tab = fkv.fkv_rotation_table(60, d)
    sl, ps = torch.from_numpy(slots).view(2, 21).cuda(), torch.from_numpy(positions).view(2, 21).cuda()
    got = up(pool)
    out = fkv.fkv_page_append(got, k, v, sl, ps, tab, q=q, q_out=q)
    torch.cuda.synchronize()
    assert out is q
    ref.append(*pool, fk, fv, slots, positions, tab.cpu())
    same(got, pool, slots, page)
    assert torch.equal(flat(q), ref.turned(fq, positions, tab.cpu(), False).to(F16))
    before[:, 3:24, :heads * group, :d] = wide[:, 3:24, :heads * group, :d]
    assert torch.equal(before, wide)      # nothing else was written


def test_append_of_rows_of_no_request_and_positions_outside(fkv):
    page, heads, d = 16, 2, 32
    pool = ref.pool(6, heads, page, d, INT8, 3)
    slots = np.array([0, 1, 2, -1, -1, 5 * 16, 6 * 16 + 1, -1], np.int64)
    positions = np.array([0, 40, -3, -1, 7, 9, 3, 99], np.int32)
    k, v, q = (rows(8, heads, d, F16, s) for s in (1, 2, 3))
    tab = ref.table(10, d)
    got, bad = up(pool), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((8, heads, d), 7.0, dtype=F16, device="cuda")
    fkv.fkv_page_append(got, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(positions).cuda(), tab.cuda(),
                        q=q.cuda(), q_out=out, n_bad=bad)
    torch.cuda.synchronize()
    ref.append(*pool, k, v, slots, positions, tab)
    same(got, pool, slots, page)
    want = ref.turned(q, positions, tab, False).to(F16)
    want[3] = 7.0
    assert torch.equal(out.cpu(), want)
    assert int(bad) == 4       # 40, -3 with a slot, a slot beyond the pool, 99


def test_append_of_nothing(fkv):
    pool = up(ref.pool(2, 1, 16, 16, INT8, 0))
    before = [t.clone() for t in pool]
    none = torch.zeros((0, 1, 16), dtype=F16, device="cuda")
    out = fkv.fkv_page_append(pool, none, none, torch.zeros(0, dtype=torch.int64, device="cuda"),
                              torch.zeros(0, dtype=torch.int32, device="cuda"), fkv.fkv_rotation_table(4, 16), q=none,
                              boxes=fkv.fkv_boxes(pool))
    assert out.shape == (0, 1, 16)
    for a, b in zip(pool, before):
        assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("codes", [INT8, E4M3])
def test_append_token_by_token(fkv, codes):
    """Boxes after appending one token at a time are those of the codes that the pages then hold."""
    page, heads, d = 16, 2, 48
    pages_, g = fkv.fkv_pages(5, page, heads, d, codes), torch.Generator().manual_seed(8)
    boxes, tab = fkv.fkv_boxes(pages_), fkv.fkv_rotation_table(64, d)
    for t in range(37):
        x = (torch.randn((2, 1, heads, d), generator=g) * (0.1 + 0.3 * t)).to(BF16).cuda()
        fkv.fkv_page_append(pages_, x[0], x[1], torch.tensor([t + page], device="cuda"),
                            torch.tensor([t], dtype=torch.int32, device="cuda"), tab, boxes=boxes)
    torch.cuda.synchronize()
    k = pages_.k.cpu()
    for p, n in ((1, 16), (2, 16), (3, 5)):
        assert torch.equal(boxes[p].cpu().float(), ref.box_of(k[p], n))


def test_append_of_rows_near_the_types_ends(fkv):
    """bfloat16 rows whose rotation passes fp32's end, and rows far below what a scale can hold."""
    page, heads, d = 16, 1, 16
    x = torch.zeros((4, 1, d))
    x[0] = 3e38
    x[1] = -2e38
    x[2], x[3] = 2.0 ** -100, 1e-38
    for at, codes in (([0, 1], INT8), ([2, 3], E4M3), ([0, 3], E4M3)):
        k = x[at].to(BF16)
        pool = ref.pool(2, heads, page, d, codes, 3)
        slots, positions, tab = np.array([16, 17], np.int64), np.array([5, 6], np.int32), ref.table(8, d)
        got, boxes = up(pool), torch.zeros((2, heads, 2, d))
        gbox = boxes.to(codes).cuda()
        fkv.fkv_page_append(got, k.cuda(), k.cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(positions).cuda(), tab.cuda(),
                            boxes=gbox)
        torch.cuda.synchronize()
        ref.append(*pool, k, k, slots, positions, tab, boxes=boxes)
        same(got, pool, slots, page)
        assert torch.equal(gbox.cpu().float(), boxes)
