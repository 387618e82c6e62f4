"""Boxes of pages that are written over from their middle, as by a request whose drafted tokens were refused: those of the
tokens that the page then holds, whatever it held before."""
import numpy as np
import pytest
import torch

import select_reference as ref
from test_gpu_append import bits, rows, same, up

pytestmark = pytest.mark.gpu

INT8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def check(fkv, page, heads, d, codes, kind, rot, pairs, writes, seed=0):
    """writes: (first token, tokens, factor of the rows, a row with infinities and a NaN) of one request, one after another."""
    n_tok = max(at + n for at, n, _, _ in writes)
    n_pages = -(-n_tok // page) + 2
    _, _, ((*ids,),) = ref.slot_map([(n_tok, 0)], page, n_pages, seed)
    pool = ref.pool(n_pages, heads, page, d, codes, seed + 1)
    got, boxes = up(pool), torch.zeros((n_pages, heads, 2, d))
    gbox, tab = boxes.to(codes).cuda(), ref.table(n_tok, rot)
    for step, (at, n, factor, special) in enumerate(writes):
        p = np.arange(at, at + n)
        slots = np.array(ids, np.int64)[p // page] * page + p % page
        k, v = (rows(n, heads, d, kind, seed + 10 * step + e, special) * factor for e in (2, 3))
        fkv.fkv_page_append(got, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(p.astype(np.int32)).cuda(), tab.cuda(),
                            pairs=pairs, boxes=gbox)
        torch.cuda.synchronize()
        ref.append(*pool, k, v, slots, p, tab, pairs, boxes)
        same(got, pool, slots, page)
        assert torch.equal(gbox.cpu().float(), boxes), step
    return pool, gbox, ids


@pytest.mark.parametrize("page,heads,d,codes,kind,rot,pairs", [
    (16, 2, 64, INT8, F16, 64, False), (16, 1, 16, E4M3, BF16, 16, True), (64, 8, 128, INT8, BF16, 128, False),
    (64, 2, 80, E4M3, F16, 80, False), (48, 3, 112, INT8, F16, 32, True), (256, 2, 256, E4M3, BF16, 128, False),
    (256, 1, 256, INT8, BF16, 256, True), (128, 2, 144, INT8, F16, 96, False), (32, 2, 240, E4M3, F16, 0, False)])
def test_boxes_after_tokens_are_written_over(fkv, page, heads, d, codes, kind, rot, pairs):
    check(fkv, page, heads, d, codes, kind, rot, pairs, [
        (0, 10, 1.0, False), (5, 1, 0.5, False),                                    # the drafted ones refused, one token in their place
        (6, page + 9, 3.0, False), (page - 3, 2, 0.1, False),                       # back over a page's end
        (page - 1, 6, 8.0, False), (page + 1, 1, 0.25, False), (page + 2, 1, 0.25, False),
        (page + 1, 9, 20.0, True), (page + 2, 3, 1.0, False), (page + 15, 1, 0.0, False)], seed=d + page)


def test_a_refused_outlier_leaves_box_and_lists(fkv):
    """Ten tokens, one of them far from the others, then the fifth and later ones again: lists are those of what the pages hold."""
    page, heads, d, n = 16, 2, 64, 16 * 12
    pool, boxes, ids = check(fkv, page, heads, d, INT8, F16, 0, False, [(0, n, 0.1, False), (16 * 5 + 4, 6, 30.0, False), (16 * 5 + 4, 16 * 7 - 4, 0.1, False)])
    box = torch.zeros(boxes.shape)
    for p in ids:
        box[p] = ref.box_of(pool[0][p], page)
    assert torch.equal(boxes.cpu().float()[ids], box[ids])
    q = torch.randn((1, 2 * heads, d), generator=torch.Generator().manual_seed(3)).half()
    tables, kv, starts = torch.tensor([ids], dtype=torch.int32), torch.tensor([n], dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32)
    want = torch.zeros((1, heads, 4), dtype=torch.int32)
    ref.select(box.to(INT8), pool[2], q, tables, kv, starts, page, 4, 0, 0, True, want)
    got = fkv.fkv_page_select(up(pool), boxes, q.cuda(), tables.cuda(), kv.cuda(), starts.cuda(), 1, n, 4, keep_first=0, keep_last=0)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("codes", [INT8, E4M3])
def test_boxes_of_pages_begun_by_store(fkv, codes):
    """A page's box is formed of its codes: rows that fkv_page_store wrote before are in it."""
    page, heads, d = 32, 2, 96
    pool = fkv.fkv_pages(3, page, heads, d, codes)
    boxes = fkv.fkv_boxes(pool)
    boxes.view(torch.uint8).fill_(0x55)
    k = rows(page + 20, heads, d, F16, 1).cuda()
    slots = torch.arange(page, 2 * page + 20, device="cuda")
    fkv.fkv_page_store(pool, k[:20], k[:20], slots[:20])
    fkv.fkv_page_append(pool, k[20:], k[20:], slots[20:], boxes=boxes)
    torch.cuda.synchronize()
    codes_ = pool.k.cpu()
    assert torch.equal(boxes[1].cpu().float(), ref.box_of(codes_[1], page)) and torch.equal(boxes[2].cpu().float(), ref.box_of(codes_[2], 20))
    assert (bits(boxes[0]) == 0x55).all()
