"""Pages selected by a bound on their scores, and attention over lists of pages, on the GPU: the lists number for number,
attention against 64 bits."""
import math

import numpy as np
import pytest
import torch

import pages_reference as pages
import select_reference as ref

pytestmark = pytest.mark.gpu

INT8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def up(pool):
    return tuple(t.cuda() for t in pool)


def requests(lengths, page, n_pages, seed, width=None):
    """Block tables (CPU int32) over pages in no order, lengths and first rows of requests (tokens after, new tokens)."""
    _, _, t = ref.slot_map([(kv, 0) for kv, _ in lengths], page, n_pages, seed)
    width = width or max(1, max(len(x) for x in t))
    tables = torch.full((len(t), width), -1, dtype=torch.int32)
    for r, x in enumerate(t):
        tables[r, :len(x)] = torch.tensor(x, dtype=torch.int32)
    kv = torch.tensor([kv for kv, _ in lengths], dtype=torch.int32)
    starts = torch.tensor(np.concatenate(([0], np.cumsum([n for _, n in lengths]))), dtype=torch.int32)
    return tables, kv, starts


def boxes_of(n_pages, heads, d, codes, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n_pages, heads, 2, d), generator=g) * pages.LARGEST[codes] / 6 + torch.randn((n_pages, heads, 1, d), generator=g) * 20
    x = torch.stack((x.amin(2), x.amax(2)), 2)
    return pages.to_codes(x, codes)


# ---------------------------------------------------------------- select

def check_select(fkv, page, heads, group, d, codes, kind, lengths, n_select, keep_first, keep_last, causal=True, seed=0, change=None,
                 extra_rows=0, width=None):
    n_pages = sum(-(-kv // page) for kv, _ in lengths) + 3
    tables, kv, starts = requests(lengths, page, n_pages, seed, width)
    n = int(starts[-1]) + extra_rows
    boxes, scales = boxes_of(n_pages, heads, d, codes, seed + 1), torch.rand((n_pages, heads, 2), generator=torch.Generator().manual_seed(seed)) + 0.5
    q = torch.randn((n, heads * group, d), generator=torch.Generator().manual_seed(seed + 2)).to(kind)
    if change:
        change(boxes, scales, q, tables)
    pool = fkv.fkv_pages(n_pages, page, heads, d, codes)
    pool.scales.copy_(scales)
    max_new, max_kv = max(1, max(m for _, m in lengths)), max(x for x, _ in lengths)
    got = torch.full((n, heads, n_select), -7, dtype=torch.int32, device="cuda")
    want = got.cpu().clone()
    fkv.fkv_page_select(pool, boxes.cuda(), q.cuda(), tables.cuda(), kv.cuda(), starts.cuda(), max_new, max_kv, n_select,
                        keep_first=keep_first, keep_last=keep_last, causal=causal, selected=got)
    torch.cuda.synchronize()
    ref.select(boxes, scales, q, tables, kv, starts, page, n_select, keep_first, keep_last, causal, want)
    assert torch.equal(got.cpu(), want)
    return want


SELECTS = [
    # page, heads, group, d, codes, rows, (tokens, new) of each request, n_select, keep_first, keep_last
    (16, 1, 1, 16, INT8, F16, [(1, 1)], 1, 0, 1),
    (16, 2, 4, 64, INT8, F16, [(300, 1), (17, 1), (0, 0), (5, 2), (161, 3)], 4, 1, 1),
    (64, 8, 4, 128, INT8, BF16, [(4000, 1), (64, 1), (65, 1), (1900, 1)], 5, 1, 2),
    (32, 3, 7, 96, E4M3, F16, [(900, 4), (33, 1), (1, 1)], 6, 2, 1),
    (48, 1, 16, 80, E4M3, BF16, [(2000, 2), (97, 2)], 3, 0, 0),
    (128, 2, 20, 48, INT8, F16, [(3000, 3), (700, 1)], 7, 7, 0),
    (16, 1, 33, 32, INT8, F16, [(500, 2)], 9, 3, 3),
    (256, 2, 2, 256, INT8, F16, [(9000, 2), (1, 1)], 8, 1, 1),
    (16, 2, 5, 144, E4M3, F16, [(900, 9)], 10, 1, 1),
    (16, 2, 2, 64, INT8, F16, [(700, 150), (400, 400), (33, 33)], 8, 1, 1),      # four row tiles a wave
    (64, 4, 4, 128, INT8, BF16, [(2100, 90), (1700, 41)], 16, 1, 1),
    (32, 1, 3, 128, E4M3, F16, [(1000, 200)], 12, 0, 4),
    (16, 1, 2, 32, INT8, F16, [(16 * 70, 2)], 60, 1, 1),
    (16, 1, 2, 32, INT8, F16, [(16 * 300, 1)], 100, 1, 1),
    (16, 1, 2, 32, INT8, F16, [(16 * 513 - 5, 2)], 200, 1, 1),
    (16, 1, 1, 16, E4M3, F16, [(16 * 1500, 1), (16 * 257, 1)], 500, 2, 3),
    (16, 2, 1, 16, INT8, F16, [(16 * 2048, 1)], 33, 1, 1),
    (16, 2, 1, 16, INT8, F16, [(16 * 2049, 2), (40, 1), (16 * 2049 - 17, 1)], 33, 1, 1),   # a block a row
    (16, 1, 2, 32, E4M3, BF16, [(16 * 5000 + 3, 1)], 1500, 0, 0),
    (16, 2, 7, 96, E4M3, F16, [(16 * 300, 4), (16 * 90, 8), (50, 8)], 40, 2, 1),          # several tiles of few rows, at once
    (16, 1, 1, 64, INT8, BF16, [(16 * 200, 64), (16 * 100, 17), (30, 30)], 20, 0, 2),
    (16, 2, 16, 128, INT8, F16, [(16 * 1000, 4), (16 * 2048, 3)], 64, 1, 1),
    (16, 64, 1, 16, INT8, F16, [(16 * 2100, 1), (16 * 3000 - 3, 1), (20, 1)], 30, 1, 1),  # all of a block's waves a row
    (16, 128, 1, 16, E4M3, F16, [(16 * 16384 - 9, 1)], 100, 1, 1),
    (16, 2, 4, 128, INT8, F16, [(16 * 900, 17), (16 * 2200, 1)], 100, 1, 1),
    (16, 1, 1, 128, INT8, F16, [(16 * 512, 64)], 20, 1, 1),                               # the most of a block's LDS
    (16, 2, 4, 64, E4M3, BF16, [(16 * 90, 1), (16 * 40, 130), (700, 1), (0, 0), (16 * 33, 2)], 12, 1, 1),   # few rows and many
    (16, 2, 2, 32, INT8, F16, [(33, 0)] * 70 + [(160, 9)] + [(17, 0)] * 64 + [(100, 1), (100, 1)] + [(0, 0)] * 200 + [(90, 40)], 3, 1, 1),
    (16, 1, 20, 16, E4M3, F16, [(90, 0)] * 4100 + [(120, 3), (20, 0), (99, 1)] + [(1, 0)] * 40 + [(80, 1)], 2, 0, 1),
]


@pytest.mark.parametrize("page,heads,group,d,codes,kind,lengths,n_select,first,last", SELECTS)
@pytest.mark.parametrize("causal", [True, False])
def test_select(fkv, page, heads, group, d, codes, kind, lengths, n_select, first, last, causal):
    check_select(fkv, page, heads, group, d, codes, kind, lengths, n_select, first, last, causal, seed=d + page)


@pytest.mark.parametrize("tokens", [16 * 40, 16 * 300, 16 * 2500])
def test_select_of_equal_scores_takes_the_first(fkv, tokens):
    def same(boxes, scales, q, tables):
        boxes[:] = boxes[0]
        scales[:] = 1.0
    want = check_select(fkv, 16, 1, 2, 32, INT8, F16, [(tokens, 2)], 9, 1, 2, change=same)
    assert want[0, 0, :7].tolist() == list(range(7))

    def steps(boxes, scales, q, tables):       # few different scores, many of each
        boxes[:] = boxes[0]
        scales[:] = torch.randint(1, 4, scales.shape, generator=torch.Generator().manual_seed(3)).float()
    check_select(fkv, 16, 2, 2, 32, INT8, F16, [(tokens, 2)], 25, 1, 2, change=steps)


@pytest.mark.parametrize("tokens", [16 * 50, 16 * 2100])
def test_select_of_unusual_numbers(fkv, tokens):
    """Scales of zero, infinity and NaN, pages of no pool, rows of zeros, infinities and NaN, rows near their type's ends."""
    def change(boxes, scales, q, tables):
        g = torch.Generator().manual_seed(5)
        pick = torch.randint(0, 8, scales.shape, generator=g)
        scales[pick == 0] = 0.0
        scales[pick == 1] = math.inf
        scales[pick == 2] = math.nan
        tables[0, 3], tables[0, 7], tables[0, 11] = -1, 10 ** 6, len(boxes)
        q[0] = 0.0
        q[1, 0, 3], q[1, 1, 4], q[1, 2, 5] = math.inf, -math.inf, math.nan
        q[2, 0] *= 1e-38
        q[2, 1] *= 1e30
        q[3] *= 2.0 ** -125
        q[4] = math.nan
    check_select(fkv, 16, 2, 2, 64, INT8, BF16, [(tokens, 6)], 12, 1, 1, change=change)
    check_select(fkv, 16, 2, 2, 64, E4M3, BF16, [(tokens, 6)], 30, 0, 0, change=change)


def test_select_leaves_other_rows(fkv):
    want = check_select(fkv, 16, 2, 2, 64, INT8, F16, [(700, 3), (20, 0), (300, 5)], 6, 1, 1, extra_rows=9)
    assert (want[8:] == -7).all()
    # a request with no keys, and one whose rows outnumber its tokens
    want = check_select(fkv, 16, 2, 2, 64, INT8, F16, [(0, 3), (2, 5), (300, 1)], 6, 1, 1)
    assert (want[:3] == -1).all()


def test_select_never_misses_the_largest(fkv):
    """A page's score is no less than that of its keys' products with the rounded query: on boxes kept by append."""
    page, heads, d, n = 16, 2, 64, 640
    pool = fkv.fkv_pages(n // page, page, heads, d)
    boxes = fkv.fkv_boxes(pool)
    k = torch.randn((n, heads, d), generator=torch.Generator().manual_seed(1)).half().cuda()
    fkv.fkv_page_append(pool, k, k, torch.arange(n, device="cuda"), boxes=boxes)
    # a query that is the key of token 200, alone with a large product: its page is the one selected beside none kept
    k2 = torch.zeros_like(k)
    k2[200] = k[200] * 4
    fkv.fkv_page_append(pool, k2, k2, torch.arange(n, device="cuda"), boxes=boxes)
    got = fkv.fkv_page_select(pool, boxes, k2[200:201], torch.arange(n // page, dtype=torch.int32, device="cuda")[None],
                              torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                              1, n, 1, keep_first=0, keep_last=0)
    assert (got.cpu() == 200 // page).all()


# ---------------------------------------------------------------- attend

def lists(lengths, page, heads, n_selected, causal, seed, kind):
    """Lists of each token and KV head: `picked` as a selection gives them, `any` with repeats, holes and entries of no page."""
    rng = np.random.default_rng(seed)
    out = []
    for kv, new in lengths:
        for i in range(new):
            seen = max(0, -(-((kv - new + i + 1) if causal else kv) // page))
            for _ in range(heads):
                x = np.full(n_selected, -1, np.int32)
                if kind == "picked":
                    m = min(seen, n_selected)
                    x[:m] = np.sort(rng.choice(seen, m, replace=False)) if m else []
                    if m:
                        x[m - 1] = seen - 1
                else:
                    x[:] = rng.integers(-2, -(-kv // page) + 3, n_selected)
                    x[rng.random(n_selected) < 0.3] = -1
                    x[0] = 2 ** 31 - 1
                out.append(x)
    return torch.from_numpy(np.array(out).reshape(-1, heads, n_selected))


def check_attend(fkv, page, heads, group, d, codes, rows, lengths, n_selected, kind="picked", causal=True, seed=0, strided=False, scale=None,
                 bad_pages=False, extra_rows=0, **how):
    n_pages = sum(-(-kv // page) for kv, _ in lengths) + 3
    pool = ref.pool(n_pages, heads, page, d, codes, seed + 1)
    tables, kv, starts = requests(lengths, page, n_pages, seed)
    if bad_pages:
        tables[0, 1], tables[0, 2] = -1, n_pages
    n = int(starts[-1]) + extra_rows
    q = torch.randn((n, heads * group, d), generator=torch.Generator().manual_seed(seed + 2)).to(rows)
    selected = torch.full((n, heads, n_selected), -1, dtype=torch.int32)
    selected[:int(starts[-1])] = lists(lengths, page, heads, n_selected, causal, seed + 3, kind)
    # tokens behind a request's last one hold anything
    if codes == E4M3:
        for r, (t, _) in enumerate(lengths):
            if t % page:
                p = int(tables[r, t // page])
                if 0 <= p < n_pages:
                    pool[0].view(torch.uint8)[p, :, t % page:] = 0x7f
                    for o in range(t % page, page):
                        pool[1].view(torch.uint8)[p, :, o // 16, :, o % 16] = 0x7f
    dq = q.cuda()
    out = torch.full_like(dq, 7.0)
    if strided:
        wide = torch.zeros((n, heads * group + 2, d + 8), dtype=rows, device="cuda")
        wide[:, 1:-1, :d] = dq
        dq = wide[:, 1:-1, :d]
        out = torch.full((n, heads * group + 1, d + 16), 7.0, dtype=rows, device="cuda")[:, 1:, :d]
    lse = torch.full((n, heads * group), 7.0, device="cuda")
    max_new, max_kv = max(1, max(m for _, m in lengths)), max(x for x, _ in lengths)
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in how.items()}
    fkv.fkv_page_attend_selected(up(pool), dq, tables.cuda(), kv.cuda(), starts.cuda(), selected.cuda(), max_new, max_kv, scale=scale,
                                 causal=causal, out=out, lse=lse, **dev)
    torch.cuda.synchronize()
    scale = d ** -0.5 if scale is None else scale
    sane = (torch.nan_to_num(pool[0].float()).to(codes), torch.nan_to_num(pool[1].float()).to(codes), pool[2])
    # int8 codes are shifted where a wave has an item: of one tile, or of 2048 items
    rows_of_q, tiles = len(lengths) * max_new, -(-n_selected * (page // 16) // 4)
    items = (n if rows_of_q >= 2 * n else rows_of_q) * heads * -(-group // 16)
    shifted = tiles if codes == INT8 and (items >= 2048 or tiles == 1) else 0
    want, wlse, off, loff = ref.attend_selected(*sane, q, tables, kv, starts, selected, scale, causal=causal, shifted=shifted, **how)
    used = int(starts[-1])
    got, glse = out.cpu().double(), lse.cpu().double()
    assert torch.equal(torch.isinf(glse[:used]), torch.isinf(wlse[:used]))
    fine = ~torch.isinf(wlse[:used])
    assert ((glse - wlse)[:used][fine].abs() <= loff[:used][fine]).all()
    half = torch.finfo(rows).eps / 2
    room = off[:used] + half * (want[:used].abs() + off[:used]) + 2.0 ** -25
    worst = ((got - want)[:used].abs() / room).max() if used else 0.0
    assert worst <= 1.0, float(worst)
    assert (got[used:] == 7.0).all() and (glse[used:] == 7.0).all()


ATTENDS = [
    # page, heads, group, d, codes, rows, (tokens, new) of each request, n_selected
    (16, 1, 1, 16, INT8, F16, [(1, 1)], 1),
    (16, 2, 4, 64, INT8, F16, [(300, 1), (17, 1), (0, 0), (5, 2), (161, 3)], 4),
    (64, 8, 4, 128, INT8, BF16, [(1000, 1), (64, 1), (65, 1), (700, 1)], 5),
    (32, 3, 7, 96, E4M3, F16, [(500, 4), (33, 1), (1, 1)], 9),
    (48, 1, 16, 80, E4M3, BF16, [(700, 2), (97, 2)], 6),
    (128, 2, 20, 48, INT8, F16, [(900, 3), (700, 1)], 4),
    (16, 1, 33, 32, INT8, F16, [(300, 2)], 70),
    (256, 2, 2, 256, INT8, F16, [(1500, 2), (1, 1)], 4),
    (16, 2, 5, 144, E4M3, F16, [(300, 4)], 11),
    (64, 2, 4, 128, INT8, BF16, [(64 * 140, 1)], 130),           # split
    (16, 1, 3, 64, E4M3, F16, [(16 * 300, 1), (100, 1)], 260),
    (64, 2, 4, 128, INT8, BF16, [(64 * 60, 1), (500, 1)], 30),   # eight waves a block
    (16, 2, 3, 80, E4M3, F16, [(16 * 200, 1), (33, 2)], 100),
    (128, 1, 9, 64, E4M3, BF16, [(128 * 20, 2)], 13),
    (16, 4, 2, 64, INT8, F16, [(400, 300)], 4),                 # a wave an item
    (64, 4, 4, 128, INT8, BF16, [(700, 450), (300, 300)], 3),
    (64, 2, 4, 64, INT8, BF16, [(700, 1), (300, 200), (0, 0), (64, 1), (500, 3)], 4),   # few rows and many
    (16, 2, 2, 32, INT8, F16, [(33, 0)] * 70 + [(160, 9)] + [(17, 0)] * 64 + [(100, 1), (100, 1)] + [(0, 0)] * 200 + [(90, 40)], 3),
    (16, 1, 20, 16, E4M3, F16, [(90, 0)] * 4100 + [(120, 3), (20, 0), (99, 1)] + [(1, 0)] * 40 + [(80, 1)], 5),
]


@pytest.mark.parametrize("page,heads,group,d,codes,rows,lengths,n", ATTENDS)
@pytest.mark.parametrize("kind", ["picked", "any"])
def test_attend_selected(fkv, page, heads, group, d, codes, rows, lengths, n, kind):
    check_attend(fkv, page, heads, group, d, codes, rows, lengths, n, kind, seed=d + page)


LENGTHS = [(400, 3), (37, 2), (90, 1), (2, 4)]


@pytest.mark.parametrize("codes,rows", [(INT8, F16), (E4M3, BF16)])
@pytest.mark.parametrize("how", [
    dict(causal=False), dict(softcap=20.0), dict(softcap=500.0), dict(slopes=torch.linspace(0.01, 0.5, 6)), dict(window=70, sinks=9),
    dict(window=5, sinks=40, softcap=30.0), dict(prefix=torch.tensor([200, 10, 500, 0], dtype=torch.int32)),
    dict(first=torch.tensor([0, 50, 380, 36, 0, 64, 0, 1, 0, 5], dtype=torch.int32)), dict(scale=-0.2),
    dict(causal=False, window=60, slopes=torch.linspace(0.5, 0.01, 6)), dict(bad_pages=True), dict(strided=True), dict(extra_rows=5)])
@pytest.mark.parametrize("n", [7, 30])
def test_attend_selected_masks(fkv, codes, rows, how, n):
    check_attend(fkv, 16, 2, 3, 64, codes, rows, LENGTHS, n, "any", seed=3, **how)
    check_attend(fkv, 16, 2, 3, 64, codes, rows, LENGTHS, n, "picked", seed=4, **how)


HOWS = {
    "all": dict(causal=False), "cap": dict(softcap=20.0), "large cap": dict(softcap=500.0), "bias": dict(slopes=(0.01, 0.5)),
    "window": dict(window=70, sinks=9), "window and cap": dict(window=5, sinks=40, softcap=30.0), "prefix": dict(prefix=200),
    "first": dict(first=90), "negative": dict(scale=-0.2), "window of all": dict(causal=False, window=60, slopes=(0.5, 0.01)),
    "bad pages": dict(bad_pages=True), "strides": dict(strided=True), "more rows": dict(extra_rows=5)}


@pytest.mark.parametrize("codes,rows", [(INT8, F16), (E4M3, BF16)])
@pytest.mark.parametrize("name", HOWS)
@pytest.mark.parametrize("heads,group,d,lengths", [(2, 3, 64, LENGTHS), (16, 3, 64, [(330, 128), (70, 2)]), (16, 5, 80, [(270, 129)])])
def test_attend_selected_masks_of_whole_tiles(fkv, codes, rows, name, heads, group, d, lengths):
    """Pages of 64 tokens: of few items, and of so many that a wave has one."""
    how, n, g = dict(HOWS[name]), sum(m for _, m in lengths), torch.Generator().manual_seed(d)
    if "slopes" in how:
        how["slopes"] = torch.linspace(*how["slopes"], heads * group)
    if "prefix" in how:
        how["prefix"] = torch.randint(0, how["prefix"], (len(lengths),), generator=g, dtype=torch.int32)
    if "first" in how:
        how["first"] = torch.randint(-3, how["first"], (n,), generator=g, dtype=torch.int32)
    check_attend(fkv, 64, heads, group, d, codes, rows, lengths, 6, "any", seed=d, **how)


@pytest.mark.parametrize("kind", ["picked", "any"])
@pytest.mark.parametrize("page,heads,group,d,codes,rows,lengths,n", [
    (64, 16, 3, 80, E4M3, F16, [(500, 130)], 4),
    (128, 16, 1, 48, INT8, BF16, [(700, 130)], 3),
    (64, 16, 8, 144, INT8, F16, [(300, 129)], 3),
    (192, 16, 4, 256, E4M3, BF16, [(800, 128)], 2),
    (64, 32, 2, 16, INT8, F16, [(200, 70)], 3),
    (64, 16, 4, 96, INT8, F16, [(64 * 9, 130)], 9),
    (256, 16, 2, 112, E4M3, F16, [(900, 129)], 3),
    (48, 16, 2, 112, INT8, BF16, [(400, 129)], 5),
    (64, 3, 4, 240, E4M3, F16, [(60, 9), (130, 1)], 1),
    (64, 2, 4, 128, INT8, BF16, [(64 * 140, 1), (300, 0), (200, 3), (64 * 90, 1)], 130),   # few rows of many places, split
])
def test_attend_selected_of_many(fkv, page, heads, group, d, codes, rows, lengths, n, kind):
    check_attend(fkv, page, heads, group, d, codes, rows, lengths, n, kind, seed=d + page)


def test_attend_of_all_pages_is_attend(fkv):
    page, heads, group, d, lengths = 32, 2, 4, 64, [(1000, 3), (33, 2), (400, 1)]
    n_pages = sum(-(-kv // page) for kv, _ in lengths) + 3
    pool = up(ref.pool(n_pages, heads, page, d, INT8, 1))
    tables, kv, starts = (t.cuda() for t in requests(lengths, page, n_pages, 2))
    q = torch.randn((6, heads * group, d), generator=torch.Generator().manual_seed(1)).half().cuda()
    every = torch.arange(tables.shape[1], dtype=torch.int32, device="cuda").expand(6, heads, -1).contiguous()
    a, la = fkv.fkv_page_attend(pool, q, tables, kv, starts, 3, 1000, want_lse=True)
    b, lb = fkv.fkv_page_attend_selected(pool, q, tables, kv, starts, every, 3, 1000, want_lse=True)
    # two fp32 sums in another order, of weights rounded to 11 bits: within the bound that both keep to the exact ones
    want, _, off, loff = pages.attend(*(t.cpu() for t in pool), q.cpu(), tables.cpu(), kv.cpu(), starts.cpu(), d ** -0.5)
    assert ((a - b).cpu().double().abs() <= 2 * off + 2.0 ** -10 * (want.abs() + off)).all()
    assert ((la - lb).cpu().double().abs() <= 2 * loff).all()


def test_attend_of_lists_of_nothing(fkv):
    pool = up(ref.pool(4, 2, 16, 32, INT8, 1))
    q = torch.randn((2, 4, 32)).half().cuda()
    one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")    # noqa: E731
    for n in (1, 65, 300):
        out, lse = fkv.fkv_page_attend_selected(pool, q, one([[0, 1]]), one([20]), one([0, 2]), torch.full((2, 2, n), -1, dtype=torch.int32, device="cuda"),
                                                2, 20, want_lse=True)
        assert (out == 0).all() and (lse == -math.inf).all()
