"""The paged 8-bit cache on the GPU: block tables and slot maps against a plan made request by request, codes and
scales against the fp32 operations that define them, rows read back and attention against 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

import pages_reference as ref

pytestmark = pytest.mark.gpu

INT8, E4M3 = torch.int8, torch.float8_e4m3fn


def dev(a, dtype=None):
    return torch.as_tensor(a, dtype=dtype).cuda()


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


# ---------------------------------------------------------------- plan

def check_plan(fkv, page, kv, new, free, head, tables, n_tokens):
    want = ref.plan(page, kv, new, free, head, tables, n_tokens)
    t = dev(tables.copy(), torch.int32)
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = fkv.fkv_page_plan(page, dev(kv, torch.int32), dev(new, torch.int32), dev(free, torch.int32),
                            dev([head], torch.int32), t, n_tokens, n_bad=bad)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want["tables"])
    for name in ("slots", "positions", "q_start", "kv_end", "status"):
        assert np.array_equal(getattr(got, name).cpu().numpy(), want[name]), name
    assert int(got.head) == want["head"] and int(got.next_head) == want["next_head"]
    assert int(bad) == int((want["status"] != 0).sum())
    return want


@pytest.mark.parametrize("n_req,kv_hi,new_hi,page,free,short", [
    (0, 1, 1, 16, 1.0, 0), (1, 0, 1, 16, 1.0, 0), (1, 5, 0, 64, 1.0, 0), (7, 40, 3, 16, 1.0, 0), (16, 1023, 1, 16, 1.0, 0),
    (255, 300, 9, 48, 0.8, 0), (256, 300, 40, 16, 1.0, 5), (257, 300, 40, 32, 0.5, -7), (2048, 50, 7, 256, 1.0, 0),
    (2049, 90, 5, 16, 0.7, 0), (5000, 400, 3, 64, 0.3, 11), (3, 100, 70000, 16, 1.0, 0)])
def test_plan(fkv, n_req, kv_hi, new_hi, page, free, short):
    """`short`: rows that the step has room for fewer (or more, negative) than the requests bring."""
    rng = np.random.default_rng(n_req * 31 + page)
    kv, new = rng.integers(0, kv_hi + 1, n_req), rng.integers(0, new_hi + 1, n_req)
    if n_req > 20:
        kv[3], new[5], new[-1] = -4, -2, 10 ** 6      # the last brings more rows than the step holds
    width = -(-(kv_hi + new_hi) // page) + 1
    if n_req > 100:
        width = max(1, width - 2)     # too short for some
    old = -(-np.maximum(kv, 0) // page)
    need = int((-(-(np.maximum(kv, 0) + np.maximum(new, 0)) // page) - old)[:max(1, n_req - 1)].sum())
    tables = np.full((n_req, width), -1, np.int32)
    for r in range(n_req):
        tables[r, :min(old[r], width)] = rng.integers(0, 1 << 20, min(old[r], width))
    ids = rng.permutation(max(1, int(need * free)) + 3).astype(np.int32) + 7
    total = int(np.minimum(np.maximum(new, 0), 70000).sum()) - short
    want = check_plan(fkv, page, kv.astype(np.int32), new.astype(np.int32), ids, 3, tables, max(0, total))
    if n_req == 5000:
        assert {0, 1, 2, 3} <= set(want["status"].tolist())


def test_plan_rest_of_the_list_goes_on(fkv):
    """A request that the list has too few pages for leaves them to the next step; lengths beyond every bound."""
    kv = np.array([16, 16, 5, 2 ** 31 - 1], np.int32)
    new = np.array([16, 64, 3, 2 ** 30], np.int32)
    tables = np.full((4, 8), 99, np.int32)
    want = check_plan(fkv, 16, kv, new, np.array([4, 5, 6], np.int32), 0, tables, 83)
    assert want["status"].tolist() == [0, 1, 0, 3] and want["next_head"] == 1 and want["head"] == 5
    check_plan(fkv, 16, kv, new, np.array([4, 5, 6], np.int32), -3, tables, 83)
    check_plan(fkv, 16, kv, new, np.array([4, 5, 6], np.int32), 9, tables, 83)
    check_plan(fkv, 16, kv, new, np.zeros(0, np.int32), 0, tables, 83)


# ---------------------------------------------------------------- store, load

def make_rows(n, heads, d, dtype, seed, special=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g)
    x[:, :, :2] *= 10
    if special and n:
        x[0, 0, 3], x[-1, -1, 5], x[n // 2, 0, 0] = math.inf, -math.inf, math.nan
    return x.to(dtype)


def slot_map(lengths, page, n_pages, seed):
    """Slots of requests given as (tokens before, new tokens), on pages in no order; and the block tables."""
    rng = random.Random(seed)
    ids = list(range(n_pages))
    rng.shuffle(ids)
    slots, tables = [], []
    for kv, new in lengths:
        t = [ids.pop() for _ in range(-(-(kv + new) // page))]
        tables.append(t)
        slots += [t[p // page] * page + p % page for p in range(kv, kv + new)]
    return np.array(slots, np.int64), tables


STORES = [
    # page, heads, d, code type, row type, (before, new) of each request
    (16, 1, 16, INT8, torch.float16, [(0, 1)]),
    (16, 2, 64, INT8, torch.float16, [(0, 16), (3, 1), (15, 1), (16, 2), (7, 40), (0, 5)]),
    (16, 3, 80, E4M3, torch.bfloat16, [(1, 1), (2, 14), (0, 33), (5, 30)]),
    (48, 2, 96, INT8, torch.bfloat16, [(0, 47), (47, 2), (13, 100), (1, 1)]),
    (64, 8, 128, E4M3, torch.float16, [(0, 64), (63, 1), (10, 7), (0, 130), (61, 5)]),
    (64, 2, 128, INT8, torch.bfloat16, [(0, 200), (0, 1), (30, 3)]),
    (256, 2, 256, INT8, torch.float16, [(0, 300), (100, 90), (2, 1)]),
    (128, 1, 48, E4M3, torch.float16, [(9, 120), (0, 128), (127, 3)]),
    (16, 4, 64, INT8, torch.float16, [(5, 3)] * 400),       # more than 1024 rows
    (32, 2, 32, E4M3, torch.bfloat16, [(31, 1)] * 1100),
]


@pytest.mark.parametrize("page,heads,d,codes,rows,lengths", STORES)
@pytest.mark.parametrize("special", [False, True])
def test_store_matches_its_definition(fkv, page, heads, d, codes, rows, lengths, special):
    n_pages = sum(-(-(kv + new) // page) for kv, new in lengths) + 3
    slots, _ = slot_map(lengths, page, n_pages, d)
    g = torch.Generator().manual_seed(7)
    k = ref.to_codes(torch.randn((n_pages, heads, page, d), generator=g) * 40, codes)
    v = ref.to_codes(torch.randn((n_pages, heads, page // 16, d, 16), generator=g) * 40, codes)
    scales = torch.rand((n_pages, heads, 2), generator=g) * 0.05      # some grow, some stay
    n = len(slots)
    rk, rv = make_rows(n, heads, d, rows, 1, special), make_rows(n, heads, d, rows, 2, special)
    pages = fkv.Pages(k.cuda(), v.cuda(), scales.cuda())
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    sent = slots.copy()
    if n > 4:
        sent = np.concatenate((slots, [-1, n_pages * page, -9]))
        rk, rv = torch.cat((rk, rk[:3])), torch.cat((rv, rv[:3]))
    fkv.fkv_page_store(pages, rk.cuda(), rv.cuda(), dev(sent), n_bad=bad)
    torch.cuda.synchronize()
    assert int(bad) == (n > 4)
    was = k.clone()
    ref.store(k, v, scales, rk, rv, sent)
    written = torch.zeros((n_pages, page), dtype=torch.bool)          # tokens that the step leaves valid
    for i, m in ref.runs(slots, page):
        p, o = divmod(int(slots[i]), page)
        written[p, :o + m] = True
    untouched = ~written.any(1)
    assert torch.equal(bits(pages.scales), bits(scales))
    got_k, got_v = pages.k.cpu().view(torch.uint8), pages.v.cpu().view(torch.uint8).transpose(-1, -2).reshape(k.shape)
    want_k, want_v = k.view(torch.uint8), v.view(torch.uint8).transpose(-1, -2).reshape(k.shape)
    seen = written[:, None, :, None]
    assert torch.equal(torch.where(seen, got_k, 0), torch.where(seen, want_k, 0))
    assert torch.equal(torch.where(seen, got_v, 0), torch.where(seen, want_v, 0))
    assert torch.equal(got_k[untouched], was.view(torch.uint8)[untouched])
    # and against the rows themselves: half a step of the format, in 64 bits
    if not special:
        kk, vv = ref.values(pages.k.cpu(), pages.v.cpu(), pages.scales.cpu())
        p, o = torch.from_numpy(slots // page), torch.from_numpy(slots % page)
        for got, x, which in ((kk, rk, 0), (vv, rv, 1)):
            err = (got[p, :, o] - x[:n].double()).abs()
            s = scales[p][:, :, which, None].double()
            # int8: half a step; 8-bit floats: 2^-4 of the element, or half the least step; 2^-16 for the fp32 steps
            most = s * 0.5 if codes == INT8 else torch.maximum(x[:n].double().abs() * 2.0 ** -4, s * 2.0 ** -10)
            assert (err <= most * (1 + 2.0 ** -12) + s * 127 * 2.0 ** -20).all()


def test_store_tiny_and_zero_rows(fkv):
    """Pages of zeros and of elements below 2^-90 hold zeros; the largest bfloat16 elements keep their size."""
    pages = fkv.fkv_pages(4, 16, 1, 16, INT8)
    x = torch.zeros((64, 1, 16), dtype=torch.bfloat16)
    x[16:32] = 2.0 ** -100
    x[32:48] = 3.0e38
    x[48:64, :, 0] = 2.0 ** -80
    fkv.fkv_page_store(pages, x.cuda(), x.cuda(), torch.arange(64, device="cuda"))
    k, v = fkv.fkv_page_load(pages, torch.arange(64, device="cuda"), torch.bfloat16)
    assert not k[:32].any() and torch.equal(k, v) and not pages.scales[:2].any()
    assert torch.equal(k[32:].cpu(), x[32:])


@pytest.mark.parametrize("rows", [torch.float16, torch.bfloat16])
def test_store_layouts(fkv, rows):
    """Slices of a fused projection, head-major streams and plain rows give the same pages; and rows that come back."""
    b, t, heads, d, page = 3, 37, 4, 64, 16
    n_pages = 12
    slots, _ = slot_map([(0, t)] * b, page, n_pages, 3)
    fused = make_rows(b * t, 5 * heads, d, rows, 5).cuda()
    k, v = fused[:, 3 * heads:4 * heads], fused[:, 4 * heads:]
    want = fkv.fkv_pages(n_pages, page, heads, d)
    fkv.fkv_page_store(want, k.contiguous(), v.contiguous(), dev(slots))
    a = fkv.fkv_pages(n_pages, page, heads, d)
    fkv.fkv_page_store(a, k, v, dev(slots))
    c = fkv.fkv_pages(n_pages, page, heads, d)
    streams = torch.stack([x.reshape(b, t, heads, d).transpose(1, 2) for x in (k, v)])
    fkv.fkv_page_store(c, streams[0], streams[1], dev(slots.reshape(b, t)))
    for other in (a, c):
        for x, y in zip(want, other):
            assert torch.equal(bits(x), bits(y))
    back = torch.empty((2, b, heads, t, d), dtype=rows, device="cuda")
    fkv.fkv_page_load(want, dev(slots.reshape(b, t)), k=back[0], v=back[1])
    k2, v2 = fkv.fkv_page_load(want, dev(slots), rows)
    assert torch.equal(back[0].transpose(1, 2).reshape(b * t, heads, d), k2)
    assert torch.equal(back[1].transpose(1, 2).reshape(b * t, heads, d), v2)
    only = torch.zeros_like(v2)
    assert fkv.fkv_page_load(want, dev(slots), v=only)[0] is None
    assert torch.equal(only, v2)


@pytest.mark.parametrize("page,heads,d,codes", [(16, 3, 64, INT8), (48, 2, 80, E4M3), (64, 8, 128, INT8), (256, 1, 256, E4M3),
                                               (32, 5, 16, INT8)])
@pytest.mark.parametrize("rows", [torch.float16, torch.bfloat16])
def test_load(fkv, page, heads, d, codes, rows):
    """Rows in order, from any offset, in no order, twice, and slots of no page."""
    g = torch.Generator().manual_seed(d)
    n_pages = 9
    k = ref.to_codes(torch.randn((n_pages, heads, page, d), generator=g) * 40, codes)
    v = ref.to_codes(torch.randn((n_pages, heads, page // 16, d, 16), generator=g) * 40, codes)
    scales = torch.rand((n_pages, heads, 2), generator=g) * 2.0 ** -4 + 2.0 ** -9
    pages = fkv.Pages(k.cuda(), v.cuda(), scales.cuda())
    kk, vv = ref.values(k, v, scales)
    rng = np.random.default_rng(page)
    pool = n_pages * page
    for slots in (np.arange(pool), np.arange(4, pool - 3), np.arange(7, pool - 9)[1::1], np.arange(9, 10),
                  rng.integers(-3, pool + 3, 203), np.arange(pool)[::-1].copy(), np.zeros(0, np.int64)):
        gk, gv = fkv.fkv_page_load(pages, dev(slots, torch.int64), rows)
        ok = torch.from_numpy((slots >= 0) & (slots < pool))
        p, o = torch.from_numpy(np.clip(slots, 0, pool - 1) // page), torch.from_numpy(np.clip(slots, 0, pool - 1) % page)
        for got, all_rows in ((gk, kk), (gv, vv)):
            want = torch.where(ok[:, None, None], all_rows[p, :, o], 0.0)
            u = 2.0 ** -11 if rows == torch.float16 else 2.0 ** -8
            assert ((got.cpu().double() - want).abs() <= want.abs() * (u + 2.0 ** -23) + 2.0 ** -25).all()


# ---------------------------------------------------------------- attend

def make_pool(lengths, page, heads, d, codes, seed, garbage=True):
    """A pool whose rows are what a prompt's are like; what no request holds is anything, in 8-bit floats NaN too."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + 3
    x = torch.randn((n_pages, heads, page, d), generator=g)
    x[:, :, :, :3] *= 6
    y = torch.randn((n_pages, heads, page // 16, d, 16), generator=g) * (10.0 ** torch.randint(-3, 2, (n_pages, 1, 1, 1, 1), generator=g))
    scales = torch.stack((x.abs().amax((2, 3)), y.abs().amax((2, 3, 4))), 2) / ref.LARGEST[codes]
    k = ref.to_codes(x / scales[:, :, 0, None, None], codes).view(torch.uint8)
    v = ref.to_codes(y / scales[:, :, 1, None, None, None], codes).view(torch.uint8)
    order = torch.randperm(n_pages, generator=g)
    width = max(need + [1]) + 2
    tables = torch.randint(-5, 2 ** 31 - 1, (len(lengths), width), generator=g, dtype=torch.int64).to(torch.int32)
    at = 0
    used = torch.zeros((n_pages, page), dtype=torch.bool)
    for r, n in enumerate(lengths):
        tables[r, :need[r]] = order[at:at + need[r]].int()
        for p in range(need[r]):
            used[order[at + p], :min(page, n - p * page)] = True
        at += need[r]
    if garbage:
        fill = 0x80 if codes == INT8 else 0x7f
        k = torch.where(used[:, None, :, None], k, fill)
        v = torch.where(used.view(n_pages, 1, page // 16, 1, 16), v, fill)
        scales[~used.any(1)] = math.nan
    return k.view(codes), v.view(codes), scales, tables


def check_attend(fkv, lengths, new, page, heads, group, d, codes, rows, seed=0, strided=False, q_scale=1.0, **opt):
    k, v, scales, tables = make_pool(lengths, page, heads, d, codes, seed)
    g = torch.Generator().manual_seed(seed + 1)
    n = sum(new)
    q = (torch.randn((n, heads * group, d), generator=g) * q_scale).to(rows)
    q_start = torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32)
    kv = torch.tensor(lengths, dtype=torch.int32)
    clean_k, clean_v = k.clone(), v.clone()
    if codes == E4M3:      # the reference looks at valid keys only, but a product with a NaN is one
        for c in (clean_k, clean_v):
            b = c.view(torch.uint8)
            b[b == 0x7f] = 0
    scale = opt.pop("scale", d ** -0.5)
    out, lse, off, loff = ref.attend(clean_k, clean_v, torch.nan_to_num(scales), q, tables, kv, q_start, scale, **opt)
    if strided:
        big = torch.full((n, heads * group + 3, d + 8), 7.0, dtype=rows, device="cuda")
        qd, od = big[:, 1:-2, :d], torch.full((n, 2 * heads * group, d), 5.0, dtype=rows, device="cuda")[:, ::2]
        qd.copy_(q)
    else:
        qd, od = q.cuda(), None
    dopt = {name: (x.cuda() if isinstance(x, torch.Tensor) else x) for name, x in opt.items()}
    got, glse = fkv.fkv_page_attend(fkv.Pages(k.cuda(), v.cuda(), scales.cuda()), qd, tables.cuda(), kv.cuda(), q_start.cuda(),
                                    max(new + [1]), max(lengths + [0]), scale=scale, out=od, want_lse=True, **dopt)
    torch.cuda.synchronize()
    got, glse = got.cpu().double(), glse.cpu().double()
    u = 2.0 ** -11 if rows == torch.float16 else 2.0 ** -8
    empty = lse == -math.inf
    assert torch.equal(glse == -math.inf, empty) and not got[empty].any()
    diff = (got - out).abs()
    worst = (diff / (off + u * (out.abs() + off) + 2.0 ** -24)).max() if diff.numel() else 0
    assert worst <= 1, float(worst)
    assert ((glse - lse).abs()[~empty] <= loff[~empty]).all()
    return got, glse


ATTEND = [
    # lengths, new, page, heads, group, d
    ([1], [1], 16, 1, 1, 64),
    ([0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300], [1] * 12, 16, 2, 1, 64),
    ([5, 700, 0, 64, 191, 1000], [1, 1, 0, 1, 1, 1], 48, 2, 4, 96),
    ([257, 1, 513], [1, 1, 1], 64, 3, 8, 128),
    ([130, 1030], [2, 2], 256, 1, 7, 256),
    ([333, 20], [5, 3], 32, 2, 3, 80),
    ([70, 40], [1, 1], 128, 1, 16, 16),
    ([70, 400, 3], [70, 1, 3], 16, 2, 1, 64),
    ([129, 200, 64, 0, 1], [129, 77, 64, 0, 1], 48, 2, 2, 80),
    ([300, 90], [33, 90], 64, 2, 4, 128),
    ([150], [130], 16, 1, 1, 256),
    ([100, 31], [100, 31], 32, 1, 5, 48),
    ([4, 30], [9, 40], 16, 1, 2, 32),            # more rows than tokens: the first see nothing
    ([2, 30], [3, 2], 16, 1, 4, 32),
]


@pytest.mark.parametrize("lengths,new,page,heads,group,d", ATTEND)
@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16), (INT8, torch.bfloat16), (E4M3, torch.float16)])
def test_attend_causal(fkv, lengths, new, page, heads, group, d, codes, rows):
    check_attend(fkv, lengths, new, page, heads, group, d, codes, rows, seed=d, strided=codes == E4M3)


def _slopes(n):
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / n) for i in range(n)])


OPTIONS = [
    dict(softcap=30.0), dict(slopes=True), dict(softcap=5.0, slopes=True), dict(causal=False), dict(window=7, sinks=0),
    dict(window=20, sinks=4), dict(window=70, sinks=100), dict(window=1, sinks=0), dict(prefix=True), dict(first=True),
    dict(first=True, window=33, sinks=9, softcap=20.0), dict(causal=False, window=40, sinks=3, slopes=True),
    dict(prefix=True, window=25, sinks=2, first=True, slopes=True, softcap=11.0), dict(scale=0.0), dict(scale=-0.3),
]


@pytest.mark.parametrize("opt", OPTIONS)
@pytest.mark.parametrize("shape", [([400, 33, 1, 260], [1, 1, 1, 1], 16, 2, 4, 64), ([400, 33, 150], [160, 33, 7], 48, 2, 2, 80),
                                   ([300, 200], [200, 3], 64, 1, 8, 128)])
@pytest.mark.parametrize("codes,rows", [(INT8, torch.float16), (E4M3, torch.bfloat16)])
def test_attend_scores_and_masks(fkv, opt, shape, codes, rows):
    lengths, new, page, heads, group, d = shape
    opt = dict(opt)
    rng = np.random.default_rng(d)
    if opt.pop("slopes", False):
        opt["slopes"] = _slopes(heads * group)
    if opt.pop("prefix", False):
        opt["prefix"] = torch.tensor([rng.integers(0, n + 30) for n in lengths], dtype=torch.int32)
    if opt.pop("first", False):
        # documents, out of order too, one that begins after every key and one before the first
        opt["first"] = torch.tensor(rng.integers(-5, max(lengths) + 20, sum(new)), dtype=torch.int32)
    check_attend(fkv, lengths, new, page, heads, group, d, codes, rows, seed=3, **opt)


@pytest.mark.parametrize("codes,rows", [(INT8, torch.bfloat16), (E4M3, torch.float16)])
@pytest.mark.parametrize("new", [[1, 1], [9, 40]])
def test_attend_long_axis_is_split(fkv, codes, rows, new):
    """Long requests beside a short one: several splits, most of the short one's empty."""
    check_attend(fkv, [9000, 70], new, 64, 2, 4, 64, codes, rows, seed=5)
    check_attend(fkv, [9000, 70], new, 64, 2, 4, 64, codes, rows, seed=5, window=300, sinks=5)


@pytest.mark.parametrize("rows", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_scale", [1e-6, 1e3])
def test_attend_small_and_large_queries(fkv, rows, q_scale):
    """Rows far from 1: the binary16 operand of a bfloat16 row keeps its bits."""
    for new in ([1], [40]):
        check_attend(fkv, [200], new, 16, 1, 1, 64, INT8, rows, q_scale=q_scale, scale=0.125 / q_scale)


def test_attend_pages_of_no_pool_are_not_seen(fkv):
    """Table entries outside the pool hide their keys, a request with no valid page is empty."""
    for new in ([1, 1], [20, 20]):
        k, v, scales, tables = make_pool([100, 100], 16, 1, 64, INT8, 1, garbage=False)
        tables[0, 2], tables[0, 4], tables[1] = -1, k.shape[0], 2 ** 31 - 1
        q = torch.randn((sum(new), 2, 64)).to(torch.float16)
        q_start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32)
        kv = torch.tensor([100, 100], dtype=torch.int32)
        out, lse, off, loff = ref.attend(k, v, scales, q, tables, kv, q_start, 0.125)
        got, glse = fkv.fkv_page_attend((k.cuda(), v.cuda(), scales.cuda()), q.cuda(), tables.cuda(), kv.cuda(), q_start.cuda(),
                                        max(new), 100, want_lse=True)
        assert ((got.cpu().double() - out).abs() <= off + 2.0 ** -11 * (out.abs() + off) + 2.0 ** -24).all()
        assert not got[new[0]:].any() and (glse[new[0]:] == -math.inf).all()


def test_attend_not_a_number_in_a_query_stays_in_its_row(fkv):
    for new in (3, 40):
        k, v, scales, tables = make_pool([100], 16, 1, 64, INT8, 1)
        q = torch.randn((new, 2, 64)).to(torch.float16)
        q[1, 0, 5], q[2, 1, 7] = math.nan, math.inf
        args = ((k.cuda(), v.cuda(), scales.cuda()), q.cuda(), tables.cuda(), dev([100], torch.int32), dev([0, new], torch.int32), new, 100)
        got, _ = fkv.fkv_page_attend(*args)
        bad = torch.zeros((new, 2), dtype=torch.bool)
        bad[1, 0] = bad[2, 1] = True
        assert got[bad.cuda()].isnan().all() and got[~bad.cuda()].isfinite().all()


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_beyond_32_bits(fkv, new):
    """A pool of more than 4 GiB of keys: the last pages are stored, attended to and read back like any."""
    heads, page, d = 2, 64, 128
    n_pages = (1 << 32) // (heads * page * d) + 300
    pages = fkv.fkv_pages(n_pages, page, heads, d)
    ids = np.arange(n_pages - 4, n_pages)
    slots = (ids[:, None] * page + np.arange(page)).reshape(-1)
    rk, rv = make_rows(256, heads, d, torch.float16, 1).cuda(), make_rows(256, heads, d, torch.float16, 2).cuda()
    fkv.fkv_page_store(pages, rk, rv, dev(slots))
    small = fkv.fkv_pages(4, page, heads, d)
    fkv.fkv_page_store(small, rk, rv, torch.arange(256, device="cuda"))
    for a, b in zip(pages, small):
        assert torch.equal(bits(a[-4:]), bits(b))
    for a, b in zip(fkv.fkv_page_load(pages, dev(slots)), fkv.fkv_page_load(small, torch.arange(256, device="cuda"))):
        assert torch.equal(a, b)
    q = make_rows(new, 4, d, torch.float16, 3).cuda()
    got = [fkv.fkv_page_attend(p, q, dev(t, torch.int32), dev([250], torch.int32), dev([0, new], torch.int32), new, 250, want_lse=True)
           for p, t in ((pages, ids[None]), (small, np.arange(4)[None]))]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


# ---------------------------------------------------------------- streams, graphs, repetition

def _step(fkv, pages, st):
    p = fkv.fkv_page_plan(16, st["kv"], st["new"], st["free"], st["head"], st["tables"], st["k"].shape[0])
    fkv.fkv_page_store(pages, st["k"], st["v"], p.slots)
    out, lse = fkv.fkv_page_attend(pages, st["q"], st["tables"], p.kv_end, p.q_start, st["max_new"], st["max_kv"], want_lse=True)
    return p, out, lse


def _state(fkv, new, kv=(40, 3000, 7), heads=2, group=4, d=64):
    n = sum(new)
    need = sum(-(-(a + b) // 16) for a, b in zip(kv, new))
    pages = fkv.fkv_pages(need + 4, 16, heads, d)
    ids = torch.randperm(need, device="cuda", dtype=torch.int32)
    width = -(-(max(kv) + max(new)) // 16)
    tables = torch.zeros((len(kv), width), dtype=torch.int32, device="cuda")
    zero = torch.zeros(len(kv), dtype=torch.int32, device="cuda")
    p = fkv.fkv_page_plan(16, zero, dev(kv, torch.int32), ids, None, tables, sum(kv))
    fkv.fkv_page_store(pages, make_rows(sum(kv), heads, d, torch.float16, 1).cuda(), make_rows(sum(kv), heads, d, torch.float16, 2).cuda(), p.slots)
    return pages, dict(kv=dev(kv, torch.int32), new=dev(new, torch.int32), free=ids, head=p.next_head, tables=tables,
                       k=make_rows(n, heads, d, torch.float16, 3).cuda(), v=make_rows(n, heads, d, torch.float16, 4).cuda(),
                       q=make_rows(n, heads * group, d, torch.float16, 5).cuda(), max_new=max(new), max_kv=max(kv) + max(new))


@pytest.mark.parametrize("new", [(1, 1, 1), (30, 5, 12)])
def test_same_bits_every_time_and_on_another_stream(fkv, new):
    pages, st = _state(fkv, new)
    p, out, lse = _step(fkv, pages, st)
    kept = [bits(x) for x in (*pages, out, lse, p.slots)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = _step(fkv, pages, st)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, bits(b)) for a, b in zip(kept, (*pages, again[1], again[2], again[0].slots)))
    # by its handle: the scratch comes from that stream, or from the caller
    out2, lse2 = fkv.fkv_page_attend(pages, st["q"], st["tables"], p.kv_end, p.q_start, st["max_new"], st["max_kv"], want_lse=True,
                                     stream=side.cuda_stream)
    side.synchronize()
    need = fkv.fkv_page_attend_workspace(pages, st["q"], 3, st["tables"].shape[1], st["max_new"], st["max_kv"])
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    out3, lse3 = fkv.fkv_page_attend(pages, st["q"], st["tables"], p.kv_end, p.q_start, st["max_new"], st["max_kv"], want_lse=True, workspace=work)
    assert need > 0 and torch.equal(out2, out) and torch.equal(lse2, lse) and torch.equal(out3, out) and torch.equal(lse3, lse)
    with pytest.raises(fkv.FkvError):
        fkv.fkv_page_attend(pages, st["q"], st["tables"], p.kv_end, p.q_start, st["max_new"], st["max_kv"], workspace=work[:need - 16])


def test_a_step_in_a_graph(fkv):
    """plan, store and attend captured once; replays with other rows and lengths give the eager results."""
    pages, st = _state(fkv, (1, 1, 1))
    _step(fkv, pages, st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p, out, lse = _step(fkv, pages, st)
    for i in range(4):
        st["k"].copy_(make_rows(3, 2, 64, torch.float16, 50 + i))
        st["q"].copy_(make_rows(3, 8, 64, torch.float16, 60 + i))
        st["kv"].copy_(torch.tensor([30 + i, 2990 - 300 * i, 3 + i]))
        before = [x.clone() for x in pages]
        g.replay()
        torch.cuda.synchronize()
        kept = [bits(x) for x in (*pages, out, lse, p.slots)]
        for x, y in zip(pages, before):
            x.copy_(y)
        want = _step(fkv, pages, st)
        assert all(torch.equal(a, bits(b)) for a, b in zip(kept, (*pages, want[1], want[2], want[0].slots))), i


# ---------------------------------------------------------------- refusals of the binding

def test_binding_refuses(fkv):
    pages = fkv.fkv_pages(4, 16, 2, 64)
    slots = torch.arange(8, device="cuda")
    rows = torch.zeros((8, 2, 64), dtype=torch.float16, device="cuda")
    for bad in (rows.float(), rows.transpose(1, 2), rows[:, :, ::2], rows.cpu()):
        with pytest.raises((TypeError, ValueError)):
            fkv.fkv_page_store(pages, bad, rows, slots)
    with pytest.raises(ValueError):
        fkv.fkv_page_store(pages, rows[:7], rows, slots)
    with pytest.raises(fkv.FkvError):
        fkv.fkv_page_store(pages, rows, rows.bfloat16(), slots)
    with pytest.raises(fkv.FkvError):      # not 16-byte aligned
        fkv.fkv_page_store(pages, torch.zeros(8 * 128 + 8, dtype=torch.float16, device="cuda")[1:1025].view(8, 2, 64), rows, slots)
    with pytest.raises(TypeError):
        fkv.fkv_page_store(pages, rows, rows, slots.int())
    with pytest.raises((TypeError, ValueError)):
        fkv.fkv_page_store((pages.k, pages.v[:2], pages.scales), rows, rows, slots)
    with pytest.raises(TypeError):
        fkv.fkv_page_load((pages.k.float(), pages.v, pages.scales), slots)
    q = torch.zeros((8, 4, 64), dtype=torch.float16, device="cuda")
    t, kv, qs = dev([[0, 1]], torch.int32), dev([8], torch.int32), dev([0, 8], torch.int32)
    fkv.fkv_page_attend(pages, q, t, kv, qs, 8, 8)
    for kw in (dict(slopes=torch.zeros(3, device="cuda")), dict(prefix=dev([1, 2], torch.int32)), dict(first=dev([1], torch.int32)),
               dict(out=q.bfloat16()), dict(out=q[:7])):
        with pytest.raises((TypeError, ValueError)):
            fkv.fkv_page_attend(pages, q, t, kv, qs, 8, 8, **kw)
    for kw in (dict(softcap=-1.0), dict(window=-1), dict(sinks=-1), dict(scale=math.nan), dict(softcap=math.inf)):
        with pytest.raises(fkv.FkvError):
            fkv.fkv_page_attend(pages, q, t, kv, qs, 8, 8, **kw)
    with pytest.raises(fkv.FkvError):      # 3 query heads over 2 KV heads
        fkv.fkv_page_attend(pages, q[:, :3].contiguous(), t, kv, qs, 8, 8)
    assert fkv.fkv_page_attend(pages, q[:0], t, kv, qs, 8, 8)[0].shape == (0, 4, 64)
