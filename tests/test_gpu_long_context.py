"""The calls for long contexts as a server makes them: rows appended, pages selected and the lists attended to, prompt and
decoding steps in turn, on other streams, captured and replayed, in padded batches and in scratch that the caller keeps."""
import numpy as np
import pytest
import torch

import select_reference as ref

pytestmark = pytest.mark.gpu

INT8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def dev(a, dtype=torch.int32):
    return torch.as_tensor(a, dtype=dtype).cuda()


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


def some(n, heads, d, kind, seed):
    return torch.randn((n, heads, d), generator=torch.Generator().manual_seed(seed)).to(kind).cuda()


class Server:
    """A pool, its boxes and the requests' state; a step plans, appends, selects and attends."""

    def __init__(self, fkv, page, heads, group, d, codes, kind, most, n_select, pairs=False):
        self.fkv, self.page, self.heads, self.group, self.d, self.kind, self.n_select, self.pairs = fkv, page, heads, group, d, kind, n_select, pairs
        n_req, width = len(most), -(-max(most) // page)
        need = sum(-(-m // page) for m in most) + 2
        self.pool = fkv.fkv_pages(need, page, heads, d, codes)
        self.boxes = fkv.fkv_boxes(self.pool)
        self.table = fkv.fkv_rotation_table(max(most), d)
        self.free = torch.randperm(need, generator=torch.Generator().manual_seed(1)).int().cuda()
        self.head, self.kv = None, torch.zeros(n_req, dtype=torch.int32, device="cuda")
        self.tables = torch.zeros((n_req, width), dtype=torch.int32, device="cuda")

    def rows(self, n, seed):
        return (some(n, self.heads * self.group, self.d, self.kind, seed), some(n, self.heads, self.d, self.kind, seed + 1),
                some(n, self.heads, self.d, self.kind, seed + 2))

    def step(self, new, q, k, v, max_new, max_kv, **how):
        fkv = self.fkv
        p = fkv.fkv_page_plan(self.page, self.kv, new, self.free, self.head, self.tables, len(q), stream=how.get("stream"))
        stream = how.get("stream")
        turned = fkv.fkv_page_append(self.pool, k, v, p.slots, p.positions, self.table, q=q, pairs=self.pairs, boxes=self.boxes, stream=stream)
        lists = fkv.fkv_page_select(self.pool, self.boxes, turned, self.tables, p.kv_end, p.q_start, max_new, max_kv, self.n_select,
                                    workspace=how.get("select_work"), selected=how.get("selected"), stream=stream)
        out, lse = fkv.fkv_page_attend_selected(self.pool, turned, self.tables, p.kv_end, p.q_start, lists, max_new, max_kv, want_lse=True,
                                                out=how.get("out"), workspace=how.get("attend_work"), stream=stream)
        return p, turned, lists, out, lse

    def next(self, p):
        self.kv, self.head = p.kv_end, p.next_head


@pytest.mark.parametrize("page,heads,group,d,codes,kind,pairs", [(16, 2, 4, 64, INT8, F16, False), (64, 1, 7, 128, E4M3, BF16, True),
                                                                 (32, 3, 1, 80, INT8, BF16, False)])
def test_prompts_and_tokens_in_turn(fkv, page, heads, group, d, codes, kind, pairs):
    """Every step against the plain forms on the rows that the steps before left."""
    prompts, steps = [5 * page + 3, 1, 9 * page, 2 * page - 1], 4
    s = Server(fkv, page, heads, group, d, codes, kind, [m + 2 * steps for m in prompts], 4, pairs)
    cpu = [t.cpu() for t in s.pool]
    box = torch.zeros(s.boxes.shape)
    tab = s.table.cpu()
    kv = np.zeros(len(prompts), int)
    for i in range(steps + 1):
        new = np.array(prompts if i == 0 else [1, 1, 0, 2] if i == 2 else [1] * len(prompts))
        q, k, v = s.rows(int(new.sum()), 100 + 10 * i)
        kv = kv + new
        p, turned, lists, out, lse = s.step(dev(new), q, k, v, int(new.max()), int(kv.max()))
        torch.cuda.synchronize()
        slots, positions, starts = (t.cpu() for t in (p.slots, p.positions, p.q_start))
        ref.append(*cpu, k.cpu(), v.cpu(), slots.numpy(), positions, tab, pairs, box)
        assert p.kv_end.tolist() == kv.tolist()
        used = torch.unique(slots // page)
        assert torch.equal(bits(s.pool.scales), bits(cpu[2]))
        assert torch.equal(s.boxes.cpu().float()[used], box[used])
        want_q = ref.turned(q.cpu(), positions, tab, pairs).to(kind)
        assert torch.equal(turned.cpu(), want_q)
        tables, ends = s.tables.cpu(), torch.from_numpy(kv)
        want = torch.full((len(q), heads, 4), -9, dtype=torch.int32)
        ref.select(box.to(codes), cpu[2], want_q, tables, ends, starts, page, 4, 1, 1, True, want)
        assert torch.equal(lists.cpu(), want)
        exact, elog, off, loff = ref.attend_selected(*cpu, want_q, tables, ends, starts, want, d ** -0.5,
                                                     shifted=int(codes == INT8 and page == 16))
        half = torch.finfo(kind).eps / 2
        assert ((out.cpu().double() - exact).abs() <= off + half * (exact.abs() + off) + 2.0 ** -25).all()
        assert ((lse.cpu().double() - elog).abs() <= loff).all()
        s.next(p)


def serving(fkv, new=(1, 1, 1), padded=0):
    s = Server(fkv, 16, 2, 4, 64, INT8, F16, [3100, 700, 60], 24)
    before = [3000, 600, 7]
    p, *_ = s.step(dev(before), *s.rows(sum(before), 5), 3000, 3000)
    s.next(p)
    return s, s.rows(sum(new) + padded, 50)


def results(s, step):
    return [bits(x) for x in (*s.pool, s.boxes, *step[1:])]


@pytest.mark.parametrize("new", [(1, 1, 1), (40, 3, 17)])
def test_other_streams_and_kept_scratch(fkv, new):
    s, rows = serving(fkv, new)
    first = [x.clone() for x in (*s.pool, s.boxes)]
    args = (dev(new), *rows, max(new), 3000 + max(new))

    def back():
        for x, y in zip((*s.pool, s.boxes), first):
            x.copy_(y)

    want = results(s, s.step(*args))
    back()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = s.step(*args)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, results(s, got)))
    back()
    torch.cuda.synchronize()
    got = s.step(*args, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, results(s, got)))
    back()
    q, shape = rows[0], (3, s.tables.shape[1], max(new), 3000 + max(new), s.n_select)
    sizes = [fkv.fkv_page_select_workspace(s.pool, q, *shape), fkv.fkv_page_attend_selected_workspace(s.pool, q, *shape)]
    work = [torch.randint(0, 256, (max(1, n),), dtype=torch.uint8, device="cuda") for n in sizes]
    got = s.step(*args, select_work=work[0], attend_work=work[1], out=torch.full_like(q, float("nan")),
                 selected=torch.full((len(q), 2, s.n_select), 9, dtype=torch.int32, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(want, results(s, got)))


def test_two_streams_at_once(fkv):
    """Selection and attention of the same pool by two streams, each with scratch of its own."""
    s, rows = serving(fkv)
    p, turned, lists, out, lse = s.step(dev([1, 1, 1]), *rows, 1, 3001)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(20):
        for side in streams:
            with torch.cuda.stream(side):
                again = fkv.fkv_page_select(s.pool, s.boxes, turned, s.tables, p.kv_end, p.q_start, 1, 3001, s.n_select)
                got.append((again, *fkv.fkv_page_attend_selected(s.pool, turned, s.tables, p.kv_end, p.q_start, again, 1, 3001, want_lse=True)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, lists) and torch.equal(b, out) and torch.equal(c, lse) for a, b, c in got)


@pytest.mark.parametrize("n_select", [24, 190])
@pytest.mark.parametrize("padded", [0, 5])
def test_a_step_in_a_graph(fkv, padded, n_select):
    """A decoding step captured once, some rows of no request behind the last one: replays with other rows, lengths and numbers
    of tokens give the eager results, and two graphs of the same calls do not disturb each other."""
    s, rows = serving(fkv, padded=padded)
    s.n_select = n_select
    new, kv = dev([1, 1, 1]), s.kv.clone()
    s.kv = kv
    s.step(new, *rows, 1, 3050)
    torch.cuda.synchronize()
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append(s.step(new, *rows, 1, 3050))
    lengths = [[3000, 600, 7], [2990, 580, 0], [2999, 1, 5], [16, 300, 3], [2047, 0, 1]]
    tokens = [[1, 1, 1], [1, 1, 1], [1, 0, 1], [1, 1, 0], [1, 0, 1]]
    for i, (a, b) in enumerate(zip(lengths, tokens)):
        for x, y in zip(rows, s.rows(3 + padded, 60 + 3 * i)):
            x.copy_(y)
        kv.copy_(dev(a))
        new.copy_(dev(b))
        used = sum(b)
        before = [x.clone() for x in (*s.pool, s.boxes)]
        kept = []
        for g, step in zip(graphs, held):
            for x, y in zip((*s.pool, s.boxes), before):
                x.copy_(y)
            g.replay()
            torch.cuda.synchronize()
            kept.append([bits(x) for x in (*s.pool, s.boxes)] + [bits(x[:used]) for x in step[1:]])
        for x, y in zip((*s.pool, s.boxes), before):
            x.copy_(y)
        want = s.step(new, *rows, 1, 3050)
        want = [bits(x) for x in (*s.pool, s.boxes)] + [bits(x[:used]) for x in want[1:]]
        for x, y in zip((*s.pool, s.boxes), before):
            x.copy_(y)
        for replay in kept:
            assert all(torch.equal(x, y) for x, y in zip(replay, want)), i


def test_same_page_in_several_requests(fkv):
    """Requests that share their prompt's pages, and a request listed twice."""
    s, _ = serving(fkv)
    tables, kv = s.tables[[0, 0, 1, 0]].contiguous(), dev([3000, 3000, 600, 1500])
    q = some(4, 8, 64, F16, 9)
    q[1] = q[0]
    qs = dev([0, 1, 2, 3, 4])
    lists = fkv.fkv_page_select(s.pool, s.boxes, q, tables, kv, qs, 1, 3000, 24)
    out, lse = fkv.fkv_page_attend_selected(s.pool, q, tables, kv, qs, lists, 1, 3000, want_lse=True)
    assert torch.equal(lists[0], lists[1]) and torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
    alone = [fkv.fkv_page_select(s.pool, s.boxes, q[i:i + 1], tables[i:i + 1], kv[i:i + 1], qs[:2], 1, 3000, 24) for i in range(4)]
    assert torch.equal(lists, torch.cat(alone))


def test_binding_refuses(fkv):
    pool = fkv.fkv_pages(4, 16, 2, 64)
    boxes = fkv.fkv_boxes(pool)
    rows, q = (torch.zeros((8, h, 64), dtype=torch.float16, device="cuda") for h in (2, 4))
    slots, positions, table = torch.arange(8, device="cuda"), torch.arange(8, device="cuda").int(), fkv.fkv_rotation_table(8, 64)
    Errors = (TypeError, ValueError)
    fkv.fkv_page_append(pool, rows, rows, slots, positions, table, q=q, boxes=boxes)
    for kw in (dict(positions=None), dict(positions=positions.long()), dict(positions=positions[:7]), dict(table=table.double()),
               dict(table=table[..., 0]), dict(q=q[:7]), dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:, :, ::2]), dict(q=q[0]),
               dict(q_out=q[:, :3]), dict(q=None, q_out=q), dict(boxes=boxes[:3]), dict(boxes=boxes.float()), dict(boxes=boxes.cpu()),
               dict(k=rows.transpose(1, 2)), dict(v=rows[:7]), dict(slots=slots.int()), dict(n_bad=slots)):
        args = {**dict(k=rows, v=rows, slots=slots, positions=positions, table=table, q=q, boxes=boxes), **kw}
        with pytest.raises(Errors):
            fkv.fkv_page_append(pool, **args)
    for kw in (dict(q_out=q.bfloat16()), dict(v=rows.bfloat16()), dict(table=fkv.fkv_rotation_table(8, 80)),
               dict(table=torch.zeros((8, 5, 2), device="cuda"))):
        args = {**dict(k=rows, v=rows, slots=slots, positions=positions, table=table, q=q, boxes=boxes), **kw}
        with pytest.raises(fkv.FkvError):
            fkv.fkv_page_append(pool, **args)
    t, kv, qs = dev([[0, 1]]), dev([8]), dev([0, 8])
    lists = fkv.fkv_page_select(pool, boxes, q, t, kv, qs, 8, 8, 2)
    for kw in (dict(boxes=boxes[:3]), dict(boxes=boxes.view(torch.float8_e4m3fn)), dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()),
               dict(q=q[:, :, :32]), dict(tables=t[0]), dict(tables=t.long()), dict(kv_len=dev([8, 8])), dict(q_start=dev([0])),
               dict(selected=lists[:7]), dict(selected=lists.long()), dict(selected=lists[:, :, :1]), dict(workspace=lists)):
        args = {**dict(boxes=boxes, q=q, tables=t, kv_len=kv, q_start=qs, max_new=8, max_kv=8, n_select=2), **kw}
        with pytest.raises(Errors):
            fkv.fkv_page_select(pool, **args)
    for kw in (dict(n_select=0), dict(n_select=-1), dict(keep_first=2), dict(keep_last=-1), dict(max_new=0), dict(max_kv=-1)):
        with pytest.raises(fkv.FkvError):
            fkv.fkv_page_select(pool, **{**dict(boxes=boxes, q=q, tables=t, kv_len=kv, q_start=qs, max_new=8, max_kv=8, n_select=2), **kw})
    with pytest.raises(fkv.FkvError):
        fkv.fkv_page_select(pool, boxes, q[:, :3].contiguous(), t, kv, qs, 8, 8, 2)
    for kw in (dict(selected=lists[:7]), dict(selected=lists.long()), dict(selected=lists[:, :1].contiguous()), dict(selected=lists[0]),
               dict(q=q.float()), dict(out=q.bfloat16()), dict(out=q[:7]), dict(lse=torch.zeros(3, device="cuda")),
               dict(slopes=torch.zeros(3, device="cuda")), dict(prefix=dev([1, 2])), dict(first=dev([1]))):
        args = {**dict(q=q, tables=t, kv_len=kv, q_start=qs, selected=lists, max_new=8, max_kv=8), **kw}
        with pytest.raises(Errors):
            fkv.fkv_page_attend_selected(pool, **args)
    for kw in (dict(softcap=-1.0), dict(window=-1), dict(scale=float("inf")), dict(selected=lists[:, :, :0])):
        with pytest.raises(fkv.FkvError):
            fkv.fkv_page_attend_selected(pool, **{**dict(q=q, tables=t, kv_len=kv, q_start=qs, selected=lists, max_new=8, max_kv=8), **kw})
    assert fkv.fkv_page_select(pool, boxes, q[:0], t, kv, qs, 8, 8, 2).shape == (0, 2, 2)
    assert fkv.fkv_page_attend_selected(pool, q[:0], t, kv, qs, lists[:0], 8, 8)[0].shape == (0, 4, 64)


@pytest.mark.parametrize("new", [3, 70])
def test_pages_beyond_32_bits(fkv, new):
    """The last pages of a pool of more than 2^32 bytes of keys give what the same pages of a small one give."""
    page, heads, group, d, kv = 256, 16, 2, 256, 900
    n = 4500                          # 4.7 GB of keys, as much of values
    results = []
    for n_pages, ids in ((n, [n - 1, n - 3, n - 2, n - 4]), (4, [3, 1, 2, 0])):
        pool = fkv.fkv_pages(n_pages, page, heads, d)
        boxes, table = fkv.fkv_boxes(pool), fkv.fkv_rotation_table(1024, d)
        tables = dev([ids])
        for start, rows in ((0, kv), (kv, new)):
            at = torch.arange(start, start + rows)
            slots = (torch.tensor(ids)[at // page] * page + at % page).cuda()
            k, v, q = some(rows, heads, d, BF16, start), some(rows, heads, d, BF16, start + 1), some(rows, heads * group, d, BF16, start + 2)
            q = fkv.fkv_page_append(pool, k, v, slots, at.int().cuda(), table, q=q, boxes=boxes)
        lists = fkv.fkv_page_select(pool, boxes, q, tables, dev([kv + new]), dev([0, new]), new, kv + new, 2)
        out, lse = fkv.fkv_page_attend_selected(pool, q, tables, dev([kv + new]), dev([0, new]), lists, new, kv + new, want_lse=True)
        ids = torch.tensor(ids).cuda()
        results.append([bits(x) for x in (pool.k[ids], pool.v[ids], pool.scales[ids], boxes[ids], q, lists, out, lse)])
        del pool
    assert all(torch.equal(a, b) for a, b in zip(*results))
