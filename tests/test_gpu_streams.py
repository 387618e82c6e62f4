"""Calls by a stream's handle: what they make lies in that stream's memory and is cleared on it, whatever the current stream is
at."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream whose memory a tensor lies in."""
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]


def busy():
    """Some milliseconds of work on the current stream."""
    x = torch.ones((8192, 8192), dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    for _ in range(20):
        torch.mm(x, x, out=y)
    return x, y


def rows(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).half().cuda()


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("max_new", [1, 200])
def test_paged_calls_make_their_results_on_their_stream(fkv, max_new):
    page, heads, d = 64, 2, 64
    side = torch.cuda.Stream()
    how = dict(stream=side.cuda_stream)
    pool = fkv.fkv_pages(300, page, heads, d)
    boxes, table = fkv.fkv_boxes(pool), fkv.fkv_rotation_table(20000, d)
    tables, free = torch.zeros((1, 300), dtype=torch.int32, device="cuda"), torch.arange(300, dtype=torch.int32, device="cuda")
    q, k, v = rows(max_new, 4, d), rows(max_new, heads, d, seed=1), rows(max_new, heads, d, seed=2)
    kv = 130 * page
    torch.cuda.synchronize()
    p = fkv.fkv_page_plan(page, dev([kv]), dev([max_new]), free, None, tables, max_new, **how)
    turned = fkv.fkv_page_append(pool, k, v, p.slots, p.positions, table, q=q, boxes=boxes, **how)
    lists = fkv.fkv_page_select(pool, boxes, turned, tables, p.kv_end, p.q_start, max_new, kv + max_new, 70, **how)
    out = fkv.fkv_page_attend_selected(pool, turned, tables, p.kv_end, p.q_start, lists, max_new, kv + max_new, want_lse=True, **how)
    full = fkv.fkv_page_attend(pool, turned, tables, p.kv_end, p.q_start, max_new, kv + max_new, want_lse=True, **how)
    back = fkv.fkv_page_load(pool, p.slots, **how)
    side.synchronize()
    for t in (*p, turned, lists, *out, *full, *back):
        assert stream_of(t) == side.cuda_stream
    here = torch.cuda.current_stream().cuda_stream
    assert stream_of(fkv.fkv_page_load(pool, p.slots)[0]) == here != side.cuda_stream


def test_archive_calls_make_their_results_on_their_stream(fkv):
    ns, T, d, S, K = 4, 300, 64, 3, 32
    side = torch.cuda.Stream()
    how = dict(stream=side.cuda_stream)
    x, books, sb = rows(ns, T, d), rows(2, S, K, d, seed=1), dev([0, 1, 1, 0])
    codec = fkv.Codec(K)
    codec.table(x.device)
    torch.cuda.synchronize()
    sym, residual = fkv.fkv_rvq_assign(x, books, sb, 0, T, want_residual=True, **how)
    points = fkv.fkv_cgr_encode_spans(codec, sym, **how)
    decoded = fkv.fkv_cgr_decode_spans(codec, points, T * S, **how)
    found = fkv.fkv_span_lookup(codec, points, T * S, S, sb, sb, **how)
    again = fkv.fkv_rehydrate(codec, points, T * S, S, books, sb, sb, sb, **how)
    traj = fkv.fkv_trajectory(codec, sym, **how)
    side.synchronize()
    assert torch.equal(decoded, sym)
    for t in (sym, residual, points, decoded, found, again, traj):
        assert stream_of(t) == side.cuda_stream


def test_what_a_call_clears_it_clears_on_its_stream(fkv):
    """The search's counters and the update's sums, while the current stream has work of its own."""
    ns, T, d, S, K = 4, 300, 64, 3, 32
    x, books, sb = rows(ns, T, d), rows(2, S, K, d, seed=1), dev([0, 1, 1, 0])
    codec = fkv.Codec(K)
    sym, _ = fkv.fkv_rvq_assign(x, books, sb, 0, T)
    traj = fkv.fkv_trajectory(codec, sym)
    query = sym[1, 100:108].contiguous()
    side, one, two = torch.cuda.Stream(), books.clone(), books.clone()
    sums, counts = (torch.full(s, 7, dtype=t, device="cuda") for s, t in (((2, K, d), torch.int64), ((2, K), torch.int32)))
    hits, n_hits, n_candidates = fkv.fkv_suffix_search(codec, traj, query)
    _, want = fkv.fkv_kmeans_step(x, one, sb, 0, T, sym, 1)
    three = books.clone()
    torch.cuda.synchronize()
    work = busy()
    found = fkv.fkv_suffix_search(codec, traj, query, stream=side.cuda_stream)
    _, made = fkv.fkv_kmeans_step(x, two, sb, 0, T, sym, 1, stream=side.cuda_stream)
    _, given = fkv.fkv_kmeans_step(x, three, sb, 0, T, sym, 1, sums=sums, counts=counts, stream=side.cuda_stream)
    side.synchronize()
    got = [t.cpu() for t in (*found, made, given, two, three)]
    torch.cuda.synchronize()
    del work
    assert int(got[1]) == int(n_hits) >= 1 and int(got[2]) == int(n_candidates)
    hit = lambda h: sorted(map(tuple, h[:int(n_hits)].tolist()))     # noqa: E731
    assert hit(got[0]) == hit(hits.cpu())
    assert torch.equal(got[3], want.cpu()) and torch.equal(got[4], want.cpu())
    assert np.array_equal(got[5].view(torch.int16), one.cpu().view(torch.int16)) and np.array_equal(got[6].view(torch.int16), one.cpu().view(torch.int16))


def test_the_default_streams_handle(fkv):
    """0 is the default stream's handle, whatever stream is current."""
    ns, T, d, S, K = 4, 300, 64, 3, 32
    x, books, sb = rows(ns, T, d), rows(2, S, K, d, seed=1), dev([0, 1, 1, 0])
    pool, slots = fkv.fkv_pages(2, 16, 2, 64), torch.arange(4, device="cuda")
    side = torch.cuda.Stream()
    sym, _ = fkv.fkv_rvq_assign(x, books, sb, 0, T)
    one, two = books.clone(), books.clone()
    _, want = fkv.fkv_kmeans_step(x, one, sb, 0, T, sym, 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        work = busy()
        k, v = fkv.fkv_page_load(pool, slots, stream=0)
        _, counts = fkv.fkv_kmeans_step(x, two, sb, 0, T, sym, 1, stream=torch.cuda.default_stream().cuda_stream)
    torch.cuda.synchronize()
    del work
    assert torch.cuda.default_stream().cuda_stream == 0
    assert stream_of(k) == stream_of(v) == stream_of(counts) == 0 != side.cuda_stream
    assert torch.equal(counts, want) and torch.equal(one.view(torch.int16), two.view(torch.int16))
