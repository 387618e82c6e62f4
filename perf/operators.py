"""Performance cases of the paged 8-bit KV cache: the calls that a serving program makes around the archive, with
their plain forms.

  plan    block tables and slot maps of a step, from the requests' lengths
  store   a step's K/V rows written into 8-bit pages, and the touched pages' rows as attention will see them
  load    rows of a context read back, as the archive's assignment takes them
  attend  attention over the pages: single tokens, prompts and chunks of prompts

Pages hold `page` tokens of every KV head, keys as [page][d], values as [page/16][d][16], with one scale for each
page, head and K or V; a request's pages lie anywhere in the pool, in the order of its block table.
"""
import math
import random

import numpy as np
import torch

own = False

OUTLIERS, OUTLIER_SCALE = 4, 10.0      # strong key channels, as in the archive's synthetic workloads
SMALLEST = 2.0 ** -90                  # a page whose largest element is below this is stored as zeros
MOST_SCORES = 32 * 4096 * 32768        # rows x heads x keys of a drawn attention case at most
MOST_CODES = 64 * 8 * 32768 * 128      # padded key elements of a drawn attention case at most
MOST_PAIRS = 4 * 128 * 32 * 4096 * 30000


def listed():
    return [
        # a decoding step of 16 sequences of up to 1024 tokens: the smallest plan, where launches count
        dict(name="plan_decode_b16", op="plan", requests=16, kv_lo=100, kv_hi=1023, new_lo=1, new_hi=1, page=16,
             free=1.0, mix=1),
        # admission of 2048 prompts and continuations of all lengths, the free pages running out on the way
        dict(name="plan_prompts", op="plan", requests=2048, kv_lo=1, kv_hi=32768, new_lo=1, new_hi=2048, page=64,
             free=0.9, mix=2),
        # one layer's rows of a decoding step, batch 16, GPT-2 heads; most pages are part full
        dict(name="store_decode_b16", op="store", requests=16, kv_lo=100, kv_hi=1023, new_lo=1, new_hi=1, heads=12,
             d=64, page=16, dtype="float16", codes="int8", layout="fused", mix=3),
        # one layer's rows of a 32,768-token prompt (8 KV heads of 128), out of the fused projection
        dict(name="store_long", op="store", requests=1, kv_lo=0, kv_hi=0, new_lo=32768, new_hi=32768, heads=8, d=128,
             page=64, dtype="bfloat16", codes="int8", layout="fused", mix=4),
        # the 988 positions between the sinks and the recent window, 16 contexts, to be archived
        dict(name="load_archive_b16", op="load", requests=16, kv=1024, t0=4, t1=992, heads=12, d=64, page=16,
             dtype="float16", codes="int8", mix=5),
        # the same of four 32,768-token contexts
        dict(name="load_archive_long", op="load", requests=4, kv=32768, t0=4, t1=32736, heads=8, d=128, page=64,
             dtype="float16", codes="int8", mix=6),
        # single-token attention: one GPT-2-shaped sequence, the smallest call
        dict(name="attend_gpt2", op="attend", requests=1, kv_lo=1024, kv_hi=1024, new_lo=1, new_hi=1, heads=12, group=1,
             d=64, page=16, dtype="float16", codes="int8", softcap=0.0, slopes=False, docs=0, prefix=False, window=0,
             sinks=0, causal=True, mix=7),
        # ... 64 ragged sequences over 8-bit floats, capped scores, a distance bias
        dict(name="attend_ragged_b64", op="attend", requests=64, kv_lo=1, kv_hi=32768, new_lo=1, new_hi=1, heads=8,
             group=4, d=128, page=64, dtype="float16", codes="e4m3", softcap=50.0, slopes=True, docs=0, prefix=False,
             window=0, sinks=0, causal=True, mix=8),
        # ... four 32,768-token contexts of the grouped-KV model
        dict(name="attend_long_b4", op="attend", requests=4, kv_lo=32768, kv_hi=32768, new_lo=1, new_hi=1, heads=8,
             group=4, d=128, page=64, dtype="bfloat16", codes="int8", softcap=0.0, slopes=False, docs=0, prefix=False,
             window=0, sinks=0, causal=True, mix=9),
        # 16 prompts of packed documents, of all lengths up to 1024
        dict(name="attend_docs_b16", op="attend", requests=16, kv_lo=100, kv_hi=1024, new_lo=1024, new_hi=1024,
             heads=12, group=1, d=64, page=16, dtype="float16", codes="int8", softcap=0.0, slopes=False, docs=3,
             prefix=False, window=0, sinks=0, causal=True, mix=10),
        # eight prompts whose first part sees itself whole, behind earlier turns, bfloat16 rows, capped scores
        dict(name="attend_prefix_b8", op="attend", requests=8, kv_lo=2000, kv_hi=8000, new_lo=500, new_hi=2000,
             heads=8, group=4, d=128, page=64, dtype="bfloat16", codes="e4m3", softcap=30.0, slopes=False, docs=0,
             prefix=True, window=0, sinks=0, causal=True, mix=11),
        # the largest: the last 4096 tokens of a 32,768-token prompt
        dict(name="attend_chunk_long", op="attend", requests=1, kv_lo=32768, kv_hi=32768, new_lo=4096, new_hi=4096,
             heads=8, group=4, d=128, page=64, dtype="bfloat16", codes="int8", softcap=0.0, slopes=False, docs=0,
             prefix=False, window=0, sinks=0, causal=True, mix=12),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + (n == 1024 * 3 and n < hi)


def draw(rng):
    """A case of the listed ones' ranges, odd sizes among them."""
    op = rng.choice(("plan", "store", "load", "attend", "attend", "attend"))
    mix, page = rng.randint(100, 10 ** 6), rng.choice((16, 16, 32, 48, 64, 64, 128))
    if op == "plan":
        new = rng.choice((1, 1, _log(rng, 2, 2048)))
        return dict(op=op, requests=_log(rng, 1, 2048), kv_lo=rng.choice((0, 1, 100)), kv_hi=_log(rng, 200, 32768),
                    new_lo=rng.choice((0, 1)) if new > 1 else 1, new_hi=new, page=page,
                    free=rng.choice((1.0, 1.0, 0.7)), mix=mix)
    heads, group, d = rng.choice((4, 8, 8, 12)), rng.choice((1, 1, 2, 4, 4, 7, 8)), rng.choice((64, 64, 80, 96, 128, 128))
    dtype, codes = rng.choice(("float16", "bfloat16")), rng.choice(("int8", "int8", "e4m3"))
    shape = dict(heads=heads, d=d, page=page, dtype=dtype, codes=codes)
    if op == "store":
        if rng.random() < 0.5:
            return dict(op=op, requests=_log(rng, 1, 512), kv_lo=rng.choice((0, 1, 100)), kv_hi=_log(rng, 200, 2048),
                        new_lo=1, new_hi=rng.choice((1, 1, 4)), layout="fused", mix=mix, **shape)
        requests = _log(rng, 1, 16)
        new = _log(rng, 16, 32768 // requests)
        same = rng.random() < 0.5
        return dict(op=op, requests=requests, kv_lo=0, kv_hi=rng.choice((0, 1000)), new_lo=new if same else 1, new_hi=new,
                    layout=rng.choice(("fused", "streams")) if same else "fused", mix=mix, **shape)
    if op == "load":
        requests = _log(rng, 1, 32)
        kv = _log(rng, 40, 131072 // requests)
        t0 = rng.choice((0, 4, rng.randrange(kv)))
        return dict(op=op, requests=requests, kv=kv, t0=t0, t1=rng.randint(t0 + 1, max(t0 + 1, kv - rng.choice((0, 32)))),
                    mix=mix, **shape)
    if heads * group * d == 1024 * 3:
        group = 7
    if rng.random() < 0.5:                       # a few tokens a request
        new_lo, new_hi, requests = 1, rng.choice((1, 1, 1, 2, 5)), _log(rng, 1, 128)
        kv_hi = _log(rng, 64, min(65536, MOST_CODES // (requests * heads * d)))
        kv_lo = rng.choice((1, kv_hi))
    else:                                        # prompts and chunks of prompts
        requests = _log(rng, 1, 16)
        kv_hi = _log(rng, 64, 32768 // requests)
        new_hi = rng.choice((kv_hi, _log(rng, 6, kv_hi)))
        kv_lo, new_lo = rng.choice((max(1, kv_hi // 20), kv_hi)), rng.choice((1, new_hi))
    while requests * heads * group * new_hi * kv_hi > MOST_SCORES // 2:
        new_hi, kv_hi = max(1, new_hi // 2), kv_hi - kv_hi // 4 - 1
        kv_lo, new_lo = min(kv_lo, kv_hi), min(new_lo, new_hi)
    window = rng.choice((0, 0, 0, 32, _log(rng, 16, 4096)))
    causal = rng.random() < 0.9
    case = dict(op=op, requests=requests, kv_lo=kv_lo, kv_hi=kv_hi, new_lo=new_lo, new_hi=new_hi, group=group,
                softcap=rng.choice((0.0, 0.0, 30.0, 50.0)), slopes=rng.random() < 0.3, docs=rng.choice((0, 0, 0, 4)),
                prefix=causal and rng.random() < 0.2, window=window, sinks=4 if window else 0, causal=causal, mix=mix,
                **shape)
    return case


# ---------------------------------------------------------------- a case's lengths

def _lengths(case, lo, hi, salt):
    """One length a request, spread over the logarithm of the range, the largest among them."""
    rng = random.Random(case["mix"] * 16 + salt)
    n = [hi if lo >= hi else min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 0.7)), math.log(hi + 0.4))))))
         for _ in range(case["requests"])]
    n[rng.randrange(len(n))] = hi
    return np.array(n, np.int64)


def _kv_new(case):
    """Tokens in the cache before the call (attend: after it) and the step's own, a request each."""
    kv, new = _lengths(case, case["kv_lo"], case["kv_hi"], 1), _lengths(case, case["new_lo"], case["new_hi"], 2)
    return kv, np.minimum(new, kv) if case["op"] == "attend" else new


def _starts(n):
    return np.concatenate(([0], np.cumsum(n)))


def _first(case, kv, new):
    """The first position of each query token's document."""
    rng = random.Random(case["mix"] * 16 + 3)
    out = []
    for k, n in zip(kv.tolist(), new.tolist()):
        cuts = np.array(sorted({0, *(rng.randrange(k) for _ in range(case["docs"]))}))
        pos = np.arange(k - n, k)
        out.append(cuts[np.searchsorted(cuts, pos, side="right") - 1])
    return np.concatenate(out)


def _prefix(case, kv):
    rng = random.Random(case["mix"] * 16 + 4)
    return np.array([rng.randint(0, int(k) // 2 + 1) for k in kv])


def _slopes(case):
    n = case["heads"] * case["group"]
    return 2.0 ** (-8.0 * np.arange(1, n + 1) / n)


def _pages(n, page):
    return -(-n // page)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return getattr(torch, case["dtype"])


def _largest(case):
    return 127.0 if case["codes"] == "int8" else 448.0


def _key_scale(case, seed):
    rng = np.random.default_rng(int(seed))
    s = np.ones((case["heads"], case["d"]), np.float32)
    for h in range(case["heads"]):
        s[h, rng.choice(case["d"], OUTLIERS, replace=False)] = OUTLIER_SCALE
    return torch.from_numpy(s).cuda()


def _to_codes(x, largest):
    x = x.clamp_(-largest, largest)
    return x.round_().to(torch.int8) if largest == 127.0 else x.to(torch.float8_e4m3fn)


def _pool(case, n_pages, seed):
    """A pool of pages that hold rounded rows: (keys, values, scales)."""
    heads, page, d = case["heads"], case["page"], case["d"]
    gen, largest = _gen(seed), _largest(case)
    x = torch.randn((n_pages, heads, page, d), generator=gen, device="cuda").mul_(_key_scale(case, seed)[None, :, None, :])
    scales = torch.empty((n_pages, heads, 2), device="cuda")
    scales[:, :, 0] = x.abs().amax((2, 3)) / largest
    k = _to_codes(x.div_(scales[:, :, 0, None, None]), largest)
    x = torch.randn((n_pages, heads, page // 16, d, 16), generator=gen, device="cuda")
    scales[:, :, 1] = x.abs().amax((2, 3, 4)) / largest
    return k, _to_codes(x.div_(scales[:, :, 1, None, None, None]), largest), scales


def _tables(case, n, seed, width=None):
    """Block tables of requests of n tokens over a pool in no order, and the pool's number of pages."""
    need = _pages(n, case["page"])
    total = int(need.sum())
    n_pages = total + total // 8 + 1
    order = np.random.default_rng(int(seed) + 17).permutation(n_pages)[:total]
    tables = np.full((len(n), width or max(1, int(need.max()))), -1, np.int32)
    at = _starts(need)
    for r in range(len(n)):
        tables[r, :need[r]] = order[at[r]:at[r + 1]]
    return tables, n_pages


def _slots(tables, page, begin, end):
    """Slots of the positions [begin, end) of every request, in order."""
    out = [tables[r, np.arange(b, e) // page].astype(np.int64) * page + np.arange(b, e) % page
           for r, (b, e) in enumerate(zip(begin, end))]
    return np.concatenate(out)


def _up(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def prepare(case, seed):
    op, page = case["op"], case["page"]
    st = dict(case=case)
    if op == "plan":
        kv, new = _kv_new(case)
        tables, _ = _tables(case, kv, seed, _pages(case["kv_hi"] + case["new_hi"], page))
        used = int(_pages(kv, page).sum())
        need = int((_pages(kv + new, page) - _pages(kv, page)).sum())
        free = np.random.default_rng(int(seed) + 5).permutation(max(1, int(need * case["free"]))) + used
        st |= dict(kv=_up(kv, torch.int32), new=_up(new, torch.int32), tables=_up(tables, torch.int32), n=int(new.sum()),
                   free=_up(free, torch.int32), head=torch.zeros(1, dtype=torch.int32, device="cuda"))
        return st
    heads, d = case["heads"], case["d"]
    if op == "store":
        kv, new = _kv_new(case)
        tables, n_pages = _tables(case, kv + new, seed)
        st["k"], st["v"], st["scales"] = _pool(case, n_pages, seed)
        slots = _slots(tables, page, kv, kv + new)
        n, gen = len(slots), _gen(seed + 3)
        if case["layout"] == "fused":     # slices of the projection's rows: three query heads for each KV head, K, V
            rows = torch.randn((n, 5 * heads, d), generator=gen, device="cuda")
            rows[:, 3 * heads:4 * heads] *= _key_scale(case, seed)
            rows = rows.to(_dtype(case))
            st["rows_k"], st["rows_v"] = rows[:, 3 * heads:4 * heads], rows[:, 4 * heads:]
        else:                             # streams, head-major, as the archive's rows lie
            rows = torch.randn((2, case["requests"], heads, n // case["requests"], d), generator=gen, device="cuda")
            rows[0] *= _key_scale(case, seed)[:, None, :]
            rows = rows.to(_dtype(case))
            st["rows_k"], st["rows_v"] = rows[0], rows[1]
            slots = slots.reshape(case["requests"], -1)
        st["slots"] = _up(slots, torch.int64)
        st["back"] = _up(_slots(tables, page, kv // page * page, kv + new), torch.int64)
        st["touched"] = _up(np.unique(slots // page), torch.int64)
    elif op == "load":
        kv = np.full(case["requests"], case["kv"])
        tables, n_pages = _tables(case, kv, seed)
        st["k"], st["v"], st["scales"] = _pool(case, n_pages, seed)
        slots = _slots(tables, page, np.full_like(kv, case["t0"]), np.full_like(kv, case["t1"]))
        st["slots"] = _up(slots.reshape(case["requests"], -1), torch.int64)
    else:
        kv, new = _kv_new(case)
        tables, n_pages = _tables(case, kv, seed)
        st["k"], st["v"], st["scales"] = _pool(case, n_pages, seed)
        q = torch.randn((int(new.sum()), heads * case["group"], d), generator=_gen(seed + 9), device="cuda")
        st |= dict(q=q.to(_dtype(case)), tables=_up(tables, torch.int32), kv=_up(kv, torch.int32),
                   q_start=_up(_starts(new), torch.int32), max_new=int(new.max()), max_kv=int(kv.max()),
                   slopes=_up(_slopes(case), torch.float32) if case["slopes"] else None,
                   prefix=_up(_prefix(case, kv), torch.int32) if case["prefix"] else None,
                   first=_up(_first(case, kv, new), torch.int32) if case["docs"] else None)
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    return (_run_own if own else _PLAIN[case["op"]])(case, st)


def _run_own(case, st):
    from paper_2607_07144_amd import fkv
    op = case["op"]
    if op == "plan":
        p = fkv.fkv_page_plan(case["page"], st["kv"], st["new"], st["free"], st["head"], st["tables"], st["n"])
        return {"tables": st["tables"], "slots": p.slots, "positions": p.positions, "q_start": p.q_start,
                "kv_end": p.kv_end, "head": p.head, "status": p.status}
    pages = (st["k"], st["v"], st["scales"])
    if op == "store":
        fkv.fkv_page_store(pages, st["rows_k"], st["rows_v"], st["slots"])
        k, v = fkv.fkv_page_load(pages, st["back"], _dtype(case))
        return {"k": k, "v": v, "scales": st["scales"]}
    if op == "load":
        n, t = st["slots"].shape
        x = torch.empty((2, n, case["heads"], t, case["d"]), dtype=_dtype(case), device="cuda")
        fkv.fkv_page_load(pages, st["slots"], k=x[0], v=x[1])
        return {"x": x}
    out, lse = fkv.fkv_page_attend(pages, st["q"], st["tables"], st["kv"], st["q_start"], st["max_new"], st["max_kv"],
                                   softcap=case["softcap"], causal=case["causal"], window=case["window"],
                                   sinks=case["sinks"], slopes=st["slopes"], prefix=st["prefix"], first=st["first"],
                                   want_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- the plain forms, in 32 bits

def _plain_plan(case, st):
    page, kv, new, free, tables = case["page"], st["kv"].long(), st["new"].long(), st["free"], st["tables"]
    width, n = tables.shape[1], st["n"]
    old, total = (kv + page - 1) // page, (kv + new + page - 1) // page
    fits = total <= width
    need = torch.where(fits, total - old, 0)
    upto = st["head"].long() + need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= free.numel()))
    j = torch.arange(width, device="cuda")
    fresh = ok[:, None] & (j >= old[:, None]) & (j < total[:, None])
    at = ((upto - need)[:, None] + j - old[:, None]).clamp(0, free.numel() - 1)
    tables.copy_(torch.where(fresh, free[at], tables))
    q_start = torch.zeros(kv.numel() + 1, dtype=torch.int32, device="cuda")
    q_start[1:] = new.cumsum(0)
    i = torch.arange(n, device="cuda")
    r = torch.searchsorted(q_start[1:].long(), i, right=True)
    pos = kv[r] + i - q_start[r]
    slots = tables[r, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    head = torch.where(ok, upto, st["head"].long()).amax().view(1).int()
    return {"tables": tables, "slots": torch.where(ok[r], slots, -1), "positions": pos.int(), "q_start": q_start,
            "kv_end": torch.where(ok, kv + new, kv).int(), "head": head,
            "status": torch.where(ok, 0, torch.where(fits, 1, 2)).to(torch.uint8)}


def _raw(codes):
    return codes.view(torch.uint8)


def _rows(st, slots):
    """(keys, values) of flat slots as [n][heads][d] in 32 bits."""
    page = st["case"]["page"]
    p, o = slots // page, slots % page
    s = st["scales"][p]
    k = _raw(st["k"])[p, :, o].view(st["k"].dtype).float() * s[:, :, 0, None]
    v = _raw(st["v"])[p, :, o // 16, :, o % 16].view(st["v"].dtype).float() * s[:, :, 1, None]
    return k, v


def _plain_store(case, st):
    page, largest, scales, touched = case["page"], _largest(case), st["scales"], st["touched"]
    flat = st["slots"].reshape(-1)
    p, o = flat // page, flat % page
    begin = torch.full((scales.shape[0],), page, device="cuda").scatter_reduce_(0, p, o, "amin")[touched]
    kept = torch.arange(page, device="cuda") < begin[:, None]

    def write(rows, codes, which, values):
        x = rows.float() if rows.dim() == 3 else rows.float().transpose(1, 2).reshape(-1, *rows.shape[1::2])
        fine = torch.isfinite(x)
        most = torch.where(fine, x.abs(), 0.0).amax(2)
        most = torch.zeros_like(scales[:, :, 0]).scatter_reduce_(0, p[:, None].expand_as(most), most, "amax")[touched]
        s = torch.where(most < SMALLEST, 0.0, most / largest)
        was = scales[touched, :, which]
        s = torch.where(begin[:, None] > 0, torch.maximum(s, was), s)
        # what the touched pages hold before the first new token, at the new scale
        c = codes[touched].float()
        c = c * torch.where(s > 0, was / s, 1.0).reshape(*s.shape, *(1,) * (c.dim() - 2))
        c = _raw(_to_codes(c, largest))
        mask = kept.view(-1, 1, page // 16, 1, 16) if values else kept[:, None, :, None]
        _raw(codes)[touched] = torch.where(mask, c, _raw(codes)[touched])
        scales[touched, :, which] = s
        inv = torch.where(scales[:, :, which] > 0, 1.0 / scales[:, :, which], 0.0)[p][:, :, None]
        x = torch.where(fine, x * inv, torch.where(torch.isnan(x), 0.0, torch.sign(x) * largest))
        x = _raw(_to_codes(x, largest))
        if values:
            _raw(codes)[p, :, o // 16, :, o % 16] = x
        else:
            _raw(codes)[p, :, o] = x

    write(st["rows_k"], st["k"], 0, False)
    write(st["rows_v"], st["v"], 1, True)
    k, v = _rows(st, st["back"])
    return {"k": k.to(_dtype(case)), "v": v.to(_dtype(case)), "scales": scales}


def _plain_load(case, st):
    n, t = st["slots"].shape
    x = torch.empty((2, n, case["heads"], t, case["d"]), dtype=_dtype(case), device="cuda")
    k, v = _rows(st, st["slots"].reshape(-1))
    x[0] = k.view(n, t, case["heads"], case["d"]).transpose(1, 2)
    x[1] = v.view(n, t, case["heads"], case["d"]).transpose(1, 2)
    return {"x": x}


def _plain_attend(case, st):
    heads, group, d = case["heads"], case["group"], case["d"]
    q, kv, q_start = st["q"], st["kv"].long(), st["q_start"].long()
    R, nq, n = kv.numel(), st["max_new"], q.shape[0]
    # the requests' keys and values, padded to the longest
    table = st["tables"].long().clamp(min=0)
    s = st["scales"][table]
    k = _raw(st["k"])[table].view(st["k"].dtype).float() * s[..., 0, None, None]
    v = _raw(st["v"])[table].view(st["v"].dtype).float() * s[..., 1, None, None, None]
    k = k.transpose(1, 2).reshape(R, heads, -1, d)[:, :, :st["max_kv"]]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(R, heads, -1, d)[:, :, :st["max_kv"]]
    # their query tokens, padded to the most
    new = q_start[1:] - q_start[:-1]
    i = torch.arange(nq, device="cuda")
    token = (q_start[:-1, None] + i).clamp(max=n - 1)
    rows = q[token].float().view(R, nq, heads, group, d).permute(0, 2, 1, 3, 4).reshape(R, heads, nq * group, d)
    z = torch.matmul(rows, k.transpose(2, 3).contiguous()).view(R, heads, nq, group, -1)
    z.mul_(d ** -0.5)
    if case["softcap"]:
        z.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    pos = (kv - new)[:, None] + i
    j = torch.arange(z.shape[-1], device="cuda")
    if st["slopes"] is not None:
        far = (j - pos[:, :, None]).abs().float()
        z.addcmul_(far[:, None, :, None], st["slopes"].view(1, heads, 1, group, 1), value=-1.0)
    seen = (j < kv[:, None, None]).expand(R, nq, -1)
    if case["causal"]:
        past = j <= pos[:, :, None]
        seen = seen & (past if st["prefix"] is None else past | (j < st["prefix"][:, None, None]))
    if case["window"]:
        seen = seen & ((j > pos[:, :, None] - case["window"]) | (j < case["sinks"]))
    if st["first"] is not None:
        seen = seen & (j >= st["first"][token][:, :, None])
    z.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    out = torch.matmul(z.view(R, heads, nq * group, -1), v).view(R, heads, nq, group, d)
    out = torch.where(total > 0, out / total, 0.0)
    lse = (top + total.log()).squeeze(-1)
    # and back to one row a token
    t = torch.arange(n, device="cuda")
    r = torch.searchsorted(q_start[1:], t, right=True)
    i = t - q_start[r]
    return {"out": out.permute(0, 2, 1, 3, 4)[r, i].reshape(n, heads * group, d).to(q.dtype),
            "lse": lse.permute(0, 2, 1, 3)[r, i].reshape(n, heads * group)}


_PLAIN = {"plan": _plain_plan, "store": _plain_store, "load": _plain_load, "attend": _plain_attend}


# ---------------------------------------------------------------- floor

def _seen(case, kv, new):
    """(visible pairs of a query token and a key, keys that some token of the request sees), over all requests."""
    first = np.split(_first(case, kv, new), _starts(new)[1:-1]) if case["docs"] else None
    prefix = _prefix(case, kv) if case["prefix"] else None
    pairs = keys = 0
    for r, (k, n) in enumerate(zip(kv.tolist(), new.tolist())):
        pos = np.arange(k - n, k)
        end = np.full(n, k) if not case["causal"] else pos + 1 if prefix is None else np.minimum(k, np.maximum(pos + 1, prefix[r]))
        low = first[r] if first is not None else np.zeros(n, np.int64)
        begin = np.maximum(low, pos + 1 - case["window"]) if case["window"] else low
        sinks = np.maximum(0, np.minimum(np.minimum(case["sinks"], begin), end) - low) if case["window"] else 0
        pairs += int((np.maximum(0, end - begin) + sinks).sum())
        keys += min(k, int(end.max() - begin.min() + (np.max(sinks) if case["window"] else 0)))
    return pairs, keys


def work(case):
    if case["op"] == "load":
        n = case["requests"] * (case["t1"] - case["t0"]) * case["heads"] * case["d"]
        pages = case["requests"] * (_pages(case["t1"], case["page"]) - case["t0"] // case["page"])
        return {"bytes": 6 * n + 8 * pages * case["heads"] + 8 * case["requests"] * (case["t1"] - case["t0"]), "flops": 2 * n}
    kv, new = _kv_new(case)
    page = case["page"]
    if case["op"] == "plan":
        need = int((_pages(kv + new, page) - _pages(kv, page)).sum() * case["free"])
        return {"bytes": 17 * case["requests"] + 12 * int(new.sum()) + 8 * need, "flops": 0}
    if case["op"] == "store":
        # the rows, the codes they become, what the part-full pages hold before them, and the rows that come back
        n, old = int(new.sum()), int((kv % page).sum())
        pages = int((_pages(kv + new, page) - kv // page).sum())
        per = case["heads"] * case["d"]
        return {"bytes": (4 * n + 2 * n + 2 * old + 6 * (n + old)) * per + 24 * pages * case["heads"] + 16 * n + 8 * old,
                "flops": 8 * n * per}
    pairs, keys = _seen(case, kv, new)
    heads, rows, d = case["heads"], int(new.sum()) * case["heads"] * case["group"], case["d"]
    return {"bytes": 2 * keys * heads * d + 8 * _pages(keys, page) * heads + rows * (4 * d + 4) + 8 * case["requests"],
            "flops": 4 * pairs * heads * case["group"] * d}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def exact(case, seed):
    st, op, page = prepare(case, seed), case["op"], case["page"]
    if op == "plan":
        return None      # whole numbers throughout
    k, v, scales = st["k"].double(), st["v"].double(), st["scales"].double()
    if op == "load":
        x = torch.empty((2, case["requests"], case["heads"], case["t1"] - case["t0"], case["d"]), dtype=torch.float64, device="cuda")
        for r in range(case["requests"]):
            p, o = st["slots"][r] // page, st["slots"][r] % page
            x[0, r] = (k[p, :, o] * scales[p][:, :, 0, None]).transpose(0, 1)
            x[1, r] = (v[p, :, o // 16, :, o % 16] * scales[p][:, :, 1, None]).transpose(0, 1)
        return {"x": x}
    if op == "store":
        largest = _largest(case)
        v = v.transpose(3, 4).reshape(k.shape)
        rows = [x.double() if x.dim() == 3 else x.double().transpose(1, 2).flatten(0, 1) for x in (st["rows_k"], st["rows_v"])]
        slots = st["slots"].reshape(-1).cpu().numpy()
        if len(np.unique(slots // page)) > 4000:
            return None

        def near(x):
            return x.round() if largest == 127.0 else x.float().to(torch.float8_e4m3fn).double()

        cuts = np.flatnonzero((np.diff(slots) != 1) | (slots[1:] % page == 0)) + 1
        for run_ in np.split(np.arange(len(slots)), cuts):
            p, o, a, b = int(slots[run_[0]]) // page, int(slots[run_[0]]) % page, int(run_[0]), int(run_[-1]) + 1
            for which, (codes, x) in enumerate(zip((k, v), rows)):
                x = x[a:b].transpose(0, 1)
                s = x.abs().amax((1, 2)) / largest
                if o:
                    s = torch.maximum(s, scales[p, :, which])
                    grow = (scales[p, :, which] / s)[:, None, None]
                    codes[p, :, :o] = torch.where(grow < 1, near(codes[p, :, :o] * grow), codes[p, :, :o])
                scales[p, :, which] = s
                codes[p, :, o:o + b - a] = near(x / s[:, None, None])
        p, o = st["back"] // page, st["back"] % page
        return {"k": k[p, :, o] * scales[p][:, :, 0, None], "v": v[p, :, o] * scales[p][:, :, 1, None], "scales": scales}
    kv, new = _kv_new(case)
    heads, group, d = case["heads"], case["group"], case["d"]
    if _seen(case, kv, new)[0] * heads * group * d * 4 > 2 * MOST_PAIRS:
        return None
    start = _starts(new)
    out = torch.zeros((int(new.sum()), heads * group, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        n, m, a = int(kv[r]), int(new[r]), int(start[r])
        t = st["tables"][r, :_pages(n, page)].long()
        keys = (k[t] * scales[t][:, :, 0, None, None]).transpose(0, 1).reshape(heads, -1, d)[:, :n]
        values = (v[t] * scales[t][:, :, 1, None, None, None]).permute(1, 0, 2, 4, 3).reshape(heads, -1, d)[:, :n]
        j = torch.arange(n, device="cuda")
        pos = torch.arange(n - m, n, device="cuda")[:, None]
        hide = torch.zeros((m, n), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hide |= (j > pos) & (j >= (int(st["prefix"][r]) if case["prefix"] else 0))
        if case["window"]:
            hide |= (pos - j >= case["window"]) & (j >= case["sinks"])
        if case["docs"]:
            hide |= j < st["first"][a:a + m, None]
        for h in range(heads * group):
            x = torch.mm(st["q"][a:a + m, h].double(), keys[h // group].t().contiguous()) / math.sqrt(d)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            if case["slopes"]:
                x = x - float(st["slopes"][h]) * (pos - j).abs()
            x.masked_fill_(hide, -math.inf)
            lse[a:a + m, h] = torch.logsumexp(x, 1)
            x = torch.nan_to_num(torch.exp(x - lse[a:a + m, h, None]), nan=0.0)
            out[a:a + m, h] = torch.mm(x, values[h // group])
    return {"out": out, "lse": lse}
