"""Plain forms of the paged 8-bit cache in 64 bits (and, where a result is defined bit for bit, in the fp32
operations that define it), on the CPU, from the definitions in include/fkv.h."""
import math

import numpy as np
import torch

LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def plan(page, kv, new, free, head, tables, n_tokens):
    """One request after another.  tables is updated; returns a dict of the outputs."""
    tables = tables.copy()
    width = tables.shape[1]
    slots, positions = np.full(n_tokens, -1, np.int64), np.full(n_tokens, -1, np.int32)
    status, end, start = [], [], [0]
    head = min(max(head, 0), len(free))
    asked, taken, mark, row = head, head, head, 0
    for r, (k, n) in enumerate(zip(kv.tolist(), new.tolist())):
        rows = max(n, 0)
        old, total = -(-max(k, 0) // page), -(-(max(k, 0) + rows) // page)
        st = 3 if k < 0 or n < 0 or row + rows > n_tokens else 2 if total > width or k + rows > 2 ** 31 - 1 else 0
        need = total - old if st == 0 else 0
        asked += need
        if st == 0 and need and asked > len(free):
            st = 1
        if st == 0:
            mark = max(mark, asked)
            if need:
                taken = asked
                tables[r, old:total] = free[asked - need:asked]
        for i in range(min(rows, max(0, n_tokens - row))):
            positions[row + i] = max(k, 0) + i
            if st == 0:
                slots[row + i] = int(tables[r, (k + i) // page]) * page + (k + i) % page
        row += rows
        start.append(min(row, n_tokens))
        status.append(st)
        end.append(k + n if st == 0 else k)
    return dict(tables=tables, slots=slots, positions=positions, q_start=np.array(start, np.int32),
                kv_end=np.array(end, np.int32), head=mark, next_head=taken, status=np.array(status, np.uint8))


def to_codes(x, dtype):
    """fp32 values to codes, to nearest, ties to even."""
    x = x.clamp(-LARGEST[dtype], LARGEST[dtype])
    return x.round().to(torch.int8) if dtype == torch.int8 else x.to(torch.float8_e4m3fn)


def runs(slots, page):
    """(first row, rows) of each run of a flat slot map."""
    out, i = [], 0
    while i < len(slots):
        n = 1
        if slots[i] >= 0:
            while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] % page:
                n += 1
            out.append((i, n))
        i += n
    return out


def store(k, v, scales, rows_k, rows_v, slots):
    """CPU tensors; k, v, scales are updated.  rows [n][heads][d].  Every value as the fp32 operations give it."""
    n_pages, heads, page, d = k.shape
    inv_largest = np.float32(1.0) / np.float32(LARGEST[k.dtype])
    for i, n in runs(slots, page):
        p, o = divmod(int(slots[i]), page)
        if p >= n_pages:
            continue
        for which, (codes, rows) in enumerate(((k, rows_k), (v, rows_v))):
            c = codes[p] if which == 0 else codes[p].transpose(-1, -2).reshape(heads, page, d)
            c = c.float()
            x = rows[i:i + n].float().transpose(0, 1)
            fine = torch.isfinite(x)
            a = torch.where(fine, x.abs(), 0.0).amax((1, 2))
            s = torch.where(a < 2.0 ** -90, 0.0, a * float(inv_largest))
            if o:
                was = scales[p, :, which].clone()
                s = torch.maximum(s, was)
                grown = to_codes(c[:, :o] * torch.where(s > 0, was / s, 1.0)[:, None, None], k.dtype).float()
                c[:, :o] = torch.where((s > was)[:, None, None], grown, c[:, :o])
            inv = torch.where(s > 0, 1.0 / s, 0.0)[:, None, None]
            y = torch.where(fine, x * inv, torch.where(x.isnan(), 0.0, x.sign() * LARGEST[k.dtype]))
            c[:, o:o + n] = to_codes(y, k.dtype).float()
            scales[p, :, which] = s
            c = c.to(k.dtype)
            if which == 0:
                codes[p] = c
            else:
                codes[p] = c.view(torch.uint8).reshape(heads, page // 16, 16, d).transpose(-1, -2).contiguous().view(k.dtype)


def values(k, v, scales):
    """All rows of the pool in 64 bits: two tensors [n_pages][heads][page][d]."""
    n_pages, heads, page, d = k.shape
    kk = k.double() * scales[:, :, 0, None, None].double()
    vv = v.double().transpose(-1, -2).reshape(k.shape) * scales[:, :, 1, None, None].double()
    return kk, vv


def attend(k, v, scales, q, tables, kv_len, q_start, scale, softcap=0.0, causal=True, window=0, sinks=0, slopes=None,
           prefix=None, first=None):
    """Returns (out, lse, bound on |out| errors, bound on lse errors) in 64 bits, CPU.

    The bounds hold for fp32 scores and sums and weights rounded to binary16: a dot product of d terms in fp32 is
    within (d + 8) 2^-24 sum |q k| of exact, tanh, the bias and the change to base 2 within 2^-21 of their own sizes;
    a score error e changes a weight by a factor within 1 +- 2e (e < 1/4), and a rounding to binary16 by 1 +- 2^-11."""
    n_pages, heads, page, d = k.shape
    kk, vv = values(k, v, scales)
    n, q_heads, _ = q.shape
    group = q_heads // heads
    out, lse = torch.zeros((n, q_heads, d), dtype=torch.float64), torch.full((n, q_heads), -math.inf, dtype=torch.float64)
    off, loff = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(len(kv_len)):
        kv, b, e = int(kv_len[r]), int(q_start[r]), int(q_start[r + 1])
        if kv == 0 or b == e:
            continue
        t = tables[r, :-(-kv // page)].long()
        there = ((t >= 0) & (t < n_pages)).repeat_interleave(page)[:kv]
        t = t.clamp(0, n_pages - 1)
        keys = kk[t].transpose(0, 1).reshape(heads, -1, d)[:, :kv]
        vals = torch.where(there[None, :, None], vv[t].transpose(0, 1).reshape(heads, -1, d)[:, :kv], 0.0)
        keys = torch.where(there[None, :, None], keys, 0.0)
        j = torch.arange(kv)
        for i in range(b, e):
            pos = kv - (e - b) + (i - b)
            see = there.clone()
            if causal:
                see &= (j <= pos) | (j < (int(prefix[r]) if prefix is not None else 0))
            if window:
                see &= (j > pos - window) | (j < sinks)
            if first is not None:
                see &= j >= int(first[i])
            if not see.any():
                continue
            ks, vs = keys[:, see].repeat_interleave(group, 0), vals[:, see].repeat_interleave(group, 0)
            x = q[i].double()
            z = (ks @ x[:, :, None])[..., 0] * scale
            err = (ks.abs() @ x.abs()[:, :, None])[..., 0] * abs(scale) * (d + 8) * 2.0 ** -24
            if softcap:
                z = softcap * torch.tanh(z / softcap)
                err = err + softcap * 2.0 ** -21
            if slopes is not None:
                bias = slopes.double()[:, None] * (j[see] - pos).abs()
                z = z - bias
                err = err + bias * 2.0 ** -21
            err = err + z.abs() * 2.0 ** -21
            m = z.amax(1, keepdim=True)
            w = torch.exp(z - m)
            total = w.sum(1, keepdim=True)
            w = w / total
            lse[i] = (m + total.log())[:, 0]
            out[i] = (w[:, None] @ vs)[:, 0]
            # keys whose weight is below 2^-30 of all do not count, whatever their scores' error
            big = torch.where(w > 2.0 ** -30, err, 0.0).amax(1)
            assert big.max() < 0.25
            off[i] = (2.0 ** -11 + 4 * big[:, None] + 2.0 ** -18) * (w[:, None] @ vs.abs())[:, 0]
            loff[i] = 2 * big + lse[i].abs() * 2.0 ** -20 + 2.0 ** -18
    return out, lse, off, loff
