"""Plain forms of the calls for long contexts on the paged cache (rotated rows, boxes, selection, attention over selected
pages), on the CPU, from the definitions in include/fkv.h: in the fp32 operations that define a result bit for bit where
there are such, else in 64 bits."""
import math
import random

import numpy as np
import torch

import pages_reference as pages


def slot_map(lengths, page, n_pages, seed):
    """(slots, positions, tables) of requests given as (tokens before, new tokens), on pages in no order."""
    ids = list(range(n_pages))
    random.Random(seed).shuffle(ids)
    slots, positions, tables = [], [], []
    for kv, new in lengths:
        t = [ids.pop() for _ in range(-(-(kv + new) // page))]
        tables.append(t)
        slots += [t[p // page] * page + p % page for p in range(kv, kv + new)]
        positions += range(kv, kv + new)
    return np.array(slots, np.int64), np.array(positions, np.int32), tables


def pool(n_pages, heads, page, d, dtype, seed):
    """Codes and scales of any pages, CPU: (k, v, scales)."""
    g = torch.Generator().manual_seed(seed)
    most = pages.LARGEST[dtype]
    k = pages.to_codes(torch.randn((n_pages, heads, page, d), generator=g) * most / 4, dtype)
    v = pages.to_codes(torch.randn((n_pages, heads, page // 16, d, 16), generator=g) * most / 4, dtype)
    return k, v, torch.rand((n_pages, heads, 2), generator=g) * (4 / most) + 0.5 / most


def table(n_pos, rot, base=10000.0):
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.stack((a.cos(), a.sin()), -1).float()


def turned(x, positions, tab, pairs):
    """Rows [n][heads][d] in fp32, the table's channels turned: each product and sum rounded to fp32."""
    rot = 2 * tab.shape[1]
    cs = tab[torch.as_tensor(positions).long().clamp(0, len(tab) - 1)][:, None]
    c, s = cs[..., 0], cs[..., 1]
    y = x.float().clone()
    at = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = y[..., at[0]].clone(), y[..., at[1]].clone()
    y[..., at[0]] = torch.sub(torch.mul(a, c), torch.mul(b, s))
    y[..., at[1]] = torch.add(torch.mul(b, c), torch.mul(a, s))
    return y


def box_of(k, tokens):
    """The box [heads][2][d] of a page's codes [heads][page][d] over its first tokens, as fp32."""
    f = k[:, :tokens].float()
    return torch.stack((f.amin(1), f.amax(1)), 1)


def append(k, v, scales, rows_k, rows_v, slots, positions=None, tab=None, pairs=False, boxes=None):
    """CPU tensors; k, v, scales and boxes (fp32 values of codes) are updated."""
    rows_k = rows_k.float() if tab is None else turned(rows_k, positions, tab, pairs)
    pages.store(k, v, scales, rows_k, rows_v, slots)
    if boxes is not None:
        for i, n in pages.runs(slots, k.shape[2]):
            p, o = divmod(int(slots[i]), k.shape[2])
            if 0 <= p < k.shape[0]:
                boxes[p] = box_of(k[p], o + n)


# ---------------------------------------------------------------- selection

def whole_rows(q):
    """Rows [..][d] as whole numbers, and the exponents e of their powers of two."""
    x = q.float()
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), 0.0).amax(-1)
    ex = (most.contiguous().view(torch.int32) >> 23) & 0xff
    e = torch.where(ex == 0, 0, (133 - ex).clamp(max=126))
    w = torch.where(x.isnan(), 0.0, (x.double() * 2.0 ** e[..., None].double()).clamp(-127, 127).round())
    return w.long(), e


def select(boxes, scales, q, tables, kv_len, q_start, page, n_select, keep_first, keep_last, causal, out):
    """boxes: codes, CPU; out [n_tokens][heads][n_select] is updated."""
    n_pages, heads, _, d = boxes.shape
    group = q.shape[1] // heads
    box = boxes.float()
    if boxes.dtype != torch.int8:
        box = torch.stack((torch.floor(box[:, :, 0] / 4), torch.ceil(box[:, :, 1] / 4)), 2)
    box = box.long()
    w, e = whole_rows(q)
    for r in range(len(kv_len)):
        kv, b, end = int(kv_len[r]), int(q_start[r]), int(q_start[r + 1])
        for i in range(b, end):
            pos = kv - (end - b) + (i - b)
            seen = max(0, -(-(min(pos + 1, kv) if causal else kv) // page))
            out[i] = -1
            if seen <= n_select:
                out[i, :, :seen] = torch.arange(seen, dtype=torch.int32)
                continue
            t = tables[r, :seen].long()
            there = (t >= 0) & (t < n_pages)
            t = torch.where(there, t, 0)
            for h in range(heads):
                best = torch.full((seen,), -math.inf)
                for g in range(h * group, (h + 1) * group):
                    s = torch.maximum(box[t, h, 0] * w[i, g], box[t, h, 1] * w[i, g]).sum(-1)
                    x = (s.float() * scales[t, h, 0]) * torch.tensor(2.0 ** -int(e[i, g]), dtype=torch.float32)
                    best = torch.maximum(best, torch.where(x.isnan() | ~there, -math.inf, x))
                kept = list(range(keep_first)) + list(range(seen - keep_last, seen))
                rest = sorted(range(keep_first, seen - keep_last), key=lambda p: (-float(best[p]), p))
                out[i, h] = torch.tensor(sorted(kept + rest[:n_select - keep_first - keep_last]), dtype=torch.int32)


# ---------------------------------------------------------------- attention to lists

def attend_selected(k, v, scales, q, tables, kv_len, q_start, selected, scale, softcap=0.0, causal=True, window=0, sinks=0,
                    slopes=None, prefix=None, first=None, shifted=0):
    """As pages_reference.attend, whose bounds hold here too, over the listed pages' keys, each as often as listed.

    shifted: tiles of 64 keys of a list whose int8 codes are summed as c + 128, at most 255, and 128 times the other factors'
    sum taken off.  A score's d + 8 roundings are then of sums up to 255 scale sum |q|; those of the values, 64 a tile and 16
    at the end, of sums up to 255 of the weights times value scales, and as many of 128 times those."""
    n_pages, heads, page, d = k.shape
    kk, vv = pages.values(k, v, scales)
    n, q_heads, _ = q.shape
    group = q_heads // heads
    out, lse = torch.zeros((n, q_heads, d), dtype=torch.float64), torch.full((n, q_heads), -math.inf, dtype=torch.float64)
    off, loff = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(len(kv_len)):
        kv, b, e = int(kv_len[r]), int(q_start[r]), int(q_start[r + 1])
        for i in range(b, e):
            pos = kv - (e - b) + (i - b)
            for h in range(heads):
                column = selected[i, h].long()
                column = column[(column >= 0) & (column < -(-kv // page))]
                column = column[(tables[r, column] >= 0) & (tables[r, column] < n_pages)]
                if not len(column):
                    continue
                ids = tables[r, column].long()
                j = (column[:, None] * page + torch.arange(page)).flatten()
                see = j < kv
                if causal:
                    see &= (j <= pos) | (j < (int(prefix[r]) if prefix is not None else 0))
                if window:
                    see &= (j > pos - window) | (j < sinks)
                if first is not None:
                    see &= j >= int(first[i])
                if not see.any():
                    continue
                ks, vs = kk[ids, h].reshape(-1, d)[see], vv[ids, h].reshape(-1, d)[see]
                for hq in range(h * group, (h + 1) * group):
                    x = q[i, hq].double()
                    z = ks @ x * scale
                    err = (ks.abs() @ x.abs()) * abs(scale) * (d + 8) * 2.0 ** -24
                    if shifted:
                        both = scales[ids, h].double().repeat_interleave(page, 0)[see]
                        err = both[:, 0] * x.abs().sum() * 255 * abs(scale) * (d + 8) * 2.0 ** -24
                    if softcap:
                        z = softcap * torch.tanh(z / softcap)
                        err = err + softcap * 2.0 ** -21
                    if slopes is not None:
                        bias = float(slopes[hq]) * (j[see] - pos).abs().double()
                        z = z - bias
                        err = err + bias * 2.0 ** -21
                    err = err + z.abs() * 2.0 ** -21
                    m = z.max()
                    w = torch.exp(z - m)
                    total = w.sum()
                    w = w / total
                    lse[i, hq] = m + total.log()
                    out[i, hq] = w @ vs
                    big = torch.where(w > 2.0 ** -30, err, 0.0).max()
                    assert big < 0.25
                    off[i, hq] = (2.0 ** -11 + 4 * big + 2.0 ** -18) * (w @ vs.abs())
                    if shifted:
                        off[i, hq] += (64 * shifted + 16) * 2.0 ** -24 * (255 + 128) * (w @ both[:, 1])
                    loff[i, hq] = 2 * big + lse[i, hq].abs() * 2.0 ** -20 + 2.0 ** -18
    return out, lse, off, loff
