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
