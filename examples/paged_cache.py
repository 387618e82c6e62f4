"""A serving loop around the archive: prompts and decoding steps on the paged 8-bit cache, then the old positions
from the pages into the archive, and back from the archive into pages.

    python examples/paged_cache.py

One layer of a small model, random K/V rows and queries.  A batch of prompts of different lengths is planned
(block tables and slots from the lengths, on the GPU), stored and attended to; decoding steps add one token a
sequence; the positions between the sinks and the recent window are loaded from the pages, assigned and encoded
by the archive, rehydrated from it, and stored into fresh pages, over which the last step's attention is taken
again.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2607_07144_amd import fkv
from paper_2607_07144_amd.workloads import RECENT, SINKS

HEADS, GROUP, D, PAGE = 4, 2, 64, 16           # KV heads, query heads of each, channels, tokens of a page
STAGES, CODEWORDS, ALPHABET = 4, 256, 256      # the archive's quantizer


def rows(gen, n, heads):
    return torch.randn((n, heads, D), generator=gen, device="cuda").to(torch.float16)


class Cache:
    """What a program keeps between steps: the pool, the block tables, the lengths and the free list."""

    def __init__(self, lengths, steps, dtype=torch.int8):
        batch, most = len(lengths), max(lengths) + steps
        self.width = -(-most // PAGE)
        self.pages = fkv.fkv_pages(batch * self.width, PAGE, HEADS, D, dtype)
        self.tables = torch.full((batch, self.width), -1, dtype=torch.int32, device="cuda")
        self.kv = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(batch * self.width, device="cuda").to(torch.int32)
        self.head = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.most = most

    def step(self, new, n, max_new, k, v, q, **scores):
        """One step: new[r] tokens of every sequence, n in all, at most max_new of one."""
        p = fkv.fkv_page_plan(PAGE, self.kv, new, self.free, self.head, self.tables, n)
        fkv.fkv_page_store(self.pages, k, v, p.slots)
        out, _ = fkv.fkv_page_attend(self.pages, q, self.tables, p.kv_end, p.q_start, max_new, self.most, **scores)
        self.kv, self.head = p.kv_end, p.next_head
        return out, p

    def slots(self, r, begin, end):
        t = torch.arange(begin, end, device="cuda")
        return self.tables[r].long()[t // PAGE] * PAGE + t % PAGE


def archive(x, seed=5):
    """Archives streams x f16 [n_streams][T][d] and gives back their reconstruction, from the archive alone."""
    ns, T, d = x.shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pick = torch.stack([torch.randperm(T, generator=gen, device="cuda").repeat(-(-CODEWORDS // T))[:CODEWORDS]
                        for _ in range(ns)])
    books = torch.zeros((ns, STAGES, CODEWORDS, d), dtype=torch.float16, device="cuda")
    books[:, 0] = x[torch.arange(ns, device="cuda")[:, None], pick]
    for s in range(1, STAGES):
        books[:, s] = books[:, 0] * 0.5 ** (s + 1)
    sb = torch.arange(ns, dtype=torch.int32, device="cuda")
    for stage in range(STAGES):                 # a Lloyd iteration a stage
        sym, _ = fkv.fkv_rvq_assign(x, books, sb, 0, T)
        fkv.fkv_kmeans_step(x, books, sb, 0, T, sym, stage)
    codec = fkv.Codec(ALPHABET)
    _, points, _ = fkv.fkv_rvq_assign_encode(codec, x, books, sb, 0, T)
    qs = torch.arange(ns, device="cuda", dtype=torch.int32).repeat_interleave(T)
    qt = torch.arange(T, device="cuda", dtype=torch.int32).repeat(ns)
    back = fkv.fkv_rehydrate(codec, points, T * STAGES, STAGES, books, sb, qs, qt)
    return back.view(ns, T, d), points


def main(lengths=(200, 75, 310), steps=8, seed=1, dtype=torch.int8):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    batch = len(lengths)
    cache = Cache(lengths, steps, dtype)
    # the prompts: every sequence's rows behind one another, its first 16 tokens seen by all of it
    new = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    n = sum(lengths)
    k, v, q = rows(gen, n, HEADS), rows(gen, n, HEADS), rows(gen, n, HEADS * GROUP)
    kept = [[k[sum(lengths[:r]):sum(lengths[:r + 1])]] for r in range(batch)], \
           [[v[sum(lengths[:r]):sum(lengths[:r + 1])]] for r in range(batch)]
    prompt, _ = cache.step(new, n, max(lengths), k, v, q, prefix=torch.full_like(new, 16), softcap=50.0)
    print("prompts of %s tokens: %d rows of attention" % (", ".join(map(str, lengths)), prompt.shape[0]))
    # decoding, a token a sequence
    one = torch.ones_like(new)
    for _ in range(steps):
        k, v, q = rows(gen, batch, HEADS), rows(gen, batch, HEADS), rows(gen, batch, HEADS * GROUP)
        for r in range(batch):
            kept[0][r].append(k[r:r + 1]), kept[1][r].append(v[r:r + 1])
        out, plan = cache.step(one, batch, 1, k, v, q)
    print("%d decoding steps, %d of %d pages in use" % (steps, int(cache.head), cache.free.numel()))
    # one sequence's old positions into the archive and back, into pages of their own
    r = max(range(batch), key=lambda i: lengths[i])
    T = lengths[r] + steps
    begin, end = SINKS, T - RECENT
    x = torch.empty((2, 1, HEADS, end - begin, D), dtype=torch.float16, device="cuda")
    fkv.fkv_page_load(cache.pages, cache.slots(r, begin, end)[None], k=x[0], v=x[1])
    back, points = archive(x.view(2 * HEADS, end - begin, D))
    whole = torch.empty((2, 1, HEADS, T, D), dtype=torch.float16, device="cuda")
    fkv.fkv_page_load(cache.pages, cache.slots(r, 0, T)[None], k=whole[0], v=whole[1])   # sinks and window as they are
    whole[:, 0, :, begin:end] = back.view(2, HEADS, end - begin, D)
    again = Cache((T,), 0, dtype)
    p = fkv.fkv_page_plan(PAGE, again.kv, torch.tensor([T], dtype=torch.int32, device="cuda"), again.free, None,
                          again.tables, T)
    fkv.fkv_page_store(again.pages, whole[0], whole[1], p.slots[None])
    last = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    restored, _ = fkv.fkv_page_attend(again.pages, q[r:r + 1], again.tables, p.kv_end, last, 1, T)
    off = float((restored.float() - out[r:r + 1].float()).norm() / out[r].float().norm())
    print("sequence %d: positions %d to %d archived in %d bytes of points (%d in the pages), "
          "attention over the restored rows %.2f off" % (r, begin, end - 1, points.numel() * 8,
                                                        2 * HEADS * (end - begin) * D, off))
    return dict(prompt=prompt, out=out, q=q, restored=restored, off=off, kept=kept, cache=cache, row=r, plan=plan)


if __name__ == "__main__":
    main()
