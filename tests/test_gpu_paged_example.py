"""The serving loop of examples/paged_cache.py: its last decoding step against attention over the rows themselves,
and the archive's way back."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_serving_loop(fkv, dtype):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import paged_cache
    finally:
        sys.path.pop(0)
    r = paged_cache.main(lengths=(70, 33, 150), steps=5, dtype=dtype)
    kv = r["cache"].kv.tolist()
    assert kv == [75, 38, 155] and r["plan"].status.tolist() == [0, 0, 0]
    group, d = paged_cache.GROUP, paged_cache.D
    for s in range(3):
        k = torch.cat(r["kept"][0][s]).double().cpu().repeat_interleave(group, 1)
        v = torch.cat(r["kept"][1][s]).double().cpu().repeat_interleave(group, 1)
        z = torch.einsum("hd,thd->ht", r["q"][s].double().cpu(), k) / math.sqrt(d)
        want = torch.einsum("ht,thd->hd", z.softmax(1), v)
        # rows held in 8 bits: half a step of 1/127 of a page's largest element (about 4), or 2^-4 of an
        # element, in keys and values; an error e of the keys moves a score by |q| e / 8, about 1 e at random
        got = r["out"][s].double().cpu()
        assert (got - want).norm() / want.norm() < (0.05 if dtype == torch.int8 else 0.15)
    # 4 x 256 codewords for 119 tokens of each stream reconstruct them closely
    assert r["off"] < 0.3 and torch.isfinite(r["restored"]).all()


def test_prompt_step_in_a_graph(fkv):
    """plan, store and the attention of prompts captured once; replays with other rows give the eager results."""
    from test_gpu_pages import _state, _step, bits, make_rows
    new = (30, 5, 12)
    pages, st = _state(fkv, new)
    _step(fkv, pages, st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p, out, lse = _step(fkv, pages, st)
    for i in range(4):
        st["k"].copy_(make_rows(47, 2, 64, torch.float16, 50 + i))
        st["q"].copy_(make_rows(47, 8, 64, torch.float16, 60 + i))
        st["kv"].copy_(torch.tensor([30 + i, 2990 - 300 * i, 3 + i]))
        before = [x.clone() for x in pages]
        g.replay()
        torch.cuda.synchronize()
        kept = [bits(x) for x in (*pages, out, lse, p.slots)]
        for x, y in zip(pages, before):
            x.copy_(y)
        want = _step(fkv, pages, st)
        assert all(torch.equal(a, bits(b)) for a, b in zip(kept, (*pages, want[1], want[2], want[0].slots))), i
