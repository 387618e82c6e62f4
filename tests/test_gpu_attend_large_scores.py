"""Attention to all pages where scores are far beyond what an exponential holds: finite, and a row's best key has all the
weight."""
import pytest
import torch

from test_gpu_attend_selected_ranges import best, inputs, up

pytestmark = pytest.mark.gpu

INT8, E4M3, F16 = torch.int8, torch.float8_e4m3fn, torch.float16


@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("page,heads,group,d", [(64, 2, 3, 128), (64, 2, 8, 64), (16, 1, 4, 80), (48, 2, 1, 256)])
@pytest.mark.parametrize("lengths", [[(200, 2), (130, 1)], [(330, 128), (70, 3)], [(3000, 40)]])
@pytest.mark.parametrize("how", [{}, dict(slopes=0.01), dict(softcap=1e36)])
@pytest.mark.parametrize("power", [22, 111])
def test_large_scores(fkv, codes, page, heads, group, d, lengths, how, power):
    pool, tables, kv, starts, q, _ = inputs(page, heads, group, d, codes, F16, lengths, 4, d + page)
    pool[2][:, :, 0] *= 2.0 ** power
    q = torch.where(q.abs() < 2.0 ** -5, 2.0 ** -5, q).to(F16)
    out, lse = fkv.fkv_page_attend(up(pool), q.cuda(), tables.cuda(), kv.cuda(), starts.cuda(), max(n for _, n in lengths),
                                   max(t for t, _ in lengths), want_lse=True, scale=2.0 ** -3,
                                   **{k: torch.full((heads * group,), x, device="cuda") if k == "slopes" else x for k, x in how.items()})
    got, lse = out.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all() and torch.isfinite(lse).all()
    every = torch.arange(tables.shape[1], dtype=torch.int32).repeat(len(q), heads, 1)
    for r in range(len(kv)):
        every[int(starts[r]):int(starts[r + 1])][every[int(starts[r]):int(starts[r + 1])] * page >= int(kv[r])] = -1
    want, top, err, sure = best(pool, tables, kv, starts, q, every, 2.0 ** -3, gap=40.0 + 0.01 * max(t for t, _ in lengths))
    # (best's errors take sums of 255 units of a scale, which sums of codes stay below; a bias is 0.01 a token; a cap keeps the
    # order and takes t^2 / 3 of a score, less than 2^-12 of those up to 0.027 of it; a weight of 1 times its value scale is
    # rounded to 11 bits, and of 3000 other keys' weights less than e^-40 each is left)
    assert top.max() < 2.7e34 and sure.float().mean() > 0.5
    half = torch.finfo(F16).eps / 2
    assert ((got - want).abs() <= (half + 2.0 ** -11 + 2.0 ** -18) * want.abs() + 2.0 ** -25)[sure].all()
    assert ((lse - top).abs() <= err + top.abs() * 2.0 ** -12 + 30)[sure].all()
