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


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("heads,group,new", [(1, 2, 1), (2, 4, 40), (16, 3, 130), (16, 5, 130)])
@pytest.mark.parametrize("codes", [INT8, E4M3])
@pytest.mark.parametrize("level", [2.0 ** 24 * 1.5, 2.0 ** 25 * 1.5, 2.0 ** 26 * 1.5])
def test_tiles_a_rounding_apart(fkv, listed, heads, group, new, codes, level):
    """Scores of 2^24 and more, where fp32's steps are 2, 4 and 8, the second tile's 8 above the first's in base 2: all values
    are alike, so the result is that value."""
    page, d, kv = 64, 16, 320
    k, v = torch.zeros((5, heads, page, d)), torch.full((5, heads, page // 16, d, 16), 96.0)
    k[:, :, :, 0] = 96.0
    k[1:, :, :, 1] = 1.0
    scales = torch.tensor([32.0, 0.25]).repeat(5, heads, 1)
    q = torch.zeros((new, heads * group, d))
    q[:, :, 0], q[:, :, 1] = level / (96 * 32), 0.25
    assert q.half().float().equal(q)
    pool = (k.to(codes).cuda(), v.to(codes).cuda(), scales.cuda())
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    args = (pool, q.half().cuda(), i32([[0, 1, 2, 3, 4]]), i32([kv]), i32([0, new]))
    how = dict(scale=0.6931472, causal=False, want_lse=True)
    if listed:
        every = torch.arange(5, dtype=torch.int32, device="cuda").repeat(new, heads, 1)
        out, lse = fkv.fkv_page_attend_selected(*args, every, new, kv, **how)
    else:
        out, lse = fkv.fkv_page_attend(*args, new, kv, **how)
    # weights of 11 bits, their sums and what binary16 holds of 24
    assert ((out.cpu().double() - 24).abs() <= 24 * (2.0 ** -11 + 2.0 ** -11 + 2.0 ** -16)).all()
    assert torch.isfinite(lse).all()
