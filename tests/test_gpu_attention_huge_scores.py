"""Scores far beyond what an exponent's rounding allows: the largest probability is still one.

Scores are exact by construction (one column, powers of two and small whole numbers), so the softmax is: equal shares for
the keys with the largest score that a row sees, nothing for all others, which lie at least 2^24 below.  What may be off is
the mean of up to n values (n 2^-24 of their largest, and the unit of a probability where it is rounded to 16 bits) and the
output's rounding; of lse 3 units of 2^-24 of itself."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests.attention_reference import UNIT, visible

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dt,up", [(F32, 30), (F32, 60), (BF16, 30), (BF16, 60), (F16, 24), (F16, 27)])
@pytest.mark.parametrize("b,n,d,row", [(3, 12, 32, 32), (3, 40, 64, 64), (2, 100, 128, 128), (2, 40, 64, 65), (2, 300, 64, 64),
                                       (2, 300, 128, 128), (2, 200, 64, 65), (40, 150, 64, 64), (2, 20, 128, 128)])
@pytest.mark.parametrize("window", [(-1, 0), (3, 3), (-1, -1)])
def test_largest_scores_share_the_row(b, n, d, row, window, dt, up):
    gen = torch.Generator(device="cuda").manual_seed(n + up)
    room = torch.zeros((3, b, n, 2, row), dtype=dt, device="cuda")
    q, k, v = room[0, ..., :d], room[1, ..., :d], room[2, ..., :d]
    ranks = torch.randint(-8, 8, (b, n, 2), generator=gen, device="cuda")
    half = min(up // 2, 12)                                # 15 * 2^12 is within binary16
    q[..., 1] = 2.0 ** (up - half)
    k[..., 1] = (ranks * 2 + 1).to(dt) * 2.0 ** half
    v.copy_(torch.randn((b, n, 2, d), generator=gen, device="cuda"))
    out, lse = B.gs_attention_forward(q, k, v, scale=1.0, window=window)
    see = visible(n, n, n, n, window, "cuda")
    s = (ranks * 2 + 1).double().permute(0, 2, 1)[:, :, None, :].expand(b, 2, n, n).masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s == top).double()
    count = p.sum(-1, keepdim=True)
    vd = v.double().permute(0, 2, 1, 3)
    want = (p / count) @ vd
    bound = (n + 4) * 2.0 ** -24 * (p / count) @ vd.abs() + UNIT[dt] * want.abs()
    if dt != F32:
        bound = bound + 2 * UNIT[dt] * (p / count) @ vd.abs()
    if dt == F16:
        bound = bound + 2.0 ** -25
    off = (out.double().permute(0, 2, 1, 3) - want).abs()
    assert not torch.isnan(out).any() and (off <= bound).all(), (off - bound).max().item()
    lse_want = top.squeeze(-1) * 2.0 ** up + count.squeeze(-1).log()
    assert ((lse.double() - lse_want).abs() <= 3 * 2.0 ** -24 * lse_want.abs()).all()
    assert not torch.isinf(lse).any()
