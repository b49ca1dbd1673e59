"""How fp32 sums over positions are rounded where the products are the tensor cores'."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("row", [0, 1], ids=["tma", "no_tma"])
def test_sums_over_key_blocks_are_rounded_to_nearest(d, row):
    """Equal scores: every probability is one before the quotient, and n = 128 makes the quotient exact.  A value
    1 + 2^-12 - 2^-23 splits into 1 and eleven bits below; sixteen of them add up exactly in 24 bits.  What may be off is
    the addition of eight blocks: half a unit, 2^-24, of running sums of 16, 32, .. 128, against a result of 128 values:
    16 * 36 / 128 = 4.5 times 2^-24.  One running sum on the tensor cores, which round
    towards zero, was off by 20 times 2^-24."""
    n, value = 128, 1.0 + 2.0 ** -12 - 2.0 ** -23
    room = torch.zeros((3, 4, n, 2, d + row), device="cuda")
    q, k, v = room[0, ..., :d], room[1, ..., :d], room[2, ..., :d]
    k.normal_()
    v.fill_(value)
    out, lse = B.gs_attention_forward(q, k, v)
    off = (out.double() - value).abs().max().item()
    assert off <= 4.5 * 2.0 ** -24 * value, off / 2.0 ** -24
    assert (lse.double() - math.log(n)).abs().max().item() <= 4 * 2.0 ** -24 * math.log(n)
