"""The order of the sums of the gradient norm, and their rounding at the edges of a chunk.

Tolerance: a square is rounded once and up to 18 of them are added in fp32 by fused operations, 18 roundings of 2^-24 at
most; fp64 from there.  The root halves the relative error and is rounded to fp32: (18 / 2 + 1) 2^-24 of the norm."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TOL = 10 * 2.0 ** -24


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_the_norm_does_not_depend_on_where_the_result_goes(dt):
    gen = torch.Generator(device="cuda").manual_seed(5)
    room = torch.empty(70_000, dtype=F32, device="cuda")
    for shift in range(9):
        g = torch.randn(60_011 + shift, generator=gen, device="cuda").to(dt)[shift:]
        alone = B.gs_gradient_norm([g])
        norms = [B.gs_clip_gradients([g], 1.0, out=[room[at:at + g.numel()]]) for at in range(5)]
        norms.append(B.gs_clip_gradients([g], 1.0, out=[torch.empty_like(g)]))
        norms.append(B.gs_clip_gradients([g], 1.0))                       # in place, the last call
        assert all(torch.equal(alone, n) for n in norms), (shift, alone, norms)


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("first", range(4))
def test_the_norm_does_not_depend_on_where_the_result_goes_to_the_last_bit(first, dt):
    # one element in four is 1, the others' squares are 2^-24: whether fp32 sums see them depends on the order
    g = torch.full((8192,), 2.0 ** -12, device="cuda").to(dt)
    g[first::4] = 1.0
    room = torch.empty(8200, dtype=F32, device="cuda")
    alone = B.gs_gradient_norm([g])
    for at in range(8):
        assert torch.equal(alone, B.gs_clip_gradients([g], 1e9, out=[room[at:at + g.numel()]])), at


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [4095, 4096, 4097, 8191, 8193, 12289])
def test_chunk_edges_at_every_offset(size, dt):
    gen = torch.Generator(device="cuda").manual_seed(size)
    for shift in range(9):
        g = (torch.randn(size + shift, generator=gen, device="cuda") * 3).to(dt)[shift:]
        for x in (g, g[:1], g[-1:]):
            want = math.sqrt(x.double().square().sum().item())
            assert abs(B.gs_gradient_norm([x]).item() - want) <= TOL * want
        # every element once: an odd one out among zeros at each end and at the seam of two chunks
        z = torch.zeros(size + shift, dtype=dt, device="cuda")[shift:]
        for at in (0, 1, 7, 8, size // 2, 4094, size - 2, size - 1):
            z[at] = 4.0
            assert B.gs_gradient_norm([z]).item() == 4.0
            z[at] = 0.0
