"""Activations in 8 bits against the definition: whole numbers and scales are equal, values are their product."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests import layers_reference as R

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def check(x):
    packed, scales = B.gs_checkpoint_pack(x)
    flat = x.reshape(-1, x.shape[-1])
    q, s = R.checkpoint(flat)
    assert same(scales.view(s.shape), s)
    fine = torch.isfinite(s).repeat_interleave(128, -1)[:, :q.shape[1]]
    assert torch.equal(packed.view(q.shape).double()[fine], q[fine])
    for dtype in (F32, F16, BF16):
        got = B.gs_checkpoint_unpack(packed, scales, dtype)
        assert same(got, R.checkpoint_values(packed, scales).to(dtype))
    return packed, scales


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("columns", [1, 3, 4, 8, 100, 127, 128, 129, 136, 256, 300, 1001, 4096])
def test_against_the_definition(columns, dtype):
    gen = torch.Generator("cuda").manual_seed(columns)
    for rows in (1, 2, 77, 2500):
        x = torch.randn((rows, columns), generator=gen, device="cuda") * torch.exp(3 * torch.randn((rows, 1), generator=gen, device="cuda"))
        check(x.to(dtype))


def test_every_place_between_two_whole_numbers():
    # quotients on ties and one fp32 step to either side of them, for many scales
    gen = torch.Generator("cuda").manual_seed(1)
    top = torch.exp(4 * torch.randn((2000, 1), generator=gen, device="cuda"))
    s = R.checkpoint(top)[1]
    k = torch.arange(127, device="cuda")[None] + 0.5
    tie = (s.double() * k).float()
    for x in (tie, torch.nextafter(tie, tie + 1), torch.nextafter(tie, tie - 1)):
        check(torch.cat([top, x], 1))
        check(-torch.cat([top, x], 1))
    for dtype in (F16, BF16):                                                     # tops of 127 steps: exact ties
        top = 127 * 2.0 ** torch.arange(-6, 6, device="cuda").float()[:, None]
        check(torch.cat([top, (top / 127) * k], 1).to(dtype))


@pytest.mark.parametrize("power", [-149, -146, -143, -142, -140, -130, -126, -110, -100, -61, -60, -59, 0, 100, 126, 127])
def test_magnitudes(power):
    gen = torch.Generator("cuda").manual_seed(3)
    x = (torch.rand((50, 128), generator=gen, device="cuda", dtype=torch.float64) * 4 - 2) * 2.0 ** power
    check(x.clamp(-3.4e38, 3.4e38).float())


def test_largest_and_zero_blocks():
    x = torch.zeros((3, 256), device="cuda")
    x[0, :128] = torch.finfo(F32).max
    x[1, 5] = -torch.finfo(F32).max
    packed, scales = check(x)
    assert torch.isfinite(B.gs_checkpoint_unpack(packed, scales)).all()
    x = torch.zeros((2, 200), dtype=F16, device="cuda")
    x[0, 7] = torch.finfo(F16).max
    back = B.gs_checkpoint_unpack(*check(x), F16)
    assert torch.isfinite(back).all() and back[0, 7] == torch.finfo(F16).max and (back[1] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_bad_value_marks_its_block(bad):
    for columns in (384, 383):
        x = torch.randn((4, columns), device="cuda")
        x[2, 130] = bad
        packed, scales = check(x)
        back = B.gs_checkpoint_unpack(packed, scales)
        assert torch.isnan(back[2, 128:256]).all() and torch.isnan(back).sum() == 128
        assert torch.isnan(scales).sum() == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_apart(dtype):
    for columns, width, at in ((256, 272, 8), (200, 203, 1), (128, 130, 0)):
        room = torch.full((90, width), 7.0, dtype=dtype, device="cuda")
        x = room[:, at:at + columns]
        x.copy_(torch.randn((90, columns), device="cuda"))
        packed, scales = check(x)
        out = torch.full_like(room, 7.0)
        B.gs_checkpoint_unpack(packed, scales, out=out[:, at:at + columns])
        assert torch.equal(out[:, at:at + columns], B.gs_checkpoint_unpack(packed, scales, dtype))
        assert (out == 7).sum() >= 90 * (width - columns)


def test_shapes():
    for shape in ((5,), (2, 3, 4, 130), (0, 8), (4, 0), (0,)):
        x = torch.randn(shape, device="cuda")
        packed, scales = B.gs_checkpoint_pack(x)
        back = B.gs_checkpoint_unpack(packed, scales)
        assert packed.shape == back.shape == x.shape
        if x.numel():
            assert ((back - x).abs() <= 0.5001 * scales.repeat_interleave(128, -1)[..., :shape[-1]]).all()


def test_offsets_beyond_32_bits():
    rows, columns = 2 ** 19 + 100, 4096
    x = torch.randn((64, columns), device="cuda", dtype=BF16).repeat(rows // 64 + 1, 1)[:rows]
    packed, scales = B.gs_checkpoint_pack(x)
    q, s = R.checkpoint(x[:64])
    for at in (0, rows // 64 // 2 * 64, (rows // 64 - 1) * 64):
        assert torch.equal(packed[at:at + 64].double(), q) and torch.equal(scales[at:at + 64], s)
    back = B.gs_checkpoint_unpack(packed, scales, BF16)
    assert torch.equal(back[-36:], back[(rows - 36) % 64:][:36]) and torch.equal(back[:64], R.checkpoint_values(packed[:64], s).to(BF16))


def test_captured_and_on_another_stream():
    x = torch.randn((300, 384), device="cuda")
    B.gs_checkpoint_pack(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        packed, scales = B.gs_checkpoint_pack(x)
        back = B.gs_checkpoint_unpack(packed, scales)
    x.copy_(torch.randn_like(x))
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert torch.equal(B.gs_checkpoint_unpack(*B.gs_checkpoint_pack(x)), back)
