"""Layer norm and its gradient against the 64-bit definition, within bounds derived there."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests import layers_reference as R

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def tensors(b, n, c, dtype, wdtype, seed=0, ragged=True):
    gen = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")                   # noqa: E731
    x = ((rand(b, n, c) + rand(c)) * torch.exp(0.5 * rand(c))).to(dtype)
    dy = rand(b, n, c).to(dtype)
    lens = torch.randint(-1, n + 2, (b,), generator=gen, device="cuda", dtype=torch.int32) if ragged else None
    if ragged and b > 1:
        lens[0], lens[1] = n, 0
    return x, dy, (1 + 0.3 * rand(c)).to(wdtype), rand(c).to(wdtype), lens


def check(x, dy, w, bias, lens, eps=1e-5):
    y, stats = B.gs_layer_norm_forward(x, w, bias, eps, lens)
    want = R.layer_norm(x, w, bias, eps, lens)
    R.within(y, want["y"], want["y_bound"], "y")
    R.within(stats, want["stats"], want["stats_bound"], "stats")
    got = B.gs_layer_norm_backward(dy, x, w, bias, stats, lens)
    wdtype = F32 if w is None and bias is None else (w if w is not None else bias).dtype
    want = R.layer_norm_backward(dy, x, w, stats, lens, wdtype)
    for name, g, there in zip(("dx", "dweight", "dbias"), got, (x, w, bias)):
        assert (g is None) == (there is None)
        if g is not None:
            R.within(g, want[name], want[name + "_bound"], name)
    return y, stats, got


# every team: parts of a warp, a warp with one to sixteen pieces a thread, blocks, blocks of wide rows; one column; odd widths
COLUMNS = [1, 2, 7, 8, 24, 32, 33, 64, 96, 128, 129, 200, 256, 384, 512, 520, 777, 1000, 1001, 2048, 4104, 8192, 8200, 8191, 16384, 16383]


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (F16, F32), (F16, F16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("columns", COLUMNS)
def test_against_the_definition(columns, dtype, wdtype):
    rows = 5 if columns > 600 else 37
    check(*tensors(3, rows, columns, dtype, wdtype, columns))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("columns", [64, 100, 128, 512, 1500, 4096])
def test_many_rows(columns, dtype):
    # more rows than the grid has teams: every team goes through several, the sums over rows too
    check(*tensors(5, 3001 if columns < 1000 else 701, columns, dtype, F32, 1))


@pytest.mark.parametrize("b,n", [(1, 1), (1, 2), (7, 1), (1, 5000), (2500, 2)])
def test_shapes_of_the_batch(b, n):
    check(*tensors(b, n, 72, BF16, F32, 3))
    check(*tensors(b, n, 72, F32, F32, 4, ragged=False))


@pytest.mark.parametrize("which", ["weight", "bias", "neither"])
def test_without_weight_or_bias(which):
    for c in (65, 128, 1024, 9000):
        x, dy, w, bias, lens = tensors(2, 9, c, BF16, BF16, c)
        check(x, dy, w if which == "weight" else None, bias if which == "bias" else None, lens)


@pytest.mark.parametrize("columns", [48, 1024])
def test_a_mean_far_from_zero(columns):
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn((1, 64, columns), generator=gen, device="cuda") + 1e4
    check(x, torch.randn_like(x), None, None, None)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("columns", [520, 1024, 4096, 8192])
def test_a_few_columns_far_from_the_rest(columns, dtype):
    gen = torch.Generator("cuda").manual_seed(6)
    for first, count, value in ((0, 1, 1e4), (0, 8, 1e4), (256, 8, -3e4), (columns - 8, 8, 2e3), (0, 200, 500.0)):
        x = torch.randn((1, 20, columns), generator=gen, device="cuda")
        x[..., first:first + count] += value
        check(x.to(dtype), torch.randn_like(x).to(dtype), None, None, None)


def test_constant_rows_and_zero_eps():
    x = torch.full((1, 4, 40), 3.0, device="cuda")
    y, stats = B.gs_layer_norm_forward(x, None, torch.full((40,), 0.5, device="cuda"))
    assert (y == 0.5).all() and (stats[..., 0] == 3).all()
    x[0, 1] = torch.arange(40.0, device="cuda")
    y, _ = B.gs_layer_norm_forward(x, eps=0.0)
    assert torch.isfinite(y[0, 1]).all() and torch.isnan(y[0, 0]).all()           # 0 / 0, as the formula has it


@pytest.mark.parametrize("columns", [64, 1024, 9000, 33])
def test_positions_behind_the_end_are_never_used(columns):
    x, dy, w, bias, lens = tensors(6, 11, columns, F16, F32, 8)
    clean = check(x, dy, w, bias, lens)
    behind = ~R.valid_rows(lens, 6, 11, "cuda").expand_as(x)
    for poison in (float("nan"), float("inf"), torch.finfo(F16).min):
        y, stats, got = check(x.masked_fill(behind, poison), dy.masked_fill(behind, poison), w, bias, lens)
        assert torch.equal(y, clean[0]) and torch.equal(stats, clean[1]) and all(torch.equal(a, b) for a, b in zip(got, clean[2]))
        assert (y[behind] == 0).all() and (got[0][behind] == 0).all()


def test_a_bad_row_stays_alone():
    x, dy, w, bias, _ = tensors(1, 20, 128, F32, F32, 9)
    y0, _ = B.gs_layer_norm_forward(x, w, bias)
    x[0, 7, 3] = float("inf")
    x[0, 12, 100] = float("nan")
    y, stats = B.gs_layer_norm_forward(x, w, bias)
    other = [i for i in range(20) if i not in (7, 12)]
    assert torch.equal(y[0, other], y0[0, other]) and torch.isnan(y[0, [7, 12]]).all()
    dx, dw, _ = B.gs_layer_norm_backward(dy, x, w, bias, stats)
    assert torch.isfinite(dx[0, other]).all() and torch.isnan(dx[0, [7, 12]]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("columns", [96, 1024])
def test_strides(columns, dtype):
    x, dy, w, bias, lens = tensors(4, 10, columns, dtype, F32, 10)
    want = check(x, dy, w, bias, lens)
    wide = torch.full((4, 13, columns + 24), 7.0, dtype=dtype, device="cuda")
    odd = torch.full((10, 4, columns + 3), 7.0, dtype=dtype, device="cuda")
    for make in (lambda: wide.clone()[:, 2:12, 8:8 + columns], lambda: odd.clone().transpose(0, 1)[:, :, 1:1 + columns],
                 lambda: wide.clone()[:, 1:11, 5:5 + columns]):
        xs, ys, dys, dxs = make(), make(), make(), make()
        xs.copy_(x)
        dys.copy_(dy)
        y, stats = B.gs_layer_norm_forward(xs, w, bias, 1e-5, lens, y=ys)
        full = R.layer_norm(x, w, bias, 1e-5, lens)
        R.within(ys, full["y"], full["y_bound"], "y")
        got = B.gs_layer_norm_backward(dys, xs, w, bias, stats, lens, dx=dxs)
        full = R.layer_norm_backward(dy, x, w, stats, lens)
        for name, g in zip(("dx", "dweight", "dbias"), got):
            R.within(g, full[name], full[name + "_bound"], name)
        assert (ys._base == 7).sum() >= ys._base.numel() - ys.numel()             # nothing beside the view was written
        assert (dxs._base == 7).sum() >= dxs._base.numel() - dxs.numel()
    shared = x[:1].expand(4, -1, -1)                                              # broadcast input
    y, _ = B.gs_layer_norm_forward(shared, w, bias)
    assert torch.equal(y, y[:1].expand_as(y))
    assert want[0].shape == y.shape


@pytest.mark.parametrize("columns", [40, 128, 256, 512, 2000, 4096, 9008, 1001, 60])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_checkpoint(columns, dtype):
    x, dy, w, bias, lens = tensors(3, 8, columns, dtype, F32, 11)
    y, stats, packed, scales = B.gs_layer_norm_forward(x, w, bias, 1e-5, lens, checkpoint=True)
    plain = B.gs_layer_norm_forward(x, w, bias, 1e-5, lens)
    assert torch.equal(y, plain[0]) and torch.equal(stats, plain[1])
    on = R.valid_rows(lens, 3, 8, "cuda")
    q, s = R.checkpoint(x.masked_fill(~on, 0.0).view(24, columns))
    assert torch.equal(packed.view(24, columns).double(), q) and torch.equal(scales.view(24, -1), s)
    got = B.gs_layer_norm_backward(dy, packed, w, bias, stats, lens, scales)
    want = R.layer_norm_backward(dy, R.checkpoint_values(packed, scales), w, stats, lens)
    for name, g in zip(("dx", "dweight", "dbias"), got):
        R.within(g, want[name], want[name + "_bound"], name)


def test_sums_over_rows_are_whole():
    # whole numbers, exact in fp32: a row that is missed or taken twice shows
    for c, n in ((64, 100_003), (128, 70_001), (1000, 5003), (4096, 3001), (9000, 1009)):
        dy = torch.randint(-8, 9, (1, n, c), device="cuda").to(BF16)
        stats = torch.tensor([0.0, 1.0], device="cuda").repeat(1, n, 1)
        x = torch.randint(-4, 5, (1, n, c), device="cuda").to(BF16)
        w = torch.ones(c, device="cuda")
        _, dw, db = B.gs_layer_norm_backward(dy, x, w, w, stats)
        assert torch.equal(db.double(), dy.double().sum((0, 1))) and torch.equal(dw.double(), (dy.double() * x.double()).sum((0, 1)))


def test_gradient_against_differences():
    gen = torch.Generator("cuda").manual_seed(2)
    x, dy = (torch.randn((1, 3, 20), generator=gen, device="cuda") for _ in range(2))
    w, bias = (torch.randn(20, generator=gen, device="cuda") for _ in range(2))

    def value(x, w, bias):
        v = x.double()
        v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()
        return ((v * w + bias) * dy).sum()
    _, stats = B.gs_layer_norm_forward(x, w, bias)
    got = B.gs_layer_norm_backward(dy, x, w, bias, stats)
    step = 1e-5                                                                   # error of a central difference ~ step^2
    for i, t in enumerate((x, w, bias)):
        for at in range(0, t.numel(), 3):
            args = [a.double().clone() for a in (x, w, bias)]
            args[i].view(-1)[at] += step
            up = value(*args)
            args[i].view(-1)[at] -= 2 * step
            assert abs((up - value(*args)) / (2 * step) - got[i].view(-1)[at]) <= 1e-4


def test_repeatable_and_on_any_stream():
    x, dy, w, bias, lens = tensors(9, 501, 200, BF16, F32, 12)
    y, stats = B.gs_layer_norm_forward(x, w, bias, 1e-5, lens)
    want = B.gs_layer_norm_backward(dy, x, w, bias, stats, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(B.gs_layer_norm_forward(x, w, bias, 1e-5, lens)[0], y)
        got = B.gs_layer_norm_backward(dy, x, w, bias, stats, lens)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed():
    x, dy, w, bias, lens = tensors(4, 33, 320, F16, F16, 13)
    B.gs_layer_norm_forward(x, w, bias, 1e-5, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, stats, packed, scales = B.gs_layer_norm_forward(x, w, bias, 1e-5, lens, checkpoint=True)
        got = B.gs_layer_norm_backward(dy, packed, w, bias, stats, lens, scales)
    for seed in (14, 15):
        for old, new in zip((x, dy, w, bias, lens), tensors(4, 33, 320, F16, F16, seed)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = B.gs_layer_norm_forward(x, w, bias, 1e-5, lens, checkpoint=True)
        assert torch.equal(y, want[0])
        assert all(torch.equal(a, b) for a, b in zip(got, B.gs_layer_norm_backward(dy, want[2], w, bias, want[1], lens, want[3])))


def test_offsets_beyond_32_bits():
    c = 4096
    far = 2 ** 31 // c + 5
    x = torch.empty((2, 1, c), dtype=BF16, device="cuda").as_strided((2, 1, c), (c, c, 1))
    room = torch.zeros(far * c + c, dtype=BF16, device="cuda")
    x = room.as_strided((2, 3, c), ((far - 2) * c, c, 1))
    x.copy_(torch.randn((2, 3, c), device="cuda"))
    y, stats = B.gs_layer_norm_forward(x)
    want = R.layer_norm(x, None, None, 1e-5)
    R.within(y, want["y"], want["y_bound"], "y")
    out = torch.zeros_like(room).as_strided((2, 3, c), ((far - 2) * c, c, 1))
    B.gs_layer_norm_forward(x, y=out)
    assert torch.equal(out, y)


def test_empty():
    w = torch.ones(16, device="cuda")
    for b, n in ((0, 5), (5, 0)):
        x = torch.empty((b, n, 16), device="cuda")
        y, stats = B.gs_layer_norm_forward(x, w, w)
        dx, dw, db = B.gs_layer_norm_backward(x, x, w, w, stats)
        assert y.shape == dx.shape == x.shape and (dw == 0).all() and (db == 0).all()
