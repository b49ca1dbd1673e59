"""The gated linear recurrence and its gradient against the 64-bit definition, within bounds derived there."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests import layers_reference as R

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def tensors(b, n, c, dtype, seed=0, ragged=True, start=True):
    gen = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")                   # noqa: E731
    slow = 6 * torch.rand(c, generator=gen, device="cuda") - 1
    gate, x, dout = (rand(b, n, c) + slow).to(dtype), rand(b, n, c).to(dtype), rand(b, n, c).to(dtype)
    lens = torch.randint(-1, n + 2, (b,), generator=gen, device="cuda", dtype=torch.int32) if ragged else None
    if ragged and b > 1:
        lens[0], lens[1] = n, 0
    return gate, x, dout, rand(b, c) if start else None, rand(b, c) if start else None, lens


def check(gate, x, dout, h0, dfinal, lens):
    out, final, states = B.gs_recurrence_forward(gate, x, h0, lens)
    got = B.gs_recurrence_backward(dout, gate, x, h0, states, dfinal, lens)
    want = R.recurrence(gate, x, h0, lens, dout, dfinal)
    for name, g in zip(("out", "final", "states", "dgate", "dx", "dh0"), (out, final, states, *got)):
        R.within(g, want[name], want[name + "_bound"], name)
    return out, final, states, got


# one stretch, several, a whole span, spans of one window, several windows, and the places next to their borders
LENGTHS = [1, 2, 10, 15, 16, 17, 40, 80, 127, 128, 129, 130, 255, 257, 640, 1023, 1024, 1025, 1153, 2050]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("length", LENGTHS)
def test_against_the_definition(length, dtype):
    check(*tensors(3, length, 70, dtype, length))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("channels", [1, 2, 3, 31, 32, 33, 63, 64, 65, 66, 128, 130])
def test_channels(channels, dtype):
    for n in (5, 150):
        check(*tensors(2, n, channels, dtype, channels))


@pytest.mark.parametrize("start,ragged", [(False, False), (False, True), (True, False)])
def test_without_states_or_lengths(start, ragged):
    for n in (20, 300):
        check(*tensors(4, n, 64, BF16, 5, ragged, start))


def test_many_walks():
    for dtype, n in ((BF16, 40), (F16, 10), (F32, 80), (BF16, 100), (F32, 65)):
        check(*tensors(700, n, 66, dtype, n))


def test_long():
    check(*tensors(1, 9001, 34, F32, 1))
    check(*tensors(2, 6000, 64, BF16, 2))


@pytest.mark.parametrize("b,n,c,dtype", [(460, 140, 64, BF16), (310, 300, 32, F32), (230, 300, 40, F16), (120, 600, 50, BF16), (60, 700, 96, F32)])
def test_clusters_of_every_size(b, n, c, dtype):
    # as many chains as leave 1, 2, 4 and 8 blocks to each of them
    check(*tensors(b, n, c, dtype, b))


@pytest.mark.parametrize("b,n,c,dtype", [(1, 8193, 64, BF16), (1, 9300, 33, F32), (2, 8500, 16, F16), (1, 12300, 130, F32)])
def test_chains_that_several_clusters_share(b, n, c, dtype):
    args = gate, x, dout, h0, dfinal, lens = tensors(b, n, c, dtype, n, ragged=b > 1)
    out, final, _, _ = check(*args)
    state = h0.clone()                                                             # the final state in the place of the first
    again, _, _ = B.gs_recurrence_forward(gate, x, state, lens, final=state)
    assert torch.equal(again, out) and torch.equal(state, final)
    if n == 8193:
        check(gate, x, dout, None, None, torch.full((b,), n - 5000, dtype=torch.int32, device="cuda"))


def test_no_incoming_gradient():
    gate, x, dout, h0, dfinal, lens = tensors(3, 200, 40, F32, 6)
    _, _, states = B.gs_recurrence_forward(gate, x, h0, lens)
    got = B.gs_recurrence_backward(None, gate, x, h0, states, dfinal, lens)
    want = R.recurrence(gate, x, h0, lens, None, dfinal)
    for name, g in zip(("dgate", "dx", "dh0"), got):
        R.within(g, want[name], want[name + "_bound"], name)
    assert all((g == 0).all() for g in B.gs_recurrence_backward(None, gate, x, h0, states, None, lens))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gates_that_are_shut_or_open(dtype):
    gate, x, dout, h0, dfinal, _ = tensors(2, 300, 64, dtype, 7)
    for z in (-200.0, -30.0, 0.0, 10.0, 30.0, 200.0, float("inf"), float("-inf")):
        gate.fill_(z)
        out, final, _, got = check(gate, x, dout, h0, dfinal, None)
        if z >= 200:
            assert torch.equal(final, h0) and (got[1] == 0).all()
        if z <= -200:
            assert torch.equal(out, x)
    # slow channels: a state that forgets one part in 20000 a step keeps that rate
    gate = torch.full((1, 1500, 32), 9.9, device="cuda")
    x = torch.ones_like(gate)
    out, _, _ = B.gs_recurrence_forward(gate, x)
    want = R.recurrence(gate, x)["out"]
    assert ((out.double() - want).abs() <= 1e-5 * want).all()


@pytest.mark.parametrize("length", [40, 700])
def test_positions_behind_the_end_are_never_used(length):
    gate, x, dout, h0, dfinal, lens = tensors(6, length, 66, F16, 8)
    clean = check(gate, x, dout, h0, dfinal, lens)
    behind = ~R.valid_rows(lens, 6, length, "cuda").expand_as(x)
    for poison in (float("nan"), float("inf"), torch.finfo(F16).min):
        got = check(*(t.masked_fill(behind, poison) for t in (gate, x, dout)), h0, dfinal, lens)
        assert all(torch.equal(a, b) for a, b in zip(got[:3] + got[3], clean[:3] + clean[3]))
        assert (got[0][behind] == 0).all() and (got[3][0][behind] == 0).all() and (got[3][1][behind] == 0).all()


def test_a_bad_value_reaches_what_follows_it_in_its_channel_and_nothing_else():
    gate, x, dout, h0, dfinal, _ = tensors(2, 300, 64, F32, 9)
    out0, _, states0 = B.gs_recurrence_forward(gate, x, h0)
    x[1, 200, 5] = float("nan")
    out, final, states = B.gs_recurrence_forward(gate, x, h0)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[1, 200:, 5] = True
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], out0[~hit]) and torch.isnan(final).sum() == 1
    dgate, dx, dh0 = B.gs_recurrence_backward(dout, gate, x, h0, states, dfinal)
    assert torch.isfinite(dx).all() and torch.isfinite(dh0).all() and torch.equal(torch.isnan(dgate), hit)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length", [40, 300])
def test_strides(length, dtype):
    c = 66
    args = gate, x, dout, h0, dfinal, lens = tensors(4, length, c, dtype, 10)
    check(*args)
    room = torch.full((4, length + 3, 3 * c + 2), 7.0, dtype=dtype, device="cuda")
    odd = torch.full((length, 4, c + 3), 7.0, dtype=dtype, device="cuda")
    want = R.recurrence(gate, x, h0, lens, dout, dfinal)
    for make in (lambda: room.clone()[:, 2:-1, c:2 * c], lambda: room.clone()[:, 1:-2, 3:3 + c],
                 lambda: odd.clone().transpose(0, 1)[:, :, 1:1 + c]):
        views = [make() for _ in range(6)]
        for v, t in zip(views, (gate, x, dout)):
            v.copy_(t)
        o, dg, dxs = views[3:]
        _, final, states = B.gs_recurrence_forward(views[0], views[1], h0, lens, out=o)
        B.gs_recurrence_backward(views[2], views[0], views[1], h0, states, dfinal, lens, dgate=dg, dx=dxs)
        for name, g in (("out", o), ("final", final), ("dgate", dg), ("dx", dxs)):
            R.within(g, want[name], want[name + "_bound"], name)
        for v in (o, dg, dxs):
            assert (v._base == 7).sum() >= v._base.numel() - v.numel()
    both = torch.cat([gate, x], -1)                                                # halves of one projection
    check(both[..., :c], both[..., c:], dout[:, :1].expand(-1, length, -1), h0, dfinal, lens)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_continued_in_pieces_and_step_by_step(dtype):
    gate, x, _, h0, _, _ = tensors(5, 300, 64, dtype, 11, ragged=False)
    want = R.recurrence(gate, x, h0)
    for cuts in ([0, 1, 2, 3, 130, 300], list(range(0, 41)) + [300]):
        state, outs = h0.clone(), []
        for i, j in zip(cuts, cuts[1:]):
            out, same, states = B.gs_recurrence_forward(gate[:, i:j], x[:, i:j], state, keep=False, final=state)
            assert same is state and states is None
            outs.append(out)
        R.within(torch.cat(outs, 1), want["out"], 2 * want["out_bound"], "out")     # another split of the same sums
        R.within(state, want["final"], 2 * want["final_bound"], "final")


def test_in_place_state_of_long_sequences():
    gate, x, _, h0, _, lens = tensors(40, 2500, 64, BF16, 12)
    want = B.gs_recurrence_forward(gate, x, h0, lens)
    for _ in range(5):
        state = h0.clone()
        out, _, _ = B.gs_recurrence_forward(gate, x, state, lens, final=state)
        assert torch.equal(out, want[0]) and torch.equal(state, want[1])


def test_gradient_against_differences():
    gen = torch.Generator("cuda").manual_seed(2)
    gate, x, dout = (torch.randn((1, 9, 3), generator=gen, device="cuda") for _ in range(3))
    h0, dfinal = (torch.randn((1, 3), generator=gen, device="cuda") for _ in range(2))

    def value(gate, x, h0):
        r = R.recurrence(gate, x, h0)
        return (r["out"] * dout).sum() + (r["final"] * dfinal).sum()
    _, _, states = B.gs_recurrence_forward(gate, x, h0)
    got = B.gs_recurrence_backward(dout, gate, x, h0, states, dfinal)
    step = 1e-5
    for i, t in enumerate((gate, x, h0)):
        for at in range(t.numel()):
            args = [a.double().clone() for a in (gate, x, h0)]
            args[i].view(-1)[at] += step
            up = value(*args)
            args[i].view(-1)[at] -= 2 * step
            assert abs((up - value(*args)) / (2 * step) - got[i].view(-1)[at]) <= 1e-4


def test_repeatable_and_on_any_stream():
    gate, x, dout, h0, dfinal, lens = tensors(9, 1300, 200, BF16, 12)
    want = B.gs_recurrence_forward(gate, x, h0, lens)
    back = B.gs_recurrence_backward(dout, gate, x, h0, want[2], dfinal, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.gs_recurrence_forward(gate, x, h0, lens)
        again = B.gs_recurrence_backward(dout, gate, x, h0, got[2], dfinal, lens)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + again, want + back))


def test_captured_and_replayed():
    args = gate, x, dout, h0, dfinal, lens = tensors(4, 333, 96, F16, 13)
    B.gs_recurrence_forward(gate, x, h0, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, final, states = B.gs_recurrence_forward(gate, x, h0, lens)
        got = B.gs_recurrence_backward(dout, gate, x, h0, states, dfinal, lens)
    for seed in (14, 15):
        for old, new in zip(args, tensors(4, 333, 96, F16, seed)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = B.gs_recurrence_forward(gate, x, h0, lens)
        assert torch.equal(out, want[0]) and torch.equal(final, want[1])
        assert all(torch.equal(a, b) for a, b in zip(got, B.gs_recurrence_backward(dout, gate, x, h0, want[2], dfinal, lens)))


def test_offsets_beyond_32_bits():
    c, n = 64, 200
    far = 2 ** 31 + 4096
    room = torch.zeros(far + n * c, dtype=BF16, device="cuda")
    gate, x, dout, h0, dfinal, _ = tensors(2, n, c, BF16, 16)
    views = []
    for t in (gate, x):
        v = room.clone().as_strided((2, n, c), (far, c, 1))
        v.copy_(t)
        views.append(v)
    out = room.as_strided((2, n, c), (far, c, 1))
    want = B.gs_recurrence_forward(gate, x, h0)
    got = B.gs_recurrence_forward(views[0], views[1], h0, out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dx = out.zero_()
    B.gs_recurrence_backward(dout, views[0], views[1], h0, got[2], dfinal, dx=dx)
    assert torch.equal(dx, B.gs_recurrence_backward(dout, gate, x, h0, want[2], dfinal)[1])


def test_a_wait_that_ran_out_fails_the_next_long_call():
    gate, x, _, h0, _, _ = tensors(1, 300, 16, F32, 17)
    B.gs_stall_drill()
    torch.cuda.synchronize()
    with pytest.raises(B.GsError, match="gave up a wait"):
        B.gs_recurrence_forward(gate, x, h0)
    B.gs_recurrence_forward(gate[:, :128], x[:, :128], h0)                         # short ones wait for nobody
    assert B.gs_stalled_kernels(clear=True) == 1
    B.gs_recurrence_forward(gate, x, h0)
    assert B.gs_stalled_kernels() == 0


def test_empty():
    for b, n in ((0, 5), (3, 0), (0, 0)):
        x = torch.empty((b, n, 16), device="cuda")
        h0 = torch.randn((b, 16), device="cuda")
        out, final, states = B.gs_recurrence_forward(x, x, h0)
        assert out.shape == x.shape and torch.equal(final, h0)
        assert torch.equal(B.gs_recurrence_backward(x, x, x, h0, states, h0)[2], h0)
        assert (B.gs_recurrence_forward(x, x)[1] == 0).all() and (B.gs_recurrence_backward(x, x, x, None, states)[2] == 0).all()
