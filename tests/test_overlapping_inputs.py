"""Inputs whose positions share memory (windows that slide over one sequence): results have a layout of their own."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.layers import gated_recurrence, layer_norm

pytestmark = pytest.mark.gpu


def _windows(batch, positions, columns, dtype, seed, by=1):
    """[batch, positions, columns]: position t holds the columns values from t * by on."""
    gen = torch.Generator("cuda").manual_seed(seed)
    n = (positions - 1) * by + columns
    return torch.randn((batch, n), generator=gen, device="cuda").to(dtype).as_strided((batch, positions, columns), (n, by, 1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,positions,columns,by", [(2, 3, 8, 1), (1, 5, 64, 1), (3, 40, 7, 1), (2, 3, 8, 0), (2, 3, 16, 4), (1, 200, 33, 1)])
def test_windows_of_a_sequence(batch, positions, columns, by, dtype):
    x, gate, dy = (_windows(batch, positions, columns, dtype, s, by) for s in range(3))
    cx, cgate, cdy = (t.contiguous() for t in (x, gate, dy))
    w = torch.ones(columns, device="cuda")

    y, stats, packed, scales = B.gs_layer_norm_forward(x, w, w, checkpoint=True)
    want = B.gs_layer_norm_forward(cx, w, w, checkpoint=True)
    # other alignments may sum in another order: compared within two steps of 32-bit sums over the row, and of the result's rounding
    size = 2 * torch.finfo(dtype).eps + 8 * columns * 2.0 ** -24
    close = lambda a, c: ((a.double() - c.double()).abs() <= size * (1 + c.double().abs().max())).all()           # noqa: E731
    assert close(y, want[0]) and close(stats, want[1]) and torch.equal(packed, want[2]) and torch.equal(scales, want[3])
    for a, c in zip(B.gs_layer_norm_backward(dy, x, w, w, want[1]), B.gs_layer_norm_backward(cdy, cx, w, w, want[1])):
        assert a.shape == c.shape and close(a, c)

    out, final, states = B.gs_recurrence_forward(gate, x)
    again = B.gs_recurrence_forward(cgate, cx)
    assert close(out, again[0]) and close(final, again[1])
    for a, c in zip(B.gs_recurrence_backward(dy, gate, x, None, states), B.gs_recurrence_backward(cdy, cgate, cx, None, again[2])):
        assert a.shape == c.shape and close(a, c)


def test_gradients_of_windows():
    base, gates = (torch.randn((2, 10), device="cuda").requires_grad_(True) for _ in range(2))

    def loss(windows, norm, scan):
        out, final = scan(windows(gates), norm(windows(base)))
        return out.square().sum() + final.sum()
    got = torch.autograd.grad(loss(lambda t: t.unfold(1, 8, 1), layer_norm, gated_recurrence), [base, gates])
    want = torch.autograd.grad(loss(lambda t: t.unfold(1, 8, 1).contiguous(), layer_norm, gated_recurrence), [base, gates])
    for a, c in zip(got, want):
        assert (a - c).abs().max() <= 1e-5 * c.abs().max()
