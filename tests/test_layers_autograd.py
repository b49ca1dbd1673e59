"""What autograd may and may not do with layer norm, the gated recurrence and kept activations.  On the CPU the library
calls are stood in for by their definitions in torch, so that only the autograd functions are under test."""
import pytest
import torch

from paper_2407_15452_b200 import layers as L
from tests import layers_reference as R

E32 = 2.0 ** -24


def _norm(x, weight=None, bias=None, eps=1e-5, lens=None, checkpoint=False):
    r = R.layer_norm(x, weight, bias, eps, lens)
    y, stats = r["y"].to(x.dtype), r["stats"].float()
    if not checkpoint:
        return y, stats
    q, s = R.checkpoint(x.reshape(-1, x.shape[-1]))
    return y, stats, q.to(torch.int8).view(x.shape), s.view(*x.shape[:-1], -1)


def _norm_back(dy, x, weight, bias, stats, lens=None, scales=None):
    r = R.layer_norm_backward(dy, x if scales is None else R.checkpoint_values(x, scales), weight, stats, lens)
    return (r["dx"].to(dy.dtype), None if weight is None else r["dweight"].to(weight.dtype), None if bias is None else r["dbias"].to(bias.dtype))


def _scan(gate, x, h0=None, lens=None, keep=True):
    r = R.recurrence(gate, x, h0, lens)
    return r["out"].to(x.dtype), r["final"].float(), r["states"].float()


def _scan_back(dout, gate, x, h0=None, states=None, dfinal=None, lens=None):
    r = R.recurrence(gate, x, h0, lens, dout, dfinal)
    return r["dgate"].to(x.dtype), r["dx"].to(x.dtype), r["dh0"].float()


def _pack(x):
    q, s = R.checkpoint(x.reshape(-1, x.shape[-1]))
    return q.to(torch.int8).view(x.shape), s.view(*x.shape[:-1], -1)


def _unpack(packed, scales, dtype=torch.float32):
    return R.checkpoint_values(packed, scales).to(dtype)


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        for name, f in (("layer_norm_forward", _norm), ("layer_norm_backward", _norm_back), ("recurrence_forward", _scan),
                        ("recurrence_backward", _scan_back), ("checkpoint_pack", _pack), ("checkpoint_unpack", _unpack)):
            monkeypatch.setattr(L.B, "gs_" + name, f)
    return request.param


def _inputs(device, seed=3):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((2, 6, 24), generator=gen).to(device).requires_grad_(True)
    m = (torch.randn((24, 48), generator=gen) / 5).to(device).requires_grad_(True)
    w, b = (torch.randn(24, generator=gen).to(device).requires_grad_(True) for _ in range(2))
    lens = torch.tensor([6, 3], dtype=torch.int32, device=device)
    return x, m, w, b, lens


def _plain_layer(x, m, w, b, lens, h0=None):
    """The same layer in torch operations of 64 bits."""
    on = R.valid_rows(lens, 2, x.shape[1], x.device)
    v = x.double().masked_fill(~on, 0.0)
    v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()
    gate, value = ((v * w + b).masked_fill(~on, 0.0) @ m.double()).chunk(2, -1)
    h, outs = (0.0 if h0 is None else h0.double()) + torch.zeros(2, 24, device=x.device), []
    for t in range(x.shape[1]):
        a = torch.sigmoid(gate[:, t])
        h = torch.where(on[:, t], a * h + (1 - a) * value[:, t], h)
        outs.append(h)
    return x + torch.stack(outs, 1).masked_fill(~on, 0.0), h


def _layer(x, m, w, b, lens, h0=None, checkpoint=False):
    y = L.layer_norm(x, w, b, lens=lens, checkpoint=checkpoint)
    gate, value = (y @ m).chunk(2, -1)
    out, final = L.gated_recurrence(gate, value, h0, lens)
    return x + out, final


def _close(got, want, steps):
    for g, w in zip(got, want):
        assert (g - w).abs().max() <= steps * E32 * max(1.0, w.abs().max().item())


@pytest.mark.parametrize("start", [False, True])
def test_a_layer_and_its_gradients(device, start):
    x, m, w, b, lens = args = _inputs(device)
    h0 = torch.randn((2, 24), generator=torch.Generator().manual_seed(1)).to(device).requires_grad_(True) if start else None
    wanted = [x, m, w, b] + ([h0] if start else [])
    out, final = _layer(*args, h0)
    got = torch.autograd.grad(out.square().sum() + final.sum(), wanted)
    ref, ref_final = _plain_layer(*args, h0)
    want = torch.autograd.grad(ref.square().sum() + ref_final.sum(), wanted)
    # some hundred products of values of order one to ten, fp32 on one side
    _close([out, final], [ref, ref_final], 500)
    _close(got, want, 5000)


def test_only_one_of_the_two_results_is_used(device):
    x, m, w, b, lens = args = _inputs(device)
    for pick in (0, 1):
        got = torch.autograd.grad(_layer(*args)[pick].sum(), [x, m])
        want = torch.autograd.grad(_plain_layer(*args)[pick].sum(), [x, m])
        _close(got, want, 5000)


def test_leading_dimensions(device):
    x = torch.randn((24,), device=device, requires_grad=True)
    four = torch.randn((2, 3, 2, 24), device=device, requires_grad=True)
    for t in (x, four):
        y = L.layer_norm(t)
        assert y.shape == t.shape
        y.pow(3).sum().backward()
        v = t.detach().double().requires_grad_(True)
        ((v - v.mean(-1, keepdim=True)) / (v.var(-1, correction=0, keepdim=True) + 1e-5).sqrt()).pow(3).sum().backward()
        _close([t.grad], [v.grad], 5000)
    with pytest.raises(ValueError, match="lens"):
        L.layer_norm(x, lens=torch.ones(1, dtype=torch.int32, device=device))


def test_second_derivatives_raise(device):
    x, m, w, b, lens = args = _inputs(device)
    (g,) = torch.autograd.grad(_layer(*args)[0].pow(3).sum(), x, create_graph=True)
    for target in (m, w, x):
        with pytest.raises(RuntimeError, match="differentiable once"):
            torch.autograd.grad(g.square().sum(), target, retain_graph=True)
    (g,) = torch.autograd.grad(L.layer_norm(x, w, b).sum() + x.pow(3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(g.square().sum(), w)
    for checkpointed in (lambda: _layer(*args, checkpoint=True)[0], lambda: L.kept_in_8_bits(lambda t: t.square(), x)):
        with pytest.raises(RuntimeError, match="differentiable once"):
            torch.autograd.grad(checkpointed().sum(), x, create_graph=True)


def test_a_kept_input_gives_the_gradients_at_its_8_bits(device):
    x, m, w, b, lens = args = _inputs(device)
    got = torch.autograd.grad(L.layer_norm(x, w, b, lens=lens, checkpoint=True).square().sum(), [x, w, b])
    r = R.layer_norm(x.detach(), w.detach(), b.detach(), 1e-5, lens)
    packed, scales = _pack(x.detach())
    want = R.layer_norm_backward(2 * r["y"], R.checkpoint_values(packed, scales), w.detach(), r["stats"], lens)
    _close(got, [want["dx"], want["dweight"], want["dbias"]], 2000)


def _block(x, m, w, b, lens, scale):
    return _layer(x, m, w, b, lens)[0] * scale


def test_a_function_whose_input_is_kept_in_8_bits(device):
    x, m, w, b, lens = args = _inputs(device)
    out = L.kept_in_8_bits(_block, *args, 2.0)
    assert torch.equal(out, _block(*args, 2.0))
    out.square().sum().backward()
    got = [t.grad.clone() for t in (x, m, w, b)]
    kept = R.checkpoint_values(*_pack(x.detach())).requires_grad_(True)
    again = _block(kept, m, w, b, lens, 2.0)
    want = torch.autograd.grad(again, [kept, m, w, b], 2 * out.detach())
    _close(got, want, 100)
    y = L.kept_in_8_bits(_block, x.detach(), m, w.detach(), b, lens, 2.0)          # gradients only where they are asked for
    y.sum().backward()
    assert w.grad is not None and torch.equal(w.grad, got[2])


def test_a_function_that_hides_a_parameter_raises(device):
    x, m, w, b, lens = _inputs(device)
    out = L.kept_in_8_bits(lambda t: t @ m, x)
    with pytest.raises(RuntimeError, match="not one of its arguments"):
        out.sum().backward()
    with pytest.raises(TypeError, match="one tensor"):
        L.kept_in_8_bits(lambda t: (t, t), x)


def test_without_gradients_nothing_is_kept(device):
    x, m, w, b, lens = _inputs(device)
    with torch.no_grad():
        assert not _layer(x, m, w, b, lens)[0].requires_grad
        assert torch.equal(L.kept_in_8_bits(lambda t: t + 1, x), x + 1)
