"""What autograd may and may not do with the attention operation.  On the CPU the two library calls are stood in
for by the definition in torch, so that only the autograd function itself is under test."""
import math

import pytest
import torch

from paper_2407_15452_b200 import attention as A


def _forward(q, k, v, scale=None, window=(-1, -1), q_lens=None, k_lens=None):
    s = torch.einsum("bihd,bjhd->bhij", q, k) * (q.shape[3] ** -0.5 if scale is None else scale)
    return torch.einsum("bhij,bjhd->bihd", s.softmax(-1), v), s.logsumexp(-1)


def _backward(dout, q, k, v, out, lse, scale=None, window=(-1, -1), q_lens=None, k_lens=None):
    scale = q.shape[3] ** -0.5 if scale is None else scale
    p = (torch.einsum("bihd,bjhd->bhij", q, k) * scale - lse[..., None]).exp()
    ds = p * (torch.einsum("bihd,bjhd->bhij", dout, v) - (dout * out).sum(-1).transpose(1, 2)[..., None]) * scale
    return (torch.einsum("bhij,bjhd->bihd", ds, k), torch.einsum("bhij,bihd->bjhd", ds, q),
            torch.einsum("bhij,bihd->bjhd", p, dout))


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        monkeypatch.setattr(A.B, "gs_attention_forward", _forward)
        monkeypatch.setattr(A.B, "gs_attention_backward", _backward)
    return request.param


def _layer(device):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((2, 6, 2, 8), generator=gen).to(device).requires_grad_(True)
    w = [(torch.randn((8, 8), generator=gen) / math.sqrt(8)).to(device).requires_grad_(True) for _ in range(3)]
    return x, w


def test_first_gradient(device):
    x, w = _layer(device)
    got = torch.autograd.grad(A.attention(*(x @ m for m in w)).square().sum(), [x, *w])
    want = torch.autograd.grad(_forward(*(x @ m for m in w))[0].square().sum(), [x, *w])
    # some hundred products of values of order one, in fp32 on both sides
    for a, b in zip(got, want):
        assert (a - b).abs().max() <= 1000 * 2.0 ** -24 * max(1.0, b.abs().max().item())


def test_second_gradient_raises_instead_of_leaving_attention_out(device):
    # a residual path keeps the graph of the first gradient alive, as in a real layer
    x, w = _layer(device)
    y = x + A.attention(*(x @ m for m in w))
    (g,) = torch.autograd.grad(y.pow(3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(g.square().sum(), w, retain_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        g.square().sum().backward()


def test_second_gradient_with_a_constant_incoming_gradient_raises(device):
    # the loss is linear in the result: only q, k and v carry the second derivative
    x, w = _layer(device)
    (g,) = torch.autograd.grad(A.attention(*(x @ m for m in w)).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(g.square().sum(), w)


def test_a_kept_graph_that_nobody_differentiates_is_no_error(device):
    x, w = _layer(device)
    loss = A.attention(*(x @ m for m in w)).square().sum()
    kept = torch.autograd.grad(loss, [x, *w], create_graph=True)
    again = torch.autograd.grad(loss, [x, *w])
    assert all(torch.equal(a, b) for a, b in zip(kept, again))
