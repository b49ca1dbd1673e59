"""Functions whose input is kept in 8 bits: parameters that are not arguments, arguments written into, and the second call of the
function, which has to be the first one's.  On the CPU the library calls are stood in for by their definitions."""
import pytest
import torch

from paper_2407_15452_b200 import layers as L
from tests.test_layers_autograd import _inputs, device  # noqa: F401


def _hidden(how, m):
    """A function of one tensor that uses the parameter m without taking it as an argument, and what else to hand it."""
    if how == "module":
        linear = torch.nn.Linear(24, 24, device=m.device)
        return linear, ()
    if how == "closure":
        return (lambda t: t @ m), ()
    return (lambda t, ms: t @ ms[0]), ([m],)


@pytest.mark.parametrize("how", ["module", "closure", "list"])
def test_a_hidden_parameter_behind_an_input_without_gradient_raises(device, how):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    f, rest = _hidden(how, m)
    with pytest.raises(RuntimeError, match="not one of its arguments"):
        L.kept_in_8_bits(f, x.detach(), *rest)
    with torch.no_grad():                                   # nothing to lose
        assert torch.equal(L.kept_in_8_bits(f, x.detach(), *rest), f(x.detach(), *rest))
    m.requires_grad_(False)
    if how != "module":
        y = L.kept_in_8_bits(f, x.detach(), *rest)
        assert not y.requires_grad and torch.equal(y, f(x.detach(), *rest))
    # beside an argument that asks for a gradient the backward pass raises
    f, rest = _hidden(how, m.requires_grad_(True))
    y = L.kept_in_8_bits(lambda t, scale, *r: f(t, *r) * scale, x.detach(), w.detach()[:1].requires_grad_(True), *rest)
    with pytest.raises(RuntimeError, match="not one of its arguments"):
        y.sum().backward()


def test_a_function_that_writes_into_its_arguments_raises(device):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    for f, args in ((lambda t, m: t.add_(1.0) @ m, (x.detach().clone(), m)),
                    (lambda t, m: t[0].mul_(2.0) @ m, (x * 1.0, m.detach())),
                    (lambda t, w: w.add_(1.0) * t, (x, w.detach().clone()))):
        with pytest.raises(RuntimeError, match="wrote into"):
            L.kept_in_8_bits(f, *args)
    y = L.kept_in_8_bits(lambda t, m: (t + 0).add_(1.0) @ m, x.detach(), m)       # its own tensors it may change
    y.sum().backward()
    assert m.grad is not None


@pytest.mark.parametrize("then,later", [(True, False), (False, True), (True, True)])
def test_the_second_call_runs_under_the_first_ones_autocast(device, then, later):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    seen = []

    def f(t, m):
        y = t @ m
        seen.append(y.dtype)
        return y.float()
    with torch.autocast(device, torch.bfloat16, enabled=then):
        y = L.kept_in_8_bits(f, x, m)
    with torch.autocast(device, torch.bfloat16, enabled=later):
        y.sum().backward()
    assert seen == [torch.bfloat16 if then else torch.float32] * 2
    kept = L.B.gs_checkpoint_unpack(*L.B.gs_checkpoint_pack(x.detach())).requires_grad_(True)
    with torch.autocast(device, torch.bfloat16, enabled=then):
        again = (kept @ m).float()
    with torch.autocast(device, torch.bfloat16, enabled=later):        # as the backward pass of anything else
        want = torch.autograd.grad(again.sum(), [kept, m])
    assert torch.equal(x.grad, want[0]) and torch.equal(m.grad, want[1])


@pytest.mark.parametrize("source", ["default", "argument", "cpu"])
def test_the_second_call_draws_the_first_ones_random_numbers(device, source):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    gen = torch.Generator(device).manual_seed(5)
    seen = []

    def f(t, m, gen):
        shape, where = t.shape, "cpu" if source == "cpu" else t.device
        mask = torch.rand(shape, device=where, generator=gen if source == "argument" else None).to(t.device) < 0.5
        seen.append(mask)
        return t * mask @ m
    y = L.kept_in_8_bits(f, x, m, gen)
    draw = lambda: torch.rand(8, device=device, generator=gen if source == "argument" else None)      # noqa: E731
    states = [g.get_state() for g in (gen, torch.default_generator)]
    if device == "cuda":
        states.append(torch.cuda.get_rng_state())
    y.sum().backward()
    assert len(seen) == 2 and torch.equal(seen[0], seen[1])
    # and what is drawn afterwards is what would have been drawn
    after = [g.get_state() for g in (gen, torch.default_generator)] + ([torch.cuda.get_rng_state()] if device == "cuda" else [])
    assert all(torch.equal(a, c) for a, c in zip(states, after))
    assert not torch.equal(draw(), draw())
    kept = L.B.gs_checkpoint_unpack(*L.B.gs_checkpoint_pack(x.detach())).requires_grad_(True)
    want = torch.autograd.grad((kept * seen[0] @ m).sum(), [kept, m])
    assert torch.equal(x.grad, want[0]) and torch.equal(m.grad, want[1])


@pytest.mark.gpu
def test_random_numbers_in_a_captured_function_are_refused():
    gen = torch.Generator("cuda").manual_seed(4)
    x, m = (torch.randn(s, generator=gen, device="cuda").requires_grad_(True) for s in ((2, 6, 24), (24, 48)))

    def step(p):
        y = L.kept_in_8_bits(lambda t, m: torch.nn.functional.dropout(t, p, training=p > 0) @ m, x, m)
        return torch.autograd.grad(y.sum(), [x, m])
    want = step(0.0)
    step(0.5)                                               # eager calls may
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="random numbers"):
        with torch.cuda.graph(graph):
            step(0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(0.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_an_input_computed_in_inference_mode(device):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    with torch.inference_mode():
        features = x * 2.0
    L.kept_in_8_bits(lambda t, m: t @ m, features, m).sum().backward()
    kept = L.B.gs_checkpoint_unpack(*L.B.gs_checkpoint_pack(features.clone()))
    (want,) = torch.autograd.grad((kept @ m).sum(), m)
    assert torch.equal(m.grad, want)
