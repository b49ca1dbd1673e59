"""Where no gradient can be asked for, layers leave nothing behind for a backward pass.  On the CPU the library calls are stood in for by
their definitions."""
import pytest
import torch

from paper_2407_15452_b200 import layers as L
from tests.test_layers_autograd import _inputs, _layer, device  # noqa: F401


@pytest.fixture
def calls(monkeypatch, device):  # noqa: F811
    """What the layers ask of the library: (name, kept) of every call."""
    seen = []

    def watch(name, kept):
        f = getattr(L.B, name)
        monkeypatch.setattr(L.B, name, lambda *a, **kw: seen.append((name, kept(kw))) or f(*a, **kw))
    watch("gs_layer_norm_forward", lambda kw: kw.get("checkpoint", False))
    watch("gs_recurrence_forward", lambda kw: kw.get("keep", True))
    watch("gs_checkpoint_pack", lambda kw: True)
    return seen


def _all(x, m, w, b, lens):
    _layer(x, m, w, b, lens, checkpoint=True)
    return L.kept_in_8_bits(_layer_out, x, m, w, b, lens)


def _layer_out(*args):
    return _layer(*args, checkpoint=True)[0]


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_under_no_grad_nothing_is_kept(device, calls, mode):  # noqa: F811
    args = _inputs(device)
    want = _layer_out(*args).detach()
    calls.clear()
    with mode():
        got = _all(*args)
    assert torch.equal(got, want) and not got.requires_grad
    assert [name for name, _ in calls] == ["gs_layer_norm_forward", "gs_recurrence_forward"] * 2
    assert not any(kept for _, kept in calls)


def test_for_inputs_without_gradient_nothing_is_kept(device, calls):  # noqa: F811
    x, m, w, b, lens = _inputs(device)
    _all(*(t.detach() for t in (x, m, w, b)), lens)
    assert not any(kept for _, kept in calls)
    calls.clear()
    _all(x, m, w, b, lens).sum().backward()
    assert any(kept for _, kept in calls)
