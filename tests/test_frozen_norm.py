"""Layer norm whose weight and bias ask for no gradient: none is summed up, and no scratch is taken for it."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200 import layers as L
from tests import layers_reference as R
from tests import test_layers_autograd as A
from tests.test_layers_autograd import device  # noqa: F401


@pytest.mark.parametrize("frozen", ["both", "weight", "bias", "neither"])
def test_gradients_that_nobody_asked_for(device, frozen, monkeypatch):  # noqa: F811
    x, m, w, b, lens = A._inputs(device)
    w.requires_grad_(frozen not in ("both", "weight"))
    b.requires_grad_(frozen not in ("both", "bias"))
    asked, real = [], B.gs_layer_norm_backward

    def watch(*args, sums=True):
        asked.append(sums)
        if device == "cuda":
            return real(*args, sums=sums)
        got = A._norm_back(*args)
        return got if sums else (got[0], None, None)
    monkeypatch.setattr(L.B, "gs_layer_norm_backward", watch)
    for checkpoint in (False, True):
        wanted = [t for t in (x, w, b) if t.requires_grad]
        got = torch.autograd.grad(L.layer_norm(x, w, b, lens=lens, checkpoint=checkpoint).square().sum(), wanted)
        r = R.layer_norm(x.detach(), w.detach(), b.detach(), 1e-5, lens)
        at = R.checkpoint_values(*A._pack(x.detach())) if checkpoint else x.detach()
        want = R.layer_norm_backward(2 * r["y"], at, w.detach(), r["stats"], lens)
        A._close(got, [want[k] for k, t in (("dx", x), ("dweight", w), ("dbias", b)) if t.requires_grad], 2000)
    assert asked == [frozen != "both"] * 2


@pytest.mark.gpu
def test_no_scratch_for_a_frozen_weight():
    x = torch.randn((1, 5000, 8192), device="cuda")
    w = torch.ones(8192, device="cuda")
    _, stats = B.gs_layer_norm_forward(x, w, w)
    want = B.gs_layer_norm_backward(x, x, w, w, stats)
    for args, kw in (((w, w), dict(sums=False)), ((None, None), {})):
        dx = torch.empty_like(x)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = B.gs_layer_norm_backward(x, x, *args, stats, dx=dx, **kw)
        assert torch.cuda.max_memory_allocated() == before
        assert got[1] is None and got[2] is None and torch.equal(dx, want[0])
