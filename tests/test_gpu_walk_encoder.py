"""The differentiable attention over walks and the example that trains with it."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200 import workloads as WL
from paper_2407_15452_b200.attention import attention, walk_lengths
from tests.attention_reference import check, reference

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location(
        "walk_encoder", Path(__file__).resolve().parent.parent / "examples" / "walk_encoder.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
def test_gradients_through_autograd_on_walks_with_dead_ends(dt):
    # a graph whose odd nodes lead nowhere: walks of every length from 1 on
    n = 64
    off, cols = [0], []
    for v in range(n):
        cols += [(v + 1) % n, (v + 2) % n] if v % 8 else ([(v + 2) % n] if v % 16 else [])
        off.append(len(cols))
    g = B.gs_graph_load_csr(torch.tensor(off, dtype=torch.int64, device="cuda"),
                            torch.tensor(cols, dtype=torch.int32, device="cuda"))
    walks = B.gs_random_walks(g, None, n, 0, 20, 3)
    lens = walk_lengths(walks)
    assert lens.min() == 1 and lens.max() > 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((n, 20, 3, 2, 32), generator=gen, device="cuda").to(dt).requires_grad_(True)
    dout = torch.randn((n, 20, 2, 32), generator=gen, device="cuda").to(dt)
    out = attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], window=(-1, 0), q_lens=lens, k_lens=lens)
    out.backward(dout)
    with torch.no_grad():
        r = reference(*(qkv[:, :, i] for i in range(3)), 32 ** -0.5, (-1, 0), lens, lens, dout)
        check(out, r, "out")
        for i, name in enumerate(("dq", "dk", "dv")):
            check(qkv.grad[:, :, i], r, name)


def test_incoming_gradients_of_any_layout():
    q, k, v = (torch.randn((2, 9, 2, 16), device="cuda", requires_grad=True) for _ in range(3))
    attention(q, k, v).sum().backward()                     # an expanded gradient: every stride zero
    got = [t.grad.clone() for t in (q, k, v)]
    r = reference(q.detach(), k.detach(), v.detach(), 0.25, (-1, -1), dout=torch.ones((2, 9, 2, 16), device="cuda"))
    for name, g in zip(("dq", "dk", "dv"), got):
        check(g, r, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_learns(dtype):
    losses, norms, model = _example().train(steps=40, nodes=2000, dim=64, heads=2, dtype=dtype, walks_per_step=512, walk_len=20)
    assert torch.isfinite(losses).all() and torch.isfinite(norms).all()
    assert abs(losses[0].item() - math.log(2.0)) < 1e-3      # zero output embeddings: log 2 per term
    assert losses[-5:].mean() < losses[:5].mean() - 0.1
    total = math.sqrt(sum(p.grad.double().square().sum().item() for p in model.params.values()))
    assert total <= 1.0 + 1e-4                               # the last step's gradients are within the bound
