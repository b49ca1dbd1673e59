"""A layer of a sequence model on sampled walks: layer norm, recurrence or attention, kept activations, clipped gradients,
and the same model carried on one node at a time."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200 import workloads as WL
from paper_2407_15452_b200.layers import gated_recurrence, kept_in_8_bits, layer_norm
from tests.test_gpu_walk_encoder import _example

pytestmark = pytest.mark.gpu


def _model(dtype, **kw):
    graph = WL.chung_lu_graph(2000, 10, 2.3, seed=7)
    g = B.gs_graph_load_csr(graph.offsets.to("cuda"), graph.cols.to("cuda"), B.GS_VALIDATE)
    walks = B.gs_random_walks(g, None, 256, 0, 20, 7)
    walks[5, 9:] = -1                                       # dead ends
    walks[6, 1:] = -1
    model = _example().WalkEncoder(graph.n_nodes, 64, 2, dtype, 7, **kw)
    gen = torch.Generator("cuda").manual_seed(1)
    with torch.no_grad():
        for p in model.params.values():                     # away from the start, where gradients vanish
            p.add_(torch.randn(p.shape, generator=gen, device="cuda") * 0.05)
    negatives = torch.randint(0, graph.n_nodes, (256, 19, 5), generator=gen, device="cuda")
    return model, walks, negatives


def _plain_encode(model, walks):
    """The layer in torch operations of 64 bits."""
    p, (n, length) = {k: v.double() for k, v in model.params.items()}, walks.shape
    on = (walks >= 0)[..., None]
    x = p["nodes_in"][walks.clamp(min=0).long()]
    y = x
    if "norm_weight" in p:
        y = (x - x.mean(-1, keepdim=True)) / (x.var(-1, correction=0, keepdim=True) + 1e-5).sqrt() * p["norm_weight"] + p["norm_bias"]
    gate, value = (y @ p["gates"]).chunk(2, -1)
    h, outs = torch.zeros_like(x[:, 0]), []
    for t in range(length):
        a = torch.sigmoid(gate[:, t])
        h = torch.where(on[:, t], a * h + (1 - a) * value[:, t], h)
        outs.append(h)
    return x + torch.stack(outs, 1).masked_fill(~on, 0.0) @ p["proj"], h


def test_gradients_of_a_normalised_recurrent_layer():
    model, walks, negatives = _model(torch.float32, mixer="recurrence", norm=True)
    loss, _ = model.loss(walks, negatives)
    got = dict(zip(model.params, torch.autograd.grad(loss, list(model.params.values()))))
    model.encode = lambda w: _plain_encode(model, w)
    # the rest of the loss in fp32, from 64-bit vectors; the same loss of the plain layer
    want = dict(zip(model.params, torch.autograd.grad(_double_loss(model, walks, negatives), list(model.params.values()))))
    for k in got:
        # sums of some thousand fp32 terms on one side
        assert (got[k] - want[k]).abs().max() <= 2e-5 * want[k].abs().max() + 1e-7, k


def _double_loss(model, walks, negatives):
    h, _ = _plain_encode(model, walks)
    out = model.params["nodes_out"].double()
    h, nxt = h[:, :-1], walks[:, 1:]
    pos = (h * out[nxt.clamp(min=0).long()]).sum(-1)
    neg = torch.einsum("nld,nlkd->nlk", h, out[negatives])
    per = torch.nn.functional.softplus(-pos) + torch.nn.functional.softplus(neg).sum(-1)
    return (per * (nxt >= 0)).sum() / walks.shape[0]


@pytest.mark.parametrize("mixer", ["attention", "recurrence"])
def test_kept_activations_change_gradients_by_their_precision_only(mixer):
    model, walks, negatives = _model(torch.bfloat16, mixer=mixer, norm=True)
    grads = []
    for model.kept in (False, True):
        loss, _ = model.loss(walks, negatives)
        grads.append(torch.autograd.grad(loss, list(model.params.values())))
    # 8 bits are off by 1 / 254 of a row's largest value, here some 3 standard deviations: 1.2 % of one at most, and these errors are
    # independent over columns; gradients of the weights, which the kept values do not enter, are the same but for bf16
    for name, a, b in zip(model.params, *grads):
        assert (a - b).norm() <= 0.02 * a.norm(), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_walks_carried_on_one_node_at_a_time(dtype):
    model, walks, _ = _model(dtype, mixer="recurrence", norm=True)
    with torch.no_grad():
        whole, final = model.encode(walks)
        state, parts = None, []
        for t in range(walks.shape[1]):
            h, state = model.encode(walks[:, t:t + 1].contiguous(), state)
            parts.append(h)
        # the projections are rounded to dtype on both sides; their products may be summed in another order
        size = 2.0 ** -6 if dtype == torch.bfloat16 else 1e-4
        on = (walks >= 0)[..., None]
        assert ((torch.cat(parts, 1) - whole) * on).abs().max() <= size * whole.abs().max()
        assert (state - final).abs().max() <= size * final.abs().max()


def test_a_training_step_captured_into_a_graph():
    # layer norm from 8 bits, the recurrence and a function whose input is kept, forward and backward, replayed on other inputs
    gen = torch.Generator("cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")                   # noqa: E731
    x, m, w, b = rand(4, 150, 64), rand(64, 128) / 8, 1 + 0.1 * rand(64), 0.1 * rand(64)
    lens = torch.tensor([150, 0, 77, 149], dtype=torch.int32, device="cuda")
    wanted = [t.requires_grad_(True) for t in (x, m, w, b)]

    def block(x, m, w, b):
        gate, value = (layer_norm(x, w, b, lens=lens, checkpoint=True) @ m).chunk(2, -1)
        return gated_recurrence(gate, value, None, lens)[0]

    def step():
        y = x + block(x, m, w, b)
        y = y + kept_in_8_bits(block, y, m, w, b)
        return [y.detach(), *torch.autograd.grad(y.square().sum(), wanted)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = step()                                       # also allocates what libraries need; its results stay alive
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(2):
        with torch.no_grad():
            x.copy_(rand(4, 150, 64))
            lens.copy_(torch.tensor([[20, 150, 0, 128], [129, 1, 150, 5]][seed], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, step()):
            assert torch.equal(a, c)
    assert len(eager) == len(got)


def test_two_streams_at_once():
    gen = torch.Generator("cuda").manual_seed(5)
    make = lambda: [torch.randn((2, 9000, 64), generator=gen, device="cuda").bfloat16() for _ in range(3)]      # noqa: E731
    sets, streams = [make(), make()], [torch.cuda.Stream(), torch.cuda.Stream()]

    def both(gate, x, dout):
        out, final, states = B.gs_recurrence_forward(gate, x)
        y, stats = B.gs_layer_norm_forward(out)
        return [out, final, y, *B.gs_recurrence_backward(dout, gate, x, None, states), *B.gs_checkpoint_pack(y),
                B.gs_layer_norm_backward(dout, out, None, None, stats)[0]]
    want = [both(*s) for s in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i] = both(*sets[i])
    torch.cuda.synchronize()
    for g, r in zip(got, want):
        assert all(torch.equal(a, c) for a, c in zip(g, r))


@pytest.mark.parametrize("kw", [dict(mixer="recurrence"), dict(mixer="recurrence", norm=True), dict(norm=True, kept=True),
                                dict(mixer="recurrence", norm=True, kept=True)])
def test_example_runs(kw):
    losses, norms, model = _example().train(steps=6, nodes=2000, dim=64, heads=2, walks_per_step=128, walk_len=20, **kw)
    assert torch.isfinite(losses).all() and torch.isfinite(norms).all()
    assert abs(losses[0].item() - math.log(2.0)) < 1e-3      # zero output embeddings: log 2 per term
    total = math.sqrt(sum(p.grad.double().square().sum().item() for p in model.params.values()))
    assert total <= 1.0 + 1e-4
