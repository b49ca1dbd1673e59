"""The layers around attention as differentiable torch operations: layer norm, a gated linear recurrence, and activations
that wait for the backward pass in 8 bits.  include/gs.h has the formulas; every operation is differentiable once, a second
derivative through it raises.
"""
from __future__ import annotations

import contextlib

import torch
from torch.utils._python_dispatch import TorchDispatchMode

from . import binding as B


def _once(what):
    """A function whose gradient raises: it stands in the graph between gradients that are computed under create_graph=True and
    what they were computed from, so that a second derivative does not take them for constants.  (Where x is kept in 8 bits
    there is nothing to tie that node to, and create_graph=True itself raises.)"""

    class Gradient(torch.autograd.Function):
        @staticmethod
        def forward(ctx, call, *tensors):
            return call(*tensors)

        @staticmethod
        def backward(ctx, *grads):
            raise RuntimeError(f"{what} is differentiable once: its gradients have no gradient")

    def gradient(call, *tensors):
        return Gradient.apply(call, *tensors) if torch.is_grad_enabled() else call(*tensors)
    return gradient


def _asks(*tensors):
    """True if a gradient can be asked for; a function's needs_input_grad does not know of torch.no_grad()."""
    return torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors)


def _rows_of_columns(t):
    return t if t is None or t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


# ---------------------------------------------------------------- layer norm
_norm_gradient = _once("layer_norm")


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, lens, checkpoint):
        if checkpoint:
            y, stats, packed, scales = B.gs_layer_norm_forward(x, weight, bias, eps, lens, checkpoint=True)
            ctx.save_for_backward(packed, weight, bias, stats, lens, scales)
        else:
            y, stats = B.gs_layer_norm_forward(x, weight, bias, eps, lens)
            ctx.save_for_backward(x, weight, bias, stats, lens, None)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, stats, lens, scales = ctx.saved_tensors
        if scales is not None and torch.is_grad_enabled():
            raise RuntimeError("layer_norm with checkpoint=True is differentiable once: call backward without create_graph")

        frozen = not any(ctx.needs_input_grad[1:3]) and (weight is not None or bias is not None)

        def call(dy, weight, x, bias):
            kw = dict(sums=False) if frozen else {}
            return tuple(g for g in B.gs_layer_norm_backward(_rows_of_columns(dy), x, weight, bias, stats, lens, scales, **kw) if g is not None)
        grads = iter(_norm_gradient(call, dy, weight, x, bias))
        return next(grads), None if frozen or weight is None else next(grads), None if frozen or bias is None else next(grads), None, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, lens=None, checkpoint=False):
    """Layer norm of x[..., columns] over its columns.  lens (for x[batch, length, columns]): valid positions of each sequence; the
    others give zeros and no gradient.  checkpoint=True keeps x for the backward pass in 8 bits (a quarter or half of
    its memory; see gs_checkpoint_pack in gs.h for what that costs in precision)."""
    shape = x.shape
    if x.dim() != 3:
        if lens is not None:
            raise ValueError("lens needs x of [batch, length, columns]")
        if x.dim() == 0:
            raise ValueError("x must have at least one dimension")
        x = x.reshape(1, -1, shape[-1]) if shape[-1] else x.reshape(1, 0, 0)
    return _LayerNorm.apply(x, weight, bias, eps, lens, checkpoint and _asks(x, weight, bias)).view(shape)


# ---------------------------------------------------------------- gated linear recurrence
_recurrence_gradient = _once("gated_recurrence")


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, h0, lens, keep):
        ctx.set_materialize_grads(False)
        out, final, states = B.gs_recurrence_forward(gate, x, h0, lens, keep=keep)
        ctx.save_for_backward(gate, x, h0, lens, states)
        return out, final

    @staticmethod
    def backward(ctx, dout, dfinal):
        gate, x, h0, lens, states = ctx.saved_tensors
        if dout is None and dfinal is None:
            return None, None, None, None, None

        def call(dout, dfinal, gate, x, h0):
            return B.gs_recurrence_backward(_rows_of_columns(dout), gate, x, h0, states,
                                            None if dfinal is None else dfinal.contiguous(), lens)
        dgate, dx, dh0 = _recurrence_gradient(call, dout, dfinal, gate, x, h0)
        return dgate, dx, None if h0 is None else dh0, None, None


def gated_recurrence(gate, x, h0=None, lens=None):
    """h_t = a_t h_(t-1) + (1 - a_t) x_t with a_t = sigmoid(gate_t), along the positions of gate, x[batch, length, channels] from
    h0 float32[batch, channels] (zeros if None).  Returns (h like x, the state after each sequence's last valid
    position, float32[batch, channels]); the state, handed in as h0, continues the sequences."""
    return _Recurrence.apply(gate, x, h0, lens, _asks(gate, x, h0))


# ---------------------------------------------------------------- activations in 8 bits
def _autocast():
    """The state of autocast: (device type, enabled, dtype, cache) of the types that tensors here may have."""
    cache = torch.is_autocast_cache_enabled()
    return [(k, torch.is_autocast_enabled(k), torch.get_autocast_dtype(k), cache) for k in ("cuda", "cpu")]


@contextlib.contextmanager
def _under(states):
    """Autocast as _autocast found it then."""
    with contextlib.ExitStack() as stack:
        for then, now in zip(states, _autocast()):
            if then != now and (then[1] or now[1]):
                kind, enabled, dtype, cache = then
                stack.enter_context(torch.autocast(kind, dtype, enabled, cache))
        yield


class _NoDraws(TorchDispatchMode):
    """Refuses operations that draw random numbers."""

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if torch.Tag.nondeterministic_seeded in func.tags:
            raise RuntimeError("a function that draws random numbers cannot be captured into a CUDA graph by kept_in_8_bits: "
                               "the call in the backward pass would draw others")
        return func(*args, **(kwargs or {}))


def _generators(x, others):
    """What a function of these arguments may draw from, with the present states."""
    gens = [torch.default_generator, *(o for o in others if isinstance(o, torch.Generator))]
    if x.is_cuda:
        gens.append(torch.cuda.default_generators[x.device.index])
    return [(g, g.get_state()) for g in gens]


@contextlib.contextmanager
def _drawing_from(states):
    """The generators as they were in `states`; afterwards as they are now."""
    now = [(g, g.get_state()) for g, _ in states]
    try:
        for g, state in states:
            g.set_state(state)
        yield
    finally:
        for g, state in now:
            g.set_state(state)


def _versions(tensors):
    """What changes when a tensor is written into (tensors of inference mode count nothing, and cannot be written into outside)."""
    return [None if t.is_inference() else t._version for t in tensors]


class _Kept(torch.autograd.Function):
    @staticmethod
    def forward(ctx, function, x, *others):
        tensors = [o for o in others if isinstance(o, torch.Tensor)]
        # x and the generators as the function finds them (states of generators cannot be had while a graph is captured)
        kept, versions = B.gs_checkpoint_pack(x if x.is_contiguous() else x.contiguous()), _versions((x, *tensors))
        capturing = x.is_cuda and torch.cuda.is_current_stream_capturing()
        random = [] if capturing else _generators(x, others)
        with torch.no_grad(), _NoDraws() if capturing else contextlib.nullcontext():
            out = _one_tensor(function(x, *others))
        if versions != _versions((x, *tensors)):
            raise RuntimeError("the function wrote into one of its arguments: it would do so again in the backward pass")
        ctx.function, ctx.dtype, ctx.autocast = function, x.dtype, _autocast()
        ctx.random = random if any(not torch.equal(state, g.get_state()) for g, state in random) else []
        ctx.plain = [None if isinstance(o, torch.Tensor) else o for o in others]
        ctx.is_tensor = [isinstance(o, torch.Tensor) for o in others]
        ctx.save_for_backward(*kept, *tensors)
        return out

    @staticmethod
    def backward(ctx, dout):
        if torch.is_grad_enabled():
            raise RuntimeError("kept_in_8_bits is differentiable once: call backward without create_graph")
        packed, scales, *tensors = ctx.saved_tensors
        wanted = [n for n, t in zip(ctx.needs_input_grad[2:], ctx.is_tensor) if t]
        x = B.gs_checkpoint_unpack(packed, scales, ctx.dtype).requires_grad_(ctx.needs_input_grad[1])
        tensors = [t.detach().requires_grad_(n) for t, n in zip(tensors, wanted)]
        with torch.enable_grad():
            it = iter(tensors)
            others = [next(it) if is_tensor else p for is_tensor, p in zip(ctx.is_tensor, ctx.plain)]
            with _under(ctx.autocast), _drawing_from(ctx.random):
                out = ctx.function(x, *others)
        asked = [t for t in (x, *tensors) if t.requires_grad]
        _only_from(out, asked)
        grads = iter(torch.autograd.grad(out, asked, dout, allow_unused=True) if out.requires_grad else [None] * len(asked))
        dx = next(grads) if x.requires_grad else None
        it = iter(tensors)
        rest = []
        for is_tensor in ctx.is_tensor:
            rest.append(next(grads) if is_tensor and next(it).requires_grad else None)
        return None, dx, *rest


_HIDDEN = "the function uses a tensor that requires a gradient and is not one of its arguments"


def _one_tensor(out):
    if not isinstance(out, torch.Tensor):
        raise TypeError("the function must return one tensor")
    return out


def _only_from(out, leaves):
    """Raises if `out` was computed from tensors that ask for gradients and are not among `leaves`."""
    known, seen, todo = {id(t) for t in leaves}, set(), [out.grad_fn]
    while todo:
        node = todo.pop()
        if node is None or node in seen:
            continue
        seen.add(node)
        variable = getattr(node, "variable", None)
        if variable is not None and id(variable) not in known:
            raise RuntimeError(_HIDDEN)
        todo += [n for n, _ in node.next_functions]


def kept_in_8_bits(function, x, *others):
    """function(x, *others), of which nothing but x in 8 bits (and the tensors among `others`: weights, lengths) is kept for the
    backward pass; that calls the function again, on x as the 8 bits have it, and differentiates it.  The result is exact, the
    gradients are those at the kept x.  The second call runs under the first one's autocast and draws the same random numbers (from
    torch's own generators and from arguments that are generators; while a CUDA graph is captured, a function that draws raises).  The
    function must return one tensor, give the same result when it is called again otherwise, leave
    its arguments as they are (this call raises if they changed) and take every tensor that requires a gradient as an argument itself, not
    in a list, a module or a closure: otherwise the backward pass raises, and this call does where no argument requires a gradient, so
    that there would be no backward pass."""
    if _asks(x, *others):
        return _Kept.apply(function, x, *others)
    out = _one_tensor(function(x, *others))
    if torch.is_grad_enabled() and out.requires_grad:
        raise RuntimeError(_HIDDEN)
    return out
