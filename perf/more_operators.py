"""What is measured of the layers around attention: layer norm (forward and backward), a gated linear
recurrence (forward, backward, one position at a time) and activation checkpoints in 8 bits.

`own = False` computes them in elementary torch operations in 32 bits, rounded once at the end;
`own = True` calls the library through `paper_2407_15452_b200.binding`.

Tensors are [batch, length, columns].  Sequence b holds `lens[b]` valid positions (a walk that met a dead end
is shorter than walk_len, one from a refused start is empty); positions behind them give zeros and no gradient.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
LARGEST = 4 * 8192 * 2048            # elements of the largest listed cases
EPS = 1e-5
SPAN = 128                           # positions between two kept states of the recurrence
BLOCK = 128                          # columns that share a scale of a checkpoint


def _norm(name, op, dtype, batch, length, columns, ragged, weights="f32"):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "length": length, "columns": columns,
            "ragged": ragged, "weights": weights}


def _recurrence(name, op, dtype, batch, length, columns, ragged, start=False):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "length": length, "columns": columns,
            "ragged": ragged, "start": start}


def listed():
    return [
        # the paper's batch of 512 walks with the 10-node walks and dim 64 of the tiny DeepWalk workload: all latency
        _norm("norm_fwd_walk10_f32", "norm_forward", "f32", 512, 10, 64, False),
        # a wide layer of a deep sequence model
        _norm("norm_fwd_wide_bf16", "norm_forward", "bf16", 4, 4096, 4096, False),
        # a training batch of the 1M-node DeepWalk workload (40 nodes, dim 128), walks cut by dead ends
        _norm("norm_bwd_walk40_bf16", "norm_backward", "bf16", 16384, 40, 128, True),
        # rows that no vector access fits: an odd number of columns, weights of the tensors' type
        _norm("norm_bwd_odd1001_f16", "norm_backward", "f16", 16, 1250, 1001, False, "same"),
        # forward that keeps its input in 8 bits, and the backward pass from it
        _norm("norm_checkpoint_wide_bf16", "norm_checkpoint", "bf16", 4, 4096, 4096, False),
        # one more position for many open sequences: all latency
        _recurrence("scan_step_bf16", "scan_forward", "bf16", 256, 1, 1024, False, True),
        # training passes over the walks of the 1M-node and of the node2vec workload (80 nodes)
        _recurrence("scan_fwd_walk40_bf16", "scan_forward", "bf16", 16384, 40, 128, True),
        _recurrence("scan_bwd_walk80_f16", "scan_backward", "f16", 8192, 80, 128, True),
        # long sequences of a wide model, both directions
        _recurrence("scan_fwd_long_bf16", "scan_forward", "bf16", 4, 8192, 2048, False),
        _recurrence("scan_bwd_long_bf16", "scan_backward", "bf16", 4, 8192, 2048, False),
        # an odd, ragged batch in full precision that goes on from given states
        _recurrence("scan_bwd_ragged5003_f32", "scan_backward", "f32", 3, 5003, 777, True, True),
        # activations of the paper's batch kept in 8 bits and brought back
        {"name": "checkpoint_walk40_f32", "op": "checkpoint", "dtype": "f32", "batch": 512, "length": 40, "columns": 128},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "norm_checkpoint", "scan_forward", "scan_forward", "scan_backward",
                     "scan_backward", "checkpoint"])
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    most = LARGEST if case["dtype"] != "f32" else LARGEST // 2
    if op.startswith("scan"):
        kind = rng.choice(["walks", "walks", "long", "long", "step"])
        case["columns"] = rng.choice([64, 128, 128, 256, _log_int(rng, 16, 300)])
        if kind == "walks":
            case["batch"], case["length"] = _log_int(rng, 64, 16384), _log_int(rng, 2, 128)
        elif kind == "long":
            case["batch"], case["length"] = _log_int(rng, 1, 8), _log_int(rng, 129, 32768)
            case["columns"] = rng.choice([64 * _log_int(rng, 1, 64), _log_int(rng, 33, 4096)])
        else:
            case["batch"], case["length"] = _log_int(rng, 1, 1024), 1
            case["columns"] = 64 * _log_int(rng, 1, 64)
        case["ragged"], case["start"] = kind != "step" and rng.random() < 0.5, kind == "step" or rng.random() < 0.3
    else:
        case["batch"], case["length"] = _log_int(rng, 1, 2048), _log_int(rng, 1, 512)
        case["columns"] = rng.choice([64, 128, 256, 32 * _log_int(rng, 1, 256), _log_int(rng, 3, 8192)])
        if op != "checkpoint":
            case["ragged"], case["weights"] = rng.random() < 0.4, rng.choice(["f32", "same"])
    while case["batch"] * case["length"] * case["columns"] > most:
        if case["batch"] > 1:
            case["batch"] = (case["batch"] + 1) // 2
        else:
            case["length"] = (case["length"] + 1) // 2
    return case


# ------------------------------------------------------------------ inputs
def _lengths(case, gen, device):
    if not case.get("ragged"):
        return None
    b, n = case["batch"], case["length"]
    u = torch.rand(b, generator=gen, device=device)
    cut = torch.rand(b, generator=gen, device=device)
    if n <= 128:        # walks: four in five are complete, the others end early, some before they began
        lens = torch.where(u < 0.8, torch.full_like(u, float(n)), torch.floor(cut * n))
    else:               # documents padded to the longest
        lens = torch.ceil((0.3 + 0.7 * cut) * n)
        lens[0] = n
    return lens.to(torch.int32)


def prepare(case, seed):
    device = torch.device("cuda")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    shape = b, n, c = case["batch"], case["length"], case["columns"]
    rand = lambda *size: torch.randn(size, generator=gen, device=device)                     # noqa: E731
    state = {"case": case, "lens": _lengths(case, gen, device)}
    if case["op"].startswith("scan"):
        # gates of channels that forget within a position or two up to such that remember hundreds
        slow = torch.rand(c, generator=gen, device=device).mul_(6.0).sub_(1.0)
        state["gate"] = rand(*shape).add_(slow).to(dt)
        state["x"] = rand(*shape).to(dt)
        state["start"] = rand(b, c) if case["start"] else None
        if case["op"] == "scan_backward":
            state["dout"] = rand(*shape).mul_(0.05).to(dt)
            state["dfinal"] = rand(b, c).mul_(0.05) if case["start"] else None
            state["states"] = _plain_scan(state)[2]
        return state
    # activations: columns of their own mean and spread, a few of them an order of magnitude larger
    spread = torch.exp(rand(c) * 0.3) * (1.0 + 9.0 * (torch.rand(c, generator=gen, device=device) < 0.01))
    state["x"] = rand(*shape).add_(rand(c) * 0.5).mul_(spread).to(dt)
    if case["op"] == "checkpoint":
        return state
    wt = dt if case["weights"] == "same" else torch.float32
    state["weight"] = rand(c).mul_(0.2).add_(1.0).to(wt)
    state["bias"] = rand(c).mul_(0.2).to(wt)
    if case["op"] != "norm_forward":
        state["dy"] = rand(*shape).mul_(0.05).to(dt)
    if case["op"] == "norm_backward":                  # what the forward pass left behind
        state["stats"] = _plain_norm(state)[1]
    return state


# ------------------------------------------------------------------ plain forms, 32 bits
def _valid(state):
    """[batch, length, 1] truth values, or None where every position is valid."""
    lens, n = state["lens"], state["case"]["length"]
    return None if lens is None else (torch.arange(n, device=lens.device) < lens[:, None])[:, :, None]


def _hide(x, valid):
    return x if valid is None else x.masked_fill_(~valid, 0.0)


def _plain_norm(state):
    x, valid = state["x"].float(), _valid(state)
    mean = x.mean(dim=-1, keepdim=True)
    x = x - mean
    rstd = (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
    y = (x * rstd).mul_(state["weight"].float()).add_(state["bias"].float())
    return _hide(y, valid).to(state["x"].dtype), _hide(torch.cat([mean, rstd], dim=-1), valid)


def _plain_norm_backward(state, x, stats):
    dy, valid, w = state["dy"].float(), _valid(state), state["weight"].float()
    xh = _hide((x - stats[..., :1]).mul_(stats[..., 1:]), valid)
    dy = dy if valid is None else dy.masked_fill(~valid, 0.0)
    dw, db = (dy * xh).sum(dim=(0, 1)), dy.sum(dim=(0, 1))
    g = dy * w
    dx = g - g.mean(dim=-1, keepdim=True)
    dx.sub_(xh * (g.mul_(xh)).mean(dim=-1, keepdim=True)).mul_(stats[..., 1:])
    return _hide(dx, valid).to(state["x"].dtype), dw.to(state["weight"].dtype), db.to(state["bias"].dtype)


def _plain_checkpoint(x):
    """The values that the 8 bits stand for, in fp32: blocks of 128 columns, steps of amax / 127 rounded towards zero
    to fp32, the nearest whole number of steps (decided in 64 bits: a quotient must not be rounded onto a tie)."""
    c = x.shape[-1]
    v = torch.nn.functional.pad(x.float(), (0, -c % BLOCK)).unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(dim=-1, keepdim=True).double()
    step = (amax / 127).float()
    step = torch.where(step.double() * 127 > amax, torch.nextafter(step, torch.zeros_like(step)), step)
    q = (v / step.double()).round_().clamp_(-127, 127)
    return torch.where(step == 0, 0.0, q.float() * step).flatten(-2)[..., :c]


def _shifted(a, by, fill):
    """a moved by `by` positions towards the end (towards the start if negative), `fill` in the places left."""
    n = a.shape[1]
    out = torch.full_like(a, fill)
    if by > 0:
        out[:, by:] = a[:, :n - by]
    else:
        out[:, :n + by] = a[:, -by:]
    return out


def _plain_linear(a, b, sign):
    """y_t = a_t y_(t - sign) + b_t from zero, by doubling; overwrites both."""
    by = 1
    while by < a.shape[1]:
        b.addcmul_(a, _shifted(b, sign * by, 0.0))
        a.mul_(_shifted(a, sign * by, 1.0))
        by *= 2
    return b


def _plain_gates(state):
    z, valid = state["gate"].float(), _valid(state)
    a, u = 1.0 / (1.0 + torch.exp(-z)), 1.0 / (1.0 + torch.exp(z))
    if valid is not None:              # the state passes through positions behind the end
        a, u = a.masked_fill_(~valid, 1.0), u.masked_fill_(~valid, 0.0)
    return a, u


def _plain_states(state, a, u):
    b = u * _hide(state["x"].float(), _valid(state))
    if state["start"] is not None:
        b[:, 0].addcmul_(a[:, 0], state["start"])
    return _plain_linear(a.clone(), b, 1)


def _plain_scan(state):
    a, u = _plain_gates(state)
    h = _plain_states(state, a, u)
    final = h[:, -1].clone()
    kept = h[:, SPAN - 1:-1:SPAN].contiguous()
    return _hide(h, _valid(state)).to(state["x"].dtype), final, kept


def _plain_scan_backward(state):
    valid = _valid(state)
    a, u = _plain_gates(state)
    before = _shifted(_plain_states(state, a, u), 1, 0.0)
    if state["start"] is not None:
        before[:, 0] = state["start"]
    dout = state["dout"].float()
    dout = dout if valid is None else dout.masked_fill(~valid, 0.0)
    if state["dfinal"] is not None:
        dout[:, -1] += state["dfinal"]
    g = _plain_linear(_shifted(a, -1, 0.0), dout.clone(), -1)
    dstart = a[:, 0] * g[:, 0]
    dx = g * u
    dgate = before.sub_(_hide(state["x"].float(), valid)).mul_(dx).mul_(a)
    dt = state["x"].dtype
    return _hide(dgate, valid).to(dt), _hide(dx, valid).to(dt), dstart


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if not own:
        if op == "norm_forward":
            return _plain_norm(state)
        if op == "norm_backward":
            return _plain_norm_backward(state, state["x"].float(), state["stats"])
        if op == "norm_checkpoint":
            y, stats = _plain_norm(state)
            return (y,) + _plain_norm_backward(state, _plain_checkpoint(state["x"]), stats)
        if op == "scan_forward":
            return _plain_scan(state)
        if op == "scan_backward":
            return _plain_scan_backward(state)
        return _plain_checkpoint(state["x"]).to(state["x"].dtype)
    from paper_2407_15452_b200 import binding as B
    x, lens = state["x"], state["lens"]
    if op == "norm_forward":
        return B.gs_layer_norm_forward(x, state["weight"], state["bias"], EPS, lens)
    if op == "norm_backward":
        return B.gs_layer_norm_backward(state["dy"], x, state["weight"], state["bias"], state["stats"], lens)
    if op == "norm_checkpoint":
        y, stats, packed, scales = B.gs_layer_norm_forward(x, state["weight"], state["bias"], EPS, lens, checkpoint=True)
        return (y,) + B.gs_layer_norm_backward(state["dy"], packed, state["weight"], state["bias"], stats, lens,
                                               scales=scales)
    if op == "scan_forward":
        return B.gs_recurrence_forward(state["gate"], x, state["start"], lens)
    if op == "scan_backward":
        return B.gs_recurrence_backward(state["dout"], state["gate"], x, state["start"], state["states"],
                                        state["dfinal"], lens)
    return B.gs_checkpoint_unpack(*B.gs_checkpoint_pack(x), x.dtype)


def work(case):
    b, n, c, es = case["batch"], case["length"], case["columns"], BYTES[case["dtype"]]
    # lengths of a ragged batch by their mean: 0.8 + 0.2 / 2 of a walk, 0.65 of a document
    share = 1.0 if not case.get("ragged") else 0.9 if n <= 128 else 0.65
    whole = b * n * c                          # outputs are written at every position
    read = whole * share
    if case["op"] == "checkpoint":
        kept = whole + 4 * b * n * -(-c // BLOCK)
        return {"bytes": 2 * es * whole + 2 * kept, "flops": 4 * whole}
    if case["op"].startswith("scan"):
        states = 4 * b * c * ((n - 1) // SPAN)
        ends = 4 * b * c * (2 if case["start"] else 1)
        if case["op"] == "scan_forward":
            return {"bytes": int(es * (2 * read + whole) + states + ends), "flops": int(8 * read)}
        return {"bytes": int(es * (3 * read + 2 * whole) + states + 2 * ends), "flops": int(16 * read)}
    stats, vectors = 8 * b * n, 2 * c * (4 if case["weights"] == "f32" else es)
    forward = es * (read + whole) + stats + vectors
    backward = es * (2 * read + whole) + stats + 2 * vectors
    if case["op"] == "norm_forward":
        return {"bytes": int(forward), "flops": int(8 * read)}
    if case["op"] == "norm_backward":
        return {"bytes": int(backward), "flops": int(14 * read)}
    kept = whole + 4 * b * n * -(-c // BLOCK)
    return {"bytes": int(forward + backward - es * read + 2 * kept), "flops": int(26 * read)}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_kept(x):
    """Values of a checkpoint, block by block of columns."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[-1], BLOCK):
        v = x[..., at:at + BLOCK].double()
        top = v.abs().max(dim=-1, keepdim=True).values
        s = (top / 127.0).float().double()
        below = torch.nextafter(s.float(), torch.tensor(0.0, device=x.device)).double()
        s = torch.where(s * 127.0 <= top, s, below)
        steps = torch.clamp(torch.round(v / s), -127, 127)
        out[..., at:at + BLOCK] = torch.where(s > 0, steps * s, torch.zeros_like(v))
    return out


def _exact_norm(case, state, real):
    """y, stats and the gradients; the gradients from the checkpoint where the case keeps one."""
    x = state["x"].double()
    mean = x.mean(-1)
    var = torch.var(x, dim=-1, correction=0)
    rstd = 1.0 / torch.sqrt(var + EPS)
    w, b = state["weight"].double(), state["bias"].double()
    stats = torch.stack([mean, rstd], -1) * real[..., None]
    if case["op"] == "norm_forward":
        y = torch.addcmul(b, (x - mean[..., None]) * rstd[..., None], w)
        return y * real[..., None], stats
    y = None
    if case["op"] == "norm_checkpoint":
        y = torch.addcmul(b, (x - mean[..., None]) * rstd[..., None], w) * real[..., None]
        x = _exact_kept(state["x"])
    hat = (x - mean[..., None]) * (rstd * real)[..., None]
    dy = state["dy"].double() * real[..., None]
    dw, db = torch.einsum("bnc,bnc->c", dy, hat), torch.einsum("bnc->c", dy)
    m1 = torch.einsum("bnc,c->bn", dy, w) / case["columns"]
    m2 = torch.einsum("bnc,bnc,c->bn", dy, hat, w) / case["columns"]
    dx = (dy * w - m1[..., None] - hat * m2[..., None]) * (rstd * real)[..., None]
    return (dx, dw, db) if y is None else (y, dx, dw, db)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "checkpoint":
        return _exact_kept(state["x"])
    x, b, n, c = state["x"], case["batch"], case["length"], case["columns"]
    lens = torch.full((b,), n, device=x.device) if state["lens"] is None else state["lens"].long()
    real = (torch.arange(n, device=x.device)[None, :] < lens[:, None]).double()
    if not case["op"].startswith("scan"):
        return _exact_norm(case, state, real)
    # position by position
    rows = dict(dtype=torch.float64, device=x.device)
    h = torch.zeros((b, c), **rows) if state["start"] is None else state["start"].double()
    if case["op"] == "scan_forward":
        out, kept = torch.empty((b, n, c), **rows), torch.empty((b, (n - 1) // SPAN, c), **rows)
        for t in range(n):
            if t and t % SPAN == 0:
                kept[:, t // SPAN - 1] = h
            on = real[:, t, None]
            a = torch.sigmoid(state["gate"][:, t].double())
            h = torch.where(on > 0, a * h + (1.0 - a) * x[:, t].double(), h)
            out[:, t] = h * on
        return out, h, kept
    was = torch.empty((b, n, c), **rows)
    for t in range(n):
        was[:, t] = h
        a = torch.sigmoid(state["gate"][:, t].double())
        h = torch.where(real[:, t, None] > 0, a * h + (1.0 - a) * x[:, t].double(), h)
    dgate, dx = torch.empty((b, n, c), **rows), torch.empty((b, n, c), **rows)
    g = torch.zeros((b, c), **rows) if state["dfinal"] is None else state["dfinal"].double()
    for t in range(n - 1, -1, -1):
        on = real[:, t, None]
        z = state["gate"][:, t].double()
        a, u = torch.sigmoid(z), torch.sigmoid(-z)
        full = g + state["dout"][:, t].double() * on
        dx[:, t] = full * u * on
        dgate[:, t] = full * (was[:, t] - x[:, t].double()) * a * u * on
        g = torch.where(on > 0, full * a, g)
    return dgate, dx, g
