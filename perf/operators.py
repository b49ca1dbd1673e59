"""What is measured of the sequence-model operators: attention over walks (forward and backward)
and the global gradient norm with clipping.

`own = False` computes them in elementary torch operations in 32 bits, rounded once at the end;
`own = True` calls the library through `paper_2407_15452_b200.binding`.

Sequence j of a batch holds `lens[j]` valid positions (a walk that met a dead end is shorter than
walk_len; one from a refused start is empty).  Key j is visible to query i where
-window_left <= j - i <= window_right, a negative bound meaning none.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
LARGEST = 16 * 8192 * 8192           # head-pairs of the largest listed case


def _attention(name, op, dtype, batch, length, q_heads, kv_heads, head_dim, left, right, ragged):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "length": length,
            "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "left": left, "right": right, "ragged": ragged}


def listed():
    return [
        # the paper's synchronous batch of 512 walks with the 10-node walks, dim 64 and window 5 of
        # the tiny DeepWalk workload: all latency
        _attention("fwd_walk10_f32", "forward", "f32", 512, 10, 2, 2, 32, 5, 5, False),
        # a training batch of the 1M-node DeepWalk workload (40 nodes, dim 128, window 10), walks cut by dead ends
        _attention("fwd_walk40_bf16", "forward", "bf16", 16384, 40, 4, 4, 32, 10, 10, True),
        # next-token training of a sequence model with shared key/value heads
        _attention("fwd_causal2048_bf16", "forward", "bf16", 4, 2048, 16, 4, 128, -1, 0, False),
        # an odd, ragged batch of long sequences, every position sees every other
        _attention("fwd_ragged5003_f16", "forward", "f16", 3, 5003, 12, 12, 64, -1, -1, True),
        # the backward passes that belong to them
        _attention("bwd_walk10_f32", "backward", "f32", 512, 10, 2, 2, 32, 5, 5, False),
        # 80-node walks of the node2vec workload (dim 128, window 10)
        _attention("bwd_walk80_f16", "backward", "f16", 8192, 80, 4, 4, 32, 10, 10, True),
        # full precision, odd length, causal: a small model checked against its half-precision run
        _attention("bwd_causal333_f32", "backward", "f32", 8, 333, 4, 4, 64, -1, 0, False),
        _attention("bwd_causal2048_bf16", "backward", "bf16", 4, 2048, 16, 4, 128, -1, 0, False),
        # the longest: 8192 positions, all visible
        _attention("bwd_full8192_bf16", "backward", "bf16", 1, 8192, 16, 16, 128, -1, -1, False),
        # gradients of a one-layer walk encoder of dim 128, already within the bound: all latency
        {"name": "clip_encoder_f32", "op": "clip", "kind": "within", "dtype": "f32", "out": "same",
         "tensors": 14, "numel": 200_000},
        # the two dense table gradients of the 1M-node workload, clipped into the optimizer's buffers
        {"name": "clip_tables_f32", "op": "clip", "kind": "over", "dtype": "f32", "out": "f32",
         "tensors": 2, "numel": 256_000_000},
        # many odd-sized half-precision tensors of a deep model, clipped into full-precision gradients
        {"name": "clip_layers_bf16", "op": "clip", "kind": "over", "dtype": "bf16", "out": "f32",
         "tensors": 61, "numel": 150_000_000},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "clip"])
    if op == "clip":
        dtype = rng.choice(["f32", "f16", "bf16"])
        kind = rng.choice(["within", "over", "over"])
        return {"op": "clip", "kind": kind, "dtype": dtype,
                "out": "same" if kind == "within" else rng.choice(["f32", dtype]),
                "tensors": _log_int(rng, 1, 60), "numel": _log_int(rng, 20_000, 250_000_000)}
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]),
            "head_dim": rng.choice([32, 64, 64, 128, 128, 16, 80]), "ragged": rng.random() < 0.5}
    if rng.random() < 0.4:                                     # many short walks
        case["length"] = _log_int(rng, 2, 128)
        case["batch"] = _log_int(rng, 64, 16384)
        case["q_heads"] = case["kv_heads"] = rng.choice([1, 2, 4])
        case["left"] = case["right"] = rng.choice([3, 5, 10, -1])
        while case["batch"] * case["length"] * case["q_heads"] * case["head_dim"] > 1 << 27:
            case["batch"] = max(1, case["batch"] // 2)
    else:                                                      # fewer, longer sequences
        case["length"] = _log_int(rng, 1, 8192 if case["dtype"] != "f32" else 1500)
        case["batch"] = _log_int(rng, 1, 16)
        case["kv_heads"] = rng.choice([1, 2, 4, 8])
        case["q_heads"] = case["kv_heads"] * rng.choice([1, 1, 2, 4])
        case["left"], case["right"] = rng.choice([(-1, 0), (-1, 0), (-1, -1), (_log_int(rng, 16, 2048), 0)])
        most = LARGEST if case["dtype"] != "f32" else LARGEST // 64
        while case["batch"] > 1 and case["batch"] * case["q_heads"] * case["length"] ** 2 > most:
            case["batch"] //= 2
    return case


# ------------------------------------------------------------------ inputs
def _lengths(case, gen, device):
    if not case["ragged"]:
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


def _sizes(case):
    """Uneven tensor sizes, odd ones among them, that sum to case["numel"]: a pattern of large
    matrices and small vectors."""
    n, total = case["tensors"], case["numel"]
    weights = [(1.0 + (i * 7 % 11)) if i % 2 == 0 else 0.01 * (1 + i % 3) for i in range(n)]
    if n == 2:
        weights = [1.0, 1.0]
    s = sum(weights)
    sizes = [max(1, int(total * w / s)) | (1 if n > 2 else 0) for w in weights]
    return sizes


def prepare(case, seed):
    device = torch.device("cuda")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "clip":
        sizes = _sizes(case)
        grads = [torch.randn(s, generator=gen, device=device).mul_(1e-3 * (1 + i % 5)).to(dt)
                 for i, s in enumerate(sizes)]
        rms = math.sqrt(sum(s * (1 + i % 5) ** 2 for i, s in enumerate(sizes))) * 1e-3
        out = None if case["out"] == "same" else [torch.empty_like(g, dtype=DTYPES[case["out"]]) for g in grads]
        return {"case": case, "grads": grads, "out": out,
                "max_norm": rms * (4.0 if case["kind"] == "within" else 0.25)}
    b, n, hq, hk, d = (case[x] for x in ("batch", "length", "q_heads", "kv_heads", "head_dim"))
    state = {"case": case, "scale": 1.0 / math.sqrt(d), "window": (case["left"], case["right"]),
             "lens": _lengths(case, gen, device)}
    state["q"] = torch.randn((b, n, hq, d), generator=gen, device=device).to(dt)
    state["k"] = torch.randn((b, n, hk, d), generator=gen, device=device).to(dt)
    state["v"] = torch.randn((b, n, hk, d), generator=gen, device=device).to(dt)
    if case["op"] == "backward":       # what the forward pass left behind, and the gradient that arrives
        state["dout"] = torch.randn((b, n, hq, d), generator=gen, device=device).mul_(0.05).to(dt)
        state["out"], state["lse"] = _plain_forward(state)
    return state


# ------------------------------------------------------------------ plain forms, 32 bits
def _visible(case, lens, device):
    """[batch or 1, 1, length, length] truth values: query i sees key j."""
    n = case["length"]
    i = torch.arange(n, device=device)[:, None]
    j = torch.arange(n, device=device)[None, :]
    see = torch.ones((n, n), dtype=torch.bool, device=device)
    if case["left"] >= 0:
        see = see & (j >= i - case["left"])
    if case["right"] >= 0:
        see = see & (j <= i + case["right"])
    if lens is None:
        return see[None, None]
    m = lens[:, None, None]
    return (see[None] & (i[None] < m) & (j[None] < m))[:, None]


def _heads_first(x, group):
    x = x.float().permute(0, 2, 1, 3)
    return x if group == 1 else x.repeat_interleave(group, dim=1)


def _probabilities(state, q, k):
    see = _visible(state["case"], state["lens"], q.device)
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(state["scale"]).masked_fill_(~see, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    return p.div_(torch.where(total == 0, torch.ones_like(total), total)), lse


def _plain_forward(state):
    dt = state["q"].dtype
    group = state["case"]["q_heads"] // state["case"]["kv_heads"]
    q = _heads_first(state["q"], 1)
    k, v = _heads_first(state["k"], group), _heads_first(state["v"], group)
    p, lse = _probabilities(state, q, k)
    return torch.matmul(p, v).permute(0, 2, 1, 3).to(dt).contiguous(), lse


def _plain_backward(state):
    case, dt = state["case"], state["q"].dtype
    group = case["q_heads"] // case["kv_heads"]
    q, do = _heads_first(state["q"], 1), _heads_first(state["dout"], 1)
    k, v = _heads_first(state["k"], group), _heads_first(state["v"], group)
    p, _ = _probabilities(state, q, k)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2))
    ds = ds.sub_((p * ds).sum(dim=-1, keepdim=True)).mul_(p).mul_(state["scale"])
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q)
    if group > 1:
        b, _, n, d = dk.shape
        dk = dk.view(b, case["kv_heads"], group, n, d).sum(dim=2)
        dv = dv.view(b, case["kv_heads"], group, n, d).sum(dim=2)
    return tuple(x.permute(0, 2, 1, 3).to(dt).contiguous() for x in (dq, dk, dv))


def _plain_clip(state):
    grads, out = state["grads"], state["out"]
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    factor = torch.where(torch.isfinite(norm) & (norm > state["max_norm"]),
                         state["max_norm"] / norm, torch.ones_like(norm))
    targets = grads if out is None else out
    [t.copy_(g.float() * factor) for g, t in zip(grads, targets)]
    return norm.reshape(1), targets


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if not own:
        return {"forward": _plain_forward, "backward": _plain_backward, "clip": _plain_clip}[op](state)
    from paper_2407_15452_b200 import binding as B
    if op == "clip":
        norm = B.gs_clip_gradients(state["grads"], state["max_norm"], out=state["out"])
        return norm, state["grads"] if state["out"] is None else state["out"]
    how = {"scale": state["scale"], "window": state["window"], "q_lens": state["lens"], "k_lens": state["lens"]}
    if op == "forward":
        return B.gs_attention_forward(state["q"], state["k"], state["v"], **how)
    return B.gs_attention_backward(state["dout"], state["q"], state["k"], state["v"], state["out"],
                                   state["lse"], **how)


def _pairs(case):
    """Visible (query, key) pairs of one full-length sequence."""
    n, left, right = case["length"], case["left"], case["right"]
    left, right = (n if left < 0 else left), (n if right < 0 else right)
    return sum(min(n - 1, i + right) - max(0, i - left) + 1 for i in range(n))


def work(case):
    if case["op"] == "clip":
        n = sum(_sizes(case))
        wrote = 0 if case["kind"] == "within" else n * BYTES[case["out"]]
        return {"bytes": n * BYTES[case["dtype"]] + wrote + 4, "flops": 2 * n if case["kind"] == "within" else 3 * n}
    b, n, hq, hk, d = (case[x] for x in ("batch", "length", "q_heads", "kv_heads", "head_dim"))
    # lengths of a ragged batch by their mean: 0.8 + 0.2 / 2 of a walk, 0.65 of a document
    share = 1.0 if not case["ragged"] else 0.9 if n <= 128 else 0.65
    pairs = b * hq * _pairs(case) * (share if case["left"] >= 0 or not case["ragged"] else share * share + 0.04)
    es, rows_q, rows_k = BYTES[case["dtype"]], b * n * hq * d, b * n * hk * d
    if case["op"] == "forward":
        moved = es * (rows_q * (share + 1) + 2 * rows_k * share) + 4 * b * n * hq
        return {"bytes": int(moved), "flops": int(4 * d * pairs)}
    moved = es * (rows_q * (3 * share + 1) + rows_k * (2 * share + 2)) + 4 * b * n * hq * share
    return {"bytes": int(moved), "flops": int(10 * d * pairs)}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_slice(q, k, v, do, scale, left, right, n_valid):
    """One stack of sequences [s, heads, n, d] that share a length: rows and keys below n_valid."""
    s, h, n, d = q.shape
    score = torch.einsum("shid,shjd->shij", q, k) * scale
    dist = torch.arange(n, device=q.device)[None, :] - torch.arange(n, device=q.device)[:, None]
    hidden = torch.zeros((n, n), dtype=torch.bool, device=q.device)
    if left >= 0:
        hidden |= dist < -left
    if right >= 0:
        hidden |= dist > right
    pos = torch.arange(n, device=q.device)[None, :] >= n_valid[:, None]
    hidden = hidden[None, None] | pos[:, None, None, :] | pos[:, None, :, None]
    score[hidden.expand_as(score)] = -math.inf
    lse = torch.logsumexp(score, dim=-1)
    base = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
    prob = torch.exp(score - base[..., None])
    out = torch.einsum("shij,shjd->shid", prob, v)
    if do is None:
        return out, lse
    del score
    dprob = torch.einsum("shid,shjd->shij", do, v)
    dscore = prob * (dprob - (do * out).sum(-1, keepdim=True))
    del dprob
    return (torch.einsum("shij,shjd->shid", dscore, k) * scale,
            torch.einsum("shij,shid->shjd", dscore, q) * scale,
            torch.einsum("shij,shid->shjd", prob, do))


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "clip":
        norm = torch.sqrt(sum(torch.dot(g.double(), g.double()) for g in state["grads"]))
        # within the bound the gradients stay as they are
        factor = min(1.0, state["max_norm"] / float(norm))
        return norm.reshape(1), [g.double() * factor for g in state["grads"]]
    b, n, hq, hk, d = (case[x] for x in ("batch", "length", "q_heads", "kv_heads", "head_dim"))
    backward = case["op"] == "backward"
    dev = state["q"].device
    lens = state["lens"]
    lens = torch.full((b,), n, device=dev) if lens is None else lens.long()
    as64 = lambda x: x.double().transpose(1, 2)                                     # noqa: E731
    rows = dict(dtype=torch.float64, device=dev)
    if backward:
        got = [torch.zeros((b, n, h, d), **rows) for h in (hq, hk, hk)]
    else:
        got = [torch.zeros((b, n, hq, d), **rows), torch.zeros((b, hq, n), **rows)]
    step = max(1, (1 << 27) // (n * n))                       # sequences at a time, one query head each
    for h in range(hq):
        g = h // (hq // hk)
        for at in range(0, b, step):
            sl = slice(at, min(b, at + step))
            q, k, v = as64(state["q"][sl, :, h:h + 1]), as64(state["k"][sl, :, g:g + 1]), as64(state["v"][sl, :, g:g + 1])
            do = as64(state["dout"][sl, :, h:h + 1]) if backward else None
            part = _exact_slice(q, k, v, do, state["scale"], case["left"], case["right"], lens[sl])
            if backward:
                got[0][sl, :, h] = part[0][:, 0]
                got[1][sl, :, g] += part[1][:, 0]
                got[2][sl, :, g] += part[2][:, 0]
            else:
                got[0][sl, :, h] = part[0][:, 0]
                got[1][sl, h] = part[1][:, 0]
    return tuple(got)
