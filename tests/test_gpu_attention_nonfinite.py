"""Infinities and NaN at valid positions: what a row sees it must show, what it does not see it must not.

The definition is taken literally, in 64 bits and with every sum over visible positions only, so that a hidden
infinity or NaN has no factor of zero to meet.  A row whose every score is -infinity has lse -infinity and counts as
one that sees nothing.  Results must be NaN, +inf and -inf exactly where the definition is; all
other elements are checked against bounds made like those of tests/attention_reference.py."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests.attention_reference import E32, UNIT, visible

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ALL, CAUSAL = (-1, -1), (-1, 0)
INF, NAN = math.inf, math.nan
DEV = "cuda"


def finite(x):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x))


def pair_sum(w, x, see):
    """sum_j w[i, j] x[j, c] over the pairs that are seen"""
    return torch.where(see[:, :, None], w[:, :, None] * x[None], torch.zeros((), dtype=w.dtype, device=w.device)).sum(1)


def dots(x, y):
    return (x[:, None] * y[None]).sum(-1)


def literal_forward(q, k, v, scale, see, dt):
    """One head: out, lse and their bounds."""
    d, lk = q.shape[1], k.shape[0]
    u, u_p = UNIT[dt], 0.0 if dt == F32 else 2 * UNIT[dt]
    s = (dots(q, k) * scale).masked_fill(~see, -INF)
    es = ((d + 4) * E32 * scale * dots(finite(q).abs(), finite(k).abs())).masked_fill(~see, 0.0)
    lse = torch.logsumexp(s, -1)
    p = torch.where(torch.isneginf(lse)[:, None], torch.zeros_like(s), torch.exp(s - lse[:, None]))
    ep = 2 * es.amax(-1, keepdim=True) + (lk + 16) * E32 + 2 * E32 * finite(lse).abs()[:, None]
    out = pair_sum(p, v, see)
    a = pair_sum(finite(p), finite(v).abs(), see)
    tiny = 2.0 ** -24 if dt == F16 else 0.0
    b_out = (ep + lk * E32 + u_p) * a + u * finite(out).abs() + tiny * (see.double() @ finite(v).abs()) + 1e-30
    if dt == F16:
        b_out = b_out + 2.0 ** -25
    return out, lse, p, ep, b_out, ep.squeeze(-1) + 2 * E32 * finite(lse).abs()


def literal_backward(q, k, v, do, out, lse, b_out, p, ep, scale, see, dt):
    d, lk, lq = q.shape[1], k.shape[0], q.shape[0]
    u, u_p = UNIT[dt], 0.0 if dt == F32 else 2 * UNIT[dt]
    dp = dots(do, v)
    nothing = torch.zeros((), dtype=p.dtype, device=p.device)
    gives = ~torch.isneginf(lse)
    delta = torch.where(gives, (do * out).sum(-1), nothing)[:, None]
    ds = torch.where(see & gives[:, None], p * (dp - delta), nothing)
    fdo, fv, fout = finite(do).abs(), finite(v).abs(), finite(out).abs()
    e_delta = (d + 2) * E32 * (fdo * fout).sum(-1, keepdim=True) + (fdo * finite(b_out)).sum(-1, keepdim=True)
    e_dp = (d + 2) * E32 * dots(fdo, fv)
    fp, fds = finite(p).abs(), finite(ds).abs()
    e_ds = (fds * (ep + u_p) + fp * (e_dp + e_delta)) * (1 + u_p)
    e_pp = fp * (ep + u_p)
    if dt == F16:
        top = (fdo.norm(dim=-1).amax() * fv.norm(dim=-1).amax()).item()
        e_ds = e_ds + 2.0 ** -24 * top * see
        e_pp = e_pp + 2.0 ** -24 * see
    dq = pair_sum(ds, k, see & gives[:, None]) * scale
    b_dq = (e_ds + lk * E32 * fds) @ finite(k).abs() * scale + u * finite(dq).abs()
    t, n = (see & gives[:, None]).transpose(0, 1), lq
    dk = pair_sum(ds.transpose(0, 1), q, t) * scale
    b_dk = ((e_ds + n * E32 * fds) * see).transpose(0, 1) @ finite(q).abs() * scale
    dv = pair_sum(p.transpose(0, 1), do, t)
    b_dv = ((e_pp + n * E32 * fp) * see).transpose(0, 1) @ finite(do).abs()
    return (dq, b_dq), (dk, b_dk), (dv, b_dv)


def same(got, want, bound, what, factor=1.0):
    """`factor`: what the kernels multiply the finished fp32 sum by; where the sum itself is beyond fp32, nothing is asked."""
    got, want = got.double(), want.double()
    beyond = torch.isfinite(want) & (want.abs() >= factor * torch.finfo(F32).max)
    got, want = got.masked_fill(beyond, 0.0), want.masked_fill(beyond, 0.0)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), \
        f"{what}: NaN in {torch.isnan(got).sum().item()} places, in {torch.isnan(want).sum().item()} by definition"
    odd = (torch.isinf(got) | torch.isinf(want)) & (got != want)
    assert not odd.any(), f"{what}: {got[odd][:4].tolist()} where the definition has {want[odd][:4].tolist()}, {odd.sum().item()} in all"
    ok = torch.isfinite(want)
    off = (got - want).abs()[ok] - bound.expand_as(want)[ok]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: beyond its bound by {off.max().item():.3e}"


def run(q, k, v, do, window, lens=None):
    b, lq, hq, d = q.shape
    lk, hk, dt = k.shape[1], k.shape[2], q.dtype
    group, scale = hq // hk, d ** -0.5
    out, lse = B.gs_attention_forward(q, k, v, scale, window, lens, lens)
    dq, dk, dv = B.gs_attention_backward(do, q, k, v, out, lse, scale, window, lens, lens)
    tail = 2.0 ** -25 if dt == F16 else 1e-30
    u = UNIT[dt]
    for s in range(b):
        n = lq if lens is None else int(lens[s])
        see = visible(n, n, lq, lk, window, DEV)[:n, :n]
        for g in range(hk if n else 0):
            K, V = k[s, :n, g].double(), v[s, :n, g].double()
            total = {"dk": [0.0, 0.0], "dv": [0.0, 0.0]}
            for h in range(g * group, (g + 1) * group):
                Q, DO = q[s, :n, h].double(), do[s, :n, h].double()
                o, ls, p, ep, b_o, b_l = literal_forward(Q, K, V, scale, see, dt)
                same(out[s, :n, h], o, b_o, f"out[{s}, :, {h}]")
                same(lse[s, h, :n], ls, b_l, f"lse[{s}, {h}]")
                (x, bx), *kv = literal_backward(Q, K, V, DO, o, ls, b_o, p, ep, scale, see, dt)
                same(dq[s, :n, h], x, bx + tail, f"dq[{s}, :, {h}]", scale)
                for name, (y, by) in zip(("dk", "dv"), kv):
                    total[name][0] = total[name][0] + y
                    total[name][1] = total[name][1] + by
            for name, got in (("dk", dk), ("dv", dv)):
                y, by = total[name]
                same(got[s, :n, g], y, by + u * finite(y).abs() + tail, f"{name}[{s}, :, {g}]", scale if name == "dk" else 1.0)
        for name, got in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert not got[s, n:].any(), f"{name}: padding"
        assert torch.isneginf(lse[s, :, n:]).all()


def tensors(b, n, hq, hk, d, dt, seed, wide=False):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def make(h, gain=1.0):
        x = (torch.randn((b, n, h, d), generator=gen, device=DEV) * gain).to(dt)
        if wide:                                           # rows that TMA cannot address
            room = torch.full((b, n, h, d + 1), NAN, dtype=dt, device=DEV)
            room[..., :d] = x
            x = room[..., :d]
        return x
    return make(hq), make(hk), make(hk), make(hq, 0.25)


# batch, length, query heads, key/value heads, head_dim, rows without TMA: one for each kernel that a type may reach
SHAPES = {
    "walk12x32": (3, 12, 2, 2, 32, False), "walk40x16": (2, 40, 2, 1, 16, False), "walk70x64": (2, 70, 4, 2, 64, False),
    "walk100x128": (2, 100, 2, 2, 128, False), "odd40x32": (2, 40, 2, 2, 32, True), "long200x64": (2, 200, 2, 1, 64, False),
    "long300x128": (1, 300, 2, 2, 128, False), "odd200x64": (2, 200, 2, 2, 64, True), "many150x64": (40, 150, 4, 4, 64, False),
    "many90x32": (75, 90, 2, 2, 32, False),
}
PLANTS = {
    "v_inf": lambda q, k, v, do, at: v[:, at, :, 3].fill_(INF),
    "v_inf_both_signs": lambda q, k, v, do, at: (v[:, at, :, 3].fill_(INF), v[:, at + 2, :, 3].fill_(-INF)),
    "v_nan": lambda q, k, v, do, at: v[:, at].fill_(NAN),
    "k_nan": lambda q, k, v, do, at: k[:, at].fill_(NAN),
    "k_inf": lambda q, k, v, do, at: k[:, at, :, 1].fill_(INF),            # scores of either sign, by q's
    "k_scores_minus_inf": lambda q, k, v, do, at: (k[:, at, :, 1].fill_(-INF), q[..., 1].abs_().add_(0.5)),
    "q_nan": lambda q, k, v, do, at: q[:, at].fill_(NAN),
    "q_inf": lambda q, k, v, do, at: q[:, at, :, 2].fill_(INF),
    "do_inf": lambda q, k, v, do, at: do[:, at, :, 0].fill_(-INF),
    "do_nan": lambda q, k, v, do, at: do[:, at].fill_(NAN),
}


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("plant", list(PLANTS))
@pytest.mark.parametrize("shape", list(SHAPES))
def test_only_what_is_seen(shape, plant, dt):
    b, n, hq, hk, d, wide = SHAPES[shape]
    for window, lens in ((CAUSAL, None), ((2, 2), None), (CAUSAL, "ragged")):
        if lens and b > 8:
            continue
        q, k, v, do = tensors(b, n, hq, hk, d, dt, seed=n, wide=wide)
        if b > 8:                                          # a few of many sequences
            q1, k1, v1, do1 = (t[5:7] for t in (q, k, v, do))
        else:
            q1, k1, v1, do1 = q, k, v, do
        PLANTS[plant](q1, k1, v1, do1, n // 2)
        m = None
        if lens:
            m = torch.tensor([n - 3, n // 2 + 1, 0][:b], dtype=torch.int32, device=DEV)
            for s in range(b):
                for t in (q, k, v, do):
                    t[s, int(m[s]):] = NAN
        run(q, k, v, do, window, m)


@pytest.mark.parametrize("shape", list(SHAPES))
def test_values_that_round_up_to_infinity_at_eleven_bits(shape):
    b, n, hq, hk, d, wide = SHAPES[shape]
    q, k, v, do = tensors(b, n, hq, hk, d, F32, seed=n, wide=wide)
    most = torch.finfo(F32).max
    k[:, n // 2, :, 1] = most
    q[..., 1] = 0.0
    v[:, n // 3, :, 0] = most
    do[..., 0] = 0.0
    q[..., 1] = 0.0
    run(q, k, v, do, CAUSAL)


def test_an_infinity_does_not_cost_other_rows_their_precision():
    # gradients that binary16 holds only when scaled, beside a row that is not finite
    for n in (40, 300):
        q, k, v, do = tensors(1, n, 2, 2, 64, F16, seed=n)
        do.mul_(2.0 ** -12)
        v[:, n - 2, :, 3] = INF
        run(q, k, v, do, CAUSAL)


@pytest.mark.parametrize("n", [40, 300])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_everything_nan(n, dt):
    q, k, v, do = tensors(2, n, 2, 2, 64, dt, seed=n)
    v.fill_(NAN)
    run(q, k, v, do, CAUSAL)
