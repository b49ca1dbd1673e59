"""Attention and its gradient in 64 bits, with bounds on what a correct kernel may be off by.

The bounds follow the kernels' arithmetic, element by element (u = unit roundoff of the tensors'
type, e = 2^-24 of fp32, n = number of keys or queries summed over, d = head_dim):
  scores      E_s  = (d + 4) e scale sum_d |q||k|                   (fp32 sums of exact products)
  p           relative E_p = 2 max_j E_s + (n + 16) e               (exponent error, exp, sum, quotient)
  out         (E_p + n e + u_p) A + u |out| + tiny,  A = sum_j p |v|, u_p = 2u for 16-bit types (p rounded once)
  delta       (d + 2) e sum_d |do||out| + (bound of out as stored) . |do|
  dp          (d + 2) e sum_d |do||v|
  ds          |ds| (E_p + u_p) + p (E_dp + E_delta)
  dq, dk, dv  the sums of those over the products, + n e of the sums, + u of the result.
binary16 loses relative precision below 2^-14: a probability is off by up to 2^-25 there (scaled so
that a row's largest is of order one in the forward pass), a score gradient by 2^-25 in its scaled form.
"""
import math

import torch

E32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def visible(nq, nk, lq, lk, window, device):
    i = torch.arange(lq, device=device)[:, None]
    j = torch.arange(lk, device=device)[None, :]
    see = (i < nq) & (j < nk)
    at = j - (i + nk - nq)
    if window[0] >= 0:
        see = see & (at >= -window[0])
    if window[1] >= 0:
        see = see & (at <= window[1])
    return see


def _clean(x, n):
    """[L, h, d] as fp64 [h, L, d]; whatever stands at or beyond n becomes zero."""
    x = x.double().clone()
    x[n:] = 0.0
    return x.transpose(0, 1)


def reference(q, k, v, scale, window, q_lens=None, k_lens=None, dout=None):
    """Returns a dict of fp64 results and `<name>_bound`: out, lse and, with dout, dq, dk, dv."""
    b, lq, hq, d = q.shape
    lk, hk = k.shape[1], k.shape[2]
    group, dt, dev = hq // hk, q.dtype, q.device
    u = UNIT[dt]
    u_p = 0.0 if dt == torch.float32 else 2 * u
    tiny_p = 2.0 ** -24 if dt == torch.float16 else 0.0
    z = dict(dtype=torch.float64, device=dev)
    r = {"out": torch.zeros((b, lq, hq, d), **z), "lse": torch.full((b, hq, lq), -math.inf, **z)}
    r["out_bound"], r["lse_bound"] = torch.zeros_like(r["out"]), torch.zeros_like(r["lse"])
    if dout is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", k)):
            r[name] = torch.zeros(like.shape, **z)
            r[name + "_bound"] = torch.zeros(like.shape, **z)
    for s in range(b):
        nq = lq if q_lens is None else int(q_lens[s].clamp(0, lq))
        nk = lk if k_lens is None else int(k_lens[s].clamp(0, lk))
        see = visible(nq, nk, lq, lk, window, dev)
        Q = _clean(q[s], nq)
        K = _clean(k[s], nk).repeat_interleave(group, 0)
        V = _clean(v[s], nk).repeat_interleave(group, 0)
        S = Q @ K.transpose(-1, -2) * scale
        Es = ((d + 4) * E32 * scale * (Q.abs() @ K.abs().transpose(-1, -2))).masked_fill(~see, 0.0)
        S = S.masked_fill(~see, -math.inf)
        lse = torch.logsumexp(S, -1)
        base = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
        P = torch.exp(S - base[..., None])
        if lk == 0:
            continue
        Ep = 2 * Es.amax(-1, keepdim=True) + (lk + 16) * E32 + 2 * E32 * base.abs()[..., None]
        out = P @ V
        A = P @ V.abs()
        u_out = (Ep + lk * E32 + u_p) * A + u * out.abs() + tiny_p * (see.double() @ V.abs()) + 1e-30
        if dt == torch.float16:
            u_out = u_out + 2.0 ** -25
        r["out"][s], r["out_bound"][s] = out.transpose(0, 1), u_out.transpose(0, 1)
        r["lse"][s] = lse
        r["lse_bound"][s] = Ep.squeeze(-1) + 2 * E32 * base.abs()
        if dout is None:
            continue
        DO = _clean(dout[s], nq)
        dP = DO @ V.transpose(-1, -2)
        delta = (DO * out).sum(-1, keepdim=True)
        E_delta = (d + 2) * E32 * (DO * out).abs().sum(-1, keepdim=True) + (DO.abs() * u_out).sum(-1, keepdim=True)
        E_dp = (d + 2) * E32 * (DO.abs() @ V.abs().transpose(-1, -2))
        dS = P * (dP - delta)
        # a 16-bit ds is rounded from an fp32 value that already carries the errors above
        E_ds = (dS.abs() * (Ep + u_p) + P * (E_dp + E_delta)) * (1 + u_p)
        E_pp = P * (Ep + u_p)
        if dt == torch.float16:
            top = (DO.norm(dim=-1).amax() * V.norm(dim=-1).amax()).item() if nk and nq else 0.0
            E_ds = E_ds + 2.0 ** -24 * top * see
            E_pp = E_pp + 2.0 ** -24 * see
        tail = 2.0 ** -25 if dt == torch.float16 else 1e-30
        dQ = dS @ K * scale
        B = (E_ds + lk * E32 * dS.abs()) @ K.abs() * scale + u * dQ.abs() + tail
        r["dq"][s], r["dq_bound"][s] = dQ.transpose(0, 1), B.transpose(0, 1)
        n = lq * group
        for name, W, EW, X, mul in (("dk", dS, E_ds, Q, scale), ("dv", P, E_pp, DO, 1.0)):
            W, EW = W * see, EW * see
            G = (W.transpose(-1, -2) @ X * mul).view(hk, group, lk, d).sum(1)
            BG = ((EW + n * E32 * W.abs()).transpose(-1, -2) @ X.abs() * mul).view(hk, group, lk, d).sum(1)
            r[name][s] = G.transpose(0, 1)
            r[name + "_bound"][s] = (BG + u * G.abs() + tail).transpose(0, 1)
    return r


def check(got, r, name):
    """Every element of `got` within its bound (infinities where the reference has them)."""
    want, bound = r[name], r[name + "_bound"]
    got = got.double()
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf), f"{name}: infinities differ"
    assert not torch.isnan(got).any(), f"{name}: NaN"
    off = torch.where(inf, torch.zeros_like(want), (got - want).abs())
    worst = (off - bound).max().item() if off.numel() else -1.0
    assert worst <= 0.0, f"{name}: off by {off.max().item():.3e}, beyond its bound by {worst:.3e}"
