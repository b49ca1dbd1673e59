"""Layer norm, the gated linear recurrence and 8-bit checkpoints in 64 bits, with bounds on what a correct kernel may be off by.

e = 2^-24 of fp32, u = unit roundoff of the tensors' type (plus 2^-25 for binary16 below its normal range).

Layer norm.  A row's sum is 32 terms of a thread at most, 5 steps of a warp and 16 warps: 53 additions, so a sum is off by
53 e of the sum of its terms' magnitudes.  Forward, with A = mean |x - mean| <= 1 / rstd:
  differences  d = x - m, m a first mean: e |d|; their mean is off by (53 + 2) e A; centred value: 2 e |x - mean| + 55 e A + e |..|
  variance     (53 + 3) e relative + 2 (55 e A) A / var <= 170 e;  rstd: half of that + 2 ulp of rsqrt (4 e) + e: 90 e relative
  xh           (95 |xh| + 56) e;  y: |weight| of that + 2 e (|weight xh| + |bias|) + u |y|
  mean, rstd   57 e A + 2 e |mean|, 90 e rstd
Backward, from given statistics, X = mean |g xh|, G = mean |g|:
  xh 2 e, g e, sums 55 e G and 58 e X; dx: rstd (6 e (|g| + |s1| + |xh s2|) + 55 e G + 60 e |xh| X) + u |dx|
  dweight, dbias: rows of a team (148 blocks at least, or one row each) <= rows / 148 + 1, then 32 teams, 148 eighths of the
  blocks and 8 of those: (rows / 148 + 190 + 4) e of the sum of magnitudes, + u of the result.

Recurrence.  m = min(a, 1 - a) is off by 10 e of itself (exp 2 ulp, quotient 2 ulp, sum), for 16-bit tensors by 2 |z| e more (the product
z log2(e) is rounded); a step of the state by 3 e of the states' magnitudes H (recursion over magnitudes; the products of stretches and
their joins among them) and that of m (H + |x|):
  E_t = a_t E_(t-1) + 3 e (H_t + H_(t-1)) + (12 + 2 |z|) e m (H_(t-1) + |x|)
and likewise for r = a g with the magnitudes of its own recursion.  dx = (1 - a) g: (1 - a) E_g + 12 e |dx|;
dgate = a (1 - a) d g: a (1 - a) (|g| (E_h + 3 e |d|) + |d| E_g) + (25 + 4 |z|) e |dgate|; + u of each result.
"""
import torch

E32 = 2.0 ** -24
UNIT = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float64: 0.0, torch.float32: 1e-38, torch.float16: 2.0 ** -25, torch.bfloat16: 1e-38}


def rounded(x, dtype):
    """Bound of the rounding of x to dtype."""
    return UNIT[dtype] * x.abs() + LEAST[dtype]


def valid_rows(lens, b, n, device):
    if lens is None:
        return torch.ones((b, n, 1), dtype=torch.bool, device=device)
    return (torch.arange(n, device=device)[None] < lens.long().clamp(0, n)[:, None])[..., None]


def layer_norm(x, weight, bias, eps, lens=None):
    """{"y", "stats"} and bounds of x[b, n, c]."""
    b, n, c = x.shape
    on = valid_rows(lens, b, n, x.device)
    v = x.double().masked_fill(~on, 0.0)
    w = torch.ones(c, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    s = torch.zeros(c, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    mean = v.mean(-1, keepdim=True)
    d = v - mean
    rstd = (d.square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = d * rstd
    y = xh * w + s
    spread = d.abs().mean(-1, keepdim=True)
    bound = w.abs() * (95 * xh.abs() + 56) * E32 + 2 * E32 * ((w * xh).abs() + s.abs()) + rounded(y, x.dtype)
    stats = torch.cat([mean, rstd], -1)
    stats_bound = torch.cat([57 * E32 * spread + 2 * E32 * mean.abs(), 90 * E32 * rstd], -1)
    hide = lambda t: t.masked_fill(~on, 0.0)                                        # noqa: E731
    return {"y": hide(y), "y_bound": hide(bound), "stats": hide(stats), "stats_bound": hide(stats_bound)}


def layer_norm_backward(dy, x, weight, stats, lens=None, weight_dtype=torch.float32):
    """dx, dweight, dbias and bounds, from given statistics (and x as the kernel is given it, in any type)."""
    b, n, c = dy.shape
    on = valid_rows(lens, b, n, dy.device)
    w = torch.ones(c, dtype=torch.float64, device=dy.device) if weight is None else weight.double()
    mean, rstd = stats.double().masked_fill(~on, 0.0).split(1, -1)
    d = dy.double().masked_fill(~on, 0.0)
    xh = (x.double().masked_fill(~on, 0.0) - mean) * rstd
    g = d * w
    s1, s2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    dx = rstd * (g - s1 - xh * s2)
    big = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True)
    r = {"dx": dx, "dx_bound": rstd * E32 * (6 * (g.abs() + s1.abs() + (xh * s2).abs()) + 55 * big[0] + 60 * xh.abs() * big[1])
         + rounded(dx, dy.dtype)}
    depth = (b * n / 148 + 194) * E32
    for name, t in (("dweight", d * xh), ("dbias", d)):
        r[name] = t.sum((0, 1))
        r[name + "_bound"] = depth * t.abs().sum((0, 1)) + rounded(r[name], weight_dtype)
    r["dx"], r["dx_bound"] = r["dx"].masked_fill(~on, 0.0), r["dx_bound"].masked_fill(~on, 0.0)
    return r


def recurrence(gate, x, h0=None, lens=None, dout=None, dfinal=None):
    """out, final, every state, and with dout or dfinal the gradients, all with bounds."""
    b, n, c = x.shape
    f64 = dict(dtype=torch.float64, device=x.device)
    on = valid_rows(lens, b, n, x.device)
    z = gate.double().masked_fill(~on, 0.0)
    a, u = torch.sigmoid(z), torch.sigmoid(-z)
    far = z.abs().clamp(max=200.0) * (0.0 if x.dtype in (torch.float32, torch.float64) else 2.0)
    m = torch.minimum(a, u) * (12 + far)
    v = x.double().masked_fill(~on, 0.0)
    h = torch.zeros((b, c), **f64) if h0 is None else h0.double()
    big, err = h.abs(), torch.zeros((b, c), **f64)
    hs, es = torch.zeros((b, n, c), **f64), torch.zeros((b, n, c), **f64)
    before, err_before = torch.zeros((b, n, c), **f64), torch.zeros((b, n, c), **f64)
    for t in range(n):
        before[:, t], err_before[:, t] = h, err
        now, size = a[:, t] * h + u[:, t] * v[:, t], a[:, t] * big + u[:, t] * v[:, t].abs()
        e = a[:, t] * err + 3 * E32 * (size + big) + E32 * m[:, t] * (big + v[:, t].abs())
        h, big, err = torch.where(on[:, t], now, h), torch.where(on[:, t], size, big), torch.where(on[:, t], e, err)
        hs[:, t], es[:, t] = h, err
    hide = lambda t: t.masked_fill(~on, 0.0)                                        # noqa: E731
    r = {"out": hide(hs), "out_bound": hide(es + rounded(hs, x.dtype)), "final": h, "final_bound": err + E32 * h.abs() + 1e-38,
         "states": hs[:, 127:-1:128], "states_bound": (es + E32 * hs.abs() + 1e-38)[:, 127:-1:128]}
    if dout is None and dfinal is None:
        return r
    do = torch.zeros((b, n, c), **f64) if dout is None else dout.double().masked_fill(~on, 0.0)
    back = torch.zeros((b, c), **f64) if dfinal is None else dfinal.double()
    big, err = back.abs(), torch.zeros((b, c), **f64)
    for name in ("dgate", "dx"):
        r[name], r[name + "_bound"] = torch.zeros((b, n, c), **f64), torch.zeros((b, n, c), **f64)
    for t in range(n - 1, -1, -1):
        g, size = do[:, t] + back, do[:, t].abs() + big
        eg = err + 2 * E32 * size
        d = before[:, t] - v[:, t]
        dx, dz = u[:, t] * g, a[:, t] * u[:, t] * d * g
        r["dx"][:, t], r["dgate"][:, t] = dx, dz
        r["dx_bound"][:, t] = u[:, t] * eg + (12 + far[:, t]) * E32 * dx.abs() + rounded(dx, x.dtype)
        r["dgate_bound"][:, t] = (a[:, t] * u[:, t] * (g.abs() * (err_before[:, t] + 3 * E32 * (before[:, t].abs() + v[:, t].abs()))
                                                       + d.abs() * eg) + (25 + 2 * far[:, t]) * E32 * dz.abs() + rounded(dz, x.dtype))
        e = a[:, t] * eg + 3 * E32 * (a[:, t] * size + size) + E32 * m[:, t] * size
        back = torch.where(on[:, t], a[:, t] * g, back)
        big, err = torch.where(on[:, t], a[:, t] * size, big), torch.where(on[:, t], e, err)
    r["dh0"], r["dh0_bound"] = back, err + E32 * back.abs() + 1e-38
    for name in ("dgate", "dx"):
        r[name], r[name + "_bound"] = hide(r[name]), hide(r[name + "_bound"])
    return r


def checkpoint(x):
    """(whole numbers, scales) of x[rows, columns] by the definition, in 64 bits."""
    rows, c = x.shape
    blocks = (c + 127) // 128
    v = torch.nn.functional.pad(x.double(), (0, blocks * 128 - c)).view(rows, blocks, 128)
    top = v.abs().amax(-1)
    s = (top / 127).float()
    s = torch.where(s.double() * 127 > top, torch.nextafter(s, torch.zeros_like(s)), s)
    steps = torch.round(v / s.double()[..., None]).clamp(-127, 127)
    steps = torch.where(s[..., None] > 0, steps, torch.zeros_like(steps))
    fine = torch.isfinite(v).all(-1)
    s = torch.where(fine, s, torch.full_like(s, float("nan")))
    steps = torch.where(fine[..., None], steps, torch.zeros_like(steps))
    return steps.reshape(rows, blocks * 128)[:, :c], s


def checkpoint_values(packed, scales):
    """What 8-bit values and scales stand for, in fp32."""
    c = packed.shape[-1]
    return packed.float() * scales.repeat_interleave(128, -1)[..., :c]


def within(got, want, bound, what=""):
    over = (got.double() - want).abs() - bound
    assert got.shape == want.shape
    assert not torch.isnan(got.double()).any(), f"{what}: NaN"
    if got.numel():
        worst = over.max().item()
        assert worst <= 0, f"{what}: off by {worst:.3e} beyond the bound at {over.argmax().item()}"
