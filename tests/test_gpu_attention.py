"""gs_attention_forward / gs_attention_backward against the 64-bit definition, element by element
within derived bounds (tests/attention_reference.py), on the sizes, masks and layouts where a kernel
can go wrong, and the calls that must be refused."""
import ctypes
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests.attention_reference import check, reference

DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ALL, CAUSAL = (-1, -1), (-1, 0)


def tensors(b, lq, lk, hq, hk, d, dt, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    make = lambda n, h: torch.randn((b, n, h, d), generator=gen, device=DEV).to(dt)       # noqa: E731
    return make(lq, hq), make(lk, hk), make(lk, hk), (make(lq, hq) * 0.25).to(dt)


def lengths(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def run_both(q, k, v, dout, window, q_lens=None, k_lens=None, scale=None):
    """One forward and backward call, each checked in full."""
    s = scale if scale is not None else 1.0 / math.sqrt(q.shape[3])
    r = reference(q, k, v, s, window, q_lens, k_lens, dout)
    out, lse = B.gs_attention_forward(q, k, v, scale, window, q_lens, k_lens)
    check(out, r, "out")
    check(lse, r, "lse")
    grads = B.gs_attention_backward(dout, q, k, v, out, lse, scale, window, q_lens, k_lens)
    for name, g in zip(("dq", "dk", "dv"), grads):
        check(g, r, name)
    return out, lse, grads


SHAPES = [
    # batch, q_len, k_len, q_heads, kv_heads, head_dim, window
    (1, 1, 1, 1, 1, 1, ALL),
    (2, 1, 37, 4, 2, 64, ALL),             # single token over a short cache
    (3, 10, 10, 2, 2, 32, (5, 5)),         # walks
    (5, 16, 16, 1, 1, 16, CAUSAL),
    (5, 17, 17, 3, 1, 40, (2, 0)),
    (2, 40, 40, 4, 4, 32, (10, 10)),
    (2, 63, 63, 2, 2, 128, CAUSAL),
    (2, 64, 64, 2, 1, 64, (0, 0)),         # every row sees one key
    (2, 65, 65, 2, 2, 80, (0, 7)),
    (2, 80, 80, 4, 4, 32, (10, 10)),
    (1, 127, 129, 2, 2, 64, ALL),
    (1, 128, 128, 4, 2, 128, CAUSAL),
    (1, 129, 127, 2, 2, 128, CAUSAL),      # more queries than keys: the first rows see nothing
    (2, 130, 300, 6, 2, 64, CAUSAL),       # a chunk of new positions after old ones
    (1, 300, 130, 2, 1, 128, ALL),
    (1, 257, 257, 3, 3, 127, (100, 30)),
    (1, 257, 257, 8, 1, 64, CAUSAL),       # one shared key/value head
    (1, 5, 700, 2, 2, 128, (-1, 0)),
    (1, 700, 5, 2, 2, 128, ALL),
    (2, 513, 513, 2, 1, 96, (64, 0)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(x) for x in s[:6]) + f"w{s[6][0]}_{s[6][1]}")
def test_matches_definition(shape, dt):
    b, lq, lk, hq, hk, d, window = shape
    run_both(*tensors(b, lq, lk, hq, hk, d, dt, seed=lq + d), window)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d,lens,window", [
    (10, 32, [10, 0, 1, 9], (5, 5)),
    (40, 32, [40, 0, 1, 33], (10, 10)),
    (80, 64, [16, 80, 0, 65], CAUSAL),
    (200, 64, [200, 0, 128, 129], ALL),
    (200, 128, [1, 200, 64, 199], CAUSAL),
    (300, 128, [257, 300, 0, 5], (40, 3)),
], ids=lambda x: str(x) if isinstance(x, int) else None)
def test_ragged_batches_never_read_the_padding(n, d, lens, window, dt):
    q, k, v, dout = tensors(4, n, n, 4, 2, d, dt, seed=n)
    m = lengths(lens)
    for t, fill in ((q, math.nan), (k, math.inf), (v, math.nan), (dout, -math.inf)):
        for s, length in enumerate(lens):
            t[s, length:] = fill
    out, lse, (dq, dk, dv) = run_both(q, k, v, dout, window, m, m)
    for s, length in enumerate(lens):                      # padding rows are zeros, not leftovers
        assert not out[s, length:].any() and not dq[s, length:].any()
        assert not dk[s, length:].any() and not dv[s, length:].any()
        assert torch.isneginf(lse[s, :, length:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,n,hq,hk,window,ragged", [
    (90, 300, 4, 2, CAUSAL, False),        # every block goes through several work items, in fixed rounds
    (90, 300, 4, 2, CAUSAL, True),         # handed out as SMs come free; some sequences empty
    (40, 700, 3, 3, (150, 0), True),
    (200, 130, 2, 1, ALL, True),
], ids=["fixed", "asked", "asked_window", "asked_short"])
def test_more_work_items_than_sms(b, n, hq, hk, window, ragged, d, dt):
    q, k, v, dout = tensors(b, n, n, hq, hk, d, dt, seed=b)
    m = None
    if ragged:
        gen = torch.Generator().manual_seed(b)
        values = torch.randint(0, n + 1, (b,), generator=gen)
        values[::7] = 0
        m = values.to(torch.int32).to(DEV)
        for s in range(b):
            v[s, int(values[s]):] = math.nan
            q[s, int(values[s]):] = math.nan
    out, lse, grads = run_both(q, k, v, dout, window, m, m)
    again = B.gs_attention_backward(dout, q, k, v, *B.gs_attention_forward(q, k, v, window=window, q_lens=m, k_lens=m),
                                    window=window, q_lens=m, k_lens=m)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))            # whoever did which item
    assert B.gs_stalled_kernels() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [40, 200])
def test_many_short_sequences(n, dt):
    # more heads than one round of resident blocks takes, with and without dead ends
    b = 3000 if n == 40 else 400
    q, k, v, dout = tensors(b, n, n, 2, 2, 32, dt, seed=n)
    values = torch.randint(0, n + 1, (b,), generator=torch.Generator().manual_seed(n))
    values[: b // 2] = n
    m = values.to(torch.int32).to(DEV)
    for lens in (None, m):
        out, lse, grads = run_both(q, k, v, dout, (10, 10), lens, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,row", [(60, 64), (100, 104), (4, 8), (20, 24)])
@pytest.mark.parametrize("n", [24, 200])
def test_head_dims_within_wider_rows(n, d, row, dt):
    # rows that TMA can address, of head_dims that are no multiple of its 16 bytes; NaN between the rows
    make = lambda t: torch.full((*t.shape[:3], row), math.nan, dtype=dt, device=DEV)      # noqa: E731
    parts = []
    for t in tensors(2, n, n, 2, 2, d, dt, seed=d):
        x = make(t)
        x[..., :d] = t
        parts.append(x[..., :d])
    q, k, v, dout = parts
    run_both(q, k, v, dout, CAUSAL)
    out, lse = B.gs_attention_forward(q, k, v, window=CAUSAL)
    room = torch.full((4, 2, n, 2, row), 7.0, dtype=dt, device=DEV)
    B.gs_attention_forward(q, k, v, window=CAUSAL, out=room[0, ..., :d])
    B.gs_attention_backward(dout, q, k, v, out, lse, window=CAUSAL, dq=room[1, ..., :d], dk=room[2, ..., :d], dv=room[3, ..., :d])
    assert torch.equal(room[0, ..., :d], out) and (room[..., d:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_query_and_key_lengths_differ_per_sequence(dt):
    q, k, v, dout = tensors(5, 70, 140, 2, 2, 64, dt, seed=3)
    # empty queries, empty keys, more queries than keys, out-of-range lengths (clamped)
    run_both(q, k, v, dout, CAUSAL, lengths([0, 70, 70, 30, 1000]), lengths([140, 0, 20, -5, 140]))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lq,lk", [(0, 5), (5, 0), (0, 0)])
def test_zero_lengths(lq, lk, dt):
    q, k, v, dout = tensors(2, lq, lk, 2, 2, 64, dt)
    out, lse = B.gs_attention_forward(q, k, v)
    assert not out.any() and torch.isneginf(lse).all()
    for g in B.gs_attention_backward(dout, q, k, v, out, lse):
        assert not g.any()
    none = [t[:0] for t in (q, k, v, dout)]
    out, lse = B.gs_attention_forward(*none[:3])
    assert out.shape[0] == 0 and lse.shape[0] == 0
    assert [g.shape[0] for g in B.gs_attention_backward(none[3], *none[:3], out, lse)] == [0, 0, 0]


def _layouts(b, n, h, d, dt, kind):
    """q, k, v, dout in another memory layout, same values whatever the layout."""
    q, k, v, dout = tensors(b, n, n, h, h, d, dt, seed=9)
    if kind == "fused":                                    # one projection's result, [b, n, 3, h, d]
        x = torch.stack([q, k, v], dim=2)
        q, k, v = x[:, :, 0], x[:, :, 1], x[:, :, 2]
    elif kind == "heads_first":
        q, k, v, dout = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, dout))
    elif kind == "odd_offset":                             # one element off every vector width
        def shifted(t):
            flat = torch.empty(t.numel() + 1, dtype=dt, device=DEV)
            flat[1:] = t.reshape(-1)
            return flat[1:].view(t.shape)
        q, k, v, dout = map(shifted, (q, k, v, dout))
    elif kind == "odd_rows":                               # head_dim + 1 values per row in memory
        def padded(t):
            x = torch.full((*t.shape[:3], d + 1), math.nan, dtype=dt, device=DEV)
            x[..., :d] = t
            return x[..., :d]
        q, k, v, dout = map(padded, (q, k, v, dout))
    elif kind == "broadcast":                              # zero strides: one key/value head for all, one gradient row
        k, v = k[:, :, :1].expand(-1, -1, h, -1), v[:, :1].expand(-1, n, -1, -1)
        dout = dout[:1, :1].expand(b, n, -1, -1)
    elif kind == "reversed_batch":                         # sequence stride below the position stride
        q, k, v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    return q, k, v, dout


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [12, 40, 150])
@pytest.mark.parametrize("kind", ["fused", "heads_first", "odd_offset", "odd_rows", "broadcast", "reversed_batch"])
def test_layouts(kind, n, dt):
    q, k, v, dout = _layouts(3, n, 2, 64, dt, kind)
    run_both(q, k, v, dout, CAUSAL)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [20, 200])
def test_strided_outputs(n, dt):
    q, k, v, dout = tensors(2, n, n, 2, 2, 64, dt, seed=1)
    r = reference(q, k, v, 0.125, CAUSAL, dout=dout)
    room = torch.full((2, n, 5, 2, 66), 7.0, dtype=dt, device=DEV)
    out, dq, dk, dv = (room[:, :, i, :, :64] for i in range(4))
    _, lse = B.gs_attention_forward(q, k, v, window=CAUSAL, out=out)
    check(out, r, "out")
    B.gs_attention_backward(dout, q, k, v, out, lse, window=CAUSAL, dq=dq, dk=dk, dv=dv)
    for name, g in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(g, r, name)
    assert (room[:, :, 4] == 7).all() and (room[..., 64:] == 7).all()      # nothing beside them was written


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [24, 300])
@pytest.mark.parametrize("gain", [1e-3, 12.0])
def test_flat_and_peaked_scores(gain, n, dt):
    q, k, v, dout = tensors(1, n, n, 2, 2, 64, dt, seed=4)
    run_both((q * gain).to(dt), k, v, dout, CAUSAL, scale=0.125)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("n", [30, 260])
@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** 9])
def test_small_and_large_incoming_gradients(size, n, dt):
    # what a loss scale of 1 leaves in half precision, and what a large one makes of it
    q, k, v, dout = tensors(1, n, n, 2, 1, 64, dt, seed=5)
    run_both(q, k[:, :, :1], v[:, :, :1], (dout * size).to(dt), ALL)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [33, 400])
def test_rising_scores_rescale_the_running_sums(n, dt):
    # every later key beats all before it by far: the running maximum moves in every tile
    q, k, v, dout = tensors(1, n, n, 1, 1, 64, dt, seed=6)
    q = torch.ones_like(q)
    k = (torch.arange(n, device=DEV, dtype=torch.float32)[None, :, None, None] / n).expand_as(k).to(dt).contiguous()
    run_both(q, k, v, dout, ALL, scale=1.0)
    run_both(q, k.flip(1).contiguous(), v, dout, ALL, scale=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,window", [(30, (5, 5)), (300, CAUSAL)])
def test_results_repeat_bit_for_bit(n, window, dt):
    q, k, v, dout = tensors(3, n, n, 4, 2, 64, dt, seed=8)
    first = None
    for _ in range(3):
        out, lse = B.gs_attention_forward(q, k, v, window=window)
        got = (out, lse, *B.gs_attention_backward(dout, q, k, v, out, lse, window=window))
        if first is None:
            first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.gpu
@pytest.mark.parametrize("n,window", [(12, (3, 3)), (150, CAUSAL)])
def test_gradient_against_differences(n, window):
    """<gradient, direction> against the central difference of sum(out * dout) along it.  What the two
    may differ by: the rounding of both forward passes over the step (their element bounds), the step's
    truncation (the same difference in 64 bits against the 64-bit derivative) and the gradient's bounds."""
    q, k, v, dout = tensors(2, n, n, 2, 1, 32, F32, seed=12)
    k, v = k.contiguous(), v.contiguous()
    scale, h = 32 ** -0.5, 2.0 ** -6
    out, lse = B.gs_attention_forward(q, k, v, scale, window)
    grads = dict(zip("qkv", B.gs_attention_backward(dout, q, k, v, out, lse, scale, window)))
    r = reference(q, k, v, scale, window, dout=dout)
    for name in "qkv":
        ins = {"q": q, "k": k, "v": v}
        x = ins[name]
        step = torch.randn(x.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
        vals, vals64, noise = [], [], 0.0
        for sign in (1.0, -1.0):
            moved = (x + sign * h * step)
            ins[name] = moved
            o, _ = B.gs_attention_forward(ins["q"], ins["k"], ins["v"], scale, window)
            r64 = reference(ins["q"], ins["k"], ins["v"], scale, window)
            vals.append((o.double() * dout.double()).sum().item())
            vals64.append((r64["out"] * dout.double()).sum().item())
            noise += (r64["out_bound"] * dout.double().abs()).sum().item()
        width = ((x + h * step).double() - (x - h * step).double()) / (2 * h)     # the step as taken in fp32
        along = (grads[name].double() * width).sum().item()
        along64 = (r["d" + name] * width).sum().item()
        got, want = (vals[0] - vals[1]) / (2 * h), (vals64[0] - vals64[1]) / (2 * h)
        slack = noise / (2 * h) + abs(want - along64) + (r[f"d{name}_bound"] * width.abs()).sum().item()
        assert abs(got - along) <= slack, (name, got, along, slack)
        assert abs(along64) > 4 * abs(want - along64)          # the step is small enough to mean something


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_offsets_beyond_32_bits(dt):
    # two sequences 2^31 + 64 elements apart in one buffer, positions 2^25 elements apart
    n, far = 40, (1 << 31) + 64
    room = torch.zeros(far + n * (1 << 25) + 4096, dtype=dt, device=DEV)
    view = lambda at: room[at:].as_strided((2, n, 2, 64), (far, 1 << 25, 64, 1))      # noqa: E731
    q, k, v = view(0), view(128), view(256)
    dense = tensors(2, n, n, 2, 2, 64, dt, seed=7)
    for t, x in zip((q, k, v), dense):
        t.copy_(x)
    run_both(q, k, v, dense[3], CAUSAL)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [30, 260])
def test_other_streams(n):
    q, k, v, dout = tensors(2, n, n, 2, 2, 64, BF16, seed=2)
    want = B.gs_attention_forward(q, k, v)
    want_g = B.gs_attention_backward(dout, q, k, v, *want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for st in streams:                                     # at the same time on several streams: no shared scratch
        with torch.cuda.stream(st):
            o = B.gs_attention_forward(q, k, v)
            got.append((*o, *B.gs_attention_backward(dout, q, k, v, *o)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip((*want, *want_g), g))


@pytest.mark.gpu
def test_refusals_of_the_binding():
    q, k, v, dout = tensors(2, 8, 8, 4, 2, 32, BF16)
    out, lse = B.gs_attention_forward(q, k, v)
    for args, err in [
        ((q.cpu(), k, v), TypeError), ((q.double(), k, v), TypeError), ((q[0], k, v), TypeError),
        ((q, k.half(), v), TypeError), ((q, k, v[:, :4]), ValueError), ((q, k[..., :16], v), ValueError),
        ((q.transpose(2, 3).contiguous().transpose(2, 3), k, v), ValueError),
    ]:
        with pytest.raises(err):
            B.gs_attention_forward(*args)
    with pytest.raises(TypeError):
        B.gs_attention_forward(q, k, v, q_lens=torch.ones(2, device=DEV))
    with pytest.raises(TypeError):
        B.gs_attention_forward(q, k, v, k_lens=torch.ones(3, dtype=torch.int32, device=DEV))
    for kw in ({"scale": 0.0}, {"scale": -1.0}, {"scale": math.inf}, {"scale": math.nan}):
        with pytest.raises(B.GsError) as e:
            B.gs_attention_forward(q, k, v, **kw)
        assert e.value.status == -1 and "scale" in str(e.value)
    with pytest.raises(B.GsError) as e:                    # 4 query heads over 3
        B.gs_attention_forward(q, *(torch.zeros((2, 8, 3, 32), dtype=BF16, device=DEV),) * 2)
    assert e.value.status == -1 and "multiple" in str(e.value)
    wide = torch.zeros((1, 4, 1, 136), dtype=BF16, device=DEV)
    with pytest.raises(B.GsError) as e:
        B.gs_attention_forward(wide, wide, wide)
    assert e.value.status == -6 and "head_dim" in str(e.value)
    with pytest.raises(B.GsError) as e:
        B.gs_attention_forward(q, k, v, out=torch.empty((2, 8, 1, 32), dtype=BF16, device=DEV).expand(-1, -1, 4, -1))
    assert e.value.status == -1 and "zero stride" in str(e.value)
    with pytest.raises(B.GsError):
        B.gs_attention_backward(dout, q, k, v, out, lse, dk=torch.empty_like(k[:1]).expand(2, -1, -1, -1))
    with pytest.raises(ValueError):
        B.gs_attention_backward(dout, q, k, v, out, lse[:, :2])
    with pytest.raises(ValueError):
        B.gs_attention_backward(dout[:, :4], q, k, v, out, lse)
    assert out.isfinite().all()


def test_refusals_of_the_library_without_a_gpu():
    from paper_2407_15452_b200.build import build_library
    build_library()
    lib = B.lib()
    assert ctypes.sizeof(B.AttentionConfig) == 4 * 4 + 8 + 6 * 4 + 2 * 8 + 8 * 3 * 8

    def cfg(**kw):
        base = dict(dtype=B.GS_TABLE_BF16, head_dim=64, q_heads=2, kv_heads=2, batch=1, q_len=4, k_len=4,
                    window_left=-1, window_right=-1, scale=0.1)
        c = B.AttentionConfig(**{**base, **kw})
        for t in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
            getattr(c, f"{t}_stride")[:] = (512, 128, 64)
        return c

    p = ctypes.c_void_p(4096)
    fwd = lambda c, *a: lib.gs_attention_forward(ctypes.byref(c), *(a or (p, p, p, p, p)), None)      # noqa: E731
    assert lib.gs_attention_forward(None, p, p, p, p, p, None) == -1
    for kw, status, text in [
        ({"dtype": 3}, -1, b"dtype"), ({"batch": -1}, -1, b"negative"), ({"q_len": -1}, -1, b"negative"),
        ({"kv_heads": 0}, -1, b"q_heads"), ({"q_heads": 3}, -1, b"q_heads"), ({"head_dim": 0}, -1, b"head_dim"),
        ({"head_dim": 129}, -6, b"head_dim"), ({"scale": 0.0}, -1, b"scale"),
        ({"q_len": (1 << 29) + 1}, -6, b"2^29"),
    ]:
        assert fwd(cfg(**kw)) == status and text in lib.gs_last_error()
    assert fwd(cfg(), None, p, p, p, p) == -1 and b"null" in lib.gs_last_error()
    assert fwd(cfg(), p, p, p, p, None) == -1
    assert fwd(cfg(), ctypes.c_void_p(4097), p, p, p, p) == -1 and b"aligned" in lib.gs_last_error()
    assert fwd(cfg(batch=0), None, None, None, None, None) == 0            # nothing to do
    bwd = [p] * 10
    for missing in range(10):
        args = list(bwd)
        args[missing] = None
        assert lib.gs_attention_backward(ctypes.byref(cfg()), *args, None) == -1


# fp32 in tiles on the tensor cores: enough heads to fill the device, head_dims of both widths, a last tile of one
# row, shared heads, empty sequences with NaN in the padding, windows that leave warps and tiles out
@pytest.mark.gpu
@pytest.mark.parametrize("d", [7, 32, 40, 64])
@pytest.mark.parametrize("n,hq,hk,window,ragged", [
    (193, 4, 4, ALL, False),
    (193, 6, 2, CAUSAL, True),
    (257, 4, 1, (40, 3), True),
    (150, 4, 4, (0, 0), False),
], ids=["all", "causal_ragged", "window_ragged", "diagonal"])
def test_many_heads_of_fp32_tiles(n, hq, hk, window, ragged, d):
    b = 32
    q, k, v, dout = tensors(b, n, n, hq, hk, d, F32, seed=n + d)
    m = None
    if ragged:
        values = torch.randint(0, n + 1, (b,), generator=torch.Generator().manual_seed(d))
        values[:4] = torch.tensor([0, 1, n, 65])
        m = values.to(torch.int32).to(DEV)
        for s, length in enumerate(values.tolist()):
            for t in (q, k, v, dout):
                t[s, length:] = math.nan
    run_both(q, k, v, dout, window, m, m)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fused", "heads_first", "odd_offset", "odd_rows", "broadcast", "reversed_batch"])
def test_layouts_of_fp32_tiles(kind):
    q, k, v, dout = _layouts(40, 150, 2, 64, F32, kind)
    run_both(q, k, v, dout, CAUSAL)


@pytest.mark.gpu
def test_fp32_tiles_of_unequal_lengths():
    q, k, v, dout = tensors(40, 70, 140, 2, 2, 64, F32, seed=3)
    run_both(q, k, v, dout, CAUSAL)
    run_both(q, k, v, dout, CAUSAL, lengths([0, 70, 70, 30, 1000] * 8), lengths([140, 0, 20, -5, 140] * 8))
