"""gs_gradient_norm / gs_clip_gradients against 64-bit sums.

Tolerance of the norm: squares are rounded once (2^-24 each), 32 of them summed in fp32 (31 more
roundings), the rest in fp64, the root halves the relative error and is rounded to fp32: below
(32 / 2 + 1) 2^-24 of the norm.  A clipped value is g * (max_norm / norm): that error, the quotient's and the
product's rounding, and one rounding to the output's type."""
import ctypes
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B

DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NORM_TOL = 17 * 2.0 ** -24
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


def make(sizes, types, seed=0, gain=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n, generator=gen, device=DEV) * gain).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def norm64(grads):
    return math.sqrt(sum(g.double().square().sum().item() for g in grads))


def check_clip(grads, max_norm, out=None):
    before = [g.clone() for g in grads]
    want = norm64(before)
    norm = B.gs_clip_gradients(grads, max_norm, out=out)
    assert norm.shape == (1,) and norm.dtype == F32
    assert abs(norm.item() - want) <= NORM_TOL * want
    factor = min(1.0, max_norm / want) if want > 0 else 1.0
    for g, b, o in zip(grads, before, grads if out is None else out):
        if out is not None and o is not g:
            assert torch.equal(g, b)                                   # inputs untouched
        w = b.double() * factor
        tiny = 2.0 ** -25 if o.dtype == F16 else 2.0 ** -134 if o.dtype == BF16 else 2.0 ** -150
        bound = w.abs() * (NORM_TOL + 2 * 2.0 ** -24 + UNIT[o.dtype]) + tiny
        assert ((o.double() - w).abs() <= bound).all()


SIZE_SETS = {
    "one": [1],
    "vector_edges": [1, 2, 3, 7, 8, 9, 15, 31, 255, 256, 257],
    "chunk_edges": [8191, 8192, 8193, 16384, 40000, 12345],
    "with_empty": [0, 5, 0, 100, 0],
    "encoder": [16384] * 4 + [65536, 65536, 512, 128, 128, 128, 128, 128],
    "past_one_list": [3 + i % 50 for i in range(65)],
    "many": [1 + (i * 37) % 300 for i in range(2000)],
    "large": [5_000_001, 3],
}


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(F32,), (F16,), (BF16,), (F32, BF16, F16)], ids=["f32", "f16", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", list(SIZE_SETS))
def test_norm_and_clip(sizes, types):
    sizes = SIZE_SETS[sizes]
    grads = make(sizes, types, seed=len(sizes))
    want = norm64(grads)
    assert abs(B.gs_gradient_norm(grads).item() - want) <= NORM_TOL * want
    check_clip(grads, 2 * want)                                        # within: values keep their bits
    for g, b in zip(grads, make(sizes, types, seed=len(sizes))):
        assert torch.equal(g, b)
    check_clip(grads, 0.3 * want)                                      # in place
    for out_type in (F32, F16, BF16):
        grads = make(sizes, types, seed=1)
        out = [torch.full_like(g, math.nan, dtype=out_type) for g in grads]
        check_clip(grads, 0.3 * want, out)
        check_clip(grads, 5 * want, out)                               # within, into other buffers: a plain cast


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,)], ids=["f32", "bf16", "f16"])
def test_odd_addresses(types):
    # every offset of the input against the vector width, outputs with the same and with another one
    for shift in range(9):
        for shift_out in (shift, 0, 3):
            base = make([9000 + shift], types, seed=shift)[0]
            room = torch.full((9020,), 5.0, dtype=F32, device=DEV)
            g, o = base[shift:], room[shift_out:shift_out + 9000]
            check_clip([g], 0.5, [o])
            assert (room[:shift_out] == 5).all() and (room[shift_out + 9000:] == 5).all()
    base = make([20001], types)[0]
    rest = base[:1].clone()
    check_clip([base[1:]], 0.5)
    assert torch.equal(base[:1], rest)


@pytest.mark.gpu
def test_no_tensors_and_zeros():
    assert B.gs_gradient_norm([]).item() == 0.0
    assert B.gs_clip_gradients([], 1.0).item() == 0.0
    z = [torch.zeros(100, device=DEV), torch.zeros(3, device=DEV, dtype=BF16)]
    check_clip(z, 1.0)
    check_clip(z, 0.0)
    g = make([100], (F32,))
    B.gs_clip_gradients(g, 0.0)
    assert not g[0].any()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3e19])
def test_norms_that_are_not_finite_leave_the_gradients(value):
    g = make([5000, 10], (F32, BF16))
    g[0][4321] = value
    keep = [x.clone() for x in g]
    out = [torch.empty_like(x) for x in g]
    for norm in (B.gs_gradient_norm(g), B.gs_clip_gradients(g, 1.0), B.gs_clip_gradients(g, 1.0, out=out)):
        assert not math.isfinite(norm.item())
    for x, k, o in zip(g, keep, out):
        assert torch.equal(x.isnan(), k.isnan()) and torch.equal(x.nan_to_num(), k.nan_to_num())
        assert torch.equal(o.isnan(), k.isnan()) and torch.equal(o.nan_to_num(), k.nan_to_num())


@pytest.mark.gpu
def test_small_and_large_values():
    check_clip(make([10000], (F32,), gain=1e-15), 1e-14)
    check_clip(make([10000], (F32,), gain=1e15), 1e10)
    check_clip(make([10000], (F16,), gain=1e4), 1.0)


@pytest.mark.gpu
def test_results_repeat_bit_for_bit_on_any_stream():
    g = make([100_003, 7, 50_000], (F32, BF16))
    want = B.gs_gradient_norm(g)
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        with torch.cuda.stream(torch.cuda.Stream()):
            out = [torch.empty_like(x) for x in g]
            got.append((B.gs_gradient_norm(g), B.gs_clip_gradients(g, 1.0, out=out), out))
    torch.cuda.synchronize()
    for a, b, out in got:
        assert torch.equal(a, want) and torch.equal(b, want)
        assert all(torch.equal(x, y) for x, y in zip(out, got[0][2]))


@pytest.mark.gpu
def test_tensor_beyond_32_bit_offsets():
    n = (1 << 32) + 9
    g = torch.zeros(n, dtype=BF16, device=DEV)
    g[-1], g[0], g[1 << 31] = 3.0, 4.0, 12.0
    assert B.gs_clip_gradients([g], 6.5).item() == 13.0
    assert g[-1].item() == 1.5 and g[0].item() == 2.0 and g[1 << 31].item() == 6.0


@pytest.mark.gpu
def test_refusals_of_the_binding():
    g = make([10, 20], (F32,))
    for wrong in ([g[0].cpu()], [g[0].double()], [g[0][::2]], [g[0].int()]):
        with pytest.raises(TypeError):
            B.gs_gradient_norm(wrong)
    with pytest.raises(ValueError):
        B.gs_clip_gradients(g, 1.0, out=g[:1])
    for max_norm in (-1.0, math.nan, math.inf):
        with pytest.raises(B.GsError) as e:
            B.gs_clip_gradients(g, max_norm)
        assert e.value.status == -1 and "max_norm" in str(e.value)
    with pytest.raises(B.GsError) as e:
        B.gs_clip_gradients(g, 1.0, out=[g[1], g[0]])
    assert e.value.status == -1 and "another size" in str(e.value)


def test_refusals_of_the_library_without_a_gpu():
    from paper_2407_15452_b200.build import build_library
    build_library()
    lib = B.lib()
    assert ctypes.sizeof(B.TensorEntry) == 24
    p = ctypes.c_void_p(4096)
    norm = lambda t, n, work=p, out=p: lib.gs_gradient_norm(t, ctypes.c_int64(n), work, out, None)      # noqa: E731
    assert norm(None, 1) == -1 and norm(None, -1) == -1
    one = (B.TensorEntry * 1)(B.TensorEntry(4096, 8, B.GS_TABLE_F32))
    assert norm(one, 1, work=None) == -1 and norm(one, 1, out=None) == -1
    for entry in (B.TensorEntry(None, 8, 0), B.TensorEntry(4096, -1, 0), B.TensorEntry(4096, 8, 3),
                  B.TensorEntry(4098, 8, 0), B.TensorEntry(4097, 8, 1)):
        assert norm((B.TensorEntry * 1)(entry), 1) == -1 and b"gradient 0" in lib.gs_last_error()
    assert lib.gs_gradient_norm_work(ctypes.c_int64(0)) > 0
    assert lib.gs_gradient_norm_work(ctypes.c_int64(5000)) > lib.gs_gradient_norm_work(ctypes.c_int64(5))
