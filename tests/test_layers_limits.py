"""Calls of layer norm, the recurrence and 8-bit checkpoints that are refused before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.build import build_library

P = ctypes.c_void_p(4096)
INVALID, UNSUPPORTED = -1, -6


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B.lib()


def norm(**kw):
    strides = kw.pop("strides", {})
    c = B.LayerNormConfig(**{**dict(dtype=B.GS_TABLE_BF16, weight_dtype=B.GS_TABLE_F32, batch=2, length=3, columns=64, eps=1e-5), **kw})
    for t in ("x", "y", "dy", "dx"):
        getattr(c, f"{t}_stride")[:] = strides.get(t, (192, 64))
    return ctypes.byref(c)


def scan(**kw):
    strides = kw.pop("strides", {})
    c = B.RecurrenceConfig(**{**dict(dtype=B.GS_TABLE_BF16, batch=2, length=300, channels=64), **kw})
    for t in ("gate", "x", "out", "dout", "dgate", "dx"):
        getattr(c, f"{t}_stride")[:] = strides.get(t, (19200, 64))
    return ctypes.byref(c)


def refused(lib, status, want, word):
    assert status == want and word in lib.gs_last_error().decode(), (status, lib.gs_last_error())


@pytest.mark.parametrize("kw,want,word", [
    (dict(dtype=3), INVALID, "dtype"), (dict(dtype=-1), INVALID, "dtype"), (dict(weight_dtype=B.GS_TABLE_F16), INVALID, "weight_dtype"),
    (dict(batch=-1), INVALID, "batch"), (dict(length=-1), INVALID, "length"), (dict(columns=0), INVALID, "columns"),
    (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
    (dict(columns=16385), UNSUPPORTED, "columns"), (dict(batch=1 << 21, length=1 << 20), UNSUPPORTED, "rows"),
    (dict(batch=1 << 62, length=1 << 62), UNSUPPORTED, "rows"),
])
def test_layer_norm_configurations(lib, kw, want, word):
    refused(lib, lib.gs_layer_norm_forward(norm(**kw), *(P,) * 7, None), want, word)
    refused(lib, lib.gs_layer_norm_backward(norm(**kw), *(P,) * 10, None), want, word)
    assert lib.gs_layer_norm_backward_work(norm(**kw)) == -1


def test_layer_norm_pointers(lib):
    forward, backward = lib.gs_layer_norm_forward, lib.gs_layer_norm_backward
    refused(lib, forward(None, *(P,) * 7, None), INVALID, "NULL")
    refused(lib, forward(norm(), None, P, P, P, P, None, None, None), INVALID, "null")
    refused(lib, forward(norm(), P, P, P, None, P, None, None, None), INVALID, "null")
    refused(lib, forward(norm(), ctypes.c_void_p(4097), P, P, P, P, None, None, None), INVALID, "aligned")
    refused(lib, forward(norm(), P, P, P, P, P, P, None, None), INVALID, "together")
    refused(lib, forward(norm(), P, P, P, P, P, None, P, None), INVALID, "together")
    refused(lib, forward(norm(strides={"y": (0, 64)}), P, P, P, P, P, None, None, None), INVALID, "zero stride")
    refused(lib, forward(norm(strides={"y": (64, 0)}), P, P, P, P, P, None, None, None), INVALID, "zero stride")
    refused(lib, forward(norm(), P, ctypes.c_void_p(4098), P, P, P, None, None, None), INVALID, "aligned")
    refused(lib, forward(norm(), P, P, P, P, ctypes.c_void_p(4100), None, None, None), INVALID, "8 bytes")
    refused(lib, forward(norm(), P, P, P, P, P, P, ctypes.c_void_p(4098), None), INVALID, "aligned")
    refused(lib, backward(norm(), P, P, None, None, P, P, ctypes.c_void_p(4098), P, P, P, None), INVALID, "aligned")
    refused(lib, backward(norm(), P, P, P, P, P, P, P, P, P, P, None), INVALID, "either")
    refused(lib, backward(norm(), P, None, None, None, P, P, P, P, P, P, None), INVALID, "either")
    refused(lib, backward(norm(), P, None, P, None, P, P, P, P, P, P, None), INVALID, "either")
    refused(lib, backward(norm(), P, P, None, None, P, None, P, P, P, P, None), INVALID, "null")
    refused(lib, backward(norm(), P, P, None, None, P, P, None, P, P, P, None), INVALID, "null")
    refused(lib, backward(norm(), None, P, None, None, P, P, P, P, P, P, None), INVALID, "null")
    refused(lib, backward(norm(strides={"dx": (192, 0)}), P, P, None, None, P, P, P, P, P, P, None), INVALID, "zero stride")


@pytest.mark.parametrize("kw,want,word", [
    (dict(dtype=7), INVALID, "dtype"), (dict(batch=-1), INVALID, "batch"), (dict(length=-1), INVALID, "length"),
    (dict(channels=0), INVALID, "channels"), (dict(length=(1 << 30) + 1), UNSUPPORTED, "positions"),
    (dict(channels=(1 << 30) + 1), UNSUPPORTED, "channels"), (dict(batch=1 << 40, channels=2), UNSUPPORTED, "states"),
    (dict(batch=1 << 62, channels=1 << 31), UNSUPPORTED, "states"), (dict(batch=1 << 32, channels=64), UNSUPPORTED, "one launch"),
])
def test_recurrence_configurations(lib, kw, want, word):
    refused(lib, lib.gs_recurrence_forward(scan(**kw), *(P,) * 6, None, None), want, word)
    refused(lib, lib.gs_recurrence_backward(scan(**kw), *(P,) * 9, None, None), want, word)
    if word != "one launch":
        assert lib.gs_recurrence_states(scan(**kw)) == -1 and lib.gs_recurrence_work(scan(**kw)) == -1


def test_recurrence_pointers(lib):
    forward, backward = lib.gs_recurrence_forward, lib.gs_recurrence_backward
    refused(lib, forward(None, *(P,) * 6, None, None), INVALID, "NULL")
    for missing in (0, 1, 3):
        refused(lib, forward(scan(), *(None if i == missing else P for i in range(6)), None, None), INVALID, "null")
    refused(lib, forward(scan(), P, ctypes.c_void_p(4099), P, P, P, P, None, None), INVALID, "aligned")
    refused(lib, forward(scan(strides={"out": (0, 64)}), *(P,) * 6, None, None), INVALID, "zero stride")
    for missing, word in ((2, "null"), (3, "null"), (5, "d_states"), (6, "null"), (7, "null")):
        refused(lib, backward(scan(), *(None if i == missing else P for i in range(9)), None, None), INVALID, word)
    refused(lib, backward(scan(strides={"dgate": (19200, 0)}), *(P,) * 9, None, None), INVALID, "zero stride")
    assert lib.gs_recurrence_states(scan()) == 2 * 2 * 64
    refused(lib, forward(scan(), *(P,) * 6, ctypes.c_void_p(4104), None), INVALID, "16 bytes")
    refused(lib, backward(scan(), *(P,) * 9, ctypes.c_void_p(4104), None), INVALID, "16 bytes")
    refused(lib, forward(scan(), P, P, ctypes.c_void_p(4098), P, P, P, None, None), INVALID, "aligned")
    for length, kept in ((0, 0), (1, 0), (128, 0), (129, 1), (256, 1), (257, 2)):
        assert lib.gs_recurrence_states(scan(length=length)) == 2 * 64 * kept


def test_checkpoints(lib):
    pack, unpack = lib.gs_checkpoint_pack, lib.gs_checkpoint_unpack
    for call in (lambda *a: pack(a[0], a[1], a[2], a[3], a[4], a[5], a[6], None), lambda *a: unpack(a[0], a[5], a[6], a[2], a[3], a[4], a[1], None)):
        refused(lib, call(5, P, 4, 64, 64, P, P), INVALID, "dtype")
        refused(lib, call(0, P, -1, 64, 64, P, P), INVALID, "negative")
        refused(lib, call(0, P, 4, -64, 64, P, P), INVALID, "negative")
        refused(lib, call(0, P, (1 << 40) + 1, 1, 1, P, P), UNSUPPORTED, "rows")
        refused(lib, call(0, P, 1, 1 << 31, 1, P, P), UNSUPPORTED, "columns")
        refused(lib, call(0, P, 1 << 30, 1 << 20, 1, P, P), UNSUPPORTED, "values")
        for missing in (1, 5, 6):
            refused(lib, call(*(None if i == missing else a for i, a in enumerate((0, P, 4, 64, 64, P, P)))), INVALID, "null")
        refused(lib, call(0, ctypes.c_void_p(4098), 4, 64, 64, P, P), INVALID, "aligned")
        assert call(0, None, 0, 64, 64, None, None) == 0 and call(0, None, 4, 0, 64, None, None) == 0
    refused(lib, unpack(0, P, P, 4, 64, 0, P, None), INVALID, "zero stride")


def test_struct_layouts_match_header():
    assert ctypes.sizeof(B.LayerNormConfig) == len(B._pack_norm(0, 0, 0, 0, 0, 0.0, 0, *[0] * 8)) == 104
    assert ctypes.sizeof(B.RecurrenceConfig) == len(B._pack_recurrence(0, 0, 0, 0, 0, *[0] * 12)) == 128


def test_the_binding_takes_cuda_tensors_only():
    x = torch.zeros((2, 3, 64))
    for call in (lambda: B.gs_layer_norm_forward(x), lambda: B.gs_layer_norm_backward(x, x, None, None, x), lambda: B.gs_recurrence_forward(x, x),
                 lambda: B.gs_recurrence_backward(x, x, x), lambda: B.gs_checkpoint_pack(x), lambda: B.gs_checkpoint_unpack(x.to(torch.int8), x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_what_the_binding_refuses():
    x = torch.zeros((2, 300, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    y, stats = B.gs_layer_norm_forward(x, w, w)
    out, final, states = B.gs_recurrence_forward(x, x)
    packed, scales = B.gs_checkpoint_pack(x)
    lens = torch.ones(2, dtype=torch.int32, device="cuda")
    for call in (
            lambda: B.gs_layer_norm_forward(x[0]), lambda: B.gs_layer_norm_forward(x.double()), lambda: B.gs_layer_norm_forward(x.transpose(1, 2)),
            lambda: B.gs_layer_norm_forward(x, w[:32]), lambda: B.gs_layer_norm_forward(x, w, w.half()),
            lambda: B.gs_layer_norm_forward(x, w.double()), lambda: B.gs_layer_norm_forward(x, w.cpu()), lambda: B.gs_layer_norm_forward(x, w, lens=lens.long()),
            lambda: B.gs_layer_norm_forward(x, w, lens=lens[:1]), lambda: B.gs_layer_norm_forward(x, y=y[:1]), lambda: B.gs_layer_norm_forward(x, y=y.half()),
            lambda: B.gs_layer_norm_backward(x, x, w, w, stats[:1]), lambda: B.gs_layer_norm_backward(x, x.half(), w, w, stats),
            lambda: B.gs_layer_norm_backward(x, packed, w, w, stats), lambda: B.gs_layer_norm_backward(x, x, w, w, stats, scales=scales),
            lambda: B.gs_layer_norm_backward(x, packed, w, w, stats, scales=scales[:1]),
            lambda: B.gs_recurrence_forward(x, x[:1]), lambda: B.gs_recurrence_forward(x.half(), x), lambda: B.gs_recurrence_forward(x, x, final[:1]),
            lambda: B.gs_recurrence_forward(x, x, final.half()), lambda: B.gs_recurrence_forward(x, x, lens=lens.cpu()),
            lambda: B.gs_recurrence_backward(x, x, x, None, None), lambda: B.gs_recurrence_backward(x, x, x, None, states[:, :1]),
            lambda: B.gs_recurrence_backward(x, x, x, None, states, final[:1]), lambda: B.gs_recurrence_backward(x[:, :1], x, x, None, states),
            lambda: B.gs_checkpoint_pack(x.transpose(1, 2)), lambda: B.gs_checkpoint_pack(x[:, ::2]), lambda: B.gs_checkpoint_pack(x.int()),
            lambda: B.gs_checkpoint_unpack(packed, scales[:1]), lambda: B.gs_checkpoint_unpack(packed, scales, torch.float64),
            lambda: B.gs_checkpoint_unpack(packed, scales, out=x[:1])):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(B.GsError, match="16384"):
        B.gs_layer_norm_forward(torch.zeros((1, 1, 16385), device="cuda"))
    with pytest.raises(B.GsError, match="zero stride"):
        B.gs_recurrence_forward(x, x, out=x[:1].expand(2, -1, -1))
    with pytest.raises(B.GsError, match="eps"):
        B.gs_layer_norm_forward(x, eps=-1.0)
