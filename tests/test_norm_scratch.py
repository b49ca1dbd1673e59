"""Scratch of layer norm's backward pass: what the launch writes, no more asked for and nothing written behind it."""
import ctypes

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.build import build_library


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B.lib()


def _floats(lib, dtype, batch, length, columns):
    c = B.LayerNormConfig(dtype=dtype, weight_dtype=dtype, batch=batch, length=length, columns=columns, eps=0.0)
    return lib.gs_layer_norm_backward_work(ctypes.byref(c))


@pytest.mark.parametrize("dtype", [B.GS_TABLE_F32, B.GS_TABLE_F16, B.GS_TABLE_BF16])
@pytest.mark.parametrize("columns", [1, 24, 128, 512, 513, 1001, 2048, 4096, 8192, 16383, 16384])
def test_scratch_follows_the_rows_and_what_the_device_holds(lib, columns, dtype):
    one = 2 * columns                                       # sums for weight and bias of one block
    assert _floats(lib, dtype, 0, 5, columns) == 0
    assert _floats(lib, dtype, 1, 1, columns) == one
    assert _floats(lib, dtype, 3, 2, columns) <= 6 * one
    sizes = [_floats(lib, dtype, 1, rows, columns) for rows in (1, 2, 100, 1000, 10 ** 5, 10 ** 9)]
    assert sizes == sorted(sizes) and sizes[-1] % one == 0
    # blocks an SM by registers: of 256 threads for the parts of a warp, of as many as a row takes beyond; rows that wide accesses do
    # not fit go by blocks of 64 threads and more
    blocks = {1: 2, 24: 2, 128: 2, 512: 2, 513: 8, 1001: 8, 2048: 4, 4096: 2, 8192: 1, 16383: 1, 16384: 1}[columns]
    sms = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 148
    assert sizes[-1] == sms * blocks * one


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("columns", [7, 24, 64, 128, 512, 520, 1001, 2048, 4096, 8192, 9000, 16383, 16384])
@pytest.mark.parametrize("rows", [1, 3, 40, 3001])
def test_nothing_is_written_behind_it(lib, rows, columns, dtype):
    if rows * columns > 1 << 24:
        rows = 700
    gen = torch.Generator("cuda").manual_seed(columns)
    whole = lambda n, lo, hi, **kw: torch.randint(lo, hi, n, generator=gen, device="cuda", **kw).to(dtype)      # noqa: E731
    for odd in (0, 1):                                      # rows that wide accesses fit, and such that they do not
        x, dy, dx = (t[odd:odd + rows * columns].view(rows, columns) for t in
                     (whole((rows * columns + 1,), -2, 3), whole((rows * columns + 1,), -2, 3), whole((rows * columns + 1,), 0, 1)))
        stats = torch.tensor([0.0, 1.0], device="cuda").repeat(rows, 1)
        code = B._TABLE_DTYPE[dtype]
        n = _floats(lib, code, 1, rows, columns)
        work = torch.full((n + 4096,), 7.0, device="cuda")
        dw, db = torch.empty(columns, device="cuda"), torch.empty(columns, device="cuda")
        c = B.LayerNormConfig(dtype=code, weight_dtype=B.GS_TABLE_F32, batch=1, length=rows, columns=columns, eps=0.0)
        for t in ("x", "y", "dy", "dx"):
            getattr(c, f"{t}_stride")[:] = (rows * columns, columns)
        assert lib.gs_layer_norm_backward(ctypes.byref(c), *(t.data_ptr() for t in (dy, x)), None, None, None, *(
            t.data_ptr() for t in (stats, work, dx, dw, db)), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert (work[n:] == 7.0).all()
        # whole numbers, exact in fp32
        assert torch.equal(db.double(), dy.double().sum(0)) and torch.equal(dw.double(), (dy.double() * x.double()).sum(0))
