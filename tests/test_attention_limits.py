"""Attention configurations that are refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.build import build_library

P = ctypes.c_void_p(4096)


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B.lib()


def config(**kw):
    base = dict(dtype=B.GS_TABLE_BF16, head_dim=64, q_heads=2, kv_heads=2, batch=1, q_len=4, k_len=4,
                window_left=-1, window_right=-1, scale=0.1)
    c = B.AttentionConfig(**{**base, **kw})
    for t in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        getattr(c, f"{t}_stride")[:] = (512, 128, 64)
    return c


@pytest.mark.parametrize("kw", [
    dict(batch=1 << 31, q_heads=1 << 20, kv_heads=1 << 20, q_len=1 << 29, k_len=1 << 29),
    dict(batch=1 << 31, q_heads=1 << 20, kv_heads=1, q_len=1 << 13, k_len=1 << 13),       # 2^64 rows: nothing, modulo 2^64
    dict(batch=1 << 31, q_heads=1 << 5, kv_heads=1, q_len=1, k_len=1 << 29),
])
def test_row_counts_beyond_64_bits(lib, kw):
    c = config(**kw)
    assert lib.gs_attention_backward_work(ctypes.byref(c)) == -1
    assert lib.gs_attention_forward(ctypes.byref(c), P, P, P, P, P, None) == -6 and b"rows" in lib.gs_last_error()
    assert lib.gs_attention_backward(ctypes.byref(c), *(P,) * 10, None) == -6 and b"rows" in lib.gs_last_error()


def test_scratch_of_ordinary_configurations_is_given(lib):
    for kw, least in (({}, 8), (dict(batch=0), 0), (dict(q_len=0), 0), (dict(batch=3, q_heads=4, kv_heads=2, q_len=5000), 60000),
                      (dict(batch=1 << 31, q_heads=1, kv_heads=1, q_len=128, k_len=128), 1 << 38)):
        assert lib.gs_attention_backward_work(ctypes.byref(config(**kw))) >= least
