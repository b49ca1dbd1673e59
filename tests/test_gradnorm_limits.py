"""Lists of tensors that gs_gradient_norm and gs_clip_gradients refuse before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.build import build_library

P = ctypes.c_void_p(4096)


@pytest.fixture(scope="module")
def lib():
    build_library()
    return B.lib()


def entries(*sizes, dtype=B.GS_TABLE_BF16, at=4096):
    return (B.TensorEntry * len(sizes))(*(B.TensorEntry(at, n, dtype) for n in sizes))


@pytest.mark.parametrize("sizes", [(1 << 43,), ((1 << 42) + 1,), (1 << 41, 1 << 41, 1), (1 << 42, 1 << 42), (1 << 62,)],
                         ids=["2^43", "2^42+1", "sum", "two", "2^62"])
def test_more_elements_than_chunk_indexes_reach(lib, sizes):
    t = entries(*sizes)
    assert lib.gs_gradient_norm(t, len(sizes), P, P, None) == -1
    assert lib.gs_clip_gradients(t, None, len(sizes), 1.0, P, P, None) == -1
    assert lib.gs_clip_gradients(t, t, len(sizes), 1.0, P, P, None) == -1


def test_a_gradient_scaled_in_place_into_another_type(lib):
    # a chunk's results would land on elements that another block has yet to read
    t = entries(8, 8)
    for wrong in (entries(8, 8, dtype=B.GS_TABLE_F32), entries(8, 8, dtype=B.GS_TABLE_F16)):
        assert lib.gs_clip_gradients(t, wrong, 2, 1.0, P, P, None) == -1
        assert b"another type" in lib.gs_last_error()
