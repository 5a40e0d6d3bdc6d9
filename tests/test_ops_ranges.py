"""Arguments that the operators around the V step refuse because a result would leave float32, without a GPU."""
import ctypes

import pytest

from paper_2405_14852_amd import binding, load_library

INVALID = 1
A, B, P = 4096, 8192, 12288          # addresses that are never followed
F32 = 0


@pytest.fixture(scope="module")
def lib():
    if not binding.library_path().exists():
        import __graft_entry__
        __graft_entry__.build()
    return load_library()


@pytest.mark.parametrize("t", [2.0 ** -149, 2.0 ** -127, 2.0 ** 63 * 1.01, 3e38])
def test_temperatures_whose_reciprocal_or_square_leaves_float32(lib, t):
    buf = ctypes.create_string_buffer(1 << 16)
    h = ctypes.cast(buf, ctypes.c_void_p)
    assert lib.pv_distill_topk(h, 2, 9, 2, F32, A, 9, P, P, t, P, P, P, B, 9) == INVALID
    assert b"temperature" in lib.pv_last_error(h)
    assert lib.pv_distill_topk_backward(h, 2, 9, 2, F32, A, 9, P, P, t, P, P, B, 9) == INVALID
    assert b"temperature" in lib.pv_last_error(h)
