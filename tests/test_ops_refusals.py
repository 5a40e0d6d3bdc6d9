"""What the operators around the V step refuse, without a GPU: the library checks its arguments before it touches the
device, so a zeroed context is enough to ask it."""
import ctypes
import math

import pytest
import torch

from paper_2405_14852_amd import PVContext, binding, load_library, mx_shapes

OK, INVALID, SHAPE = 0, 1, 2
BIG = 1 << 31


@pytest.fixture(scope="module")
def lib():
    path = binding.library_path()
    if not path.exists():
        import __graft_entry__
        __graft_entry__.build()
    return load_library()


@pytest.fixture
def handle():
    """A context that holds nothing: enough to refuse a call."""
    buf = ctypes.create_string_buffer(1 << 16)
    return ctypes.cast(buf, ctypes.c_void_p), buf


P, ODD = 4096, 4100          # addresses that are never followed: an aligned one and one that is not
F32, BF16 = 0, 1
E2M1, E4M3 = 0, 1


def refused(lib, handle, name, args, status):
    h = handle[0]
    assert getattr(lib, name)(None, *args) == INVALID
    assert getattr(lib, name)(h, *args) == status, lib.pv_last_error(h)
    assert len(lib.pv_last_error(h)) > 5


@pytest.mark.parametrize("args,status", [
    ((-1, 4, E2M1, F32, P, P, P), SHAPE), ((4, -1, E2M1, F32, P, P, P), SHAPE), ((BIG, 4, E2M1, F32, P, P, P), SHAPE),
    ((4, BIG, E2M1, F32, P, P, P), SHAPE), ((1 << 30, 1 << 30, E2M1, F32, P, P, P), SHAPE), ((4, 4, 2, F32, P, P, P), INVALID),
    ((4, 4, E2M1, 3, P, P, P), INVALID), ((4, 4, E2M1, F32, None, P, P), INVALID), ((4, 4, E2M1, F32, P, None, P), INVALID),
    ((4, 4, E2M1, F32, P, P, None), INVALID), ((4, 4, E2M1, F32, ODD, P, P), INVALID), ((4, 4, E2M1, F32, P, ODD, P), INVALID)])
def test_quantize(lib, handle, args, status):
    refused(lib, handle, "pv_quantize_mx", args, status)
    rows, cols, fmt, t, x, c, s = args
    refused(lib, handle, "pv_dequantize_mx", (rows, cols, fmt, c, s, t, x), status)


@pytest.mark.parametrize("args,status", [
    ((-1, 4, 4, E4M3, P, P, P, P, F32, P), SHAPE), ((4, -1, 4, E4M3, P, P, P, P, F32, P), SHAPE),
    ((4, 4, -1, E4M3, P, P, P, P, F32, P), SHAPE), ((BIG, 4, 4, E4M3, P, P, P, P, F32, P), SHAPE),
    ((4, 4, 4, 7, P, P, P, P, F32, P), INVALID), ((4, 4, 4, E4M3, P, P, P, P, -1, P), INVALID),
    ((4, 4, 4, E4M3, None, P, P, P, F32, P), INVALID), ((4, 4, 4, E4M3, P, None, P, P, F32, P), INVALID),
    ((4, 4, 4, E4M3, P, P, None, P, F32, P), INVALID), ((4, 4, 4, E4M3, P, P, P, None, F32, P), INVALID),
    ((4, 4, 4, E4M3, P, P, P, P, F32, None), INVALID), ((4, 4, 4, E4M3, ODD, P, P, P, F32, P), INVALID),
    ((4, 4, 4, E4M3, P, P, ODD, P, F32, P), INVALID), ((4, 4, 4, E4M3, P, P, P, P, F32, ODD), INVALID)])
def test_product(lib, handle, args, status):
    refused(lib, handle, "pv_mx_product", args, status)


A, B, C = 4096, 8192, 12288


@pytest.mark.parametrize("args,status", [
    ((-1, 4, 4, E4M3, P, P, P, P, A, F32, B, C), SHAPE), ((4, 4, BIG, E4M3, P, P, P, P, A, F32, B, C), SHAPE),
    ((4, 4, 4, 2, P, P, P, P, A, F32, B, C), INVALID), ((4, 4, 4, E4M3, P, P, P, P, A, 5, B, C), INVALID),
    ((4, 4, 4, E4M3, P, P, P, P, A, F32, None, None), INVALID), ((4, 4, 4, E4M3, P, P, P, P, None, F32, B, C), INVALID),
    ((4, 4, 4, E4M3, None, P, P, P, A, F32, B, C), INVALID), ((4, 4, 4, E4M3, P, P, None, P, A, F32, B, None), INVALID),
    ((4, 4, 4, E4M3, P, P, P, P, A, F32, B, B), INVALID), ((4, 4, 4, E4M3, P, P, P, P, A, F32, A, C), INVALID),
    ((4, 4, 4, E4M3, P, P, P, P, A, F32, B, A), INVALID), ((4, 4, 4, E4M3, P, P, P, P, ODD, F32, B, C), INVALID)])
def test_product_grads(lib, handle, args, status):
    refused(lib, handle, "pv_mx_product_grads", args, status)


@pytest.mark.parametrize("args,status", [
    ((-1, 4, F32, P, P, P, 1e-5, A, B, E4M3, P, P, P), SHAPE), ((4, BIG, F32, P, P, P, 1e-5, A, B, E4M3, P, P, P), SHAPE),
    ((4, 4, 9, P, P, P, 1e-5, A, B, E4M3, P, P, P), INVALID), ((4, 4, F32, P, P, P, 1e-5, A, B, 9, P, P, P), INVALID),
    ((4, 4, F32, P, P, P, -1.0, A, B, E4M3, P, P, P), INVALID), ((4, 4, F32, P, P, P, math.nan, A, B, E4M3, P, P, P), INVALID),
    ((4, 4, F32, P, P, P, math.inf, A, B, E4M3, P, P, P), INVALID), ((4, 4, F32, P, P, P, 1e-5, None, None, E4M3, None, None, None), INVALID),
    ((4, 4, F32, P, P, P, 1e-5, A, B, E4M3, P, None, P), INVALID), ((4, 4, F32, P, P, P, 1e-5, A, B, E4M3, None, P, P), INVALID),
    ((4, 4, F32, None, P, P, 1e-5, A, B, E4M3, P, P, P), INVALID), ((4, 4, F32, P, P, None, 1e-5, A, B, E4M3, P, P, P), INVALID),
    ((4, 4, F32, P, P, P, 1e-5, A, A, E4M3, P, P, P), INVALID), ((4, 4, F32, P, ODD, P, 1e-5, A, B, E4M3, P, P, P), INVALID)])
def test_rms_norm(lib, handle, args, status):
    refused(lib, handle, "pv_rms_norm", args, status)


@pytest.mark.parametrize("args,status", [
    ((-1, 4, F32, P, P, P, P, P, A, B), SHAPE), ((4, 4, 3, P, P, P, P, P, A, B), INVALID), ((4, 4, F32, P, P, P, P, P, None, None), INVALID),
    ((4, 4, F32, None, P, P, P, P, A, B), INVALID), ((4, 4, F32, P, P, None, P, P, A, B), INVALID), ((4, 4, F32, P, P, P, None, P, A, B), INVALID),
    ((4, 4, F32, P, P, P, P, None, A, B), INVALID), ((4, 4, F32, P, ODD, P, P, P, A, B), INVALID), ((4, 4, F32, P, P, P, P, P, A, ODD), INVALID)])
def test_rms_norm_backward(lib, handle, args, status):
    refused(lib, handle, "pv_rms_norm_backward", args, status)


@pytest.mark.parametrize("rows,vocab,k,t,z,ld,ids,top,temp,grad,grad_ld,status", [
    (-1, 9, 2, F32, A, 9, P, P, 1.0, B, 9, SHAPE), (2, 0, 2, F32, A, 9, P, P, 1.0, B, 9, SHAPE),
    (2, (1 << 20) + 1, 2, F32, A, 1 << 21, P, P, 1.0, B, 1 << 21, SHAPE), (2, 9, -1, F32, A, 9, P, P, 1.0, B, 9, INVALID),
    (2, 9, 1025, F32, A, 9, P, P, 1.0, B, 9, INVALID), (2, 9, 2, 4, A, 9, P, P, 1.0, B, 9, INVALID),
    (2, 9, 2, F32, A, 8, P, P, 1.0, B, 9, SHAPE), (2, 9, 2, F32, A, 9, P, P, 1.0, B, 8, SHAPE),
    (2, 9, 2, F32, A, 1 << 41, P, P, 1.0, B, 9, SHAPE), (2, 9, 2, F32, A, 9, P, P, 0.0, B, 9, INVALID),
    (2, 9, 2, F32, A, 9, P, P, -1.0, B, 9, INVALID), (2, 9, 2, F32, A, 9, P, P, math.nan, B, 9, INVALID),
    (2, 9, 2, F32, A, 9, P, P, math.inf, B, 9, INVALID), (2, 9, 2, F32, None, 9, P, P, 1.0, B, 9, INVALID),
    (2, 9, 2, F32, A, 9, None, P, 1.0, B, 9, INVALID), (2, 9, 2, F32, A, 9, P, None, 1.0, B, 9, INVALID),
    (2, 9, 2, F32, A, 9, P, P, 1.0, A, 10, INVALID), (2, 9, 2, F32, ODD, 9, P, P, 1.0, B, 9, INVALID)])
def test_distill(lib, handle, rows, vocab, k, t, z, ld, ids, top, temp, grad, grad_ld, status):
    refused(lib, handle, "pv_distill_topk", (rows, vocab, k, t, z, ld, ids, top, temp, P, P, P, grad, grad_ld), status)
    refused(lib, handle, "pv_distill_topk_backward", (rows, vocab, k, t, z, ld, ids, top, temp, P, P, grad, grad_ld), status)


def test_distill_outputs(lib, handle):
    refused(lib, handle, "pv_distill_topk", (2, 9, 2, F32, A, 9, P, P, 1.0, P, None, P, B, 9), INVALID)
    refused(lib, handle, "pv_distill_topk_backward", (2, 9, 2, F32, A, 9, P, P, 1.0, None, P, B, 9), INVALID)
    refused(lib, handle, "pv_distill_topk_backward", (2, 9, 2, F32, A, 9, P, P, 1.0, P, None, B, 9), INVALID)
    refused(lib, handle, "pv_distill_topk_backward", (2, 9, 2, F32, A, 9, P, P, 1.0, P, P, None, 9), INVALID)


def test_rows_of_16_mib_are_refused_before_anything_is_enqueued(lib, handle):
    h, big, unsupported = handle[0], 1 << 24, 3
    for args in ((17, 4, big, E4M3, P, P, P, P, BF16, P), (17, 4, 2 * big, E2M1, P, P, P, P, F32, P), (17, 4, big // 2, E4M3, P, P, P, P, F32, P)):
        assert lib.pv_mx_product(h, *args) in (unsupported, 5)       # 5: there is no device here to make the context's
    assert lib.pv_mx_product_grads(h, 4, big // 2, 4, E4M3, P, P, P, P, A, F32, B, None) in (unsupported, 5)
    assert lib.pv_mx_product_grads(h, big // 2, 4, 4, E4M3, P, P, P, P, A, F32, None, C) in (unsupported, 5)


def test_nothing_to_do_is_no_error(lib, handle):
    h = handle[0]
    assert lib.pv_quantize_mx(h, 0, 4, E2M1, F32, None, None, None) == OK
    assert lib.pv_mx_product(h, 0, 4, 4, E4M3, None, None, None, None, F32, None) == OK
    assert lib.pv_rms_norm(h, 0, 4, F32, None, None, None, 1e-5, P, None, E4M3, None, None, None) == OK
    assert lib.pv_distill_topk(h, 0, 9, 0, F32, None, 9, None, None, 1.0, None, None, None, None, 9) == OK


def test_shapes_of_codes_and_scales():
    assert mx_shapes(3, 33, "e2m1") == ((3, 32), (3, 2))
    assert mx_shapes(3, 33, "e4m3") == ((3, 64), (3, 2))
    assert mx_shapes(0, 0, "e4m3") == ((0, 0), (0, 0))
    with pytest.raises(ValueError):
        mx_shapes(1, 1, "e5m2")


def test_the_binding_refuses_host_tensors_and_types():
    ctx = object.__new__(PVContext)
    ctx._h, ctx.device, ctx._lib = None, 0, None
    x, c, s = torch.zeros(4, 32), torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    with pytest.raises(TypeError, match="CUDA"):
        ctx.pv_quantize_mx(4, 32, "e2m1", x, c, s)
    with pytest.raises(TypeError, match="X must be"):
        ctx.pv_quantize_mx(4, 32, "e2m1", x.double(), c, s)
    with pytest.raises(TypeError):
        ctx.pv_distill_topk(4, 32, 0, x, None, None, 1.0, loss=torch.zeros(4))
    with pytest.raises(TypeError):
        ctx.pv_rms_norm(4, 32, None, None, x[0], 1e-5, y=x)
