"""Microscaled formats and the product with 4-bit weights against plain 64-bit implementations."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import PVContext, mx_shapes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    c = PVContext(0)
    yield c
    c.close()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def coded(rows, cols, fmt, device=DEV):
    return [torch.full(s, 0xA5, dtype=torch.uint8, device=device) for s in mx_shapes(rows, cols, fmt)]


def wild(rows, cols, dtype, seed):
    """Values over many powers of two, rows of zeros, ties of both formats, subnormals."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    x = x * torch.exp2(torch.randint(-8, 9, (rows, 1), generator=g).double())
    ties = torch.randint(-64, 65, (rows, cols), generator=g).double() / 32
    x = torch.where(torch.rand(rows, cols, generator=g) < 0.3, ties, x)
    if rows > 2:
        x[1] = 0.0
        x[2] = x[2] * 1e-42            # subnormal in float32 and bfloat16, zero in float16
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (5, 32), (4, 33), (7, 77), (2, 512), (3, 513), (33, 2072), (6, 4099)])
def test_codes_scales_and_values_are_the_formats(ctx, rows, cols, fmt, dtype):
    x = wild(rows, cols, dtype, seed=rows * 10007 + cols)
    codes, scales = coded(rows, cols, fmt)
    ctx.pv_quantize_mx(rows, cols, fmt, x.to(DEV), codes, scales)
    want_codes, want_scales = ref.quantize(x, fmt)
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(codes.cpu(), want_codes)
    values = ref.decode(want_codes, want_scales, fmt, cols)
    for out_type in TYPES:
        out = torch.full((rows, cols), 7.0, dtype=out_type, device=DEV)
        ctx.pv_dequantize_mx(rows, cols, fmt, codes, scales, out)
        assert torch.equal(out.cpu(), values.float().to(out_type)), out_type     # float32 holds them all


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_values_at_the_ends_of_float32(ctx, fmt):
    tiny, huge = 2.0 ** -149, torch.finfo(torch.float32).max
    rows = [[huge, -huge, 1.0, tiny], [tiny, -tiny, 3 * tiny, 0.0], [2.0 ** -126, 2.0 ** -127, -0.0, 0.0], [0.0, -0.0, 0.0, 0.0],
            [math.inf, 1.0, 2.0, 3.0], [1.0, math.nan, 2.0, 3.0], [-math.inf, math.inf, math.nan, 0.0], [448.0, 464.0, 480.0, -511.0],
            [6.0, 7.0, 5.0, -7.99]]
    x = torch.zeros(len(rows), 40)
    x[:, :4] = torch.tensor(rows, dtype=torch.float64).float()
    x[:, 36:] = 1.5                      # the second block of every row is an ordinary one
    codes, scales = coded(len(rows), 40, fmt)
    ctx.pv_quantize_mx(len(rows), 40, fmt, x.to(DEV), codes, scales)
    want_codes, want_scales = ref.quantize(x, fmt)
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want_codes)
    out = torch.empty(len(rows), 40, device=DEV)
    ctx.pv_dequantize_mx(len(rows), 40, fmt, codes, scales, out)
    bad = ~torch.isfinite(x[:, :32]).all(1)
    assert torch.isnan(out[:, :32]).all(1).cpu().equal(bad) and torch.isfinite(out[:, 32:]).all()
    ref.check(out, ref.decode(want_codes, want_scales, fmt, 40), 0.0)


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_every_code_and_every_scale_is_decoded(ctx, fmt):
    n = 16 if fmt == "e2m1" else 256
    c = torch.arange(n, dtype=torch.long).repeat_interleave(1)
    c = c.repeat(32 * 8 // n + 1)[:256].view(1, 256).expand(256, 256)
    scales = torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 8).contiguous()
    codes = (c[:, 0::2] + 16 * c[:, 1::2] if fmt == "e2m1" else c).to(torch.uint8).contiguous()
    out = torch.empty(256, 256, device=DEV)
    ctx.pv_dequantize_mx(256, 256, fmt, codes.to(DEV), scales.to(DEV), out)
    assert torch.equal(out.cpu().nan_to_num(1e30), ref.decode(codes, scales, fmt, 256).float().nan_to_num(1e30))


def test_a_far_row_is_reached_with_64_bit_offsets(ctx):
    """Element offsets beyond 2^31 (and byte offsets beyond 2^32) in input, codes and output."""
    rows, cols = 16, 1 << 28
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    x[-1, -32:] = torch.arange(32, dtype=torch.float32) - 12.0
    codes, scales = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, cols, "e4m3"))
    ctx.pv_quantize_mx(rows, cols, "e4m3", x, codes, scales)
    x.fill_(7.0)
    ctx.pv_dequantize_mx(rows, cols, "e4m3", codes, scales, x)
    want = torch.arange(32, dtype=torch.float32) - 12.0
    assert torch.equal(x[-1, -32:].float().cpu(), ref.decode(*ref.quantize(want[None], "e4m3"), "e4m3", 32).float()[0])
    assert int(torch.count_nonzero(x[-1, :-32])) == 0 and int(torch.count_nonzero(x[0])) == 0


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (77, 32), (1000, 64), (33, 96), (129, 128), (5, 160), (3, 1024), (2, 1056)])
def test_rows_of_whole_blocks(ctx, rows, cols, fmt, dtype):
    """One stretch after another whatever the rows; nothing is written behind the last."""
    x = wild(rows, cols, dtype, seed=rows * 10007 + cols)
    want_codes, want_scales = ref.quantize(x, fmt)
    codes, scales = (torch.full((s[0] + 9, s[1]), 0xA5, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, cols, fmt))
    ctx.pv_quantize_mx(rows, cols, fmt, x.to(DEV), codes[:rows], scales[:rows])
    assert torch.equal(codes[:rows].cpu(), want_codes) and torch.equal(scales[:rows].cpu(), want_scales)
    assert bool((codes[rows:] == 0xA5).all()) and bool((scales[rows:] == 0xA5).all())
    out = torch.full((rows + 9, cols), 7.0, device=DEV)
    ctx.pv_dequantize_mx(rows, cols, fmt, codes[:rows], scales[:rows], out[:rows])
    assert torch.equal(out[:rows].cpu(), ref.decode(want_codes, want_scales, fmt, cols).float()) and bool((out[rows:] == 7.0).all())


def test_more_short_rows_than_one_direction_of_a_grid_holds(ctx):
    """A wave a row: 2^26 rows are 2^32 threads."""
    rows, half = (1 << 26) + 70, 1 << 25
    x = torch.randn(rows, 1, device=DEV).bfloat16()
    codes, scales = (torch.full(s, 0xA5, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, 1, "e2m1"))
    ctx.pv_quantize_mx(rows, 1, "e2m1", x, codes, scales)
    for at, n in [(0, half), (half, half), (2 * half, rows - 2 * half)]:
        c, s = coded(n, 1, "e2m1")
        ctx.pv_quantize_mx(n, 1, "e2m1", x[at:at + n], c, s)
        assert torch.equal(c, codes[at:at + n]) and torch.equal(s, scales[at:at + n])
    out = torch.empty(rows, 1, dtype=torch.bfloat16, device=DEV)
    ctx.pv_dequantize_mx(rows, 1, "e2m1", codes, scales, out)
    tail = slice(rows - 200, rows)
    assert torch.equal(out[tail].cpu(), ref.decode(*ref.quantize(x[tail].cpu(), "e2m1"), "e2m1", 1).bfloat16())
    assert float((out.float() - x.float()).abs().max()) <= float(x.float().abs().max()) / 4     # E2M1's steps are a quarter of the value at most


def operands(tokens, out, inn, fmt, seed):
    g = gen(seed)
    x = torch.randn(tokens, inn, generator=g) * torch.exp2(torch.randint(-3, 4, (tokens, 1), generator=g))
    w = torch.randn(out, inn, generator=g) * 0.02
    return [t.to(DEV) for t in (*ref.quantize(x, fmt), *ref.quantize(w, "e2m1"))]


SHAPES = [(1, 1, 1), (1, 16, 32), (3, 5, 33), (1, 129, 4096), (16, 64, 128), (17, 100, 160), (31, 33, 100), (64, 256, 512),
          (65, 250, 640), (130, 257, 1000), (200, 384, 2072), (256, 512, 1024), (300, 520, 1056), (513, 260, 96),
          # sums in several parts, the last of them with part of a step
          (17, 70, 4096), (40, 70, 5000), (129, 300, 8200)]


def product_error(xs, ws, steps, cut=False):
    """The most that sums of `steps` instructions may be off: each adds 128 (or 32) terms to a float32 sum, and may lose
    2^-22 of the magnitudes in it.  cut: products of E4M3 are added in groups of 16 aligned to the largest one, and each of
    the other 15 loses less than 2^-13 of that one."""
    err = steps * 2.0 ** -22 * (xs.abs() @ ws.abs().T)
    if cut:
        pad = (0, -xs.shape[1] % 16)
        a, b = (torch.nn.functional.pad(t.abs(), pad).view(t.shape[0], -1, 16) for t in (xs, ws))
        for i in range(a.shape[1]):
            err += 15 * 2.0 ** -13 * (a[:, None, i] * b[None, :, i]).amax(2)
    return err


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("tokens,out,inn", SHAPES)
def test_product(ctx, tokens, out, inn, fmt, dtype):
    xc, xs, wc, ws = operands(tokens, out, inn, fmt, seed=tokens + out + inn)
    y = torch.full((tokens, out), 7.0, dtype=dtype, device=DEV)
    ctx.pv_mx_product(tokens, out, inn, fmt, xc, xs, wc, ws, y)
    x, w = ref.decode(xc, xs, fmt, inn), ref.decode(wc, ws, "e2m1", inn)
    wide = dtype == torch.float32 and fmt == "e4m3"          # 32 terms an instruction, nothing cut
    want, err = x @ w.T, product_error(x, w, -(-inn // (32 if wide else 128)) + 4, cut=fmt == "e4m3" and not wide)
    ref.check(y, want, err + ref.rounding(want.abs() + err, dtype))
    # the bound is of the worst case: over all outputs it is 2e-5 on such data, and the type's rounding
    far = float((y.cpu().double() - want).norm() / want.norm())
    assert far <= 2e-5 + ref.HALF_STEP[dtype]


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.bfloat16), ("e2m1", torch.float32), ("e4m3", torch.float32)], ids=str)
@pytest.mark.parametrize("tokens,out,inn", [(1100, 4203, 300), (2100, 4203, 300), (4097, 2049, 1024)])
def test_product_in_large_tiles(ctx, tokens, out, inn, fmt, dtype):
    test_product(ctx, tokens, out, inn, fmt, dtype)


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("tokens,out,inn", [(1, 64, 256), (40, 70, 288), (257, 300, 544)])
def test_a_block_that_is_nan_reaches_its_row_and_nothing_else(ctx, tokens, out, inn, fmt):
    xc, xs, wc, ws = operands(tokens, out, inn, fmt, seed=5)
    xs[tokens // 2, 1] = 255
    ws[out - 1, -1] = 255
    y = torch.empty(tokens, out, device=DEV)
    ctx.pv_mx_product(tokens, out, inn, fmt, xc, xs, wc, ws, y)
    want = torch.zeros(tokens, out, dtype=torch.bool)
    want[tokens // 2], want[:, out - 1] = True, True
    assert torch.equal(torch.isnan(y).cpu(), want)


@pytest.mark.parametrize("fmt,dtype,scale", [("e4m3", torch.bfloat16, 250), ("e2m1", torch.float32, 250), ("e4m3", torch.float32, 246)])
def test_product_of_scales_far_apart(ctx, fmt, dtype, scale):
    """Operands near either end of float32's range whose products are ordinary."""
    tokens, out, inn = 20, 48, 128
    xc, xs, wc, ws = operands(tokens, out, inn, fmt, seed=6)
    xs[:], ws[:] = scale, 10
    y = torch.empty(tokens, out, dtype=dtype, device=DEV)
    ctx.pv_mx_product(tokens, out, inn, fmt, xc, xs, wc, ws, y)
    x, w = ref.decode(xc, xs, fmt, inn), ref.decode(wc, ws, "e2m1", inn)
    want, err = x @ w.T, product_error(x, w, 8, cut=dtype != torch.float32)
    ref.check(y, want, err + ref.rounding(want.abs() + err, dtype))


@pytest.mark.parametrize("dx_type", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("tokens,out,inn", [(1, 1, 1), (2, 32, 32), (5, 33, 70), (64, 64, 64), (33, 130, 96), (100, 257, 300),
                                            (256, 256, 512), (300, 200, 520), (129, 512, 384), (40, 4100, 70), (4100, 40, 70),
                                            (70, 4203, 2100), (2100, 96, 2101)])
def test_product_grads(ctx, tokens, out, inn, fmt, dx_type):
    xc, xs, wc, ws = operands(tokens, out, inn, fmt, seed=tokens * 3 + out + inn)
    dy = torch.randn(tokens, out, generator=gen(9)).to(torch.bfloat16)
    x, w, d = ref.decode(xc, xs, fmt, inn), ref.decode(wc, ws, "e2m1", inn), dy.double()
    dx = torch.full((tokens, inn), 7.0, dtype=dx_type, device=DEV)
    dw = torch.full((out, inn), 7.0, device=DEV)
    ctx.pv_mx_product_grads(tokens, out, inn, fmt, xc, xs, wc, ws, dy.to(DEV), dx, dw)
    want, err = d @ w, product_error(d, w.T, -(-out // 32) + 4)
    ref.check(dx, want, err + ref.rounding(want.abs() + err, dx_type), "dX")
    want, err = d.T @ x, product_error(d.T, x.T, -(-tokens // 32) + 4)
    ref.check(dw, want, err + ref.rounding(want, torch.float32), "dW")
    # one at a time, without the other's operands: the same bits
    only = torch.empty_like(dx)
    ctx.pv_mx_product_grads(tokens, out, inn, fmt, None, None, wc, ws, dy.to(DEV), dX=only)
    assert torch.equal(only, dx)
    only = torch.empty_like(dw)
    ctx.pv_mx_product_grads(tokens, out, inn, fmt, xc, xs, None, None, dy.to(DEV), dW=only)
    assert torch.equal(only, dw)


def test_gradients_are_those_of_the_product_by_differences(ctx):
    """phi = sum(R * Y): Y is linear in X and W, so a difference of products along one weight's block scale is exact up to
    the sums' rounding."""
    tokens, out, inn = 24, 40, 96
    xc, xs, wc, ws = operands(tokens, out, inn, "e4m3", seed=11)
    r = torch.randn(tokens, out, generator=gen(12)).to(torch.bfloat16).to(DEV)
    dw = torch.empty(out, inn, device=DEV)
    ctx.pv_mx_product_grads(tokens, out, inn, "e4m3", xc, xs, wc, ws, r, dW=dw)

    def phi(scales):
        y = torch.empty(tokens, out, device=DEV)
        ctx.pv_mx_product(tokens, out, inn, "e4m3", xc, xs, wc, scales, y)
        return (y.double() * r.double()).sum().item()

    w, x = ref.decode(wc, ws, "e2m1", inn), ref.decode(xc, xs, "e4m3", inn)
    most = float(((x.abs() @ w.abs().T) * r.cpu().double().abs()).sum())
    for o, b in ((0, 0), (7, 2), (39, 1)):
        up = ws.clone()
        up[o, b] += 1                                     # the block's weights are doubled
        block = slice(32 * b, 32 * b + 32)
        want = float((dw.cpu().double()[o, block] * w[o, block]).sum())
        assert abs(phi(up) - phi(ws) - want) <= 3 * 2.0 ** -20 * most


def test_empty_sides(ctx):
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    y = torch.full((3, 5), 7.0, device=DEV)
    ctx.pv_mx_product(3, 5, 0, "e4m3", e(3, 0), e(3, 0), e(5, 0), e(5, 0), y)
    assert int(torch.count_nonzero(y)) == 0
    ctx.pv_mx_product(0, 5, 32, "e4m3", e(0, 32), e(0, 1), e(5, 16), e(5, 1), e(0, 5, t=torch.float32))
    ctx.pv_quantize_mx(0, 5, "e2m1", e(0, 5, t=torch.float32), e(0, 16), e(0, 1))
    ctx.pv_dequantize_mx(4, 0, "e2m1", e(4, 0), e(4, 0), e(4, 0, t=torch.float32))
    dx, dw = torch.full((3, 32), 7.0, device=DEV), torch.full((5, 32), 7.0, device=DEV)
    ctx.pv_mx_product_grads(3, 0, 32, "e4m3", e(3, 32), e(3, 1), e(0, 16), e(0, 1), e(3, 0, t=torch.bfloat16), dx, e(0, 32, t=torch.float32))
    ctx.pv_mx_product_grads(0, 5, 32, "e4m3", e(0, 32), e(0, 1), e(5, 16), e(5, 1), e(0, 5, t=torch.bfloat16), e(0, 32, t=torch.float32), dw)
    assert int(torch.count_nonzero(dx)) == 0 and int(torch.count_nonzero(dw)) == 0
