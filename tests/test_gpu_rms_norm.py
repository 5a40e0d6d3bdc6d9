"""RMS norm with the residual's addition, its 8-bit output and its gradients against plain 64-bit implementations."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import PVContext, mx_shapes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-5
# a float32 sum of squares: at most 64 terms one after the other in a lane (128 in rows beyond 2^19 values), then 10 levels
# of a tree, relative to the sum since no term is negative; the root halves it, and three operations follow
SUM = 80 * 2.0 ** -24
RSTD = SUM / 2 + 4 * 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = PVContext(0)
    yield c
    c.close()


def draw(rows, cols, dtype, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    x, r = torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g) * 2
    return x.to(dtype), r.to(dtype), 1 + 0.2 * torch.randn(cols, generator=g)


SHAPES = [(1, 1), (3, 7), (2, 32), (5, 33), (1, 500), (4, 2072), (3, 2077), (1, 4096), (1030, 96), (1025, 520), (1024, 4096),
          (2, 8200), (3, 11008), (2, 16384), (2, 16385), (1, 40001)]


def check_y8(codes, scales, fmt, y, slack, cols):
    """Codes of y known up to `slack` (relative): the block's power of two belongs to a maximum within it, and each value is
    the nearest of the format to some value within it."""
    rows = y.shape[0]
    s = scales.cpu().long()
    pad = torch.zeros(rows, s.shape[1] * 32 - cols, dtype=torch.float64)
    big = torch.cat((y, pad), 1).view(rows, -1, 32).abs().amax(2)
    lo, hi = ((ref.exponent(big * f) - ref.EMAX[fmt]).clamp(-127, 127) + 127 for f in (1 - slack, 1 + slack))
    zero = big == 0
    assert ((s >= lo) & (s <= hi) | zero & (s == 0)).all()
    power = torch.exp2((s - 127).double()).repeat_interleave(32, 1)[:, :cols]
    v = y / power
    step = torch.exp2((torch.where(v != 0, ref.exponent(v.abs()), 0).clamp(min=ref.LOW[fmt]) - ref.MANT[fmt]).double())
    got = ref.decode(codes, scales, fmt, cols) / power
    near = (got - v.clamp(-ref.TOP[fmt], ref.TOP[fmt])).abs()
    assert (near <= step / 2 + slack * v.abs()).all()
    tail = ref.split(codes, fmt)[:, cols:]
    assert int(torch.count_nonzero(tail)) == 0


@pytest.mark.parametrize("residual", [True, False], ids=["residual", "alone"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(ctx, rows, cols, dtype, residual):
    x, r, w = draw(rows, cols, dtype, seed=rows + cols)
    r = r if residual else None
    h, rstd, y = ref.rms_norm(x, r, w, EPS, dtype)
    xd, rd, wd = x.to(DEV), None if r is None else r.to(DEV), w.to(DEV)
    out = {n: torch.full((rows, cols), 7.0, dtype=dtype, device=DEV) for n in "hy"}
    rs = torch.empty(rows, device=DEV)
    fmt = "e4m3" if cols % 2 else "e2m1"
    codes, scales = (torch.full(s, 0xA5, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, cols, fmt))
    ctx.pv_rms_norm(rows, cols, xd, rd, wd, EPS, h=out["h"], y=out["y"], fmt=fmt, codes=codes, scales=scales, rstd=rs)
    assert torch.equal(out["h"].cpu().double(), h)
    ref.check(rs, rstd, rstd * RSTD)
    err = y.abs() * (RSTD + 2 * 2.0 ** -24)
    ref.check(out["y"], y, err + ref.rounding(y.abs() + err, dtype))
    check_y8(codes, scales, fmt, y, RSTD + 2 * 2.0 ** -24, cols)
    # fewer outputs, and outputs in place of inputs: the same bits
    y2 = torch.empty_like(out["y"])
    ctx.pv_rms_norm(rows, cols, xd, rd, wd, EPS, y=y2)
    c2, s2 = torch.empty_like(codes), torch.empty_like(scales)
    ctx.pv_rms_norm(rows, cols, xd, rd, wd, EPS, fmt=fmt, codes=c2, scales=s2)
    assert torch.equal(y2, out["y"]) and torch.equal(c2, codes) and torch.equal(s2, scales)
    a, b = xd.clone(), None if rd is None else rd.clone()
    ctx.pv_rms_norm(rows, cols, a, b, wd, EPS, h=a if b is None else b, y=None if b is None else a)
    assert torch.equal(a if b is None else b, out["h"]) and (b is None or torch.equal(a, out["y"]))


def test_rows_of_zeros_and_rows_that_are_not_finite(ctx):
    cols = 70
    x = torch.ones(4, cols)
    x[1], x[2, 3], x[3, 5] = 0.0, math.inf, math.nan
    w = torch.ones(cols)
    y, rs = torch.empty(4, cols, device=DEV), torch.empty(4, device=DEV)
    codes, scales = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in mx_shapes(4, cols, "e4m3"))
    for eps in (EPS, 0.0):
        ctx.pv_rms_norm(4, cols, x.to(DEV), None, w.to(DEV), eps, y=y, codes=codes, scales=scales, rstd=rs)
        _, rstd, want = ref.rms_norm(x, None, w, eps, torch.float32)
        ref.check(rs, rstd, rstd * RSTD)
        err = want.abs() * RSTD
        ref.check(y, want, err + ref.rounding(want, torch.float32))
        assert torch.equal((scales == 255).cpu().any(1), (~torch.isfinite(want)).any(1))


@pytest.mark.parametrize("with_dh", [True, False], ids=["dh", "alone"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 33), (700, 96), (5, 2077), (9, 4096), (600, 1000), (3, 11008), (2, 16384),
                                       (2, 16385), (515, 40), (3, 40001)])
def test_backward(ctx, rows, cols, dtype, with_dh):
    h, dy, w = draw(rows, cols, dtype, seed=rows * 7 + cols)
    dh = draw(rows, cols, dtype, seed=rows + 1)[0] if with_dh else None
    _, rstd, _ = ref.rms_norm(h, None, w, EPS, dtype)
    rs = rstd.float()
    dx, dw = ref.rms_norm_backward(dy, dh, h, w, rs)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    got, gw = torch.full((rows, cols), 7.0, dtype=dtype, device=DEV), torch.full((cols,), 7.0, device=DEV)
    args = (rows, cols, dev(dy), dev(dh), dev(h), dev(w), dev(rs))
    ctx.pv_rms_norm_backward(*args, got, gw)
    d, n = dy.double(), h.double() * rs.double()[:, None]
    # the row's dot product: a float32 sum as above of terms of either sign, each a product of four factors
    dot = (d * w.double() * n).abs().mean(1, keepdim=True) * (SUM + 4 * 2.0 ** -24)
    err = rs.double()[:, None] * (n.abs() * dot + ((d * w.double()).abs() + 2 * (n * (d * w.double() * n).mean(1, keepdim=True)).abs()) * 4 * 2.0 ** -24)
    ref.check(got, dx, err + ref.rounding(dx.abs() + err, dtype) + (dx.abs() + (0 if dh is None else dh.double().abs())) * 2.0 ** -24, "dx")
    # a column: at most ceil(rows / 512) rows one after the other, an eighth of 512 sums, and 8 of those
    err = (d * n).abs().sum(0) * (-(-rows // 512) + 64 + 8 + 2) * 2.0 ** -24
    ref.check(gw, dw, err + ref.rounding(dw, torch.float32), "dweight")
    # each alone, and in place: the same bits
    a, b = torch.empty_like(got), torch.empty_like(gw)
    ctx.pv_rms_norm_backward(*args, dx=a)
    ctx.pv_rms_norm_backward(*args, dweight=b)
    assert torch.equal(a, got) and torch.equal(b, gw)
    for place in (2, 3, 4):
        if args[place] is None:
            continue
        again = [t.clone() if isinstance(t, torch.Tensor) else t for t in args]
        ctx.pv_rms_norm_backward(*again, dx=again[place])
        assert torch.equal(again[place], got)


def test_backward_by_differences(ctx):
    """phi = sum(R * y + S * h) along one direction of x and of the weight, by a central difference of the 64-bit forward."""
    rows, cols = 6, 130
    x, r, w = draw(rows, cols, torch.float32, 21)
    big_r, big_s, u = draw(rows, cols, torch.float32, 22)[0], draw(rows, cols, torch.float32, 23)[0], draw(rows, cols, torch.float32, 24)[0].double()
    uw = draw(1, cols, torch.float32, 25)[2].double()
    h, rstd = (x + r).to(DEV), torch.empty(rows, device=DEV)
    ctx.pv_rms_norm(rows, cols, x.to(DEV), r.to(DEV), w.to(DEV), EPS, rstd=rstd)
    dx, dw = torch.empty(rows, cols, device=DEV), torch.empty(cols, device=DEV)
    ctx.pv_rms_norm_backward(rows, cols, big_r.to(DEV), big_s.to(DEV), h, w.to(DEV), rstd, dx, dw)

    def phi(hh, ww):
        y = hh * (hh.square().mean(1, keepdim=True) + EPS).rsqrt() * ww
        return float((big_r.double() * y + big_s.double() * hh).sum())

    h64, w64, e = h.cpu().double(), w.double(), 1e-5
    for got, want in ((float((dx.cpu().double() * u).sum()), (phi(h64 + e * u, w64) - phi(h64 - e * u, w64)) / (2 * e)),
                      (float((dw.cpu().double() * uw).sum()), (phi(h64, w64 + e * uw) - phi(h64, w64 - e * uw)) / (2 * e))):
        # float32 gradients of 780 (130) terms of order 1; the difference's own error is of order e^2
        assert abs(got - want) <= 1e-3 * 2.0 ** -4 * max(1.0, abs(want))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(1500, 64), (1025, 128), (1027, 31), (2000, 200), (1024, 256), (17001, 72), (1030, 257)])
def test_many_short_rows(ctx, rows, cols, dtype):
    """Several rows to a wave: heads' norms."""
    test_norm(ctx, rows, cols, dtype, True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(4096, 64), (4097, 128), (4111, 7), (4100, 200), (4098, 65), (5000, 500), (4097, 520), (20011, 33)])
def test_backward_of_many_short_rows(ctx, rows, cols, dtype):
    """A column's sum: R rows at a time (R = 32 at most, 4 at least) in P <= 1024 blocks, so ceil(rows / (R P)) + R + ceil(P / 32) + 32
    additions one after the other; with P = 1024 only from 1024 R rows on.  At these shapes 86 at most (20011 rows of 33: R = 32,
    P = 626), within the bound of the others, ceil(rows / 512) + 74, which is 82 or more and there 114."""
    test_backward(ctx, rows, cols, dtype, True)


@pytest.mark.parametrize("rows,cols", [(4096, 1024), (300, 16416)])
def test_codes_are_those_of_the_formula(ctx, rows, cols):
    """A value changes its code if it lies within its error of a tie, and ties lie an eighth of the value or more apart, so with an
    error of 2^-24 of it one in 2^20 would.  The sum's error is what is left: eight terms of a lane in float32, 7 roundings of
    at most half a 2^-23 each and of either sign, averaged over cols / 8 lanes and halved by the root: below 2^-24 * 7 / 2 / sqrt(cols / 8)
    in the mean, 2^-26 here; one code in 2^22, so 1 is expected of 2^22, and 12 have a probability below 10^-8."""
    g = torch.Generator(device=DEV).manual_seed(11)
    x = (torch.randn(rows, cols, generator=g, device=DEV) * 3).bfloat16()
    weight = 1 + 0.2 * torch.randn(cols, generator=g, device=DEV)
    codes, scales = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, cols, "e4m3"))
    ctx.pv_rms_norm(rows, cols, x, None, weight, EPS, codes=codes, scales=scales)
    _, _, y = ref.rms_norm(x, None, weight, EPS, x.dtype)
    want_codes, want_scales = ref.quantize(y, "e4m3")
    assert torch.equal(scales.cpu(), want_scales)
    assert int((codes.cpu() != want_codes).sum()) <= 12


def test_more_long_rows_than_blocks(ctx):
    """Rows that no block holds in registers, more of them than a launch has blocks: the same as in parts, and in place."""
    rows, cols = 4099, 16392
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(rows, cols, generator=g, device=DEV).bfloat16()
    weight = torch.rand(cols, generator=g, device=DEV) + 0.5
    y, rstd = torch.empty_like(x), torch.empty(rows, device=DEV)
    ctx.pv_rms_norm(rows, cols, x, x, weight, EPS, y=y, rstd=rstd)
    for at, n in [(0, 2048), (2048, rows - 2048)]:
        part, r = torch.empty(n, cols, dtype=x.dtype, device=DEV), torch.empty(n, device=DEV)
        ctx.pv_rms_norm(n, cols, x[at:at + n], x[at:at + n], weight, EPS, y=part, rstd=r)
        assert torch.equal(part, y[at:at + n]) and torch.equal(r, rstd[at:at + n])
    want = ref.rms_norm(x[-3:], x[-3:], weight, EPS, x.dtype)[1]
    ref.check(rstd[-3:], want, 1e-5 * want)
    ctx.pv_rms_norm(rows, cols, x, x, weight, EPS, y=x)
    assert torch.equal(x, y)


def test_empty(ctx):
    e = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    dw = torch.full((5,), 7.0, device=DEV)
    ctx.pv_rms_norm_backward(0, 5, e(0, 5), None, e(0, 5), e(5), e(0), e(0, 5), dw)
    assert int(torch.count_nonzero(dw)) == 0
    ctx.pv_rms_norm(0, 5, e(0, 5), None, e(5), EPS, y=e(0, 5))
    ctx.pv_rms_norm(3, 0, e(3, 0), None, e(0), EPS, y=e(3, 0))
