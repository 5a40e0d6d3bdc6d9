"""RMS norm where its results leave float32, and rows of more columns than a launch counts threads for."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import PVContext, mx_shapes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = PVContext(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(3, 70), (1030, 96), (2, 4096), (2, 16400)])
def test_outputs_beyond_float32_are_infinite(ctx, rows, cols, dtype):
    """h * rstd * weight beyond the largest float32 is an infinity with its sign, in 8 bits a block that is NaN; what lies next to
    it in the row, and the row's rstd, are what they are."""
    g = torch.Generator().manual_seed(cols)
    x = torch.randn(rows, cols, generator=g).to(dtype)
    w = 1 + 0.2 * torch.randn(cols, generator=g)
    w[32:40] = torch.tensor([3.4e38, -3.4e38, 2e38, 1e38, 3e37, -1e38, 3.4e38, -3.4e38])
    x[:, 32], x[:, 33], x[:, 38], x[:, 39] = 3.0, 3.0, -3.0, -3.0
    y, rstd = torch.full((rows, cols), 7.0, dtype=dtype, device=DEV), torch.empty(rows, device=DEV)
    codes, scales = (torch.full(s, 0xA5, dtype=torch.uint8, device=DEV) for s in mx_shapes(rows, cols, "e4m3"))
    ctx.pv_rms_norm(rows, cols, x.to(DEV), None, w.to(DEV), EPS, y=y, codes=codes, scales=scales, rstd=rstd)
    _, want_rstd, want = ref.rms_norm(x, None, w, EPS, dtype)
    ref.check(rstd, want_rstd, want_rstd * 2.0 ** -21)          # eight squares, a lane, in float32; halved; three roundings
    # What rounds to an infinity begins half a step above the largest value.  A step there is eps times the power of two below:
    # bfloat16's largest is (2 - 2^-7) 2^127, its step 2^-7 2^127, so (2 - 2^-8) 2^127.  No value lies within its error of there.
    most = torch.finfo(dtype).max
    edge = most + torch.finfo(dtype).eps / 2 * 2.0 ** math.floor(math.log2(most))
    assert ((want.abs() / edge - 1).abs() > 2.0 ** -19).all()
    err = want.abs() * 2.0 ** -20
    want = torch.where(want.abs() > edge, want.sign() * math.inf, want)
    assert torch.isinf(want[:, 32]).all() and torch.isinf(want[:, 38]).all()
    fine = torch.where(torch.isinf(want), 0.0, want)
    ref.check(y, want, torch.where(torch.isinf(want), 0.0, err) + ref.rounding(fine, dtype) * (1 + 2.0 ** -19))
    assert (scales[:, 1] == 255).all() and int(torch.count_nonzero(codes[:, 32:64])) == 0
    assert (scales[:, 0] != 255).all() and (scales[:, 2:] != 255).all()


def test_gradients_of_more_columns_than_a_launch_counts_threads_for():
    """32 threads a column: 2^27 columns are 2^32.  Two rows, so a column's sum has two terms; the row's dot product has 2^27, of which
    a lane adds 2^17 one after the other."""
    rows, cols = 2, (1 << 27) + 37
    ctx = PVContext(0)
    g = torch.Generator(device=DEV).manual_seed(5)
    dy, h = (torch.randn(rows, cols, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    weight = torch.rand(cols, generator=g, device=DEV) + 0.5
    rstd = torch.tensor([0.75, 1.25], device=DEV)
    dx, dweight = torch.full_like(dy, 7.0), torch.full((cols,), 7.0, device=DEV)
    ctx.pv_rms_norm_backward(rows, cols, dy, None, h, weight, rstd, dx, dweight)
    parts = [slice(at, min(at + (1 << 24), cols)) for at in range(0, cols, 1 << 24)]
    r = rstd.double()[:, None]
    terms = [dy[:, p].double() * weight[p].double() * h[:, p].double() * r for p in parts]
    dot, size = (sum(f(t).sum(1, keepdim=True) for t in terms) / cols for f in (lambda t: t, torch.abs))
    del terms
    for p in parts:
        d, n = dy[:, p].double(), h[:, p].double() * r
        want = (d * n).sum(0)
        assert ((dweight[p].double() - want).abs() <= 3 * 2.0 ** -24 * (d * n).abs().sum(0)).all()
        want = r * (d * weight[p].double() - n * dot)
        err = r * (n.abs() * size * (2 ** 17 + 64) * 2.0 ** -24 + ((d * weight[p].double()).abs() + (n * dot).abs()) * 4 * 2.0 ** -24)
        assert ((dx[:, p].double() - want).abs() <= err + ref.rounding(want.abs() + err, torch.bfloat16)).all()
    ctx.close()
