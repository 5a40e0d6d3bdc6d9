"""Distillation of logits far from zero, of small temperatures and of far teachers: q and p depend on differences of logits alone,
so what a row may be off does not grow with its distance from zero.  Against 64-bit sums of the differences."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import PVContext

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24                      # half a step of float32


@pytest.fixture(scope="module")
def ctx():
    c = PVContext(0)
    yield c
    c.close()


def expected(z, ids, top, t, weight=None):
    """loss, lse, grad and what each may be off, row by row.  An exponent -(largest - z) / t of size d is formed by at most four
    roundings, so its exponential is off by 4 d U of itself (d counts up to 104: what lies below is less than any float32);
    a sum's terms pass as many additions as a lane has of them, and a tree's."""
    z, u, ids, rows, vocab = z.double(), top.double(), ids.long(), z.shape[0], z.shape[1]
    w = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double()
    there = (ids >= 0) & (ids < vocab)
    at = torch.where(there, ids, 0)
    u = torch.where(there, u, -math.inf)
    big_z, big_u = z.amax(1, keepdim=True), u.amax(1, keepdim=True)
    dz, du = (big_z - z) / t, torch.where(torch.isinf(u), math.inf, (big_u - u) / t)
    any_ = big_u[:, 0] > -math.inf
    sum_z, sum_u = torch.exp(-dz).sum(1, keepdim=True), torch.exp(-du).sum(1, keepdim=True)
    q, p = torch.exp(-dz) / sum_z, torch.where(any_[:, None], torch.exp(-du) / sum_u, 0.0)
    ln_q, ln_p = -dz.gather(1, at) - torch.log(sum_z), -du - torch.log(sum_u)
    ratio = torch.where(p > 2.0 ** -149, ln_p - ln_q, 0.0)
    on = (w != 0) & any_
    loss = torch.where(on, w * t * t * (p * ratio).sum(1), 0.0)
    lse = torch.where(w != 0, big_z[:, 0] / t + torch.log(sum_z)[:, 0], 0.0)
    target = torch.zeros_like(z).scatter_add(1, at, torch.where(there, p, 0.0))
    grad = torch.where(on[:, None], (w * t)[:, None] * (q - target), 0.0)
    lane = max(256, -(-vocab // 512) * 5 // 4)
    depth = lambda d: torch.where(d < 104, d, 0.0).amax(1)  # noqa: E731
    s_z, s_u = (4 * depth(dz) + lane + 24) * U, (4 * depth(du) + 40) * U
    off_lse = s_z + lse.abs() * 4 * U
    size = (p * ratio.abs()).sum(1)
    off_loss = w.abs() * t * t * (s_z + s_u + (s_u + 32 * U) * size + 8 * U * (1 + (p * torch.where(p > 2.0 ** -149, dz.gather(1, at) + du, 0.0)).sum(1)))
    off_grad = (w.abs() * t)[:, None] * ((s_z + 8 * U)[:, None] * q + (s_u + 24 * U)[:, None] * target) + 2.0 ** -120
    # nothing here allows more than a few digits of float32: no row hides behind another's size
    assert float(s_z.max()) < 2.0 ** -13 and float(s_u.max()) < 2.0 ** -14
    return (loss, lse, grad), (off_loss, off_lse, off_grad)


def compare(ctx, z, ids, top, t, weight=None, backward=True):
    rows, vocab, k, dtype = z.shape[0], z.shape[1], ids.shape[1], z.dtype
    args = (rows, vocab, k, z.to(DEV), ids.to(DEV), top.to(DEV), t)
    wd = None if weight is None else weight.to(DEV)
    (loss, lse, grad), (off_loss, off_lse, off_grad) = expected(z, ids, top, t, weight)
    got_loss, got_lse = torch.full((rows,), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
    got = torch.full((rows, vocab), 7.0, dtype=dtype, device=DEV)

    def check(got, want, off, what):
        ref.check(got, want, off + ref.rounding(want.abs() + off, got.dtype), what)

    beyond = lse.abs() > torch.finfo(torch.float32).max
    lse = torch.where(beyond, lse.sign() * math.inf, lse)
    off_lse = torch.where(beyond, 0.0, off_lse)
    for g in (got, None):
        ctx.pv_distill_topk(*args, row_weight=wd, loss=got_loss, lse=got_lse, grad=g)
        check(got_loss, loss, off_loss, "loss")
        ref.check(got_lse, lse, off_lse, "lse")
    check(got, grad, off_grad, "grad")
    if not backward:
        return
    # the two directions agree: from the saved sum, for a gradient of the loss that is this call's weight
    ctx.pv_distill_topk(*args, loss=got_loss, lse=got_lse)
    w = torch.linspace(0.5, 1.5, rows) if weight is None else weight
    (_, lse, grad), (_, _, off_grad) = expected(z, ids, top, t, w)
    # up to 256 the saved float32 sum is off by 2 U of itself, and so is every z / t: q follows
    near = torch.where(lse.abs() < 256, 2 * (lse.abs() + (lse.abs() + 104)) * 2 * U, 0.0)
    off_grad = off_grad + (w.double().abs() * t * near)[:, None] * torch.softmax((z.double() - z.double().amax(1, keepdim=True)) / t, 1)
    for place in (torch.full_like(got, 9.0), args[3]):              # (the last in place of the logits)
        ctx.pv_distill_topk_backward(*args, got_lse, w.to(DEV), place)
        check(place, grad, off_grad, "backward")


FAR = [0.0, 2000.0, -1e4, 6e4, 1e6, -1e6, -1e9, 1e9, 4e9, -1e10, -1e12, -1e20, 1e20, -1e29, 1e31, -3e38]


def far_rows(vocab, dtype, seed):
    """Two rows at each distance from zero that the type holds: of one value, and of values around it (as far as the type tells them
    apart)."""
    g = torch.Generator().manual_seed(seed)
    at = [b for b in FAR if abs(b) < torch.finfo(dtype).max]
    z = torch.cat([torch.stack((torch.full((vocab,), b, dtype=torch.float64), b + 2.5 * torch.randn(vocab, generator=g, dtype=torch.float64)))
                   for b in at]).to(dtype)
    k = min(vocab, 6)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in z]).int()
    return z, ids, torch.randn(len(z), k, generator=g) * 2


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab", [1, 50, 3001, 9000, 33000])
def test_rows_far_from_zero(ctx, vocab, dtype):
    """Rows that stay in registers."""
    compare(ctx, *far_rows(vocab, dtype, seed=vocab), 1.0, backward=False)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("t", [2.0 ** -126, 1e-30, 1e-12, 1e-9, 1e-6, 0.01, 100.0])
def test_small_and_large_temperatures(ctx, t, dtype):
    """Of the largest logits alone, or nearly uniform."""
    t = float(torch.tensor(t, dtype=torch.float32))
    z, ids, top = far_rows(700, dtype, seed=5)
    z[:, 100:103] = z.amax(1, keepdim=True)                          # some places share the probability
    compare(ctx, z, ids, top, t, backward=False)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab", [70000, 140001])
def test_long_rows_far_from_zero(ctx, vocab, dtype):
    """Rows that pass by (70000 of 16 bits still stay): the gradient belongs to the same sum as the loss."""
    compare(ctx, *far_rows(vocab, dtype, seed=vocab), 1.0, backward=False)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab,t", [(1, 1.0), (50, 1.0), (700, 1e-9), (700, 0.01), (3001, 1.0), (9000, 0.5), (70000, 1.0), (140001, 1.0)])
def test_both_directions_agree_far_from_zero(ctx, vocab, t, dtype):
    compare(ctx, *far_rows(vocab, dtype, seed=vocab + 1), float(torch.tensor(t, dtype=torch.float32)))


@pytest.mark.parametrize("t", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("vocab", [50, 70000])
def test_teachers_far_from_zero(ctx, vocab, t):
    """The teacher's logits are shifted, one value, or at either end of float32."""
    z, ids, top = far_rows(vocab, torch.float32, seed=9)
    low, high = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    for r, b in enumerate([1e3, -1e4, 1e6, -1e6, 1e9, -1e9, 1e20, -1e30]):
        top[r] = (top[r].double() + b).float()
    top[8], top[9], top[10, 1:], top[11, ::2] = low, high, low, high
    top[12, 0], top[12, 1] = high, low
    top[13], top[13, 2] = -math.inf, -1e38
    compare(ctx, z[:16], ids[:16], top[:16], t, backward=False)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab", [1003, 70001, 140003])
def test_every_row_by_its_own_measure(ctx, vocab, dtype):
    """Missing entries, places twice, masked places, rows without weight: each row's results are allowed what that row's sizes
    allow, whatever else the batch holds."""
    rows, k = 14, 24
    g = torch.Generator().manual_seed(vocab)
    z = (torch.randn(rows, vocab, generator=g) * 2.5).to(dtype)
    top, ids = torch.topk(z.float() + 0.5 * torch.randn(rows, vocab, generator=g), k, 1)
    ids = ids.int()
    weight = torch.linspace(0.25, 2.0, rows)
    weight[1] = 0.0
    ids[2] = -1
    ids[3, 5:] = -1
    ids[4, ::2] = vocab
    ids[4, 1] = -(2 ** 31)
    top[5] = -math.inf
    top[6, 3:] = -math.inf
    ids[7, :] = ids[7, 0]
    ids[8, 12:] = ids[8, :12]
    z[9, : vocab // 2] = -math.inf
    ids[9] = torch.arange(vocab - k, vocab)
    z[10, vocab - 1] = torch.finfo(dtype).min
    top[10, 0] = torch.finfo(torch.float32).min
    z[11, k:] = torch.finfo(dtype).min
    ids[11] = torch.arange(k)
    z[12, ids[12, 0]] = -math.inf                    # the teacher says nothing there either
    top[12, 0] = -math.inf
    compare(ctx, z, ids, top, 1.0, weight)
