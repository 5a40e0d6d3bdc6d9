"""Distillation from a teacher's top logits: loss and gradients against a plain 64-bit implementation."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import PVContext

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    c = PVContext(0)
    yield c
    c.close()


def draw(rows, vocab, k, dtype, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * 2.5
    k_ = min(k, vocab)
    top, ids = torch.topk(z + 0.5 * torch.randn(rows, vocab, generator=g), k_, 1)
    if k_ < k:                                  # more entries than places: some of them twice
        more = torch.randint(0, vocab, (rows, k - k_), generator=g)
        ids, top = torch.cat((ids, more), 1), torch.cat((top, torch.randn(rows, k - k_, generator=g)), 1)
    return z.to(dtype), ids.int(), top.contiguous()


def slack(z, t):
    """What float32 may be off, relative to q, to p and absolutely in a log: the exponent's argument, of size a, is off by a
    few roundings, 4 a 2^-24, and the sum over the vocabulary by one 2^-24 for each operation that a term passes: the additions
    after it in its lane and 16 levels of a tree.  A lane has at most 256 terms where the row stays in registers; where it
    passes by, at most a 512th of the row, with one multiplication (by the exponential of a difference of the
    lane's largest values, itself off by its argument and counted in 4 a) for every four of them."""
    a = float((z.double().abs().max() * 2 / t).clamp(min=1.0))
    lane = max(256, -(-z.shape[1] // 512) * 5 // 4)
    return (4 * a + lane + 24) * 2.0 ** -24


def compare(ctx, z, ids, top, t, weight, dtype, stride=None):
    rows, vocab = z.shape
    k = ids.shape[1]
    buf = torch.full((rows, stride or vocab), 3.0, dtype=dtype, device=DEV)
    zd = buf[:, :vocab]
    zd.copy_(z)
    idd, topd = ids.to(DEV), top.to(DEV)
    wd = None if weight is None else weight.to(DEV)
    loss, lse = torch.full((rows,), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
    gbuf = torch.full((rows, (stride or vocab) + 3), 5.0, dtype=dtype, device=DEV)
    grad = gbuf[:, :vocab]
    args = (rows, vocab, k, zd, idd, topd, t)
    ctx.pv_distill_topk(*args, row_weight=wd, loss=loss, lse=lse, grad=grad)
    w_loss, w_lse, w_grad = ref.distill(z, ids, top, t, weight)
    fin = torch.where(torch.isfinite(z.float()), z.float(), 0.0)
    s = slack(torch.cat((fin, top.nan_to_num(0, 0, 0)), 1) if k else fin, t)
    c = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double().abs()
    ref.check(lse, w_lse, s * 2 + w_lse.abs().nan_to_num(0, 0, 0) * 2.0 ** -23, "lse")
    ref.check(loss, w_loss, c * t * t * (2 * s + 2.0 ** -22) + w_loss.abs().nan_to_num(0, 0, 0) * 2.0 ** -20, "loss")
    target = (w_grad / torch.where(c > 0, c * t, 1.0)[:, None]).abs() + 2 * torch.softmax(fin.double() / t, 1)
    err = (c * t)[:, None] * s * target.nan_to_num(1.0)
    fine = torch.where(torch.isfinite(w_grad), w_grad, 0.0)
    ref.check(grad, w_grad, err + ref.rounding(fine.abs() + err, dtype), "grad")
    # rows end where the vocabulary does
    assert bool((gbuf[:, vocab:] == 5.0).all()) and bool((buf[:, vocab:] == 3.0).all())
    # the loss alone; the gradient in place of the logits
    l2 = torch.empty_like(loss)
    ctx.pv_distill_topk(*args, row_weight=wd, loss=l2)          # (its sums may have another order)
    ref.check(l2, w_loss, c * t * t * (2 * s + 2.0 ** -22) + w_loss.abs().nan_to_num(0, 0, 0) * 2.0 ** -20, "loss alone")
    # the gradient from the saved sum, for another gradient of the loss
    gl = torch.rand(rows, generator=torch.Generator().manual_seed(3)).to(DEV) * (1.0 if wd is None else (wd != 0).float())
    ctx.pv_distill_topk(*args, loss=l2, lse=lse)
    back = torch.full_like(grad, 9.0)
    ctx.pv_distill_topk_backward(*args, lse, gl, back)
    _, _, w_back = ref.distill(z, ids, top, t, gl.cpu())
    cg = gl.cpu().double()
    fine = torch.where(torch.isfinite(w_back), w_back, 0.0)
    # the saved sum is a float32 of size |lse|, and so is every z / t
    more = s + 2 * (float(w_lse.abs().nan_to_num(0, 0, 0).max()) + float((fin.abs().max() / t))) * 2.0 ** -23
    err = (cg * t)[:, None] * more * target.nan_to_num(1.0) * 2
    ref.check(back, w_back, err + ref.rounding(fine.abs() + err, dtype), "backward")
    ctx.pv_distill_topk(*args, row_weight=wd, loss=l2, grad=zd)
    assert torch.equal(zd.nan_to_num(1e4), grad.nan_to_num(1e4))
    return loss, grad


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,vocab,k,t", [(1, 1, 1, 1.0), (3, 7, 2, 1.0), (2, 33, 40, 2.0), (5, 1000, 64, 1.0), (4, 8193, 20, 0.5),
                                            (2, 32000, 256, 1.0), (3, 50257, 5, 4.0), (1, 65541, 1024, 2.0), (2, 131072, 64, 1.0),
                                            (1, 140001, 33, 1.0), (2, 1 << 20, 8, 1.0)])
def test_loss_and_gradients(ctx, rows, vocab, k, t, dtype):
    z, ids, top = draw(rows, vocab, k, dtype, seed=vocab + k)
    compare(ctx, z, ids, top, t, None, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab,stride", [(1000, 1024), (1003, 1005), (70001, 70016)])
def test_masked_rows_missing_entries_and_row_strides(ctx, vocab, stride, dtype):
    rows, k = 12, 24
    z, ids, top = draw(rows, vocab, k, dtype, seed=vocab)
    weight = torch.linspace(0.25, 2.0, rows)
    weight[1] = 0.0
    z[1] = math.nan                                  # a row without weight is not read
    weight[2] = 0.0
    ids[3, 5:] = -1                                  # fewer entries
    ids[4] = -1                                      # none
    ids[5, ::2] = vocab                              # places that do not exist
    ids[5, 1] = -(2 ** 31)
    top[6] = -math.inf                               # entries without probability
    top[7, 3:] = -math.inf
    ids[8, :] = ids[8, 0]                            # one place only
    ids[9, 12:] = ids[9, :12]                        # every place twice
    z[10, : vocab // 2] = -math.inf                  # masked places of the student
    ids[10] = torch.arange(vocab - k, vocab)
    z[11, vocab - 1] = torch.finfo(dtype).min        # masked by the type's lowest value
    top[11, 0] = torch.finfo(torch.float32).min
    compare(ctx, z, ids, top, 1.0, weight, dtype, stride)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab", [50, 9000, 70000])
def test_rows_masked_by_the_lowest_value(ctx, vocab, dtype):
    """All of a row, all but one place, and all of what some lanes see."""
    z, ids, top = draw(4, vocab, 3, dtype, seed=vocab)
    low = torch.finfo(dtype).min
    z[0] = low
    z[1, 1:], ids[1, 0] = low, 0
    ids[1, 1:] = -1                                  # the teacher's one place is the student's
    z[2, 7:] = -math.inf
    ids[2] = torch.arange(3)
    t = 1.0
    loss, lse, grad = torch.empty(4, device=DEV), torch.empty(4, device=DEV), torch.empty(4, vocab, dtype=dtype, device=DEV)
    args = (4, vocab, 3, z.to(DEV), ids.to(DEV), top.to(DEV), t)
    w_loss, _, w_grad = ref.distill(z, ids, top, t)
    for g in (grad, None):
        ctx.pv_distill_topk(*args, loss=loss, lse=lse, grad=g)
        # a row of equal logits is uniform, whatever they are: its logarithm is that of the vocabulary
        ref.check(loss, w_loss, 1e-4 * (1 + w_loss.abs()))
    s = slack(z[3:].float(), t)
    err = s * (w_grad.abs() + 2 * torch.softmax(z.double(), 1))
    ref.check(grad, w_grad, err + ref.rounding(w_grad.abs() + err, dtype))


def test_the_student_has_no_probability_where_the_teacher_has(ctx):
    z, ids, top = draw(3, 100, 4, torch.float32, seed=1)
    z[1, ids[1, 0]] = -math.inf
    loss, grad = compare(ctx, z, ids, top, 1.0, None, torch.float32)
    assert math.isinf(float(loss[1])) and bool(torch.isfinite(grad).all())
    top[1, 0] = -math.inf                            # nor has the teacher: the place says nothing
    loss, grad = compare(ctx, z, ids, top, 1.0, None, torch.float32)
    assert bool(torch.isfinite(loss).all())


def test_values_that_are_not_finite_show(ctx):
    z, ids, top = draw(4, 300, 4, torch.float32, seed=2)
    z[0, 7], z[1, 9], top[2, 1] = math.nan, math.inf, math.nan
    loss, grad = torch.empty(4, device=DEV), torch.empty(4, 300, device=DEV)
    ctx.pv_distill_topk(4, 300, 4, z.to(DEV), ids.to(DEV), top.to(DEV), 1.0, loss=loss, grad=grad)
    assert torch.isnan(loss).cpu().tolist() == [True, True, True, False]
    assert torch.isnan(grad).any(1).cpu().tolist() == [True, True, True, False]


def test_no_entries_at_all(ctx):
    z = torch.randn(3, 50)
    loss, lse, grad = torch.empty(3, device=DEV), torch.empty(3, device=DEV), torch.empty(3, 50, device=DEV)
    ctx.pv_distill_topk(3, 50, 0, z.to(DEV), None, None, 1.0, loss=loss, lse=lse, grad=grad)
    assert int(torch.count_nonzero(loss)) == 0 and int(torch.count_nonzero(grad)) == 0
    ref.check(lse, torch.logsumexp(z.double(), 1), 1e-5)
    ctx.pv_distill_topk(0, 50, 0, torch.empty(0, 50, device=DEV), None, None, 1.0, loss=torch.empty(0, device=DEV))


def test_more_rows_than_a_launch_has_blocks(ctx):
    """2^32 threads are 2^24 rows of 256: the same as in parts."""
    rows, half = (1 << 24) + 70, 1 << 23
    g = torch.Generator(device=DEV).manual_seed(8)
    z, top = torch.randn(rows, 3, generator=g, device=DEV), torch.randn(rows, 1, generator=g, device=DEV)
    ids = torch.randint(0, 3, (rows, 1), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(rows, generator=g, device=DEV)
    new = lambda n: (torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, 3, device=DEV))  # noqa: E731
    loss, lse, grad = new(rows)
    ctx.pv_distill_topk(rows, 3, 1, z, ids, top, 2.0, row_weight=c, loss=loss, lse=lse, grad=grad)
    back = torch.empty_like(grad)
    ctx.pv_distill_topk_backward(rows, 3, 1, z, ids, top, 2.0, lse, c, back)
    for at, n in [(0, half), (half, half), (2 * half, rows - 2 * half)]:
        s = slice(at, at + n)
        l2, e2, g2 = new(n)
        ctx.pv_distill_topk(n, 3, 1, z[s], ids[s], top[s], 2.0, row_weight=c[s], loss=l2, lse=e2, grad=g2)
        assert torch.equal(l2, loss[s]) and torch.equal(e2, lse[s]) and torch.equal(g2, grad[s])
        ctx.pv_distill_topk_backward(n, 3, 1, z[s], ids[s], top[s], 2.0, e2, c[s], g2)
        assert torch.equal(g2, back[s])


def test_gradient_by_differences(ctx):
    """A central difference of the 64-bit loss along one direction."""
    rows, vocab, k, t = 4, 60, 7, 2.0
    z, ids, top = draw(rows, vocab, k, torch.float32, seed=4)
    loss, grad = torch.empty(rows, device=DEV), torch.empty(rows, vocab, device=DEV)
    ctx.pv_distill_topk(rows, vocab, k, z.to(DEV), ids.to(DEV), top.to(DEV), t, loss=loss, grad=grad)
    u, e = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(5)).double(), 1e-5
    f = lambda zz: ref.distill(zz, ids, top, t)[0].sum()  # noqa: E731
    want = float((f(z.double() + e * u) - f(z.double() - e * u)) / (2 * e))
    # 240 float32 products of order 1, each off by some 2^-20 of itself
    assert abs(float((grad.cpu().double() * u).sum()) - want) <= 240 * 2.0 ** -20


def test_the_same_bits_every_time(ctx):
    z, ids, top = draw(40, 32000, 64, torch.bfloat16, seed=6)
    ids[:, 1::2] = ids[:, ::2]
    args = (40, 32000, 64, z.to(DEV), ids.to(DEV), top.to(DEV), 1.0)
    outs = []
    for _ in range(3):
        loss, grad = torch.empty(40, device=DEV), torch.empty(40, 32000, dtype=torch.bfloat16, device=DEV)
        ctx.pv_distill_topk(*args, loss=loss, grad=grad)
        outs.append((loss, grad))
    for loss, grad in outs[1:]:
        assert torch.equal(loss, outs[0][0]) and torch.equal(grad, outs[0][1])
