"""The operators around the V step as a fine-tuning step uses them, one after the other: norm -> 8-bit operand -> product with
4-bit weights -> distillation -> gradients of the product and of the norm -> targets -> 4-bit weights again.  Eager, captured and
replayed, on other streams, side by side."""
import pytest
import torch

import ops_reference as ref
from paper_2405_14852_amd import Layout, PVContext, PVError, mx_shapes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS, ALPHA, T = 1e-5, 0.5, 2.0


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


class Step:
    """One step on one layer and its loss: the buffers that a program keeps."""

    def __init__(self, ctx, tokens, width, vocab, k, seed):
        self.ctx, self.n, self.i, self.v, self.k = ctx, tokens, width, vocab, k
        dev = lambda t: t.to(DEV)  # noqa: E731
        e = lambda *s, t=torch.float32: torch.full(s, 7, dtype=t, device=DEV)  # noqa: E731
        self.draw(seed)
        self.norm_w = dev(1 + 0.1 * torch.randn(width, generator=gen(seed + 1)))
        self.w0 = dev(0.05 * torch.randn(vocab, width, generator=gen(seed + 2)))
        self.wc, self.ws = (e(*s, t=torch.uint8) for s in mx_shapes(vocab, width, "e2m1"))
        self.nc, self.ns = (e(*s, t=torch.uint8) for s in mx_shapes(vocab, width, "e2m1"))
        self.xc, self.xs = (e(*s, t=torch.uint8) for s in mx_shapes(tokens, width, "e4m3"))
        self.h, self.dx = e(tokens, width, t=torch.bfloat16), e(tokens, width, t=torch.bfloat16)
        self.dy, self.dh = e(tokens, width, t=torch.bfloat16), e(tokens, width, t=torch.bfloat16)
        self.rstd, self.dnorm = e(tokens), e(width)
        self.logits, self.grad = e(tokens, vocab, t=torch.bfloat16), e(tokens, vocab, t=torch.bfloat16)
        self.loss, self.dw, self.w, self.t = e(tokens), e(vocab, width), e(vocab, width), e(vocab, width)
        self.row_weight = dev((torch.arange(tokens) % 5 != 0).float())
        self.lay = Layout(vocab, width, 1, 1, 8)

    def draw(self, seed):
        """Other inputs, in place where there are some."""
        g = gen(seed)
        z = torch.randn(self.n, self.v, generator=g)
        top, ids = torch.topk(z, self.k, 1)
        new = {"x": torch.randn(self.n, self.i, generator=g).to(torch.bfloat16), "r": torch.randn(self.n, self.i, generator=g).to(torch.bfloat16),
               "up": (0.01 * torch.randn(self.n, self.i, generator=g)).to(torch.bfloat16), "ids": ids.int(), "top": top.contiguous()}
        for name, t in new.items():
            if hasattr(self, name):
                getattr(self, name).copy_(t)
            else:
                setattr(self, name, t.to(DEV))

    def run(self):
        c, n, i, v, k = self.ctx, self.n, self.i, self.v, self.k
        c.pv_quantize_mx(v, i, "e2m1", self.w0, self.wc, self.ws)
        c.pv_rms_norm(n, i, self.x, self.r, self.norm_w, EPS, h=self.h, fmt="e4m3", codes=self.xc, scales=self.xs, rstd=self.rstd)
        c.pv_mx_product(n, v, i, "e4m3", self.xc, self.xs, self.wc, self.ws, self.logits)
        c.pv_distill_topk(n, v, k, self.logits, self.ids, self.top, T, row_weight=self.row_weight, loss=self.loss, grad=self.grad)
        c.pv_mx_product_grads(n, v, i, "e4m3", self.xc, self.xs, self.wc, self.ws, self.grad, self.dy, self.dw)
        c.pv_rms_norm_backward(n, i, self.dy, self.up, self.h, self.norm_w, self.rstd, self.dx, self.dnorm)
        c.pv_dequantize_mx(v, i, "e2m1", self.wc, self.ws, self.w)
        c.pv_encode_targets(self.lay, self.w, self.dw, ALPHA, self.t)
        c.pv_quantize_mx(v, i, "e2m1", self.t, self.nc, self.ns)

    def outputs(self):
        return {name: getattr(self, name).clone() for name in
                ("wc", "ws", "xc", "xs", "h", "rstd", "logits", "loss", "grad", "dy", "dw", "dx", "dnorm", "w", "t", "nc", "ns")}


def same(a, b):
    assert a.keys() == b.keys()
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.fixture
def ctx():
    c = PVContext(0)
    yield c
    c.close()


@pytest.mark.parametrize("tokens,width,vocab,k", [(1, 64, 100, 5), (37, 96, 300, 16), (150, 264, 1000, 64)])
def test_a_step(ctx, tokens, width, vocab, k):
    """Every call's results from its own inputs, which are what the call before it left."""
    s = Step(ctx, tokens, width, vocab, k, seed=tokens)
    s.run()
    torch.cuda.synchronize()
    assert torch.equal(s.wc.cpu(), ref.quantize(s.w0, "e2m1")[0])
    h, rstd, y = ref.rms_norm(s.x, s.r, s.norm_w, EPS, torch.bfloat16)
    assert torch.equal(s.h.cpu().double(), h)
    x, w = ref.decode(s.xc, s.xs, "e4m3", width), ref.decode(s.wc, s.ws, "e2m1", width)
    # the 8-bit operand is y to half a step of its format: 2^-4 of a value, or of what is 2^-6 of the block's power of two and below
    # (values above the largest code, at most an eighth larger, become it)
    power = torch.exp2((s.xs.cpu().long() - 127).double()).repeat_interleave(32, 1)[:, :width]
    assert ((x - y).abs() <= torch.maximum(y.abs() * (2.0 ** -3 + 1e-6), power * 2.0 ** -10)).all()
    far = lambda got, want, bound: float((got.cpu().double() - want).norm()) <= bound * float(want.norm())  # noqa: E731
    assert far(s.logits, x @ w.T, 2.0 ** -8)
    loss, _, grad = ref.distill(s.logits, s.ids, s.top, T, s.row_weight)
    assert far(s.loss, loss, 1e-5) and far(s.grad, grad, 2.0 ** -8)
    g = s.grad.cpu().double()
    assert far(s.dy, g @ w, 2.0 ** -8) and far(s.dw, g.T @ x, 1e-5)
    dx, dn = ref.rms_norm_backward(s.dy, s.up, s.h, s.norm_w, s.rstd)
    assert far(s.dx, dx, 2.0 ** -8) and far(s.dnorm, dn, 1e-5)
    assert torch.equal(s.w.cpu().double(), w)
    codes, scales = ref.quantize(s.t, "e2m1")
    assert torch.equal(s.nc.cpu(), codes) and torch.equal(s.ns.cpu(), scales)
    assert far(s.t, w - ALPHA * s.dw.cpu().double(), 2.0 ** -23)


def test_a_captured_step_replays_on_new_inputs():
    side = torch.cuda.Stream(device=DEV)
    ctx = PVContext(0, stream=side)
    s, want = Step(ctx, 300, 512, 1500, 20, seed=1), {}
    torch.cuda.synchronize()
    for seed in (1, 2, 3):
        s.draw(seed)
        torch.cuda.synchronize()
        s.run()
        torch.cuda.synchronize()
        want[seed] = s.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for seed in (2, 3, 1, 2):
        s.draw(seed)
        for t in (s.logits, s.dw, s.dnorm, s.nc):
            t.fill_(3)                                   # a program's own work between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(s.outputs(), want[seed])
        s.run()                                          # and an eager step of the same context
        torch.cuda.synchronize()
        same(s.outputs(), want[seed])
    ctx.close()


def test_a_first_call_that_needs_scratch_is_refused_during_a_capture():
    side = torch.cuda.Stream(device=DEV)
    ctx = PVContext(0, stream=side)
    s = Step(ctx, 64, 128, 256, 8, seed=4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.pv_quantize_mx(s.v, s.i, "e2m1", s.w0, s.wc, s.ws)
        with pytest.raises(PVError) as error:
            ctx.pv_mx_product_grads(s.n, s.v, s.i, "e4m3", s.xc, s.xs, s.wc, s.ws, s.grad, s.dy, s.dw)
    assert error.value.status == 4 and "capture" in str(error.value)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.wc.cpu(), ref.quantize(s.w0, "e2m1")[0])
    s.run()
    torch.cuda.synchronize()
    ctx.close()


def test_a_graph_keeps_its_scratch_when_a_larger_call_needs_more():
    side = torch.cuda.Stream(device=DEV)
    ctx = PVContext(0, stream=side)
    small, large = Step(ctx, 40, 64, 200, 4, seed=5), Step(ctx, 600, 1024, 3000, 4, seed=6)
    torch.cuda.synchronize()
    small.run()
    torch.cuda.synchronize()
    want = small.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        small.run()
    for _ in range(3):
        large.run()
        torch.cuda.synchronize()
        large_out = large.outputs()
        filler = torch.full((1 << 22,), 1e30, device=DEV)         # what a freed block would be used for
        small.dw.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(small.outputs(), want)
        same(large.outputs(), large_out)
        del filler
    ctx.close()


def test_contexts_on_two_streams_side_by_side():
    streams = [torch.cuda.Stream(device=DEV) for _ in range(2)]
    steps = [Step(PVContext(0, stream=st), 200 + 50 * j, 512, 1200, 16, seed=7 + j) for j, st in enumerate(streams)]
    torch.cuda.synchronize()
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
    for _ in range(4):
        for s in steps:
            s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        same(s.outputs(), w)
        s.ctx.close()


def test_a_tensor_of_another_shape_type_or_order_is_refused(ctx):
    s = Step(ctx, 8, 64, 100, 4, seed=9)
    bad = [lambda: ctx.pv_quantize_mx(100, 64, "e2m1", s.w0.T.contiguous().T, s.wc, s.ws),
           lambda: ctx.pv_quantize_mx(100, 64, "e2m1", s.w0, s.wc[:, :-1].contiguous(), s.ws),
           lambda: ctx.pv_quantize_mx(100, 64, "e4m3", s.w0, s.wc, s.ws),
           lambda: ctx.pv_mx_product(8, 100, 64, "e4m3", s.xc, s.xs, s.wc, s.ws, s.logits.double()),
           lambda: ctx.pv_mx_product(8, 100, 64, "e4m3", s.xc, s.xs, s.wc, s.ws.int(), s.logits),
           lambda: ctx.pv_mx_product_grads(8, 100, 64, "e4m3", s.xc, s.xs, s.wc, s.ws, s.grad.float(), s.dy, s.dw),
           lambda: ctx.pv_mx_product_grads(8, 100, 64, "e4m3", None, None, s.wc, s.ws, s.grad, s.dy, s.dw),
           lambda: ctx.pv_rms_norm(8, 64, s.x, s.r.float(), s.norm_w, EPS, h=s.h),
           lambda: ctx.pv_rms_norm(8, 64, s.x, s.r, s.norm_w[:-1], EPS, h=s.h),
           lambda: ctx.pv_distill_topk(8, 100, 4, s.logits, s.ids.long(), s.top, T, loss=s.loss),
           lambda: ctx.pv_distill_topk(8, 100, 4, s.logits, s.ids, s.top, T, loss=s.loss[:-1]),
           lambda: ctx.pv_distill_topk(8, 100, 4, s.logits.T.contiguous().T, s.ids, s.top, T, loss=s.loss),
           lambda: ctx.pv_distill_topk(8, 100, 4, s.logits[:1].expand(8, 100), s.ids, s.top, T, loss=s.loss),
           lambda: ctx.pv_distill_topk(8, 100, 4, s.logits, s.ids, s.top.cpu(), T, loss=s.loss)]
    for call in bad:
        with pytest.raises((TypeError, ValueError)):
            call()
