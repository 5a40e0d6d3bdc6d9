"""Timing cases of the operators around a V step: microscaled quantisation, the product with 4-bit
weights and its gradients, RMS norm with the residual's addition, distillation from a teacher's top logits.

They are the parts of a fine-tuning step on weights that the matrix cores multiply as they are stored
(blocks of 32 values that share a power of two): the norm hands its output over in 8 bits, the product
takes it with 4-bit weights, the loss compares the logits with the teacher's, and the gradient of the
weights is what the V step's targets are formed from.

`run` computes them from their formulas in elementary torch operations, in 32 bits, or, with `own` set,
by the calls of `PVContext`.  Codes of 8 and 4 bits are returned as the values that they stand for, in
bfloat16, which holds them exactly.

Kinds of a case:
  quantize      a matrix to codes and scales, and the codes back to values
  product       Y = X W^T, tokens in 8 (or 4) bits with weights in 4
  grads         dX = dY W and dW = dY^T X of that product
  norm          h = x + r and its norm times a weight, in the input's type or in 8 bits with scales
  norm_back     gradients of the norm's input and weight
  distill       loss and gradient of the logits in one call
  distill_back  loss first, the gradient from a second call with the loss's own gradient
"""
import functools
import math

import torch

own = False

BLOCK = 32
EMAX = {"e2m1": 2, "e4m3": 8}
TOP = {"e2m1": 6.0, "e4m3": 448.0}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
SIGMA_W = 0.02


def listed():
    return [
        # a small weight matrix in 4 bits: launches and latency count
        _quantize("quantize_256x256_e2m1", 256, 256, "e2m1", "f32"),
        # activations in 8 bits, rows that end inside a block
        _quantize("quantize_1003x2077_e4m3", 1003, 2077, "e4m3", "bf16"),
        # the weights of a 14336-wide MLP after a step, in 4 bits
        _quantize("quantize_14336x4096_e2m1", 14336, 4096, "e2m1", "f32"),
        # one token through an MLP up projection: the weights' bytes count
        _product("product_1x4096x11008", 1, 4096, 11008, "e4m3", "bf16"),
        # a batch of a few sequences, both sides in 4 bits, a token count that fills no tile, a long sum
        _product("product_131x14336x4096_e2m1", 131, 14336, 4096, "e2m1", "f32"),
        # a full batch of tokens: the matrix cores' rate counts
        _product("product_4096x4096x11008", 4096, 4096, 11008, "e4m3", "bf16"),
        # backward of an attention projection
        {"name": "grads_2048x4096x4096", "kind": "grads", "tokens": 2048, "in": 4096, "out": 4096, "fmt": "e4m3"},
        # one token between two layers
        _norm("norm", "norm_1x4096_f16", 1, 4096, "f16", ""),
        # a batch of tokens, handed to the product in 8 bits
        _norm("norm", "norm_8192x4096_e4m3", 8192, 4096, "bf16", "e4m3"),
        # backward over rows that fill no tile
        _norm("norm_back", "norm_back_2047x11008", 2047, 11008, "bf16", ""),
        # the loss of a batch and the gradient of its logits, 64 teacher logits a token
        _distill("distill", "distill_2048x32000_k64", 2048, 32000, 64, "bf16", 1.0),
        # an odd vocabulary, logits in 32 bits, a softened teacher, the two directions apart
        _distill("distill_back", "distill_back_333x50257_k20", 333, 50257, 20, "f32", 2.0),
    ]


def _quantize(name, rows, cols, fmt, t):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "fmt": fmt, "type": t}


def _product(name, tokens, inn, out, fmt, t):
    return {"name": name, "kind": "product", "tokens": tokens, "in": inn, "out": out, "fmt": fmt, "type": t}


def _norm(kind, name, rows, cols, t, fmt):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "type": t, "fmt": fmt}


def _distill(kind, name, rows, vocab, k, t, temperature):
    return {"name": name, "kind": kind, "rows": rows, "vocab": vocab, "k": k, "type": t, "temperature": temperature}


# the most that a drawn case of a kind costs: the largest that is listed of it
MOST = {"quantize": 14336 * 4096, "product": 4096 * 4096 * 11008, "grads": 2048 * 4096 * 4096,
        "norm": 8192 * 4096, "norm_back": 2047 * 11008, "distill": 2048 * 32000, "distill_back": 333 * 50257}


def draw(rng):
    """One more case of these ranges: matrices and layers of 256 .. 14336 a side, batches of 1 .. 8192
    tokens, vocabularies of 1000 .. 131072 with 1 .. 256 teacher logits."""
    spread = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))  # noqa: E731
    kind = rng.choice(sorted(MOST) + ["product"])
    while True:
        c = {"kind": kind}
        if kind == "quantize":
            c.update(rows=spread(1, 14336), cols=spread(32, 14336), fmt=rng.choice(("e2m1", "e4m3")), type=rng.choice(sorted(TYPES)))
            cost = c["rows"] * c["cols"]
        elif kind in ("product", "grads"):
            inn = spread(256, 14336)
            c.update(tokens=spread(1, 4096), out=spread(256, 14336), fmt=rng.choice(("e4m3", "e4m3", "e2m1")))
            c["in"] = inn if rng.random() < 0.3 else -(-inn // 128) * 128
            if kind == "product":
                c["type"] = rng.choice(("bf16", "bf16", "f16", "f32"))
            cost = c["tokens"] * c["in"] * c["out"]
        elif kind in ("norm", "norm_back"):
            cols = spread(256, 14336)
            c.update(rows=spread(1, 8192), cols=cols if rng.random() < 0.3 else -(-cols // 64) * 64, type=rng.choice(sorted(TYPES)))
            c["fmt"] = rng.choice(("", "e4m3")) if kind == "norm" else ""
            cost = c["rows"] * c["cols"]
        else:
            c.update(rows=spread(1, 4096), vocab=spread(1000, 131072), k=spread(1, 256), type=rng.choice(sorted(TYPES)),
                     temperature=rng.choice((1.0, 1.0, 2.0, 4.0)))
            cost = c["rows"] * c["vocab"]
        if cost <= MOST[kind]:
            return c


# ---- the formats: 32 consecutive values of a row share a power of two -------------------------------

def _padded(cols):
    return -(-cols // BLOCK) * BLOCK


def _code_bytes(cols, fmt):
    return _padded(cols) // (2 if fmt == "e2m1" else 1)


def _encode(x, fmt):
    """Codes (rows of whole blocks) and scale bytes of a float32 matrix of finite values."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, _padded(cols) - cols)).view(rows, -1, BLOCK)
    scale = ((x.abs().amax(2).view(torch.int32) >> 23) - EMAX[fmt]).clamp(min=0)   # the exponent's bits: floor(log2)
    v = x * ((254 - scale) << 23).view(torch.float32)[:, :, None]
    v = v.clamp(-TOP[fmt], TOP[fmt]).reshape(rows, -1)
    if fmt == "e4m3":
        return v.to(torch.float8_e4m3fn).view(torch.uint8), scale.to(torch.uint8)
    a = v.abs()
    # ties go to the even code: 0 | .5 | 1 | 1.5 | 2 | 3 | 4 | 6
    c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    c = c + torch.signbit(v).to(torch.uint8) * 8
    return c[:, 0::2] + c[:, 1::2] * 16, scale.to(torch.uint8)


def _decode(codes, scales, fmt, cols):
    """float32 values of codes."""
    if fmt == "e4m3":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
        c = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1)
        v = table[(c & 7).int()] * (1.0 - 2.0 * (c >> 3))
    e = scales.int()
    s = torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)        # 2^(e - 127)
    return (v.view(codes.shape[0], -1, BLOCK) * s[:, :, None]).view(codes.shape[0], -1)[:, :cols]


# ---- inputs ----------------------------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    kind = case["kind"]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device=dev)  # noqa: E731
    empty = lambda *shape, t=torch.float32: torch.empty(*shape, dtype=t, device=dev)  # noqa: E731
    s = dict(case)
    if kind == "quantize":
        r, c, t = case["rows"], case["cols"], TYPES[case["type"]]
        # weights, or activations with a few large channels
        x = normal(r, c) * (SIGMA_W if case["fmt"] == "e2m1" else 1.0)
        if case["fmt"] == "e4m3":
            x = x * torch.exp(0.5 * normal(c)) * (1.0 + 20.0 * (uniform(c) < 0.002))
        s.update(x=x.to(t), codes=empty(r, _code_bytes(c, case["fmt"]), t=torch.uint8),
                 scales=empty(r, _padded(c) // BLOCK, t=torch.uint8), values=empty(r, c, t=torch.bfloat16))
    elif kind in ("product", "grads"):
        n, i, o, fmt = case["tokens"], case["in"], case["out"], case["fmt"]
        s["x_codes"], s["x_scales"] = _encode(normal(n, i), fmt)
        s["w_codes"], s["w_scales"] = _encode(normal(o, i) * SIGMA_W, "e2m1")
        if kind == "product":
            s["y"] = empty(n, o, t=TYPES[case["type"]])
        else:
            s.update(dy=(normal(n, o) * 1e-3).to(torch.bfloat16), dx=empty(n, i, t=torch.bfloat16), dw=empty(o, i))
    elif kind in ("norm", "norm_back"):
        r, c, t = case["rows"], case["cols"], TYPES[case["type"]]
        s.update(weight=1.0 + 0.2 * normal(c), rstd=empty(r), h=empty(r, c, t=t))
        if kind == "norm":
            s.update(x=normal(r, c).to(t), residual=(normal(r, c) * 2.0).to(t))
            if case["fmt"]:
                s.update(codes=empty(r, _code_bytes(c, case["fmt"]), t=torch.uint8),
                         scales=empty(r, _padded(c) // BLOCK, t=torch.uint8), values=empty(r, c, t=torch.bfloat16))
            else:
                s["y"] = empty(r, c, t=t)
        else:
            s["h"] = (normal(r, c) * 2.0).to(t)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
            s.update(dy=normal(r, c).to(t), dh=normal(r, c).to(t), dx=empty(r, c, t=t), dweight=empty(c))
    else:
        r, v, k, t = case["rows"], case["vocab"], case["k"], TYPES[case["type"]]
        # a student near its teacher: logits of a peaked distribution, and the same with noise
        z = normal(r, v) * 2.5
        top, ids = torch.topk(z + 0.5 * normal(r, v), min(k, v), 1)
        s.update(logits=z.to(t), ids=ids.int(), top=top.contiguous(), loss=empty(r), lse=empty(r), grad=empty(r, v, t=t))
        # a padded batch, summed: one row in eight has no weight
        s["row_weight"] = (uniform(r) >= 0.125).float()
        s["grad_loss"] = s["row_weight"] * (0.5 + uniform(r))
    return s


# ---- one pass --------------------------------------------------------------------------------------

@functools.cache
def _context():
    from paper_2405_14852_amd import PVContext
    return PVContext(0)


def run(s):
    return (_call if own else _plain)(s)


def _call(s):
    ctx, kind = _context(), s["kind"]
    if kind == "quantize":
        ctx.pv_quantize_mx(s["rows"], s["cols"], s["fmt"], s["x"], s["codes"], s["scales"])
        ctx.pv_dequantize_mx(s["rows"], s["cols"], s["fmt"], s["codes"], s["scales"], s["values"])
        return {"values": s["values"]}
    if kind == "product":
        ctx.pv_mx_product(s["tokens"], s["out"], s["in"], s["fmt"], s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["y"])
        return {"y": s["y"]}
    if kind == "grads":
        ctx.pv_mx_product_grads(s["tokens"], s["out"], s["in"], s["fmt"], s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"],
                                s["dy"], s["dx"], s["dw"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if kind == "norm":
        if not s["fmt"]:
            ctx.pv_rms_norm(s["rows"], s["cols"], s["x"], s["residual"], s["weight"], EPS, h=s["h"], y=s["y"], rstd=s["rstd"])
            return {"h": s["h"], "y": s["y"], "rstd": s["rstd"]}
        ctx.pv_rms_norm(s["rows"], s["cols"], s["x"], s["residual"], s["weight"], EPS, h=s["h"], fmt=s["fmt"], codes=s["codes"],
                        scales=s["scales"], rstd=s["rstd"])
        ctx.pv_dequantize_mx(s["rows"], s["cols"], s["fmt"], s["codes"], s["scales"], s["values"])
        return {"h": s["h"], "y": s["values"], "rstd": s["rstd"]}
    if kind == "norm_back":
        ctx.pv_rms_norm_backward(s["rows"], s["cols"], s["dy"], s["dh"], s["h"], s["weight"], s["rstd"], s["dx"], s["dweight"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    args = (s["rows"], s["vocab"], s["ids"].shape[1], s["logits"], s["ids"], s["top"], s["temperature"])
    if kind == "distill":
        ctx.pv_distill_topk(*args, row_weight=s["row_weight"], loss=s["loss"], grad=s["grad"])
    else:
        ctx.pv_distill_topk(*args, loss=s["loss"], lse=s["lse"])
        ctx.pv_distill_topk_backward(*args, s["lse"], s["grad_loss"], s["grad"])
    return {"loss": s["loss"], "grad": s["grad"]}


def _plain(s):
    kind = s["kind"]
    if kind == "quantize":
        return {"values": _decode(*_encode(s["x"].float(), s["fmt"]), s["fmt"], s["cols"]).to(torch.bfloat16)}
    if kind in ("product", "grads"):
        x = _decode(s["x_codes"], s["x_scales"], s["fmt"], s["in"])
        w = _decode(s["w_codes"], s["w_scales"], "e2m1", s["in"])
        if kind == "product":
            return {"y": (x @ w.T).to(s["y"].dtype)}
        dy = s["dy"].float()
        return {"dx": (dy @ w).to(torch.bfloat16), "dw": dy.T @ x}
    if kind == "norm":
        h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
        rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
        y = h.float() * rstd[:, None] * s["weight"]
        y = _decode(*_encode(y, s["fmt"]), s["fmt"], s["cols"]).to(torch.bfloat16) if s["fmt"] else y.to(h.dtype)
        return {"h": h, "y": y, "rstd": rstd}
    if kind == "norm_back":
        dy, n = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = s["dh"].float() + s["rstd"][:, None] * (g - n * (g * n).mean(1, keepdim=True))
        return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * n).sum(0)}
    t = s["temperature"]
    z, u, ids = s["logits"].float() / t, s["top"] / t, s["ids"].long()
    log_q = z - z.amax(1, keepdim=True)
    log_q = log_q - torch.log(torch.exp(log_q).sum(1, keepdim=True))
    log_p = u - u.amax(1, keepdim=True)
    log_p = log_p - torch.log(torch.exp(log_p).sum(1, keepdim=True))
    p = torch.exp(log_p)
    kl = t * t * (p * (log_p - log_q.gather(1, ids))).sum(1)
    grad = torch.exp(log_q).scatter_add_(1, ids, -p)
    if kind == "distill":
        return {"loss": s["row_weight"] * kl, "grad": (grad * (t * s["row_weight"])[:, None]).to(s["logits"].dtype)}
    return {"loss": kl, "grad": (grad * (t * s["grad_loss"])[:, None]).to(s["logits"].dtype)}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    """Every input read once, every output written once; the multiply-adds of the definition."""
    kind = case["kind"]
    coded = lambda r, c, fmt: r * _code_bytes(c, fmt) + r * _padded(c) / BLOCK  # noqa: E731
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": float(SIZE[case["type"]] * n + coded(case["rows"], case["cols"], case["fmt"]) + 2 * n), "flops": 4.0 * n}
    if kind in ("product", "grads"):
        n, i, o = case["tokens"], case["in"], case["out"]
        b = coded(n, i, case["fmt"]) + coded(o, i, "e2m1")
        if kind == "product":
            return {"bytes": float(b + SIZE[case["type"]] * n * o), "flops": 2.0 * n * i * o}
        return {"bytes": float(b + 2 * n * o + 2 * n * i + 4 * o * i), "flops": 4.0 * n * i * o}
    if kind == "norm":
        n, t = case["rows"] * case["cols"], SIZE[case["type"]]
        y = coded(case["rows"], case["cols"], case["fmt"]) + 2 * n if case["fmt"] else t * n
        return {"bytes": float(3 * t * n + y + 4 * case["cols"] + 4 * case["rows"]), "flops": 5.0 * n}
    if kind == "norm_back":
        n, t = case["rows"] * case["cols"], SIZE[case["type"]]
        return {"bytes": float(4 * t * n + 8 * case["cols"] + 4 * case["rows"]), "flops": 10.0 * n}
    n, t = case["rows"] * case["vocab"], SIZE[case["type"]]
    return {"bytes": float(2 * t * n + 8 * case["rows"] * case["k"] + 12 * case["rows"]), "flops": 6.0 * n}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _power(e):
    """2^e in float64, from the bits of the exponent."""
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def _exact_values(codes, scales, fmt, cols):
    """Values of codes from their bits: sign, exponent, mantissa."""
    c = codes.to(torch.int64)
    if fmt == "e2m1":
        c = torch.stack((c % 16, c // 16), 2).flatten(1)
    m, bias, top = (1, 1, 4) if fmt == "e2m1" else (3, 7, 16)
    sign, e, f = 1 - 2 * (c // (top << m)), c // (1 << m) % top, c % (1 << m)
    v = sign * torch.where(e > 0, f + (1 << m), f) * _power(e.clamp(min=1) - bias - m)
    s = _power(scales.to(torch.int64) - 127)
    return (v * s.repeat_interleave(BLOCK, 1))[:, :cols]


def _exact_quantized(x, fmt):
    """The nearest value of the format to each element, ties to even, under the block's power of two."""
    rows, cols = x.shape
    m, low = (1, 0) if fmt == "e2m1" else (3, -6)
    x = torch.cat((x, x.new_zeros(rows, _padded(cols) - cols)), 1)
    largest = x.abs().unflatten(1, (-1, BLOCK)).max(2).values
    e = torch.where(largest > 0, torch.frexp(largest).exponent - 1 - EMAX[fmt], -127).clamp(-127, 127)
    s = _power(e).repeat_interleave(BLOCK, 1)
    v = x / s
    step = _power((torch.frexp(v).exponent - 1).clamp(min=low) - m)
    v = (torch.round(v / step) * step).clamp(-TOP[fmt], TOP[fmt])
    return (v * s)[:, :cols]


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "quantize":
        return {"values": _exact_quantized(s["x"].double(), s["fmt"])}
    if kind in ("product", "grads"):
        x = _exact_values(s["x_codes"], s["x_scales"], s["fmt"], s["in"])
        w = _exact_values(s["w_codes"], s["w_scales"], "e2m1", s["in"])
        if kind == "product":
            return {"y": torch.matmul(x, w.t())}
        dy = s["dy"].double()
        return {"dx": torch.matmul(dy, w), "dw": torch.matmul(dy.t(), x)}
    if kind == "norm":
        total = s["x"].double() + s["residual"].double()
        h = total.to(s["x"].dtype).double()            # the stored sum is what is normed
        rstd = 1.0 / torch.sqrt(torch.sum(h * h, 1) / s["cols"] + EPS)
        y = h * rstd.unsqueeze(1) * s["weight"].double()
        return {"h": total, "y": _exact_quantized(y, s["fmt"]) if s["fmt"] else y, "rstd": rstd}
    if kind == "norm_back":
        dy, h, r, w = s["dy"].double(), s["h"].double(), s["rstd"].double().unsqueeze(1), s["weight"].double()
        along = torch.sum(dy * w * h, 1, keepdim=True)
        return {"dx": s["dh"].double() + r * dy * w - r.pow(3) * h * along / s["cols"], "dweight": torch.sum(dy * h * r, 0)}
    t = case["temperature"]
    z, u, ids = s["logits"].double(), s["top"].double(), s["ids"].long()
    q, p = torch.softmax(z / t, 1), torch.softmax(u / t, 1)
    kl = torch.sum(p * (u / t - torch.logsumexp(u / t, 1, keepdim=True)), 1)
    kl = kl - torch.sum(p * (torch.gather(z, 1, ids) / t), 1) + torch.logsumexp(z / t, 1)
    target = torch.zeros_like(q).scatter_add(1, ids, p)
    c = s["row_weight"] if kind == "distill" else s["grad_loss"]
    loss = t * t * kl * (c.double() if kind == "distill" else 1.0)
    return {"loss": loss, "grad": t * c.double().unsqueeze(1) * (q - target)}
