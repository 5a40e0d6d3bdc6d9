"""ctypes binding of libpv.so: same names as the C ABI, no arithmetic here.

Tensors are torch CUDA tensors (PyTorch is used for device memory and streams
only).  The library must have been built (see __graft_entry__.build); a missing
library is an error, there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from functools import cached_property, lru_cache
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
_LIB_PATH = _PKG / "libpv.so"
_lib = None

KERNEL_IDS = {
    "encode_targets": 0, "group_scores": 1, "select": 2, "prep": 3, "score_mfma": 4,
    "rerank": 5, "exact_scan": 6, "beam": 7, "dequantize": 8, "trust_ratio": 9, "pstep": 10, "stochastic": 13,
    "probe_copy": 11, "probe_mfma": 12,
    "mx_convert": 14, "mx_product": 15, "rms_norm": 16, "distill": 17,
}

# pv_mx_format and pv_dtype
MX_FORMATS = {"e2m1": 0, "e4m3": 1}
MX_BLOCK = 32
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class PVError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"pv status {status}: {text}")
        self.status = status


class _CLayout(ctypes.Structure):
    _fields_ = [("out_features", ctypes.c_int64), ("in_features", ctypes.c_int64),
                ("group_size", ctypes.c_int32), ("num_codebooks", ctypes.c_int32),
                ("nbits", ctypes.c_int32)]


@dataclass(frozen=True)
class Layout:
    out_features: int
    in_features: int
    group_size: int
    num_codebooks: int
    nbits: int

    @cached_property
    def _c(self) -> _CLayout:
        return _CLayout(self.out_features, self.in_features, self.group_size,
                        self.num_codebooks, self.nbits)

    def c(self) -> _CLayout:
        return self._c          # the library only reads it

    @property
    def num_groups(self) -> int:
        return self.out_features * (self.in_features // self.group_size)


def library_path() -> Path:
    return _LIB_PATH


def load_library():
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(str(_LIB_PATH))
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    lp = ctypes.POINTER(_CLayout)
    lib.pv_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, vp]
    lib.pv_destroy.argtypes = [vp]
    lib.pv_destroy.restype = None
    lib.pv_last_error.argtypes = [vp]
    lib.pv_last_error.restype = ctypes.c_char_p
    lib.pv_encode_targets.argtypes = [vp, lp, vp, vp, f32, vp]
    lib.pv_encode_targets_adam.argtypes = [vp, lp, vp, vp, vp, vp, i64, f32, f32, f32, f32, vp]
    lib.pv_select_topk_groups.argtypes = [vp, lp, vp, vp, i64, vp, vp]
    lib.pv_select_topk_groups_noalloc.argtypes = [vp, lp, vp, vp, i64, vp, vp]
    lib.pv_encode_targets_adam_select.argtypes = [vp, lp, vp, vp, vp, vp, i64, f32, f32, f32, f32, vp,
                                                  i64, vp, vp]
    lib.pv_encode_targets_select.argtypes = [vp, lp, vp, vp, f32, vp, i64, vp, vp]
    lib.pv_reencode_groups.argtypes = [vp, lp, vp, vp, vp, vp, i64, i32, vp, vp]
    lib.pv_reencode_groups_stochastic.argtypes = [vp, lp, vp, vp, vp, vp, i64, i32, ctypes.c_uint64, vp, vp]
    lib.pv_dequantize.argtypes = [vp, lp, vp, vp, vp, vp]
    lib.pv_dequantize_groups.argtypes = [vp, lp, vp, vp, vp, vp, i64, vp]
    lib.pv_codebook_grads.argtypes = [vp, lp, vp, vp, vp, vp, vp, vp]
    lib.pv_dequantize_scalar.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.pv_reencode_scalar.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp, i64, vp, vp]
    lib.pv_reencode_trust_ratio.argtypes = [vp, lp, vp, vp, vp, vp, i64, i64, ctypes.c_double, i32,
                                            vp, vp, vp, vp]
    lib.pv_set_search_mode.argtypes = [vp, ctypes.c_int]
    lib.pv_timing_enable.argtypes = [vp, ctypes.c_int]
    lib.pv_timing_reset.argtypes = [vp]
    lib.pv_timing_read.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(i64)]
    lib.pv_reencode_stats.argtypes = [vp, ctypes.POINTER(i64)]
    lib.pv_probe_copy.argtypes = [vp, vp, vp, i64]
    lib.pv_probe_mfma_f16.argtypes = [vp, i64, vp, ctypes.POINTER(i64)]
    lib.pv_quantize_mx.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp]
    lib.pv_dequantize_mx.argtypes = [vp, i64, i64, i32, vp, vp, i32, vp]
    lib.pv_mx_product.argtypes = [vp, i64, i64, i64, i32, vp, vp, vp, vp, i32, vp]
    lib.pv_mx_product_grads.argtypes = [vp, i64, i64, i64, i32, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.pv_rms_norm.argtypes = [vp, i64, i64, i32, vp, vp, vp, f32, vp, vp, i32, vp, vp, vp]
    lib.pv_rms_norm_backward.argtypes = [vp, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.pv_distill_topk.argtypes = [vp, i64, i64, i32, i32, vp, i64, vp, vp, f32, vp, vp, vp, vp, i64]
    lib.pv_distill_topk_backward.argtypes = [vp, i64, i64, i32, i32, vp, i64, vp, vp, f32, vp, vp, vp, i64]
    for name in ("pv_create", "pv_select_topk_groups_noalloc", "pv_encode_targets", "pv_encode_targets_adam", "pv_select_topk_groups",
                 "pv_encode_targets_adam_select",
                 "pv_encode_targets_select", "pv_reencode_groups", "pv_reencode_groups_stochastic",
                 "pv_reencode_trust_ratio",
                 "pv_codebook_grads", "pv_dequantize_scalar", "pv_reencode_scalar",
                 "pv_dequantize_groups",
                 "pv_dequantize", "pv_set_search_mode", "pv_timing_enable", "pv_timing_reset",
                 "pv_timing_read", "pv_reencode_stats", "pv_probe_copy", "pv_probe_mfma_f16",
                 "pv_quantize_mx", "pv_dequantize_mx", "pv_mx_product", "pv_mx_product_grads",
                 "pv_rms_norm", "pv_rms_norm_backward", "pv_distill_topk", "pv_distill_topk_backward"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _dev_ptr(t, dtype, what: str, allow_none: bool = False):
    if t is None:
        if allow_none:
            return None
        raise TypeError(f"{what} is None")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous")
    return t.data_ptr()


def _mx_format(fmt) -> int:
    if fmt not in MX_FORMATS:
        raise ValueError(f"format must be one of {sorted(MX_FORMATS)}, got {fmt!r}")
    return MX_FORMATS[fmt]


@lru_cache(maxsize=1024)
def mx_shapes(rows: int, cols: int, fmt: str):
    """Shapes of the codes and the scales (both uint8) of a [rows, cols] matrix."""
    nblk = -(-cols // MX_BLOCK)
    return (rows, nblk * (MX_BLOCK // 2 if _mx_format(fmt) == 0 else MX_BLOCK)), (rows, nblk)


class PVContext:
    """One library context bound to a device and a stream (default: torch's current stream)."""

    def __init__(self, device: int = 0, stream: "torch.cuda.Stream | None" = None):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.device = device
        with torch.cuda.device(device):
            s = stream if stream is not None else torch.cuda.current_stream(device)
        self.stream = s
        st = self._lib.pv_create(ctypes.byref(self._h), device, ctypes.c_void_p(s.cuda_stream))
        if st != 0:
            raise PVError(st, "pv_create failed")

    def close(self):
        if self._h:
            self._lib.pv_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st:
            raise PVError(st, self._lib.pv_last_error(self._h).decode())

    # ---- the four calls of the path -------------------------------------
    def pv_encode_targets(self, layout: Layout, W, G, alpha: float, T):
        lay = layout.c()
        self._check(self._lib.pv_encode_targets(
            self._h, ctypes.byref(lay), _dev_ptr(W, torch.float32, "W"),
            _dev_ptr(G, torch.float32, "G"), float(alpha), _dev_ptr(T, torch.float32, "T")))

    def pv_encode_targets_adam(self, layout: Layout, W, G, m, v, step: int, lr: float,
                               beta1: float, beta2: float, eps: float, T):
        lay = layout.c()
        self._check(self._lib.pv_encode_targets_adam(
            self._h, ctypes.byref(lay), _dev_ptr(W, torch.float32, "W"),
            _dev_ptr(G, torch.float32, "G"), _dev_ptr(m, torch.float32, "m"),
            _dev_ptr(v, torch.float32, "v"), int(step), float(lr), float(beta1), float(beta2),
            float(eps), _dev_ptr(T, torch.float32, "T")))

    def pv_encode_targets_adam_select(self, layout: Layout, W, G, m, v, step: int, lr: float,
                                      beta1: float, beta2: float, eps: float, T, k: int, out_idx,
                                      group_scores=None):
        lay = layout.c()
        self._check(self._lib.pv_encode_targets_adam_select(
            self._h, ctypes.byref(lay), _dev_ptr(W, torch.float32, "W"),
            _dev_ptr(G, torch.float32, "G"), _dev_ptr(m, torch.float32, "m"),
            _dev_ptr(v, torch.float32, "v"), int(step), float(lr), float(beta1), float(beta2),
            float(eps), _dev_ptr(T, torch.float32, "T"), int(k),
            _dev_ptr(out_idx, torch.int32, "out_idx", allow_none=(k == 0)),
            _dev_ptr(group_scores, torch.float32, "group_scores", allow_none=True)))

    def pv_select_topk_groups(self, layout: Layout, T, W, k: int, out_idx, group_scores=None):
        lay = layout.c()
        self._check(self._lib.pv_select_topk_groups(
            self._h, ctypes.byref(lay), _dev_ptr(T, torch.float32, "T"),
            _dev_ptr(W, torch.float32, "W"), int(k),
            _dev_ptr(out_idx, torch.int32, "out_idx", allow_none=(k == 0)),
            _dev_ptr(group_scores, torch.float32, "group_scores", allow_none=True)))

    def pv_select_topk_groups_noalloc(self, layout: Layout, T, W, k: int, out_idx, group_scores=None):
        lay = layout.c()
        self._check(self._lib.pv_select_topk_groups_noalloc(
            self._h, ctypes.byref(lay), _dev_ptr(T, torch.float32, "T"),
            _dev_ptr(W, torch.float32, "W"), int(k),
            _dev_ptr(out_idx, torch.int32, "out_idx", allow_none=(k == 0)),
            _dev_ptr(group_scores, torch.float32, "group_scores", allow_none=True)))

    def pv_encode_targets_select(self, layout: Layout, W, G, alpha: float, T, k: int, out_idx,
                                 group_scores=None):
        lay = layout.c()
        self._check(self._lib.pv_encode_targets_select(
            self._h, ctypes.byref(lay), _dev_ptr(W, torch.float32, "W"),
            _dev_ptr(G, torch.float32, "G"), float(alpha), _dev_ptr(T, torch.float32, "T"), int(k),
            _dev_ptr(out_idx, torch.int32, "out_idx", allow_none=(k == 0)),
            _dev_ptr(group_scores, torch.float32, "group_scores", allow_none=True)))

    def pv_reencode_groups(self, layout: Layout, T, codebooks, scales, group_idx, k: int,
                           beam_width: int, codes, num_changed=None):
        lay = layout.c()
        self._check(self._lib.pv_reencode_groups(
            self._h, ctypes.byref(lay), _dev_ptr(T, torch.float32, "T"),
            _dev_ptr(codebooks, torch.float32, "codebooks"),
            _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(group_idx, torch.int32, "group_idx", allow_none=(k == 0)), int(k),
            int(beam_width), _dev_ptr(codes, torch.uint16, "codes"),
            _dev_ptr(num_changed, torch.int64, "num_changed", allow_none=True)))

    def pv_reencode_groups_stochastic(self, layout: Layout, T, codebooks, scales, group_idx, k: int,
                                      power: int, seed: int, codes, num_changed=None):
        lay = layout.c()
        self._check(self._lib.pv_reencode_groups_stochastic(
            self._h, ctypes.byref(lay), _dev_ptr(T, torch.float32, "T"),
            _dev_ptr(codebooks, torch.float32, "codebooks"),
            _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(group_idx, torch.int32, "group_idx", allow_none=(k == 0)), int(k),
            int(power), int(seed) & (2 ** 64 - 1), _dev_ptr(codes, torch.uint16, "codes"),
            _dev_ptr(num_changed, torch.int64, "num_changed", allow_none=True)))

    def pv_reencode_trust_ratio(self, layout: Layout, T, W, codebooks, scales, k_max: int,
                                chunk: int, ratio: float, beam_width: int, codes, rank_idx,
                                num_applied, stats=None):
        lay = layout.c()
        self._check(self._lib.pv_reencode_trust_ratio(
            self._h, ctypes.byref(lay), _dev_ptr(T, torch.float32, "T"),
            _dev_ptr(W, torch.float32, "W"), _dev_ptr(codebooks, torch.float32, "codebooks"),
            _dev_ptr(scales, torch.float32, "scales"), int(k_max), int(chunk), float(ratio),
            int(beam_width), _dev_ptr(codes, torch.uint16, "codes"),
            _dev_ptr(rank_idx, torch.int32, "rank_idx", allow_none=True),
            _dev_ptr(num_applied, torch.int64, "num_applied"),
            _dev_ptr(stats, torch.float64, "stats", allow_none=True)))

    def pv_dequantize_groups(self, layout: Layout, codes, codebooks, scales, group_idx, k: int, W_out):
        lay = layout.c()
        self._check(self._lib.pv_dequantize_groups(
            self._h, ctypes.byref(lay), _dev_ptr(codes, torch.uint16, "codes"),
            _dev_ptr(codebooks, torch.float32, "codebooks"), _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(group_idx, torch.int32, "group_idx", allow_none=(k == 0)), int(k),
            _dev_ptr(W_out, torch.float32, "W_out")))

    def pv_codebook_grads(self, layout: Layout, G, codes, codebooks, scales, grad_codebooks,
                          grad_scales=None):
        lay = layout.c()
        self._check(self._lib.pv_codebook_grads(
            self._h, ctypes.byref(lay), _dev_ptr(G, torch.float32, "G"),
            _dev_ptr(codes, torch.uint16, "codes"), _dev_ptr(codebooks, torch.float32, "codebooks"),
            _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(grad_codebooks, torch.float32, "grad_codebooks"),
            _dev_ptr(grad_scales, torch.float32, "grad_scales", allow_none=True)))

    def pv_dequantize_scalar(self, out_features: int, in_features: int, block_size: int, nbits: int,
                             codes, scales, zeros, W_out):
        self._check(self._lib.pv_dequantize_scalar(
            self._h, int(out_features), int(in_features), int(block_size), int(nbits),
            _dev_ptr(codes, torch.uint8, "codes"), _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(zeros, torch.float32, "zeros"), _dev_ptr(W_out, torch.float32, "W_out")))

    def pv_reencode_scalar(self, out_features: int, in_features: int, block_size: int, nbits: int,
                           T, scales, zeros, weight_idx, k: int, codes, num_changed=None):
        self._check(self._lib.pv_reencode_scalar(
            self._h, int(out_features), int(in_features), int(block_size), int(nbits),
            _dev_ptr(T, torch.float32, "T"), _dev_ptr(scales, torch.float32, "scales"),
            _dev_ptr(zeros, torch.float32, "zeros"),
            _dev_ptr(weight_idx, torch.int32, "weight_idx", allow_none=(k == 0)), int(k),
            _dev_ptr(codes, torch.uint8, "codes"),
            _dev_ptr(num_changed, torch.int64, "num_changed", allow_none=True)))

    def pv_dequantize(self, layout: Layout, codes, codebooks, scales, W_out):
        lay = layout.c()
        self._check(self._lib.pv_dequantize(
            self._h, ctypes.byref(lay), _dev_ptr(codes, torch.uint16, "codes"),
            _dev_ptr(codebooks, torch.float32, "codebooks"),
            _dev_ptr(scales, torch.float32, "scales"), _dev_ptr(W_out, torch.float32, "W_out")))

    # ---- operators around the V step --------------------------------------
    def _tensor(self, t, dtype, shape, what: str, allow_none: bool = False):
        """Address of a dense tensor of this device, type (or one of several) and shape."""
        if t is None and allow_none:
            return None
        # the checks of a call cost as much as a small kernel: those that pass are few and cheap
        try:
            if ((t.dtype is dtype or (dtype is _DTYPES and t.dtype in dtype)) and t.shape == shape
                    and t.get_device() == self.device and t.is_contiguous()):
                return t.data_ptr()
        except AttributeError:
            pass
        types = tuple(dtype) if dtype is _DTYPES else (dtype,)
        if isinstance(t, torch.Tensor) and t.dtype not in types:
            raise TypeError(f"{what} must be {' or '.join(map(str, types))}, got {t.dtype}")
        ptr = _dev_ptr(t, getattr(t, "dtype", None), what)
        if t.get_device() != self.device:
            raise ValueError(f"{what} is on {t.device}, the context on device {self.device}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{what} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
        return ptr

    def _coded(self, rows: int, cols: int, fmt: str, codes, scales, of: str = "", allow_none: bool = False):
        of_codes, of_scales = mx_shapes(rows, cols, fmt)
        return (self._tensor(codes, torch.uint8, of_codes, of + "codes", allow_none),
                self._tensor(scales, torch.uint8, of_scales, of + "scales", allow_none))

    def pv_quantize_mx(self, rows: int, cols: int, fmt: str, X, codes, scales):
        x = self._tensor(X, _DTYPES, (rows, cols), "X")
        self._check(self._lib.pv_quantize_mx(self._h, int(rows), int(cols), _mx_format(fmt), _DTYPES[X.dtype], x,
                                             *self._coded(rows, cols, fmt, codes, scales)))

    def pv_dequantize_mx(self, rows: int, cols: int, fmt: str, codes, scales, out):
        o = self._tensor(out, _DTYPES, (rows, cols), "out")
        self._check(self._lib.pv_dequantize_mx(self._h, int(rows), int(cols), _mx_format(fmt),
                                               *self._coded(rows, cols, fmt, codes, scales), _DTYPES[out.dtype], o))

    def pv_mx_product(self, tokens: int, out_features: int, in_features: int, x_format: str, x_codes, x_scales,
                      w_codes, w_scales, Y):
        y = self._tensor(Y, _DTYPES, (tokens, out_features), "Y")
        self._check(self._lib.pv_mx_product(
            self._h, int(tokens), int(out_features), int(in_features), _mx_format(x_format),
            *self._coded(tokens, in_features, x_format, x_codes, x_scales, "x_"),
            *self._coded(out_features, in_features, "e2m1", w_codes, w_scales, "w_"), _DTYPES[Y.dtype], y))

    def pv_mx_product_grads(self, tokens: int, out_features: int, in_features: int, x_format: str, x_codes, x_scales,
                            w_codes, w_scales, dY, dX=None, dW=None):
        dx = self._tensor(dX, _DTYPES, (tokens, in_features), "dX", allow_none=True)
        self._check(self._lib.pv_mx_product_grads(
            self._h, int(tokens), int(out_features), int(in_features), _mx_format(x_format),
            *self._coded(tokens, in_features, x_format, x_codes, x_scales, "x_", allow_none=dW is None),
            *self._coded(out_features, in_features, "e2m1", w_codes, w_scales, "w_", allow_none=dX is None),
            self._tensor(dY, torch.bfloat16, (tokens, out_features), "dY"),
            _DTYPES[dX.dtype] if dX is not None else 0, dx,
            self._tensor(dW, torch.float32, (out_features, in_features), "dW", allow_none=True)))

    def pv_rms_norm(self, rows: int, cols: int, x, residual, weight, eps: float, h=None, y=None, fmt: str = "e4m3",
                    codes=None, scales=None, rstd=None):
        shape, tensor = (rows, cols), self._tensor
        xp = tensor(x, _DTYPES, shape, "x")
        dtype = x.dtype
        c, s = (None, None) if codes is None and scales is None else self._coded(rows, cols, fmt, codes, scales, allow_none=True)
        self._check(self._lib.pv_rms_norm(
            self._h, int(rows), int(cols), _DTYPES[dtype], xp, tensor(residual, dtype, shape, "residual", True),
            tensor(weight, torch.float32, (cols,), "weight"), float(eps), tensor(h, dtype, shape, "h", True),
            tensor(y, dtype, shape, "y", True), _mx_format(fmt), c, s, tensor(rstd, torch.float32, (rows,), "rstd", True)))

    def pv_rms_norm_backward(self, rows: int, cols: int, dy, dh, h, weight, rstd, dx=None, dweight=None):
        shape, tensor = (rows, cols), self._tensor
        g = tensor(dy, _DTYPES, shape, "dy")
        dtype = dy.dtype
        self._check(self._lib.pv_rms_norm_backward(
            self._h, int(rows), int(cols), _DTYPES[dtype], g, tensor(dh, dtype, shape, "dh", True), tensor(h, dtype, shape, "h"),
            tensor(weight, torch.float32, (cols,), "weight"), tensor(rstd, torch.float32, (rows,), "rstd"),
            tensor(dx, dtype, shape, "dx", True), tensor(dweight, torch.float32, (cols,), "dweight", True)))

    def _strided(self, t, dtype, rows: int, vocab: int, what: str):
        """Address and row stride of [rows, vocab] whose rows are dense."""
        if t is None:
            return None, vocab
        types = tuple(dtype) if dtype is _DTYPES else (dtype,)
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in types:
            raise TypeError(f"{what} must be a CUDA tensor of {' or '.join(map(str, types))}")
        if t.get_device() != self.device:
            raise ValueError(f"{what} is on {t.device}, the context on device {self.device}")
        if t.shape != (rows, vocab):
            raise ValueError(f"{what} must have the shape {(rows, vocab)}, got {tuple(t.shape)}")
        ld = t.stride(0) if rows > 1 else vocab
        if (vocab > 1 and t.stride(1) != 1) or ld < vocab:
            raise TypeError(f"{what} must have dense rows that do not overlap, got strides {t.stride()}")
        return t.data_ptr(), ld

    def _teacher(self, rows: int, k: int, ids, logits):
        return (self._tensor(ids, torch.int32, (rows, k), "teacher_ids", allow_none=(k == 0)),
                self._tensor(logits, torch.float32, (rows, k), "teacher_logits", allow_none=(k == 0)))

    def pv_distill_topk(self, rows: int, vocab: int, k: int, logits, teacher_ids, teacher_logits, temperature: float,
                        row_weight=None, loss=None, lse=None, grad=None):
        row = lambda t, what, none: self._tensor(t, torch.float32, (rows,), what, allow_none=none)  # noqa: E731
        if logits is None:
            raise TypeError("logits is None")
        z, ld = self._strided(logits, _DTYPES, rows, vocab, "logits")
        g, grad_ld = self._strided(grad, logits.dtype, rows, vocab, "grad")
        ids, top = self._teacher(rows, k, teacher_ids, teacher_logits)
        self._check(self._lib.pv_distill_topk(
            self._h, int(rows), int(vocab), int(k), _DTYPES[logits.dtype], z, ld, ids, top, float(temperature),
            row(row_weight, "row_weight", True), row(loss, "loss", False), row(lse, "lse", True), g, grad_ld))

    def pv_distill_topk_backward(self, rows: int, vocab: int, k: int, logits, teacher_ids, teacher_logits,
                                 temperature: float, lse, grad_loss, grad):
        row = lambda t, what: self._tensor(t, torch.float32, (rows,), what)  # noqa: E731
        if logits is None or grad is None:
            raise TypeError("logits or grad is None")
        z, ld = self._strided(logits, _DTYPES, rows, vocab, "logits")
        g, grad_ld = self._strided(grad, logits.dtype, rows, vocab, "grad")
        ids, top = self._teacher(rows, k, teacher_ids, teacher_logits)
        self._check(self._lib.pv_distill_topk_backward(
            self._h, int(rows), int(vocab), int(k), _DTYPES[logits.dtype], z, ld, ids, top, float(temperature),
            row(lse, "lse"), row(grad_loss, "grad_loss"), g, grad_ld))

    # ---- instrumentation --------------------------------------------------
    def pv_set_search_mode(self, mode: int):
        self._check(self._lib.pv_set_search_mode(self._h, int(mode)))

    def pv_timing_enable(self, on: bool):
        self._check(self._lib.pv_timing_enable(self._h, int(bool(on))))

    def pv_timing_reset(self):
        self._check(self._lib.pv_timing_reset(self._h))

    def pv_timing_read(self, kernel: "int | str"):
        kid = KERNEL_IDS[kernel] if isinstance(kernel, str) else int(kernel)
        ms, n = ctypes.c_double(0), ctypes.c_int64(0)
        self._check(self._lib.pv_timing_read(self._h, kid, ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def pv_probe_copy(self, dst, src):
        nbytes = src.numel() * src.element_size()
        if dst.numel() * dst.element_size() != nbytes:
            raise ValueError("dst and src differ in size")
        self._check(self._lib.pv_probe_copy(self._h, ctypes.c_void_p(dst.data_ptr()),
                                            ctypes.c_void_p(src.data_ptr()), int(nbytes)))

    def pv_probe_mfma_f16(self, iters: int, sink):
        waves = ctypes.c_int64(0)
        self._check(self._lib.pv_probe_mfma_f16(self._h, int(iters), _dev_ptr(sink, torch.float32, "sink"),
                                                ctypes.byref(waves)))
        return waves.value

    def pv_reencode_stats(self):
        arr = (ctypes.c_int64 * 4)()
        self._check(self._lib.pv_reencode_stats(self._h, arr))
        return {"filtered": arr[0], "fallback": arr[1], "reranked_candidates": arr[2],
                "exact": arr[3]}
