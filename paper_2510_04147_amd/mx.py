"""ctypes binding of the microscaled operators (include/ssd_mx.h): argument marshalling only.

    codes, scales = mx.quantize(weight, mx.FP4)            # once, when a model is loaded
    x = mx.norm(h, partials, gain, eps)                    # residual + RMSNorm, 8 bits
    y = mx.linear(x, (codes, scales), "bf16")

A microscaled matrix is a pair (codes, scales).  codes: torch.float8_e4m3fn [rows, cols], or uint8 [rows, cols / 2], two
4-bit values to a byte.  scales: torch.float8_e8m0fnu [groups of 128 columns, rows rounded up to 32, 4].  The calls run on
the current stream of the operands' device; operands are contiguous and on one device.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding

FP4, FP8 = 4, 8
OUT_F32, OUT_BF16, OUT_SWIGLU = range(3)
RESULTS = {"fp32": OUT_F32, "bf16": OUT_BF16, "swiglu": OUT_SWIGLU}
EXPORTS = ["ssd_mx_scale_bytes", "ssd_mx_quantize", "ssd_mx_norm", "ssd_mx_linear_workspace", "ssd_mx_linear"]

_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        l = binding.lib()
        p, i, z = C.c_void_p, C.c_int, C.c_size_t
        l.ssd_mx_scale_bytes.restype = z
        l.ssd_mx_scale_bytes.argtypes = [i, i]
        l.ssd_mx_quantize.argtypes = [p, i, i, i, i, p, p, p, p]
        l.ssd_mx_norm.argtypes = [p, p, i, p, C.c_float, i, i, p, p, p, p]
        l.ssd_mx_linear_workspace.restype = z
        l.ssd_mx_linear_workspace.argtypes = [i, i, i, i]
        l.ssd_mx_linear.argtypes = [p, p, i, p, p, i, i, i, p, p, p, z, p]
        _lib = l
    return _lib


def _chk(rc):
    if rc < 0:
        raise binding.SsdError(rc, _lib.ssd_strerror(rc).decode(), _lib.ssd_last_error(None).decode())


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _ptr(t):
    return None if t is None else t.data_ptr()


class _On:
    """The operands' device made the current one, and its stream.  `tensors`: (tensor or None, its type, its shape)."""

    def __init__(self, *tensors):
        dev = tensors[0][0].device
        for t, dtype, shape in tensors:
            if t is None:
                continue
            if not (t.device == dev and dev.type == "cuda"):
                raise ValueError(f"operands on one GPU are needed, got {t.device} and {dev}")
            if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
                raise ValueError(f"a contiguous {dtype} tensor {tuple(shape)} is needed, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}")
        self.dev = dev

    def __enter__(self):
        self.prev = torch.cuda.current_device()
        if self.prev != self.dev.index:
            torch.cuda.set_device(self.dev)
        return torch.cuda.current_stream(self.dev).cuda_stream

    def __exit__(self, *exc):
        if self.prev != self.dev.index:
            torch.cuda.set_device(self.prev)


def scale_shape(rows, cols):
    return ((cols + 127) // 128, (rows + 31) // 32 * 32, 4)


def empty(rows, cols, bits, device):
    """Uninitialised codes and scales of a microscaled matrix."""
    codes = torch.empty(rows, cols * bits // 8, dtype=torch.float8_e4m3fn if bits == FP8 else torch.uint8, device=device)
    return codes, torch.empty(scale_shape(rows, cols), dtype=torch.float8_e8m0fnu, device=device)


def _form(x, rows, cols, bits):
    """What _On checks of a microscaled matrix."""
    _need(isinstance(x, (tuple, list)) and len(x) == 2, "a microscaled matrix is a pair (codes, scales)")
    return ((x[0], torch.float8_e4m3fn if bits == FP8 else torch.uint8, (rows, cols * bits // 8)),
            (x[1], torch.float8_e8m0fnu, scale_shape(rows, cols)))


def quantize(x, bits, values=None, out=None):
    """x: float32 or bfloat16 [rows, cols], cols a multiple of 32 -> (codes, scales) of `bits` (FP4 or FP8) per value.
    values (as x, may be None) receives the rounded values; out: (codes, scales) to write to."""
    l = lib()
    _need(x.dim() == 2 and x.dtype in (torch.float32, torch.bfloat16), f"a float32 or bfloat16 matrix is needed, got {x.dtype} {tuple(x.shape)}")
    rows, cols = x.shape
    _need(rows > 0 and cols > 0 and cols % 32 == 0, f"columns in blocks of 32 are needed, got {tuple(x.shape)}")
    _need(bits in (FP4, FP8), f"bits must be 4 or 8, got {bits}")
    if out is None:
        out = empty(rows, cols, bits, x.device)
    with _On((x, x.dtype, x.shape), (values, x.dtype, x.shape), *_form(out, rows, cols, bits)) as st:
        _chk(l.ssd_mx_quantize(x.data_ptr(), binding.SSD_F32 if x.dtype == torch.float32 else binding.SSD_BF16, rows, cols, bits,
                               out[0].data_ptr(), out[1].data_ptr(), _ptr(values), st))
    return out


def norm(h, partials, gain, eps, h_out=None, out=None, keep=True):
    """h + partials (float32 [rows, cols], [n, rows, cols] or None), RMSNorm with `gain` -> (codes, scales), 8 bits.  The sum goes to
    h_out, or to h itself where h_out is None and keep is true."""
    l = lib()
    _need(h.dim() == 2 and h.shape[0] > 0 and h.shape[1] > 0 and h.shape[1] % 32 == 0, f"rows in blocks of 32 columns are needed, got {tuple(h.shape)}")
    rows, cols = h.shape
    n = 0 if partials is None else partials.shape[0]
    _need(n == 0 or partials.dim() == 3, "partial sums are [n, rows, cols]")
    if out is None:
        out = empty(rows, cols, FP8, h.device)
    f32 = torch.float32
    with _On((h, f32, h.shape), (partials if n else None, f32, (n, rows, cols)), (gain, f32, (cols,)), (h_out, f32, h.shape),
             *_form(out, rows, cols, FP8)) as st:
        to = h_out if h_out is not None else h if keep else None
        _chk(l.ssd_mx_norm(h.data_ptr(), _ptr(partials) if n else None, n, gain.data_ptr(), eps, rows, cols, _ptr(to), out[0].data_ptr(),
                           out[1].data_ptr(), st))
    return out


def linear(x, w, result="bf16", out=None, workspace=None):
    """x (8 bits, [M, K]) times w (4 bits, [N, K]) transposed.  result "bf16" or "fp32": a tensor [M, N]; "swiglu": w holds gate
    rows, then up rows, and the result is silu(gate) * up as (codes, scales) of 8 bits, [M, N / 2].  workspace: a uint8 tensor of at
    least linear_workspace(...) bytes, else one is allocated where the product needs it."""
    l = lib()
    _need(result in RESULTS, f"result must be one of {sorted(RESULTS)}, got {result!r}")
    _need(len(x) == 2 and len(w) == 2 and x[0].dim() == 2 and w[0].dim() == 2, "microscaled matrices are pairs (codes, scales)")
    M, K = x[0].shape
    N, kind = w[0].shape[0], RESULTS[result]
    _need(M > 0 and N > 0 and K > 0 and K % 32 == 0, f"rows in blocks of 32 columns are needed, got {M} x {K} and {N} rows of weights")
    _need(kind != OUT_SWIGLU or N % 64 == 0, f"gate and up rows in blocks of 32 are needed, got {N}")
    dev = x[0].device
    if kind == OUT_SWIGLU:
        if out is None:
            out = empty(M, N // 2, FP8, dev)
        to, outs = _form(out, M, N // 2, FP8), (out[0].data_ptr(), out[1].data_ptr())
    else:
        dtype = torch.float32 if kind == OUT_F32 else torch.bfloat16
        if out is None:
            out = torch.empty(M, N, dtype=dtype, device=dev)
        to, outs = ((out, dtype, (M, N)),), (out.data_ptr(), None)
    with _On(*_form(x, M, K, FP8), *_form(w, N, K, FP4), *to) as st:
        need = l.ssd_mx_linear_workspace(M, N, K, kind)
        if need and workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _need(workspace is None or (workspace.dtype == torch.uint8 and workspace.is_contiguous() and workspace.device == dev), "a contiguous uint8 workspace on the operands' device is needed")
        _chk(l.ssd_mx_linear(x[0].data_ptr(), x[1].data_ptr(), M, w[0].data_ptr(), w[1].data_ptr(), N, K, kind, *outs, _ptr(workspace),
                             workspace.numel() if workspace is not None else 0, st))
    return out


def linear_workspace(M, N, K, result="bf16"):
    """Bytes of workspace of linear()."""
    return lib().ssd_mx_linear_workspace(M, N, K, RESULTS[result])
