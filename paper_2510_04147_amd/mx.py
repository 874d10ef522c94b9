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
_MOST = (1 << 31) - 1                                   # of a C int, which ctypes would fill with the low bits of a larger number
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


# The checks below run in front of every call, whose kernel may take no longer than they do: a device is its index here.
def _bad(t, what):
    return ValueError(f"{what} is needed, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def _operand(t, index, dtype, shape):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise _bad(t, f"a contiguous {dtype} tensor {tuple(shape)} on GPU {index}")
    return t.data_ptr()


def _matrix(x, index, rows, cols, bits):
    """Pointers of a microscaled matrix."""
    codes, scales = x
    return (_operand(codes, index, torch.float8_e4m3fn, (rows, cols)) if bits == FP8 else _operand(codes, index, torch.uint8, (rows, cols // 2)),
            _operand(scales, index, torch.float8_e8m0fnu, scale_shape(rows, cols)))


def _gpu(t):
    index = t.get_device()
    if index < 0:
        raise ValueError(f"operands on a GPU are needed, got {t.device}")
    return index


def _call(index, f, *args):
    """The call on the current stream of the operands' device, which is made the current one for it."""
    if index == torch.cuda.current_device():
        rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            rc = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if rc < 0:
        raise binding.SsdError(rc, _lib.ssd_strerror(rc).decode(), _lib.ssd_last_error(None).decode())


def _beyond(who, *sizes):
    return binding.SsdError(-2, _lib.ssd_strerror(-2).decode(), f"{who}: {' x '.join(map(str, sizes))} is beyond the supported size")


def scale_shape(rows, cols):
    return ((cols + 127) // 128, (rows + 31) // 32 * 32, 4)


def empty(rows, cols, bits, device):
    """Uninitialised codes and scales of a microscaled matrix."""
    codes = torch.empty(rows, cols * bits // 8, dtype=torch.float8_e4m3fn if bits == FP8 else torch.uint8, device=device)
    return codes, torch.empty(scale_shape(rows, cols), dtype=torch.float8_e8m0fnu, device=device)


def quantize(x, bits, values=None, out=None):
    """x: float32 or bfloat16 [rows, cols], cols a multiple of 32 -> (codes, scales) of `bits` (FP4 or FP8) per value.
    values (as x, may be None) receives the rounded values; out: (codes, scales) to write to."""
    l, index, dtype, shape = lib(), _gpu(x), x.dtype, x.shape
    if len(shape) != 2 or (dtype is not torch.bfloat16 and dtype is not torch.float32):
        raise _bad(x, "a float32 or bfloat16 matrix")
    rows, cols = shape
    if rows < 1 or cols < 1 or cols % 32:
        raise _bad(x, "a matrix with columns in blocks of 32")
    if rows > _MOST or cols > _MOST:
        raise _beyond("ssd_mx_quantize", rows, cols)
    if bits != FP4 and bits != FP8:
        raise ValueError(f"bits must be 4 or 8, got {bits}")
    if out is None:
        out = empty(rows, cols, bits, x.device)
    _call(index, l.ssd_mx_quantize, _operand(x, index, dtype, shape), binding.SSD_F32 if dtype is torch.float32 else binding.SSD_BF16, rows, cols, bits,
          *_matrix(out, index, rows, cols, bits), None if values is None else _operand(values, index, dtype, shape))
    return out


def norm(h, partials, gain, eps, h_out=None, out=None, keep=True):
    """h + partials (float32 [rows, cols], [n, rows, cols] or None), RMSNorm with `gain` -> (codes, scales), 8 bits.  The sum goes to
    h_out, or to h itself where h_out is None and keep is true."""
    l, index, f32, shape = lib(), _gpu(h), torch.float32, h.shape
    if len(shape) != 2 or shape[0] < 1 or shape[1] < 1 or shape[1] % 32:
        raise _bad(h, "a matrix with columns in blocks of 32")
    rows, cols = shape
    n, parts = 0, None
    if partials is not None:
        n = partials.shape[0] if partials.dim() == 3 else -1
        parts = _operand(partials, index, f32, (n, rows, cols))
    if rows > _MOST or cols > _MOST or n > _MOST:
        raise _beyond("ssd_mx_norm", n, rows, cols)
    if out is None:
        out = empty(rows, cols, FP8, h.device)
    at = _operand(h, index, f32, shape)
    to = _operand(h_out, index, f32, shape) if h_out is not None else at if keep else None
    _call(index, l.ssd_mx_norm, at, parts, n, _operand(gain, index, f32, (cols,)), eps, rows, cols, to, *_matrix(out, index, rows, cols, FP8))
    return out


def linear(x, w, result="bf16", out=None, workspace=None):
    """x (8 bits, [M, K]) times w (4 bits, [N, K]) transposed.  result "bf16" or "fp32": a tensor [M, N]; "swiglu": w holds gate
    rows, then up rows, and the result is silu(gate) * up as (codes, scales) of 8 bits, [M, N / 2].  workspace: a uint8 tensor of at
    least linear_workspace(...) bytes, else one is allocated where the matrix has several k-slices."""
    l, kind = lib(), RESULTS.get(result)
    if kind is None:
        raise ValueError(f"result must be one of {sorted(RESULTS)}, got {result!r}")
    codes = x[0]
    index, shape, N = _gpu(codes), codes.shape, w[0].shape[0]
    if len(shape) != 2 or shape[0] < 1 or shape[1] < 1 or shape[1] % 32:
        raise _bad(codes, "a matrix with columns in blocks of 32")
    if N < 1 or (kind == OUT_SWIGLU and N % 64):
        raise ValueError(f"rows of weights are needed, gate and up rows in blocks of 32, got {N}")
    M, K = shape
    if M > _MOST or N > _MOST or K > _MOST:
        raise _beyond("ssd_mx_linear", M, N, K)
    xc, xs = _matrix(x, index, M, K, FP8)
    wc, ws = _matrix(w, index, N, K, FP4)
    if kind == OUT_SWIGLU:
        if out is None:
            out = empty(M, N // 2, FP8, codes.device)
        to, to_scales = _matrix(out, index, M, N // 2, FP8)
    else:
        dtype = torch.float32 if kind == OUT_F32 else torch.bfloat16
        if out is None:
            out = torch.empty(M, N, dtype=dtype, device=codes.device)
        to, to_scales = _operand(out, index, dtype, (M, N)), None
    at, size = None, 0
    if workspace is None:
        size = l.ssd_mx_linear_workspace(M, N, K, kind)
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=codes.device)
            at = workspace.data_ptr()
    else:
        size = workspace.numel()
        at = _operand(workspace, index, torch.uint8, (size,))
    _call(index, l.ssd_mx_linear, xc, xs, M, wc, ws, N, K, kind, to, to_scales, at, size)
    return out


def linear_workspace(M, N, K, result="bf16"):
    """Bytes of workspace of linear(): proportional to M; 0 where the matrix has one k-slice, and on a bad size."""
    return 0 if max(M, N, K) > _MOST or min(M, N, K) < 1 else lib().ssd_mx_linear_workspace(M, N, K, RESULTS[result])
