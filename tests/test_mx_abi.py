"""The microscaled operators' C ABI: symbols, sizes and refusals that reach no GPU."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2510_04147_amd import binding, mx
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_04147_amd import build
        build.build()
    return mx.lib()


def test_every_declared_symbol_is_exported(lib):
    from paper_2510_04147_amd import mx
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssd_mx.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ssd_mx_[a-z_]+)\s*\(", text))) == sorted(mx.EXPORTS)
    for s in mx.EXPORTS:
        assert hasattr(lib, s)


def test_sizes(lib):
    assert lib.ssd_mx_scale_bytes(1, 32) == 32 * 4
    assert lib.ssd_mx_scale_bytes(33, 160) == 2 * 64 * 4
    for rows, cols in ((0, 32), (1, 0), (1, 31), (-4, 64), (1, 1 << 21), ((1 << 20) + 1, 32)):
        assert lib.ssd_mx_scale_bytes(rows, cols) == 0
    assert lib.ssd_mx_linear_workspace(8, 64, 512, 1) == 0                    # one slice
    assert lib.ssd_mx_linear_workspace(8, 64, 4096, 1) == 4 * 8 * 64 * 4
    assert lib.ssd_mx_linear_workspace(8, 64, 4096, 2) == 0
    assert lib.ssd_mx_linear_workspace(8, 64, 4096, 7) == 0
    # a slice that rounding up to chunks leaves empty takes no partial sum: 9 chunks in threes
    assert lib.ssd_mx_linear_workspace(1, 32, 2304, 0) == 3 * 32 * 4


# a pointer that is never read: every one of these calls ends on the host
P16, ODD = 1 << 20, (1 << 20) + 8


@pytest.mark.parametrize("change,code,what", [
    (dict(src=None), -1, "null"), (dict(codes=None), -1, "null"), (dict(scales=None), -1, "null"), (dict(dtype=2), -1, "dtype"), (dict(dtype=9), -1, "dtype"),
    (dict(format=5), -1, "format"), (dict(rows=0), -1, "row"), (dict(rows=-1), -1, "row"), (dict(cols=0), -1, "32"), (dict(cols=48), -1, "32"),
    (dict(cols=1 << 21), -2, "beyond"), (dict(rows=(1 << 20) + 1), -2, "beyond"), (dict(src=ODD), -1, "16-byte"), (dict(codes=ODD), -1, "16-byte"),
    (dict(scales=ODD), -1, "16-byte"), (dict(values=ODD), -1, "16-byte")])
def test_quantize_refusals(lib, change, code, what):
    a = dict(src=P16, dtype=0, rows=4, cols=64, format=4, codes=P16, scales=P16, values=None)
    a.update(change)
    assert lib.ssd_mx_quantize(*a.values(), None) == code
    assert what in lib.ssd_last_error(None).decode()


@pytest.mark.parametrize("change,code,what", [
    (dict(h=None), -1, "null"), (dict(gain=None), -1, "null"), (dict(codes=None), -1, "null"), (dict(scales=None), -1, "null"),
    (dict(partials=None), -1, "null"), (dict(n_part=-1), -1, "n_part"), (dict(n_part=9), -2, "partial"), (dict(eps=-1e-5), -1, "eps"),
    (dict(eps=float("nan")), -1, "eps"), (dict(rows=0), -1, "row"), (dict(cols=40), -1, "32"), (dict(cols=8224), -2, "8192"), (dict(h=ODD), -1, "16-byte"),
    (dict(partials=ODD), -1, "16-byte"), (dict(gain=ODD), -1, "16-byte"), (dict(h_out=ODD), -1, "16-byte"), (dict(codes=ODD), -1, "16-byte")])
def test_norm_refusals(lib, change, code, what):
    a = dict(h=P16, partials=P16, n_part=2, gain=P16, eps=1e-5, rows=4, cols=64, h_out=P16, codes=P16, scales=P16)
    a.update(change)
    assert lib.ssd_mx_norm(*a.values(), None) == code
    assert what in lib.ssd_last_error(None).decode()


@pytest.mark.parametrize("change,code,what", [
    (dict(x=None), -1, "null"), (dict(xs=None), -1, "null"), (dict(w=None), -1, "null"), (dict(ws=None), -1, "null"), (dict(out=None), -1, "null"),
    (dict(result=2, out_s=None), -1, "null"), (dict(result=3), -1, "result"), (dict(result=-1), -1, "result"), (dict(M=0), -1, "row"), (dict(N=0), -1, "row"),
    (dict(K=0), -1, "32"), (dict(K=100), -1, "32"), (dict(K=1 << 21), -2, "beyond"), (dict(M=1 << 21), -2, "beyond"), (dict(N=1 << 21), -2, "beyond"),
    (dict(M=1 << 20, N=1 << 20), -2, "outputs"), (dict(result=2, N=96), -1, "64"), (dict(x=ODD), -1, "16-byte"), (dict(xs=ODD), -1, "16-byte"),
    (dict(w=ODD), -1, "16-byte"), (dict(ws=ODD), -1, "16-byte"), (dict(out=ODD), -1, "16-byte"), (dict(out_s=ODD), -1, "16-byte"),
    (dict(work=ODD), -1, "16-byte"), (dict(work=None), -3, "workspace"), (dict(size=4 * 4 * 64 * 4 - 1), -3, "workspace")])
def test_linear_refusals(lib, change, code, what):
    a = dict(x=P16, xs=P16, M=4, w=P16, ws=P16, N=64, K=4096, result=1, out=P16, out_s=P16, work=P16, size=4 * 4 * 64 * 4)
    a.update(change)
    assert lib.ssd_mx_linear(*a.values(), None) == code
    assert what in lib.ssd_last_error(None).decode()


def test_contexts(lib):
    """SSD_MXFP4 in a context's configuration: accepted where the projections have whole blocks, and smaller than bf16."""
    import ctypes
    from paper_2510_04147_amd import binding, synth
    size = lambda c: lib.ssd_workspace_bytes(ctypes.byref(c))  # noqa: E731
    bf16 = binding.make_config(synth.model_config("8b"), 1, 512, 32, 4)
    mxfp4 = binding.make_config(synth.model_config("8b", dtype="mxfp4"), 1, 512, 32, 4)
    assert mxfp4.dtype == binding.SSD_MXFP4 == 2
    L, d, F = 32, 4096, 12288
    weights = L * (3 * d * d + d * d + 3 * F * d)
    assert 0 < size(mxfp4) < size(bf16) - 2 * weights + weights * 17 // 32 + (64 << 20)
    for field, value in (("d_model", 264), ("d_ffn", 12304), ("d_ffn", 1 << 20), ("max_rows", 1 << 21), ("max_rows", 1 << 20)):
        bad = binding.make_config(synth.model_config("8b", dtype="mxfp4"), 1, 512, 32, 4)
        setattr(bad, field, value)
        assert size(bad) == 0, (field, value)
    w = binding.SsdWeights()
    # a projection off a 16-byte boundary is refused before the device is touched
    one = (ctypes.c_void_p * 32)(*[1 << 20] * 32)
    odd = (ctypes.c_void_p * 32)(*[(1 << 20) + 2] * 32)
    p = lambda a: ctypes.cast(a, ctypes.POINTER(ctypes.c_void_p))  # noqa: E731
    w = binding.SsdWeights(1 << 20, 1 << 20, 1 << 20, p(one), p(odd), p(one), p(one), p(one), p(one))
    h = ctypes.c_void_p()
    assert lib.ssd_create(ctypes.byref(mxfp4), ctypes.byref(w), ctypes.c_void_p(256), 1 << 60, None, ctypes.byref(h)) == -1
    assert b"16-byte" in lib.ssd_last_error(None)
