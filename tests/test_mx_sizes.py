"""Sizes past 31 bits reach the microscaled operators' C ABI as sizes that it refuses, not cut to their low bits."""
import pytest
import torch

from paper_2510_04147_amd import binding, mx


class Rows:
    """Stands for a GPU tensor that this machine need not hold: the calls below end on the host."""
    device = "cuda:0"

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, torch.Size(shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()


def form(rows, cols, bits):
    return (Rows(torch.float8_e4m3fn, rows, cols) if bits == mx.FP8 else Rows(torch.uint8, rows, cols // 2)), Rows(torch.float8_e8m0fnu, *mx.scale_shape(rows, cols))


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_04147_amd import build
        build.build()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)


BIG = (1 << 32) + 4


@pytest.mark.parametrize("call", [
    lambda n: mx.quantize(Rows(torch.bfloat16, n, 64), mx.FP4, out=form(n, 64, mx.FP4)),
    lambda n: mx.quantize(Rows(torch.float32, 4, n * 32), mx.FP8, out=form(4, n * 32, mx.FP8)),
    lambda n: mx.norm(Rows(torch.float32, n, 64), None, Rows(torch.float32, 64), 1e-5, out=form(n, 64, mx.FP8)),
    lambda n: mx.linear(form(n, 64, mx.FP8), form(8, 64, mx.FP4), "bf16", out=Rows(torch.bfloat16, n, 8), workspace=Rows(torch.uint8, 16)),
    lambda n: mx.linear(form(8, 64, mx.FP8), form(n, 64, mx.FP4), "fp32", out=Rows(torch.float32, 8, n)),
    lambda n: mx.linear(form(8, n * 32, mx.FP8), form(8, n * 32, mx.FP4), "fp32", out=Rows(torch.float32, 8, 8))])
@pytest.mark.parametrize("n", [BIG, 1 << 31, (1 << 20) + 1])
def test_refused(call, n):
    with pytest.raises(binding.SsdError, match="beyond the supported size") as e:
        call(n)
    assert e.value.code == -2


def test_workspace_of_a_product_beyond_the_sizes():
    assert mx.linear_workspace(8, 64, 4096) > 0
    for M, N, K in ((BIG, 64, 4096), (8, BIG * 64, 4096), (8, 64, BIG * 1024), (8 - (1 << 32), 64, 4096)):
        assert mx.linear_workspace(M, N, K) == 0


@pytest.mark.parametrize("N,K", [(64, 2304), (512, 4096), (4096, 4096), (8192, 2048), (8192, 18944)])
def test_a_workspace_for_the_most_rows_serves_fewer(N, K):
    """Whichever kernels the row counts take."""
    one = mx.linear_workspace(1, N, K)
    assert one > 0
    for M in (2, 33, 160, 1000, 9000):
        assert mx.linear_workspace(M, N, K) == mx.linear_workspace(M, N, K, "fp32") == M * one
