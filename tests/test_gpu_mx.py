"""The microscaled operators alone, against their definitions in 64 bits on the same operands (mx_plain.py)."""
import math

import pytest
import torch

import mx_plain as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    from paper_2510_04147_amd import mx
    return mx


def rand(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * std


def cuda(pair):
    return tuple(t.cuda() for t in pair)


# ---------------------------------------------------------------- quantize: nothing is left to a tolerance
def special(bits):
    """Blocks at the borders of the format: largest values at which the scale turns, ties, zeros, the smallest and the largest floats,
    infinities and NaN."""
    top = [7.0, 6.9999995, 6.0, 5.0, 7.5, 3.5, 1.75, 1.7499999] if bits == 4 else [464.0, 464.00003, 448.0, 480.0, 240.0, 232.0, 1.8125, 1.8125001]
    rows = []
    for t in top:
        b = torch.linspace(-1, 1, 32, dtype=torch.float64) * t
        rows.append(b.float())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4) if bits == 4 else torch.tensor([17, 19, 21, 23, 25, 27, 29, 31] * 4) / 16.0 * torch.tensor([1.0, 2.0, 4.0, 256.0]).repeat_interleave(8)
    rows += [ties, -ties, torch.zeros(32), -torch.zeros(32), torch.full((32,), 1e-45), torch.full((32,), 3e-39), torch.full((32,), 1.2e-38),
             torch.full((32,), torch.finfo(torch.float32).max), torch.linspace(0, 1, 32) * 1e-37]
    for v in (math.inf, -math.inf, math.nan):
        b = torch.linspace(-1, 1, 32)
        b[5] = v
        rows.append(b)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (31, 160), (33, 512), (45, 544), (65, 1504), (8, 4096), (1, 18944)])
def test_quantize(mx, dtype, bits, rows, cols):
    x = (rand(rows * cols + bits, rows, cols) * torch.exp(rand(1, 1, cols)) * torch.exp(2 * rand(2, rows, 1))).to(dtype)
    codes, s, v = P.quantize(x.double(), bits)
    values = torch.empty_like(x, device="cuda")
    got = mx.quantize(x.cuda(), bits, values=values)
    assert torch.equal(P.unpack(got[0], bits), codes)
    assert torch.equal(P.row_scales(got[1], rows, cols // 32), s)
    assert (P.padding(got[1], rows, cols // 32) == 127).all()
    assert torch.equal(values.cpu(), v.to(dtype))
    again = mx.quantize(x.cuda(), bits)                # without the values
    assert torch.equal(again[0].view(torch.uint8), got[0].view(torch.uint8)) and torch.equal(again[1].view(torch.uint8), got[1].view(torch.uint8))


@pytest.mark.parametrize("bits", [4, 8])
def test_quantize_borders_and_not_finite(mx, bits):
    x = special(bits)
    codes, s, v = P.quantize(x.double(), bits)
    values = torch.empty_like(x, device="cuda")
    got = mx.quantize(x.cuda(), bits, values=values)
    assert torch.equal(P.row_scales(got[1], len(x), 1), s)
    assert torch.equal(P.unpack(got[0], bits), codes)
    assert torch.equal(values.cpu().nan_to_num(nan=-1.25), v.float().nan_to_num(nan=-1.25))
    assert int((s == 255).sum()) == 3
    # the documented bound: half a step at the value, or of the smallest step
    fine = s[:, 0] < 255
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), (s[fine] - 127).double())
    step = x[fine].double().abs() * (2.0 ** -2 if bits == 4 else 2.0 ** -4)
    assert ((v[fine] - x[fine].double()).abs() <= torch.maximum(step, scale * (0.25 if bits == 4 else 2.0 ** -10))).all()


# ---------------------------------------------------------------- norm
@pytest.mark.parametrize("rows,cols,n_part", [(1, 32, 0), (1, 4096, 1), (8, 4096, 0), (33, 288, 3), (45, 512, 2), (160, 4096, 4), (7, 8192, 8),
                                             (40, 3584, 2), (5, 1504, 5), (2, 4128, 4), (64, 256, 6), (3, 1024, 7)])
def test_norm(mx, rows, cols, n_part):
    h, gain = rand(rows, rows, cols).float() * 3, 1 + 0.2 * rand(5, cols).float()
    parts = rand(7, n_part, rows, cols).float() if n_part else None
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    want_h, mags = h.double(), h.double().abs()
    if n_part:
        want_h, mags = want_h + parts.double().sum(0), mags + parts.double().abs().sum(0)
    h_out = torch.empty(rows, cols, device="cuda")
    got = mx.norm(dev(h), dev(parts), dev(gain), 1e-5, h_out=h_out)
    assert ((h_out.cpu().double() - want_h).abs() <= (n_part + 1) * 2.0 ** -24 * mags).all()
    # the rest from the sum that the GPU kept.  fp32: squares and their sum over the tree of lanes and waves, root, quotient and two
    # products are within 32 roundings
    kept = h_out.cpu().double()
    want = kept / torch.sqrt((kept * kept).mean(-1, keepdim=True) + 1e-5) * gain.double()
    P.check_fp8(got, want, want.abs() * 32 * 2.0 ** -24)
    in_place = dev(h)
    again = mx.norm(in_place, dev(parts), dev(gain), 1e-5)
    assert torch.equal(in_place, h_out)
    dropped = dev(h)
    third = mx.norm(dropped, dev(parts), dev(gain), 1e-5, keep=False)
    assert torch.equal(dropped.cpu(), h)
    for o in (again, third):
        assert torch.equal(o[0].view(torch.uint8), got[0].view(torch.uint8)) and torch.equal(o[1].view(torch.uint8), got[1].view(torch.uint8))


def test_norm_of_zero_and_not_finite_rows(mx):
    h = rand(3, 5, 256).float()
    h[1] = 0
    h[2, 17] = math.nan
    h[3, 200] = math.inf                              # inf / inf in that channel, zeros elsewhere
    got = mx.norm(h.cuda(), None, torch.ones(256, device="cuda"), 1e-5)
    s, codes = P.row_scales(got[1], 5, 8), P.unpack(got[0], 8)
    assert (codes[1] == 0).all() and (s[1] == 0).all()
    assert (s[2] == 255).all()
    assert s[3, 6] == 255 and (s[3, :6] == 0).all() and (codes[3] % 128 == 0).all()
    assert (s[[0, 4]] < 255).all()
    # a mean square of zero with eps = 0: 0 / 0
    got = mx.norm(torch.zeros(2, 64, device="cuda"), None, torch.ones(64, device="cuda"), 0.0)
    assert (P.row_scales(got[1], 2, 2) == 255).all()


# ---------------------------------------------------------------- linear
def operands(seed, M, N, K, fill=127):
    x, xv = P.form(rand(seed, M, K) * torch.exp(0.5 * rand(seed + 1, 1, K)), 8, fill)
    w, wv = P.form(rand(seed + 2, N, K, std=0.02), 4, fill)
    return cuda(x), xv, cuda(w), wv


# K: one block, an odd number of blocks, ends inside a step, a group and a chunk, k-slices (from 2048 on) of unequal length; M around
# tiles and passes; N odd, not a multiple of four, of 32
SHAPES = [(1, 1, 32), (1, 32, 64), (5, 33, 96), (31, 45, 160), (32, 64, 256), (33, 70, 288), (45, 130, 512), (64, 96, 992), (1, 128, 2048),
          (40, 100, 2080), (65, 64, 2176), (97, 200, 320), (129, 160, 4096), (160, 97, 544), (161, 64, 2400), (193, 320, 768), (257, 130, 224), (2, 9, 18944)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(mx, M, N, K):
    x, xv, w, wv = operands(M * 7 + N * 3 + K, M, N, K, fill=255)     # what only fills up is not read
    want, off = xv @ wv.T, P.step_error(xv, wv)
    got = mx.linear(x, w, "fp32")
    assert got.dtype == torch.float32
    err = (got.cpu().double() - want).abs()
    assert (err <= off).all(), float((err / off).max())
    half = mx.linear(x, w, "bf16").cpu().double()
    assert ((half - want).abs() <= off + (want.abs() + off) * 2.0 ** -8).all()


@pytest.mark.parametrize("M,F,K", [(1, 32, 32), (3, 64, 96), (33, 96, 256), (45, 160, 512), (64, 32, 4096), (160, 256, 544), (161, 128, 320), (200, 384, 288)])
def test_linear_channels(mx, M, F, K):
    x, xv, w, wv = operands(M + F + K, M, 2 * F, K, fill=255)
    y, off = xv @ wv.T, P.step_error(xv, wv)
    g, u, og, ou = y[:, :F], y[:, F:], off[:, :F], off[:, F:]
    want = P.silu(g) * u
    # silu's slope is at most 1.1; its hardware exponential and reciprocal are good to 2^-20
    P.check_fp8(mx.linear(x, w, "swiglu"), want, 1.1 * og * (u.abs() + ou) + P.silu(g).abs() * ou + want.abs() * 2.0 ** -20)


@pytest.mark.parametrize("N,K", [(96, 512), (130, 2112), (256, 288)])
def test_rows_do_not_depend_on_the_others(mx, N, K):
    """A row's bits are the same in every call: what makes a batched verification agree with stepwise decoding."""
    x, _, w, _ = operands(3, 700, N, K)
    for result in ("fp32", "bf16") + (("swiglu",) if N % 64 == 0 else ()):
        take = lambda o: torch.cat([o[0].view(torch.uint8), o[1].view(torch.uint8).transpose(0, 1)[:o[0].shape[0]].reshape(o[0].shape[0], -1)[:, :o[0].shape[1] // 32]], 1) if isinstance(o, tuple) else o  # noqa: E731
        whole = take(mx.linear(x, w, result))
        for a, b in ((0, 1), (0, 32), (5, 45), (32, 97), (100, 140), (64, 224), (0, 193), (300, 620), (699, 700)):
            codes, s = x[0][a:b].contiguous(), x[1].view(torch.uint8)
            part = P.lay_scales(P.row_scales(s, 700, K // 32)[a:b]).cuda().view(torch.float8_e8m0fnu)
            assert torch.equal(take(mx.linear((codes, part), w, result)), whole[a:b]), (result, a, b)


def test_linear_not_a_number(mx):
    """A NaN scale reaches the outputs of its row or its column and no others."""
    x, _, w, _ = operands(11, 40, 96, 256)
    x[1].view(torch.uint8)[1, 7, 2] = 255              # row 7, block 6
    w[1].view(torch.uint8)[0, 50, 1] = 255             # output 50, block 1
    y = mx.linear(x, w, "fp32").cpu()
    nan = torch.isnan(y)
    want = torch.zeros(40, 96, dtype=torch.bool)
    want[7], want[:, 50] = True, True
    assert torch.equal(nan, want)


# ---------------------------------------------------------------- streams, graphs, workspaces
@pytest.mark.parametrize("M,N,K", [(40, 128, 2304), (300, 4096, 2304), (9000, 130, 2304)])      # slices beside and behind each other; partial sums in the workspace
def test_streams_and_graphs(mx, M, N, K):
    """On a stream of the caller's, captured and replayed with new operands in the same buffers, between eager calls."""
    st = torch.cuda.Stream()
    h = torch.empty(M, K, device="cuda")
    gain = torch.ones(K, device="cuda")
    w = cuda(P.form(rand(1, N, K, std=0.02), 4)[0])
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    form = mx.empty(M, K, mx.FP8, "cuda")
    ws = torch.empty(mx.linear_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0

    def chain():
        mx.norm(h, None, gain, 1e-5, out=form)
        mx.linear(form, w, "bf16", out=out, workspace=ws)

    def eager(src):
        return mx.linear(mx.norm(src, None, gain, 1e-5), w, "bf16").clone()

    srcs = [rand(20 + i, M, K).float().cuda() for i in range(4)]
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        h.copy_(srcs[0])
        chain()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        chain()
    for src in srcs:
        want = eager(src)
        h.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ---------------------------------------------------------------- refusals that need tensors
def test_refusals(mx):
    from paper_2510_04147_amd.binding import SsdError
    x = torch.zeros(4, 64, device="cuda")
    f = mx.quantize(x, 8)
    w = mx.quantize(torch.zeros(64, 64, device="cuda"), 4)
    bad = [lambda: mx.quantize(x.half(), 8), lambda: mx.quantize(x[:, :40].contiguous(), 8), lambda: mx.quantize(x.t(), 8),
           lambda: mx.quantize(torch.zeros(64, 4, device="cuda").t(), 8), lambda: mx.quantize(x, 6), lambda: mx.quantize(x.cpu(), 8),
           lambda: mx.quantize(x[:0], 8), lambda: mx.norm(x, x[None, :2], torch.ones(64, device="cuda"), 1e-5), lambda: mx.quantize(x, 8, values=x.bfloat16()),
           lambda: mx.norm(x, x, torch.ones(64, device="cuda"), 1e-5), lambda: mx.norm(x, None, torch.ones(32, device="cuda"), 1e-5),
           lambda: mx.norm(x.double(), None, torch.ones(64, device="cuda"), 1e-5),
           lambda: mx.linear(f, f, "bf16"), lambda: mx.linear(w, w, "bf16"), lambda: mx.linear(f, w, "int8"), lambda: mx.linear(f, (w[0][:32], w[1]), "bf16"),
           lambda: mx.linear(f, w, "bf16", out=torch.zeros(4, 64, device="cuda")), lambda: mx.linear((f[0], f[1][:, :4]), w, "bf16"),
           lambda: mx.linear(f, mx.quantize(torch.zeros(96, 64, device="cuda"), 4), "swiglu")]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")
    odd = torch.zeros(4 * 64 + 1, device="cuda")[1:].view(4, 64)      # four bytes off a 16-byte boundary
    with pytest.raises(SsdError, match="16-byte"):
        mx.quantize(odd, 8)
    with pytest.raises(SsdError, match="at most 8192"):
        mx.norm(torch.zeros(1, 8224, device="cuda"), None, torch.ones(8224, device="cuda"), 1e-5)
    with pytest.raises(SsdError, match="eps"):
        mx.norm(x, None, torch.ones(64, device="cuda"), -1.0)
    big = mx.quantize(torch.zeros(1, 2048, device="cuda"), 8), mx.quantize(torch.zeros(64, 2048, device="cuda"), 4)
    with pytest.raises(SsdError, match="workspace") as e:
        mx.linear(*big, "bf16", workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3
