"""Every tile shape of the microscaled product, at sizes that end inside its tiles, chunks and steps (test_mx_rules.py checks that
they are taken)."""
import pytest
import torch

import mx_plain as P

# shape, rows, weight rows, columns, result.  Rows no multiple of 32, results (but for activated channels) of no multiple of four,
# columns that end in half a step; from 2048 columns on partial sums
SIZES = [(0, 5, 1, 160, "fp32"), (0, 5, 1, 160, "bf16"), (0, 2, 5, 2464, "fp32"), (1, 124, 237, 96, "fp32"), (1, 124, 237, 96, "bf16"), (1, 334, 163, 2336, "fp32"),
         (2, 363, 829, 96, "fp32"), (2, 363, 829, 96, "bf16"), (2, 1039, 75, 2400, "fp32"), (3, 65, 8273, 96, "fp32"), (3, 65, 8273, 96, "bf16"),
         (3, 1, 4098, 2336, "bf16"), (4, 261, 6545, 96, "fp32"), (4, 261, 6545, 96, "bf16"), (4, 67, 4194, 2400, "fp32"), (5, 296, 8323, 96, "fp32"),
         (5, 296, 8323, 96, "bf16"), (5, 198, 8256, 480, "swiglu"), (5, 289, 2729, 2208, "bf16"), (6, 1197, 2822, 96, "fp32"), (6, 1197, 2822, 96, "bf16"),
         (6, 135, 5429, 2144, "fp32"), (6, 604, 8512, 544, "swiglu"), (7, 1029, 7221, 96, "fp32"), (7, 1029, 7221, 96, "bf16"), (7, 263, 7367, 2080, "fp32"),
         (8, 1290, 8231, 96, "fp32"), (8, 1290, 8231, 96, "bf16"), (8, 524, 5418, 2144, "fp32"), (8, 1346, 8256, 96, "swiglu"),
         (9, 1370, 271, 2336, "fp32"), (10, 130, 4153, 2336, "fp32"), (11, 259, 5629, 2336, "fp32"), (11, 259, 5629, 2336, "bf16"),
         (12, 2, 64, 288, "swiglu"), (13, 198, 2368, 736, "swiglu"), (14, 1, 64, 96, "swiglu"), (15, 195, 8448, 416, "swiglu"), (15, 193, 8448, 96, "swiglu"), (16, 129, 21824, 736, "swiglu"),
         (17, 594, 8384, 96, "swiglu"),
         # several chunks and an end
         (0, 1, 1, 736, "fp32"), (1, 193, 1154, 736, "bf16"), (2, 1399, 323, 736, "fp32"), (3, 65, 8321, 736, "bf16"), (4, 195, 8197, 736, "fp32"), (5, 291, 8255, 736, "bf16"),
         (6, 386, 8297, 736, "fp32"), (7, 1544, 4877, 736, "bf16"), (8, 1286, 8067, 736, "fp32"), (5, 193, 8256, 736, "swiglu"), (6, 577, 8320, 736, "swiglu"),
         (8, 1155, 9408, 736, "swiglu"), (14, 264, 1920, 736, "swiglu"), (15, 390, 4672, 736, "swiglu"), (5, 1220, 3136, 736, "swiglu"), (16, 161, 24000, 1248, "swiglu"), (17, 897, 6592, 736, "swiglu"),
         # three and four slices, two of them joined by the kernel, partial sums by another
         (9, 5000, 130, 4128, "fp32"), (10, 8000, 130, 2336, "fp32"), (11, 8000, 324, 2336, "fp32")]
# Products whose slices share a work-group: kind (mx_choose_all), rows, weight rows, columns, result; three and four slices, ends inside a
# chunk and inside a step, rows of outputs that are no multiple of four, rows past a tile
ALL = [(0, 1, 4096, 4096, "bf16"), (0, 1, 33, 2048, "fp32"), (0, 5, 65, 2304, "bf16"), (0, 31, 2047, 2080, "fp32"), (0, 32, 8191, 2048, "bf16"), (2, 65, 4097, 2336, "fp32"),
       (0, 7, 1, 3104, "bf16"), (0, 1039, 75, 2400, "bf16"), (1, 33, 4097, 2336, "bf16"), (1, 64, 8191, 2048, "fp32"), (1, 129, 2047, 2080, "bf16"), (2, 37, 8190, 4128, "fp32"),
       (2, 300, 2047, 2080, "bf16"), (3, 131, 5465, 2336, "bf16"), (3, 300, 4097, 2336, "fp32"), (4, 257, 6532, 2336, "bf16"), (4, 1000, 4096, 4096, "fp32"),
       (4, 524, 5418, 2144, "fp32")]


def bits(o):
    """Rows of a result as comparable tensors."""
    if not isinstance(o, tuple):
        return o
    rows, cols = o[0].shape
    return torch.cat([o[0].view(torch.uint8), o[1].view(torch.uint8).transpose(0, 1).reshape(o[1].shape[1], -1)[:rows, :cols // 32]], 1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,M,N,K,result", SIZES + ALL)
def test_shape(kind, M, N, K, result):
    """All rows against calls of few rows, which take other shapes and must give the same bits, and some rows against 64 bits."""
    from paper_2510_04147_amd import mx
    g = torch.Generator().manual_seed(M + N + K)
    x, xv = P.form(torch.randn(M, K, generator=g, dtype=torch.float64) * torch.exp(0.5 * torch.randn(K, generator=g, dtype=torch.float64)), 8)
    w4 = mx.quantize((torch.randn(N, K, generator=g) * 0.02).cuda(), mx.FP4)
    x = tuple(t.cuda() for t in x)
    whole = mx.linear(x, w4, result)
    if result == "swiglu":
        assert (P.padding(whole[1], M, N // 64) == 127).all()
    whole = bits(whole)
    s = P.row_scales(x[1], M, K // 32)
    for a in range(0, M, 40 if M > 40 else 1):
        part = (x[0][a:a + 40].contiguous(), P.lay_scales(s[a:a + 40]).view(torch.float8_e8m0fnu).cuda())
        assert torch.equal(bits(mx.linear(part, w4, result)), whole[a:a + 40]), a
    if result != "swiglu":
        rows = sorted({0, M // 2, M - 1})
        wv = P.values(P.unpack(w4[0], 4), P.row_scales(w4[1], N, K // 32), 4)
        want, off = xv[rows] @ wv.T, P.step_error(xv[rows], wv)
        off = off if result == "fp32" else off + (want.abs() + off) * 2.0 ** -8
        assert ((whole[rows].cpu().double() - want).abs() <= off).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 50, 300, 1000, 2304])
@pytest.mark.parametrize("N,K", [(2047, 2080), (4097, 2336), (8191, 2048), (4096, 4096)])
def test_slices_in_a_work_group_equal_slices_apart(rows, N, K):
    """Rows whose slices share a work-group against the same rows among 9000, whose partial sums a second kernel adds."""
    from paper_2510_04147_amd import mx
    g = torch.Generator().manual_seed(N + K + rows)
    w = mx.quantize((torch.randn(N, K, generator=g) * 0.02).cuda(), mx.FP4)
    x = torch.randn(rows, K, generator=g).cuda()
    many = x.repeat(9000 // rows + 1, 1)[:9000].contiguous()
    for result in ("fp32", "bf16"):
        few = mx.linear(mx.quantize(x, mx.FP8), w, result)
        among = mx.linear(mx.quantize(many, mx.FP8), w, result)
        assert torch.equal(among[:rows], few) and torch.equal(among[9000 // rows * rows - rows:9000 // rows * rows], few)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,weights", [((1 << 20) - 3, 33), (3, (1 << 20) - 5)])
def test_operands_past_32_bits(rows, weights):
    """Codes of more than 4 GiB on either side: the last rows against a call of their own."""
    from paper_2510_04147_amd import mx
    K = 8224 if rows > weights else 8224 * 2
    gen = torch.Generator("cuda").manual_seed(1)

    def random_form(n, bits):
        codes, scales = mx.empty(n, K, bits, "cuda")
        c = codes.view(torch.uint8)
        for a in range(0, n, 1 << 17):                 # no NaN among the 8-bit codes: exponents below the last
            c[a:a + (1 << 17)] = torch.randint(0, 256, c[a:a + (1 << 17)].shape, generator=gen, device="cuda", dtype=torch.uint8) & (0xb7 if bits == 8 else 0xff)
        scales.view(torch.uint8).random_(120, 130, generator=gen)
        return codes, scales

    x, w = random_form(rows, 8), random_form(weights, 4)
    assert max(x[0].numel(), w[0].numel()) > 1 << 32
    whole = mx.linear(x, w, "bf16")
    for a, b in ((0, 3), (rows - 3, rows)):
        part = (x[0][a:b].contiguous(), P.lay_scales(P.row_scales(x[1][:, a // 32 * 32:].contiguous(), b - a // 32 * 32, K // 32)[a % 32:]).view(torch.float8_e8m0fnu).cuda())
        assert torch.equal(mx.linear(part, w, "bf16"), whole[a:b])
        for c, d in ((0, 40), (weights - 40 + weights % 4, weights)) if weights > 40 else ():
            four = (w[0][c:d].contiguous(), P.lay_scales(P.row_scales(w[1][:, c // 32 * 32:].contiguous(), d - c // 32 * 32, K // 32)[c % 32:]).view(torch.float8_e8m0fnu).cuda())
            # fewer weight rows are cut into more slices: the same sums in another order
            near = mx.linear(part, four, "bf16").float()
            assert torch.allclose(near, whole[a:b, c:d].float(), rtol=2.0 ** -7, atol=2.0 ** -7 * float(near.abs().max()))
