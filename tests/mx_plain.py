"""The microscaled form and its operators in 64 bits, from their definitions: what the GPU tests compare with.  CPU only."""
import torch

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
E4M3 = [m / 512 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]
GRID = {4: torch.tensor(E2M1, dtype=torch.float64), 8: torch.tensor(E4M3, dtype=torch.float64)}


def scale_codes(x, bits):
    """Codes of the scales of x (float64 [rows, cols]): the smallest power of two, at least 2^-127, for which the block's largest value
    is nearest to an element of the format (a tie past the largest element would go to the even one, 8 or 448)."""
    big = x.view(x.shape[0], -1, 32).abs().amax(-1)
    border, open_ = (7.0, True) if bits == 4 else (464.0, False)
    code = torch.zeros(big.shape, dtype=torch.long)
    for s in range(254, -1, -1):                      # the largest code that is still too small, plus one
        v = big * 2.0 ** (127 - s)
        past = v >= border if open_ else v > border
        code = torch.where((code == 0) & past, s + 1, code)
    return torch.where(torch.isfinite(big), code, 255)


def nearest(v, bits):
    """v (float64) to the nearest element, ties to the even code -> codes without sign."""
    g = GRID[bits]
    a = v.abs()
    hi = torch.searchsorted(g, a.contiguous()).clamp(1, len(g) - 1)
    below, above = a - g[hi - 1], g[hi] - a
    return torch.where((below < above) | ((below == above) & ((hi - 1) % 2 == 0)), hi - 1, hi)


def quantize(x, bits):
    """-> element codes with sign [rows, cols], scale codes [rows, blocks], values, all of float64 x."""
    rows, cols = x.shape
    s = scale_codes(x, bits)
    bad = (s == 255)[..., None]
    b = torch.where(bad, 0.0, x.view(rows, -1, 32) * torch.pow(torch.tensor(2.0, dtype=torch.float64), (127 - s.clamp(max=254)).double())[..., None])
    mag = nearest(b, bits)
    codes = mag + torch.signbit(b) * (8 if bits == 4 else 128)
    return codes.view(rows, cols), s, values(codes.view(rows, cols), s, bits)


def values(codes, s, bits):
    rows, cols = codes.shape
    sign = 8 if bits == 4 else 128
    v = GRID[bits][(codes % sign).clamp(max=len(GRID[bits]) - 1)] * torch.where(codes >= sign, -1.0, 1.0)
    p = torch.pow(torch.tensor(2.0, dtype=torch.float64), (s - 127).double())
    p = torch.where(s == 255, float("nan"), p)
    return (v.view(rows, -1, 32) * p[..., None]).view(rows, cols)


def lay_scales(s, fill=127):
    rows, blocks = s.shape
    t = torch.full(((rows + 31) // 32 * 32, (blocks + 3) // 4 * 4), fill, dtype=torch.uint8)
    t[:rows, :blocks] = s.to(torch.uint8)
    return t.view(t.shape[0], -1, 4).transpose(0, 1).contiguous()


def row_scales(t, rows, blocks):
    """[groups, rows rounded up, 4] -> codes [rows, blocks]"""
    u = t.cpu().view(torch.uint8)
    return u.transpose(0, 1).reshape(u.shape[1], -1)[:rows, :blocks].long()


def padding(t, rows, blocks):
    u = t.cpu().view(torch.uint8).transpose(0, 1)
    u = u.reshape(u.shape[0], -1)
    return torch.cat([u[rows:].flatten(), u[:rows, blocks:].flatten()])


def pack(codes, bits):
    if bits == 8:
        return codes.to(torch.uint8).view(torch.float8_e4m3fn)
    c = codes.to(torch.uint8).view(codes.shape[0], -1, 2)
    return c[..., 0] | (c[..., 1] << 4)


def unpack(t, bits):
    u = t.cpu().view(torch.uint8).long()
    return u if bits == 8 else torch.stack([u % 16, u // 16], -1).view(u.shape[0], -1)


def form(x, bits, fill=127):
    """float64 matrix -> (codes, scales) tensors as the operators take them, and the values they stand for"""
    codes, s, v = quantize(x, bits)
    return (pack(codes, bits), lay_scales(s, fill).view(torch.float8_e8m0fnu)), v


def step_error(x, w):
    """Bound on what the matrix instructions' own sums can be off by, [M, N]: the 64 products of a step are added 18 bits below the
    largest of them (so 64 x 2^-18 of it), the steps and partial sums in fp32 (2^-24 each, of the magnitudes so far)."""
    M, K = x.shape
    off = torch.zeros(M, w.shape[0], dtype=torch.float64)
    for k in range(0, K, 64):
        off += 64 * 2.0 ** -18 * (x[:, None, k:k + 64] * w[None, :, k:k + 64]).abs().amax(-1)
    steps = (K + 63) // 64 + 8
    return off + steps * 2.0 ** -24 * (x.abs() @ w.abs().T)


def silu(g):
    return g * torch.sigmoid(g)


def half_step(v, s):
    """Half a step of e4m3 at the values v under scale codes s, [rows, cols]."""
    p = torch.pow(torch.tensor(2.0, dtype=torch.float64), (s - 127).double()).repeat_interleave(32, 1)
    return torch.maximum(v.abs() * 2.0 ** -4, 2.0 ** -10 * p)


def check_fp8(got, want, off):
    """(codes, scales) of 8 bits against float64 `want`, itself known to `off`: every value within half a step, every scale that of
    a block maximum within `off`, the filling 127."""
    rows, cols = want.shape
    s = row_scales(got[1], rows, cols // 32)
    lo, hi = scale_codes((want.abs() - off).clamp(min=0), 8), scale_codes(want.abs() + off, 8)
    assert ((s >= lo) & (s <= hi)).all()
    v = values(unpack(got[0], 8), s, 8)
    bad = (v - want).abs() > half_step(want.abs() + off, s) + off
    assert not bad.any(), (int(bad.sum()), float((v - want).abs().max()))
    assert (padding(got[1], rows, cols // 32) == 127).all()
