"""SwiGLU of the microscaled product where the gate is far below zero."""
import pytest
import torch

import mx_plain as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 40, 200])
def test_far_gates(M):
    """One product per sum, exact: gates of -6 x, channels of 6 x.  Down to -84 as everywhere; from -90 on 0 with the scale of a block of
    zeros."""
    from paper_2510_04147_amd import mx
    x = torch.zeros(M, 32, dtype=torch.float64)
    x[:, 0] = torch.tensor([1.0, 12.0, 14.0, 15.0, 16.0, 20.0, 448.0], dtype=torch.float64).repeat(M)[:M]
    w = torch.zeros(64, 32, dtype=torch.float64)
    w[:32, 0], w[32:, 0] = -6.0, 6.0
    form, xv = P.form(x, 8)
    four, wv = P.form(w, 4)
    assert torch.equal(xv, x) and torch.equal(wv, w)
    got = mx.linear(tuple(t.cuda() for t in form), tuple(t.cuda() for t in four), "swiglu")
    gate, up = -6 * x[:, :1], 6 * x[:, :1]
    want = (P.silu(gate) * up).repeat(1, 32)
    far = x[:, 0] >= 15
    near = ~far
    s, v = P.row_scales(got[1], M, 1), P.values(P.unpack(got[0], 8), P.row_scales(got[1], M, 1), 8)
    # e^-g as 2^(-g log2 e): the constant's and the product's roundings, 2^-24 of an exponent of |g| log2 e, change the result by |g| 2^-24
    # each; exponential and reciprocal a unit (2^-23) each, sum and two products 2^-24 each: within (|g| + 4) 2^-23
    off = want.abs() * (gate.abs() + 4) * 2.0 ** -23
    lo, hi = P.scale_codes(want.abs() - off, 8), P.scale_codes(want.abs() + off, 8)
    assert ((s >= lo) & (s <= hi))[near].all()
    assert ((v - want).abs() <= P.half_step(want.abs() + off, s) + off)[near].all() and (v[near] != 0).all()
    assert (v[far] == 0).all() and (s[far] == 0).all()
