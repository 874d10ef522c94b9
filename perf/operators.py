"""Performance cases of the microscaled operators: what a program that decodes with 4-bit weights asks of them, call by call.

  quantize  rows to microscaled form: weights to 4 bits (e2m1) when a model is loaded, activations to 8 bits (e4m3)
  norm      the residual's addition and RMSNorm in front of a projection, with an output in 8 bits and scales
  linear    the projection itself, 8-bit activations times 4-bit weights: bf16 results, or the activated
            channels silu(gate) * up in 8 bits and scales, ready for the next projection

Blocks of 32 values of a row share one scale, a power of two in 8 bits (E8M0).  Scales lie in groups of four blocks
(128 columns): [groups, rows rounded up to 32, 4]; what pads rows and groups is 1.0.  Sizes are those of the models of synth.py
(8B and 7B class) and of the small bf16 model of the tests; the rows of a call are nodes times block length.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def case(op, rows, cols, name=None, **more):
    c = dict(op=op, rows=rows, cols=cols, **more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # attention output of one block of the paper's decoding shape, in front of the output projection: latency
        case("quantize", 8, 4096, source="bf16", bits=8, values=False, name="quantize_attention_8_rows"),
        # the same for a long prompt of a small fp32 model, no multiple of a tile
        case("quantize", 4097, 1504, source="fp32", bits=8, values=False, name="quantize_prompt_fp32"),
        # a gate/up matrix of the 7B class at load time, with the rounded values to compare with
        case("quantize", 37888, 3584, source="bf16", bits=4, values=True, name="quantize_weights_gate_up_7b"),
        # first norm of a stepwise forward, nothing to add
        case("norm", 8, 4096, partials=0, name="norm_8_rows"),
        # verification forward of the 8B class behind the down projection, four partial sums
        case("norm", 160, 4096, partials=4, name="norm_160_rows"),
        # the largest forward of the 7B class
        case("norm", 2304, 3584, partials=2, name="norm_2304_rows"),
        # a single token through an output projection
        case("linear", 1, 4096, outs=4096, result="bf16", name="linear_one_token"),
        # odd rows, a small model's vocabulary
        case("linear", 45, 512, outs=2080, result="bf16", name="linear_small_45_rows"),
        # down projection, the paper's decoding shape: 5 nodes of a block of 8
        case("linear", 40, 12288, outs=4096, result="bf16", name="linear_down_40_rows"),
        # gate/up of the headline workload: 5 nodes of a block of 32
        case("linear", 160, 4096, outs=24576, result="swiglu", name="linear_gate_up_160_rows"),
        # query, key and value projections of a 1000-token prompt
        case("linear", 1000, 4096, outs=12288, result="bf16", name="linear_qkv_prompt"),
        # gate/up of the largest forward: eight sequences, nine nodes of 32 rows
        case("linear", 2304, 3584, outs=37888, result="swiglu", name="linear_gate_up_2304_rows"),
    ]


def _log_int(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng: random.Random):
    op = rng.choice(["quantize", "norm", "linear", "linear"])
    if op == "quantize":
        cols = 32 * _log_int(rng, 4, 592)
        rows = _log_int(rng, 1, min(37888, 130_000_000 // cols))
        bits = rng.choice([4, 8])
        return case(op, rows, cols, source=rng.choice(["bf16", "fp32"]), bits=bits, values=bits == 4)
    if op == "norm":
        return case(op, _log_int(rng, 1, 2304), 32 * _log_int(rng, 8, 192), partials=rng.choice([0, 1, 2, 4]))
    rows, cols = _log_int(rng, 1, 2304), 32 * _log_int(rng, 8, 592)
    outs = _log_int(rng, 128, min(37888, 135_000_000 // cols))
    result = rng.choice(["bf16", "swiglu"])
    return case(op, rows, cols, outs=max(64, outs // 64 * 64) if result == "swiglu" else outs, result=result)


# ------------------------------------------------------------------ plain forms
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _lay_scales(s):
    """Scale codes [rows, blocks] (uint8) in the order the operators keep them: [groups, rows rounded up, 4]."""
    rows, blocks = s.shape
    t = torch.full(((rows + 31) // 32 * 32, (blocks + 3) // 4 * 4), 127, dtype=torch.uint8, device=s.device)
    t[:rows, :blocks] = s
    return t.view(t.shape[0], -1, 4).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu)


def _quantize(x, bits):
    """x fp32 [rows, cols] -> elements in units of their block's scale (fp32), scale codes [rows, blocks]."""
    b = x.view(x.shape[0], -1, 32)
    big = b.abs().amax(-1)
    # the scale: a power of two for which the largest element rounds to a finite one, 6 of e2m1 (up to 7, excluded) or
    # 448 of e4m3 (up to 464): the exponent, one more where the fraction is past that
    past, emax = (0x200000, 2) if bits == 4 else (0x17FFFF, 8)
    code = (((big.view(torch.int32) + past) >> 23) - emax).clamp(min=0)
    bad = ~torch.isfinite(big)
    code = torch.where(bad, 255, code)
    v = b * ((254 - code.clamp(max=253)) << 23).view(torch.float32)[..., None]
    v = torch.where(bad[..., None], 0.0, v)
    if bits == 4:
        step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
        v = torch.round(v / step) * step
    else:
        v = v.to(torch.float8_e4m3fn).float()
    return v.view(x.shape), code.to(torch.uint8)


def _powers(code):
    """2^(code - 127), from the bits: a library's exponential need not be exact."""
    p = torch.where(code == 0, 2.0 ** -127, (code.int() << 23).view(torch.float32))
    return torch.where(code == 255, math.nan, p)


def _pack4(v):
    """e2m1 values -> codes, two to a byte, the first in the low half."""
    code = torch.bucketize(v.abs(), torch.tensor(E2M1[1:], device=v.device), right=True) + 8 * torch.signbit(v)
    code = code.to(torch.uint8).view(v.shape[0], -1, 2)
    return code[..., 0] | (code[..., 1] << 4)


def _unpack4(codes):
    table = torch.tensor(E2M1 + tuple(-t for t in E2M1), device=codes.device)
    both = torch.stack([table.repeat(16), table.repeat_interleave(16)], -1)
    return both[codes.int()].view(codes.shape[0], -1)


def _row_scales(s, rows, blocks):
    return s.view(torch.uint8).transpose(0, 1).reshape(s.shape[1], -1)[:rows, :blocks]


def _fp32_of(values, s):
    rows, cols = values.shape
    return (values.view(rows, -1, 32) * _powers(_row_scales(s, rows, cols // 32))[..., None]).view(rows, cols)


def _plain_quantize(s):
    x = s["x"].float()
    v, code = _quantize(x, s["case"]["bits"])
    if s["case"]["values"]:
        return {"values": (v.view(x.shape[0], -1, 32) * _powers(code)[..., None]).view(x.shape).to(s["x"].dtype),
                "codes": _pack4(v), "scales": _lay_scales(code)}
    return {"codes": v.to(torch.float8_e4m3fn), "scales": _lay_scales(code)}


def _plain_norm(s):
    h = s["h"]
    if s["partials"] is not None:
        p = s["partials"]
        half = (p.shape[0] + 1) // 2
        h = h + (p[:half].sum(0) + p[half:].sum(0))
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["gain"]
    v, code = _quantize(y, 8)
    return {"h": h, "codes": v.to(torch.float8_e4m3fn), "scales": _lay_scales(code)}


def _plain_linear(s):
    c = s["case"]
    y = _fp32_of(s["x"][0].float(), s["x"][1]) @ _fp32_of(_unpack4(s["w"][0]), s["w"][1]).T
    if c["result"] == "bf16":
        return y.bfloat16()
    gate, up = y.chunk(2, -1)
    v, code = _quantize(gate / (1 + torch.exp(-gate)) * up, 8)
    return {"codes": v.to(torch.float8_e4m3fn), "scales": _lay_scales(code)}


# ------------------------------------------------------------------ the calls
def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def _activations(gen, rows, cols):
    """Normed rows: unit size, some channels several times larger than the others."""
    return _normal(gen, rows, cols) * torch.exp(0.5 * _normal(gen, cols))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, cols = case["rows"], case["cols"]
    s = dict(case=case)
    if case["op"] == "quantize":
        x = _normal(gen, rows, cols, std=0.02) if case["bits"] == 4 else _activations(gen, rows, cols)
        s["x"] = x.to(torch.float32 if case["source"] == "fp32" else torch.bfloat16)
    elif case["op"] == "norm":
        n = case["partials"]
        s["h"] = _activations(gen, rows, cols)
        s["partials"] = _normal(gen, n, rows, cols, std=0.5) if n else None
        s["gain"] = 1 + 0.1 * _normal(gen, cols)
        s["eps"] = 1e-5
    else:
        v, code = _quantize(_activations(gen, rows, cols), 8)
        s["x"] = (v.to(torch.float8_e4m3fn), _lay_scales(code))
        v, code = _quantize(_normal(gen, case["outs"], cols, std=0.02), 4)
        s["w"] = (_pack4(v), _lay_scales(code))
    # the buffers that a decoding program keeps for the results
    empty = lambda *shape, dt: torch.empty(*shape, dtype=dt, device="cuda")  # noqa: E731
    form = lambda rows, cols, bits=8: (empty(rows, cols * bits // 8, dt=torch.float8_e4m3fn if bits == 8 else torch.uint8),  # noqa: E731
                                       empty((cols + 127) // 128, (rows + 31) // 32 * 32, 4, dt=torch.float8_e8m0fnu))
    if case["op"] == "quantize":
        s["out"] = form(rows, cols, case["bits"])
        s["values"] = torch.empty_like(s["x"]) if case["values"] else None
    elif case["op"] == "norm":
        s["out"] = form(rows, cols)
        s["sum"] = torch.empty_like(s["h"]) if case["partials"] else None
    elif case["result"] == "swiglu":
        s["out"] = form(rows, case["outs"] // 2)
    else:
        s["out"] = empty(rows, case["outs"], dt=torch.bfloat16)
    return s


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"quantize": _plain_quantize, "norm": _plain_norm, "linear": _plain_linear}[op](s)
    from paper_2510_04147_amd import mx
    if op == "quantize":
        codes, scales = mx.quantize(s["x"], s["case"]["bits"], values=s["values"], out=s["out"])
        return {"codes": codes, "scales": scales} if s["values"] is None else {"values": s["values"], "codes": codes, "scales": scales}
    if op == "norm":
        codes, scales = mx.norm(s["h"], s["partials"], s["gain"], s["eps"], h_out=s["sum"], out=s["out"])
        return {"h": s["h"] if s["sum"] is None else s["sum"], "codes": codes, "scales": scales}
    out = mx.linear(s["x"], s["w"], s["case"]["result"], out=s["out"])
    return {"codes": out[0], "scales": out[1]} if s["case"]["result"] == "swiglu" else out


def work(case):
    rows, cols, op = case["rows"], case["cols"], case["op"]
    if op == "quantize":
        e = 4 if case["source"] == "fp32" else 2
        return dict(bytes=rows * cols * (e + case["bits"] / 8 + 1 / 32 + (e if case["values"] else 0)), flops=3 * rows * cols)
    if op == "norm":
        return dict(bytes=rows * cols * (4 + 4 * case["partials"] + 4 + 1 + 1 / 32) + 4 * cols, flops=(7 + case["partials"]) * rows * cols)
    outs = case["outs"]
    result = 2 * outs if case["result"] == "bf16" else outs / 2 * (1 + 1 / 32)
    return dict(bytes=outs * cols * (1 / 2 + 1 / 32) + rows * cols * (1 + 1 / 32) + rows * result, flops=2 * rows * outs * cols)


# ------------------------------------------------------------------ in 64 bits
def _grid(bits):
    """Every value an element can have, in ascending order."""
    if bits == 4:
        pos = list(E2M1)
    else:
        pos = [m / 512 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]
    return torch.tensor([-p for p in reversed(pos[1:])] + pos, dtype=torch.float64, device="cuda")


def _exact_blocks(x, bits):
    """x in 64 bits -> the nearest elements (ties to the even code) and the scales, as numbers."""
    rows, cols = x.shape
    b = x.view(rows, -1, 32)
    big = b.abs().amax(-1)
    grid = _grid(bits)
    top = grid[-1]
    last = top + (2.0 if bits == 4 else 32.0) / 2           # half a step past the largest element: odd and even code
    m, e = torch.frexp(big)                                 # big = m 2^e, m in [1/2, 1)
    unit = e - (3 if bits == 4 else 9)
    over = m * (8 if bits == 4 else 512)                    # big in units of 2^unit
    unit = torch.where((over >= last) if bits == 4 else (over > last), unit + 1, unit).clamp(min=-127)
    unit = torch.where(big == 0, -127, unit)
    scale = ((unit.long() + 1023) << 52).view(torch.float64)
    v = b / scale[..., None]
    hi = torch.searchsorted(grid, v.contiguous()).clamp(1, grid.numel() - 1)
    below, above = grid[hi - 1], grid[hi]
    nearer = (v - below) - (above - v)
    even = (hi - (grid.numel() // 2)).abs() % 2 == 0        # codes count from zero, which lies in the middle
    v = torch.where((nearer > 0) | ((nearer == 0) & even), above, below)
    return v.view(rows, cols), scale


def _exact_scales(scale):
    rows, blocks = scale.shape
    t = torch.ones((rows + 31) // 32 * 32, (blocks + 3) // 4 * 4, dtype=torch.float64, device=scale.device)
    t[:rows, :blocks] = scale
    return t.view(t.shape[0], -1, 4).transpose(0, 1).contiguous()


def _exact_product(s):
    """The product in 64 bits, a slice of the weights at a time."""
    def wide(values, scales):
        rows, cols = values.shape
        by_row = scales.double().permute(1, 0, 2).reshape(scales.shape[1], -1)[:rows, :cols // 32]
        return values.double() * by_row.repeat_interleave(32, 1)

    x, codes, scales = wide(*s["x"]), *s["w"]
    parts = []
    for n0 in range(0, codes.shape[0], 4096):
        part = codes[n0:n0 + 4096]
        elements = torch.stack([part & 15, part >> 4], -1).view(part.shape[0], -1)
        magnitude = torch.tensor(E2M1, dtype=torch.float64, device="cuda")[(elements & 7).int()]
        w = wide(torch.where(elements >= 8, -magnitude, magnitude), scales[:, n0:n0 + 4096])
        parts.append(x @ w.T)
    return torch.cat(parts, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        v, scale = _exact_blocks(s["x"].double(), case["bits"])
        if case["values"]:
            return {"values": v * scale.repeat_interleave(32, 1), "codes": None, "scales": _exact_scales(scale)}
        return {"codes": v, "scales": _exact_scales(scale)}
    if case["op"] == "norm":
        h = s["h"].double()
        if s["partials"] is not None:
            h = h + s["partials"].double().sum(0)
        v, scale = _exact_blocks(h / torch.sqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["gain"].double(), 8)
        return {"h": h, "codes": v, "scales": _exact_scales(scale)}
    y = _exact_product(s)
    if case["result"] != "swiglu":
        return y
    half = y.shape[1] // 2
    v, scale = _exact_blocks(torch.sigmoid(y[:, :half]) * y[:, :half] * y[:, half:], 8)
    return {"codes": v, "scales": _exact_scales(scale)}
