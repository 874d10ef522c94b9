"""Products of three and four k-slices whose partial sums go through memory: every tile shape that leaves them, and the forwards of a
context whose projections have them, against the slices computed one by one (test_mx_partials_rules.py checks that the shapes are taken)."""
import numpy as np
import pytest
import torch

import mx_plain as P
from paper_2510_04147_amd import synth

# shape, slices, rows, weight rows, columns: no call of them is one launch, all of them leave partial sums that a second kernel adds
SIZES = [(0, 4, 3, 40, 6176), (1, 4, 257, 227, 8288), (2, 4, 326, 335, 10464), (3, 4, 386, 619, 8224), (4, 4, 643, 743, 7840), (5, 4, 986, 657, 9120),
         (6, 4, 1354, 729, 9184), (7, 4, 2727, 643, 6240), (8, 4, 533, 4168, 11168), (9, 4, 4724, 99, 3552), (10, 4, 6830, 131, 2464), (11, 4, 6872, 265, 2464),
         (5, 3, 8205, 105, 2080), (6, 3, 7458, 133, 2272), (7, 3, 7388, 282, 2272), (8, 3, 8213, 392, 2080), (9, 3, 10899, 259, 2080), (10, 3, 7460, 142, 2272),
         (11, 3, 7396, 300, 2272)]
ONE_SLICE_FROM = 8224                                  # weight rows: a matrix with more than 8192 is not cut


def slice_length(K):
    return (K + 1023) // 1024 * 256


def slices_apart(mx, x, w, M, N, K):
    """The partial sums of four slices (or as many as hold columns), each a product of its own that is not cut."""
    length, parts = slice_length(K), []
    for a in range(0, K, length):
        b = min(K, a + length)
        xs = (x[0].view(torch.uint8)[:, a:b].contiguous().view(torch.float8_e4m3fn), x[1].view(torch.uint8)[a // 128:(b + 127) // 128].contiguous().view(torch.float8_e8m0fnu))
        codes, scales = w[0][:, a // 2:b // 2].contiguous(), w[1].view(torch.uint8)[a // 128:(b + 127) // 128].contiguous()
        if b - a >= 2048:
            codes = torch.cat([codes, codes.new_zeros(ONE_SLICE_FROM - N, codes.shape[1])])
            scales = torch.cat([scales, scales.new_full((scales.shape[0], ONE_SLICE_FROM - scales.shape[1], 4), 127)], 1)
        parts.append(mx.linear(xs, (codes, scales.view(torch.float8_e8m0fnu)), "fp32")[:, :N])
    return torch.stack([p.contiguous() for p in parts])


def by_halves(parts):
    half = (len(parts) + 1) // 2
    sums = [p[0] + p[1] if len(p) == 2 else p[0] for p in (parts[:half], parts[half:])]
    return sums[0] + sums[1]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,slices,M,N,K", SIZES)
def test_partial_sums(kind, slices, M, N, K):
    """The sum of the slices by halves, bit for bit, and some rows against 64 bits."""
    from paper_2510_04147_amd import mx
    g = torch.Generator("cuda").manual_seed(M + N + K)
    x = mx.quantize(torch.randn(M, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(K, generator=g, device="cuda")), mx.FP8)
    w = mx.quantize(torch.randn(N, K, generator=g, device="cuda") * 0.02, mx.FP4)
    whole = mx.linear(x, w, "fp32")
    parts = slices_apart(mx, x, w, M, N, K)
    assert len(parts) == slices
    want = by_halves(parts)
    assert torch.equal(whole, want)
    assert torch.equal(mx.linear(x, w, "bf16"), want.bfloat16())
    rows = sorted({0, M // 2, M - 1})
    xv = P.values(P.unpack(x[0], 8), P.row_scales(x[1], M, K // 32), 8)[rows]
    wv = P.values(P.unpack(w[0], 4), P.row_scales(w[1], N, K // 32), 4)
    assert ((whole[rows].cpu().double() - xv @ wv.T).abs() <= P.step_error(xv, wv)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("seqs,block", [(1, 24), (1, 32), (1, 64), (2, 45), (3, 64), (5, 64)])
def test_a_forward_with_slices_is_its_operators(path, seqs, block):
    """The self-drafts of masked blocks behind cached prefixes in one forward, and every block's rows through the operators by hand, the
    projections' slices one by one: four of QKV and of the attention output, three of down.  The same bits on both kernel
    paths, whose shapes leave two, three or four partial sums."""
    from paper_2510_04147_amd import binding, mx
    cfg = synth.model_config("tiny", dtype="mxfp4", n_layers=2, d_model=2048, n_q_heads=16, n_kv_heads=2, head_dim=128, d_ffn=2304, vocab=2080)
    w = synth.gen_weights(cfg, 31, device="cuda")
    for l, lw in enumerate(w["layers"]):               # gains that are not one and not each other's
        for i, n in enumerate(("norm1", "norm2")):
            lw[n] = 1 + 0.1 * torch.randn(cfg["d_model"], device="cuda", generator=torch.Generator("cuda").manual_seed(100 + 2 * l + i))
    eng = binding.SSD(cfg, w, max_seqs=seqs, max_seq_len=160, block=block, max_draft=0, max_rows=384)
    eng.set_kernel_path(path)
    prefixes = [45 + 7 * i for i in range(seqs)]
    for i, prefix in enumerate(prefixes):
        eng.prefill_kv(i, synth.gen_prompt(cfg, 9 + i, prefix), 0)
    out = eng.new_out(seqs)
    eng.draft(list(range(seqs)), [[cfg["mask_id"]] * block] * seqs, [(1 << block) - 1] * seqs, prefixes, 0, out)
    got = out.host()

    eps, nq, d, F = cfg["rms_eps"], 16 * 128, cfg["d_model"], cfg["d_ffn"]
    four = [{n: mx.quantize(lw[n], mx.FP4) for n in ("wqkv", "wo", "wgu", "wdown")} for lw in w["layers"]]
    for i, prefix in enumerate(prefixes):
        h = w["embed"][torch.full((block,), cfg["mask_id"], device="cuda")].float()
        part = None
        for l, lw in enumerate(w["layers"]):
            qkv = slices_apart(mx, mx.norm(h, part, lw["norm1"], eps), four[l]["wqkv"], block, nq + 4 * 128, d)
            assert len(qkv) == 4
            attn = torch.empty(block, nq, dtype=torch.bfloat16, device="cuda")
            eng.k_attention(l, [(i, prefix, block, 0)], qkv, 0, attn)
            o = slices_apart(mx, mx.quantize(attn, mx.FP8), four[l]["wo"], block, d, nq)
            act = mx.linear(mx.norm(h, o, lw["norm2"], eps), four[l]["wgu"], "swiglu")
            part = slices_apart(mx, act, four[l]["wdown"], block, d, F)
            assert len(o) == 4 and len(part) == 3
        x = torch.empty(block, d, dtype=torch.bfloat16, device="cuda")
        eng.k_norm(h, part, w["final_norm"], x)
        head = torch.empty(3, block, device="cuda")
        eng.k_linear(binding.LIN_LM, 0, x, head)
        head = head.cpu().numpy()
        assert np.array_equal(got["row_maxlogit"][i, 0], head[0])
        assert np.array_equal(got["row_argmax"][i, 0], head[1].astype(np.int32))
        assert np.array_equal(got["row_conf"][i, 0], head[2])
    eng.close()
