"""The microscaled operators run together: a context with 4-bit projections (SSD_MXFP4) against the same operators called one by one, against
itself (SSD decodes what stepwise decoding does, bit for bit) and against the model in 64 bits."""
import numpy as np
import pytest
import torch

import mx_plain as P
from oracle import model as oracle
from paper_2510_04147_amd import synth

pytestmark = pytest.mark.gpu


def bits(ps):
    return sum(1 << p for p in ps)


def small(head_dim, **more):
    return synth.model_config("tiny", **{**dict(dtype="mxfp4", n_layers=3, d_model=512, n_q_heads=512 // head_dim, n_kv_heads=2, head_dim=head_dim, d_ffn=1536, vocab=2080), **more})


def engine(cfg, w, **k):
    from paper_2510_04147_amd import binding
    return binding.SSD(cfg, w, **k)


@pytest.mark.parametrize("head_dim,block", [(64, 24), (128, 32), (128, 45)])
@pytest.mark.parametrize("path", [0, 1])
def test_a_forward_is_its_operators(head_dim, block, path):
    """The self-draft of a masked block behind a cached prefix, and the same rows through quantize, norm, linear, the attention step and
    the LM head called by hand: the same bits (projections of fewer than 2048 columns leave one sum)."""
    from paper_2510_04147_amd import binding, mx
    cfg = small(head_dim)
    w = synth.gen_weights(cfg, 5, device="cuda")
    for lw in w["layers"]:                             # gains that are not one
        for n in ("norm1", "norm2"):
            lw[n] = 1 + 0.1 * torch.randn(cfg["d_model"], device="cuda", generator=torch.Generator("cuda").manual_seed(hash(n) % 97))
    eng = engine(cfg, w, max_seqs=1, max_seq_len=160, block=block, max_draft=0, max_rows=128)
    eng.set_kernel_path(path)
    prefix = 45
    eng.prefill_kv(0, synth.gen_prompt(cfg, 9, prefix), 0)
    out = eng.new_out(1)
    eng.draft([0], [[cfg["mask_id"]] * block], [bits(range(block))], [prefix], 0, out)
    got = out.host()

    eps, nq = cfg["rms_eps"], cfg["n_q_heads"] * head_dim
    h = w["embed"][torch.full((block,), cfg["mask_id"], device="cuda")].float()
    part = None
    for l, lw in enumerate(w["layers"]):
        four = {n: mx.quantize(lw[n], mx.FP4) for n in ("wqkv", "wo", "wgu", "wdown")}
        qkv = mx.linear(mx.norm(h, part, lw["norm1"], eps), four["wqkv"], "fp32")
        attn = torch.empty(block, nq, dtype=torch.bfloat16, device="cuda")
        eng.k_attention(l, [(0, prefix, block, 0)], qkv[None].contiguous(), 0, attn)
        o = mx.linear(mx.quantize(attn, mx.FP8), four["wo"], "fp32")
        act = mx.linear(mx.norm(h, o[None], lw["norm2"], eps), four["wgu"], "swiglu")
        part = mx.linear(act, four["wdown"], "fp32")[None]
    x = torch.empty(block, cfg["d_model"], dtype=torch.bfloat16, device="cuda")
    eng.k_norm(h, part.contiguous(), w["final_norm"], x)
    head = torch.empty(3, block, device="cuda")
    eng.k_linear(binding.LIN_LM, 0, x, head)
    head = head.cpu().numpy()
    assert np.array_equal(got["row_maxlogit"][0, 0], head[0])
    assert np.array_equal(got["row_argmax"][0, 0], head[1].astype(np.int32))
    assert np.array_equal(got["row_conf"][0, 0], head[2])
    with pytest.raises(binding.SsdError, match="microscaled") as e:
        eng.k_linear(binding.LIN_QKV, 0, x, torch.empty(block, nq + 4 * head_dim, device="cuda"))
    assert e.value.code == -1
    eng.close()


MODELS = {"small64": small(64), "small128": small(128, n_kv_heads=4), "8b": synth.model_config("8b", n_layers=2, dtype="mxfp4"),
          "7b_gqa": synth.model_config("7b_gqa", n_layers=2, dtype="mxfp4")}


@pytest.mark.parametrize("model,seqs,block,draft", [("small64", 2, 24, 3), ("small128", 1, 32, 4), ("8b", 1, 32, 4), ("8b", 2, 8, 5), ("7b_gqa", 4, 32, 8)])
def test_ssd_decodes_what_stepwise_decoding_does(model, seqs, block, draft):
    cfg = MODELS[model]
    w = synth.gen_weights(cfg, 11, device="cuda")
    gen = block + block // 2
    prompts = [synth.gen_prompt(cfg, 30 + i, 40 + 7 * i) for i in range(seqs)]
    total = max(len(p) for p in prompts) + gen
    eng = engine(cfg, w, max_seqs=seqs, max_seq_len=total, block=block, max_draft=draft, max_rows=max(seqs * 2 * (draft + 2) * block, seqs * total))
    step = eng.generate(prompts, gen, block, 0)[0]
    assert np.array_equal(eng.generate(prompts, gen, block, draft)[0], step)
    for setter, on, off in ((eng.set_tree_mode, 1, 0), (eng.set_cross_block, 1, 0), (eng.set_boundary_fusion, 0, 1), (eng.set_graphs, 1, 0)):
        setter(on)
        assert np.array_equal(eng.generate(prompts, gen, block, draft)[0], step), setter
        setter(off)
    eng.set_cache_mode(1, 8)
    step = eng.generate(prompts, gen, block, 0)[0]
    assert np.array_equal(eng.generate(prompts, gen, block, draft)[0], step)
    eng.set_spill_over(1)
    assert np.array_equal(eng.generate(prompts, gen, block, draft)[0], step)
    eng.close()


def test_plain_path_decodes_too():
    cfg = MODELS["small64"]
    w = synth.gen_weights(cfg, 12, device="cuda")
    eng = engine(cfg, w, max_seqs=1, max_seq_len=96, block=16, max_draft=3)
    eng.set_kernel_path(0)
    prompt = [synth.gen_prompt(cfg, 3, 33)]
    assert np.array_equal(eng.generate(prompt, 32, 16, 3)[0], eng.generate(prompt, 32, 16, 0)[0])
    eng.close()


# ------------------------------------------------------------- against the model in 64 bits
def forward64(w, four, cfg, tokens, round8):
    """Logits of one segment, float64, weights the values of their 4-bit form; round8: with the operands rounded as the context
    rounds them (8 bits in front of the projections; bf16 for q, k, v, probabilities, attention output and the head's rows)."""
    act = (lambda x: P.quantize(x, 8)[2]) if round8 else (lambda x: x)
    half = (lambda x: x.bfloat16().double()) if round8 else (lambda x: x)
    ocfg = dict(cfg, operand_dtype=torch.bfloat16 if round8 else None)
    Hq, Hkv, dh, F = cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["d_ffn"]
    pos, eps = torch.arange(len(tokens)), cfg["rms_eps"]
    h = w["embed"][tokens].double()
    for lw, q4 in zip(w["layers"], four):
        qkv = act(oracle.rms_norm(h, lw["norm1"], eps)) @ q4["wqkv"].T
        q, k, v = (t.reshape(len(tokens), -1, dh) for t in qkv.split([Hq * dh, Hkv * dh, Hkv * dh], -1))
        q, k, v = half(oracle.rope(q, pos, cfg["rope_theta"])), half(oracle.rope(k, pos, cfg["rope_theta"])), half(v)
        a = half(oracle.attention(q, k, v, None, ocfg).reshape(len(tokens), -1))
        h = h + act(a) @ q4["wo"].T
        gu = act(oracle.rms_norm(h, lw["norm2"], eps)) @ q4["wgu"].T
        h = h + act(P.silu(gu[:, :F]) * gu[:, F:]) @ q4["wdown"].T
    return half(oracle.rms_norm(h, w["final_norm"], eps)) @ w["lm_head"].double().T


def test_accuracy():
    """Maximum logits of a masked block, no prefix, projections with k-slices.  The context must be as near to the exact model as an
    evaluation in 64 bits with the same roundings of the operands.  From that evaluation it may be as far as independent roundings are from
    each other: sums that differ by e (some 1e-5 relative) in front of a rounding of step u (2^-4) change a share e / u of the operands
    by u, so the operands differ by sqrt(e u) behind it; twelve roundings in a row take ln(u / e) = 8.7 to 8.7 / 2^12, that is
    e to u.  Two independent errors of rms r differ by sqrt(2) r; the rms of 42 values scatters by 1 / sqrt(2 * 42), so 1.25 of that."""
    from paper_2510_04147_amd import mx
    cfg = synth.model_config("tiny", dtype="mxfp4", n_layers=3, d_model=2048, n_q_heads=16, n_kv_heads=4, head_dim=128, d_ffn=2304, vocab=2080)
    wg = synth.gen_weights(cfg, 21, device="cuda")
    w = synth.weights_to(wg, "cpu")
    four = []
    for lw in wg["layers"]:
        four.append({})
        for n in ("wqkv", "wo", "wgu", "wdown"):
            v = torch.empty_like(lw[n])
            mx.quantize(lw[n], mx.FP4, values=v)
            four[-1][n] = v.cpu().double()
    block = 64
    eng = engine(cfg, wg, max_seqs=1, max_seq_len=block, block=block, max_draft=0, max_rows=block)
    toks = torch.from_numpy(synth.gen_prompt(cfg, 2, block).astype(np.int64))
    masked = [i for i in range(block) if i % 3]
    toks[masked] = cfg["mask_id"]
    out = eng.new_out(1)
    eng.draft([0], [toks.tolist()], [bits(masked)], [0], 0, out)
    got = torch.from_numpy(out.host()["row_maxlogit"][0, 0]).double()[masked]
    logits = [forward64(w, four, cfg, toks, r) for r in (False, True)]
    exact, twin = (l[masked].clone() for l in logits)
    for l in (exact, twin):
        l[:, cfg["mask_id"]] = -float("inf")
    exact, twin = exact.max(-1).values, twin.max(-1).values
    rms = lambda d: float(d.square().mean().sqrt())  # noqa: E731
    print(f"context off exact {rms(got - exact):.4f}, roundings in 64 bits {rms(twin - exact):.4f}, context off those {rms(got - twin):.4f}")
    assert rms(got - exact) <= 1.5 * rms(twin - exact) + 2e-3
    assert rms(got - twin) <= 1.25 * 2 ** 0.5 * rms(twin - exact)
    eng.close()
