"""The rest of the library's calls on an SSD_MXFP4 context whose projections the caller has dropped."""
import numpy as np
import pytest
import torch

from paper_2510_04147_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eng():
    from paper_2510_04147_amd import binding
    cfg = synth.model_config("tiny", dtype="mxfp4", n_layers=2, d_model=2048, n_q_heads=16, n_kv_heads=2, head_dim=128, d_ffn=2304, vocab=2080)
    w = synth.gen_weights(cfg, 41, device="cuda")
    e = binding.SSD(cfg, w, max_seqs=2, max_seq_len=160, block=32, max_draft=4, max_rows=320)
    sizes = [t.numel() for lw in w["layers"] for n, t in lw.items() if n.startswith("w")]
    del w
    over = [torch.full((n,), float("nan"), dtype=torch.bfloat16, device="cuda") for n in sizes]
    yield cfg, e
    e.close()
    del over


def test_acceptance_limit(eng):
    cfg, e = eng
    prompt = synth.gen_prompt(cfg, 7, 40)
    step = e.generate([prompt], 48, 16, 0)[0][0]
    toks, pr = e.acceptance_limit(prompt, 48, 16, 4, 5)
    assert np.array_equal(toks, step)
    assert pr["matched"][0] >= pr["rounds"] and all(a <= b for a, b in zip(pr["matched"], pr["matched"][1:]))
    again, _ = e.generate([prompt], 48, 16, 4)
    assert np.array_equal(again[0], step)


def test_kernel_paths_and_static_head(eng):
    cfg, e = eng
    prompts = [synth.gen_prompt(cfg, 60 + i, 33 + 8 * i) for i in range(2)]
    want = e.generate(prompts, 48, 24, 0)[0]
    old = e.set_kernel_path(2)
    try:
        for depth in (0, 3):
            assert np.array_equal(e.generate(prompts, 48, 24, depth)[0], want)
    finally:
        e.set_kernel_path(old)
    from paper_2510_04147_amd import binding
    x = torch.randn(70, cfg["d_model"], device="cuda", generator=torch.Generator("cuda").manual_seed(3)).bfloat16()
    a, b = torch.empty(3, 70, device="cuda"), torch.empty(3, 70, device="cuda")
    e.k_linear(binding.LIN_LM, 0, x, a)
    e.k_lm_head_static(x, b)
    assert torch.equal(a, b)


def test_profile_of_a_forward(eng):
    """Every class of kernels that a layer of the context runs is counted."""
    cfg, e = eng
    e.prefill_kv(0, synth.gen_prompt(cfg, 2, 40), 0)
    out = e.new_out(1)
    e.profile_begin()
    e.draft([0], [[cfg["mask_id"]] * 32], [(1 << 32) - 1], [40], 0, out)
    torch.cuda.synchronize()
    counts = {k: v["launches"] for k, v in e.profile_read().items()}
    e.profile_end()
    for k, n in (("rmsnorm", 5), ("gemm_qkv", 2), ("attention", 2), ("gemm_o", 2), ("gemm_gate_up_swiglu", 2), ("gemm_down", 2), ("lm_head_reduce", 1)):
        assert counts[k] == n, counts
