"""An SSD_MXFP4 context keeps 4-bit copies of the projections, not the bf16 tensors that it was made from."""
import weakref

import numpy as np
import pytest
import torch

from paper_2510_04147_amd import synth

pytestmark = pytest.mark.gpu
PROJECTIONS = ("wqkv", "wo", "wgu", "wdown")


def test_projections_end_with_the_callers_references():
    from paper_2510_04147_amd import binding
    cfg = synth.model_config("tiny", dtype="mxfp4", n_layers=3, d_model=1024, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ffn=2304, vocab=2080)
    shape = dict(max_seqs=1, max_seq_len=96, block=16, max_draft=3)
    prompt = [synth.gen_prompt(cfg, 3, 33)]
    kept = synth.gen_weights(cfg, 12, device="cuda")
    eng = binding.SSD(cfg, kept, **shape)
    want = eng.generate(prompt, 32, 16, 3)[0]
    eng.close()

    w = {k: v for k, v in kept.items() if k != "layers"}
    w["layers"] = [{n: t.clone() for n, t in lw.items()} for lw in kept["layers"]]
    refs = [weakref.ref(lw[n]) for lw in w["layers"] for n in PROJECTIONS]
    sizes = [(lw[n].numel(), lw[n].dtype) for lw in w["layers"] for n in PROJECTIONS]
    eng = binding.SSD(cfg, w, **shape)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    del w
    assert all(r() is None for r in refs)
    assert before - torch.cuda.memory_allocated() >= sum(n * 2 for n, _ in sizes)
    # what lay in their place is written over: other tensors of the same sizes, no number anywhere
    others = [torch.full((n,), float("nan"), dtype=dt, device="cuda") for n, dt in sizes]
    assert np.array_equal(eng.generate(prompt, 32, 16, 3)[0], want)
    assert len(others) == len(refs)
    eng.close()


def test_other_contexts_keep_what_they_read():
    """Every weight of a bf16 context stays: its kernels may read the caller's tensors."""
    from paper_2510_04147_amd import binding
    cfg = synth.model_config("tiny", dtype="bf16", n_layers=2)
    w = synth.gen_weights(cfg, 12, device="cuda")
    refs = [weakref.ref(t) for lw in w["layers"] for t in lw.values()] + [weakref.ref(w[n]) for n in ("embed", "lm_head", "final_norm")]
    eng = binding.SSD(cfg, w, max_seqs=1, max_seq_len=64, block=16, max_draft=1)
    del w
    assert all(r() is not None for r in refs)
    eng.close()
