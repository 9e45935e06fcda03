"""A mask table without masks: what a server has while no request is under a grammar."""
import ctypes

import numpy as np
import pytest
import torch


def test_an_empty_mask_table_is_accepted_and_a_missing_one_is_not():
    import paper_2512_22737_b200 as w
    lib = w.load_library()
    cfg = w.make_config(batch=2, window=4, vocab=100)
    p = ctypes.c_void_p(4096)
    for n_masks, allowed, workspace, want in ((0, None, 16, -3), (0, 4096, 16, -3), (1, None, 16, -1), (1, 4096, 16, -3)):
        a = w.WedlmAdjust(n_masks=n_masks, allowed=allowed, mask_index=4096)       # (-3: past the rules, stopped by the workspace)
        assert lib.wedlm_confidence_commit_adjusted(ctypes.byref(cfg), ctypes.byref(a), *([p] * 17), workspace, None, None) == want
    a = w.WedlmAdjust(n_masks=0, allowed=4096)                                      # a table that nothing points into
    assert lib.wedlm_confidence_commit_adjusted(ctypes.byref(cfg), ctypes.byref(a), *([p] * 17), 16, None, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [("bf16", 9000), ("bf16", 1003), ("f32", 5000)])
def test_no_masks_constrain_nothing_and_any_index_is_flagged(dtype, V):
    import paper_2512_22737_b200 as w
    B, W = 3, 6
    cfg = w.make_config(batch=B, window=W, vocab=V, dtype=dtype, mask_token_id=V - 1, tau=0.35, lam=0.1)
    i32 = dict(dtype=torch.int32, device="cuda")
    logits = torch.randn(B, W, V, generator=torch.Generator().manual_seed(V)).cuda().to(cfg.torch_dtype)
    index = torch.full((B, W), -1, **i32)
    index[1, 2] = -7
    rules = {"none": w.make_adjust(), "empty": w.make_adjust(allowed=torch.zeros(0, w.wedlm_token_bits_words(V), **i32), mask_index=index)}
    out = {}
    for name, r in rules.items():
        step = w.DecodeStep(cfg)
        tok, fil = torch.full((B, W), V - 1, **i32), torch.zeros(B, W, dtype=torch.uint8, device="cuda")
        pre = torch.arange(B, **i32)
        step.reorder(fil, tok, pre)
        adjusted = torch.zeros_like(logits)
        w.wedlm_logits_adjust(cfg, r, logits, adjusted, step.perm, step.n_filled, status=step.status)
        step.confidence_commit(logits, tok, fil, pre, adjust=r)
        assert int(step.status.item()) == 0
        out[name] = [adjusted, step.argmax, step.maxprob, step.entropy, step.lse, tok, fil]
    assert all(torch.equal(x, y) for x, y in zip(out["none"], out["empty"]))
    assert torch.equal(out["empty"][0], logits)
    index[0, 3] = 0                                                                 # there is no mask 0
    st = torch.zeros(1, **i32)
    w.wedlm_logits_adjust(cfg, rules["empty"], logits, adjusted, step.perm, step.n_filled, status=st)
    assert int(st.item()) == w.binding.WEDLM_STATUS_BAD_TOKEN and torch.equal(adjusted, logits)


@pytest.mark.gpu
def test_the_loop_takes_an_empty_table():
    from paper_2512_22737_b200.loop import StreamingDecoder
    from workloads.model import TINY, make_model
    texts = []
    for rules in ({}, dict(allowed=np.zeros((0, TINY.vocab), dtype=bool), mask_index=np.full((2, 4), -1, dtype=np.int32))):
        dec = StreamingDecoder(TINY, make_model(TINY), batch=2, window=4, max_total_len=60, rules=rules)
        dec.prefill(np.tile(np.arange(20, dtype=np.int32), (2, 1)))
        texts.append(dec.generate(12)["y"])
    assert texts[0] == texts[1]
