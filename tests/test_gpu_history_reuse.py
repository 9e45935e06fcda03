"""A sequence's history is emptied by clearing its row of token_bits: whatever stands in the records of tokens whose bit is
clear counts for nothing, for those who read them and for those who write them."""
import numpy as np
import pytest
import torch

from oracle import adjust_oracle as adj

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _stale(shape, seed):
    """Records that an earlier request may have left, and words that no request leaves."""
    g = np.random.default_rng(seed)
    left = g.integers(0, 40, shape)
    left[..., 1] = np.float32(g.normal(0, 3, shape[:-1])).view(np.int32)
    return _i32(np.where(g.random(shape) < 0.2, g.integers(-2 ** 31, 2 ** 31, shape), left).astype(np.int32))


def _fresh(B, V, seed, window=4, **kw):
    import paper_2512_22737_b200 as w
    cfg = w.make_config(batch=B, window=window, vocab=V, mask_token_id=V - 1, tau=0.35, lam=0.1, **kw)
    bits = torch.zeros(B, w.wedlm_token_bits_words(V), dtype=torch.int32, device="cuda")
    record = _stale((B, V, 2), seed)
    return w, cfg, bits, record, w.make_adjust(bits, record)


def _check(hist, bits, record, V):
    bits, record = bits.cpu().numpy(), record.cpu().numpy()
    for b, h in enumerate(hist):
        touched = np.zeros(V, bool)
        touched[list(h.touched())] = True
        np.testing.assert_array_equal(bits[b], adj.pack_bits(touched))
        for v in h.touched():
            want = [2 * h.generated.get(v, 0) + (v in h.prompt), int(np.float32(h.bias.get(v, 0.0)).view(np.int32))]
            assert record[b, v].tolist() == want, (b, v)


# few tokens that thousands of threads of several blocks add at once, a single one, and a vocabulary in earnest
@pytest.mark.parametrize("B,V,length", [(3, 5, 6000), (2, 1, 700), (2, 50, 33), (5, 1001, 700), (2, 151936, 5000)])
@pytest.mark.parametrize("first", ["prompt", "generated", "bias"])
def test_tokens_and_biases_start_from_nothing(B, V, length, first):
    w, cfg, bits, record, rules = _fresh(B, V, seed=V + length)
    g = np.random.default_rng(length)
    hist = [adj.History() for _ in range(B)]
    steps = {"prompt": ["prompt", "generated", "bias"], "generated": ["generated", "prompt", "generated"],
             "bias": ["bias", "generated", "prompt"]}[first]
    for step in steps:
        toks = (g.random((B, length)) ** 3 * V).astype(np.int64)
        if step == "bias":
            n = min(length, 64)
            val = np.float32(g.normal(0, 3, (B, n)))
            w.wedlm_history_bias(cfg, rules, _i32(toks[:, :n]), torch.as_tensor(val, device="cuda"))
            for b in range(B):
                hist[b].set_bias(toks[b, :n], val[b], V)
        else:
            count = g.integers(length // 2, length + 1, B)
            w.wedlm_history_add(cfg, rules, _i32(toks), _i32(count), step == "prompt")
            for b in range(B):
                hist[b].add(toks[b, :count[b]], step == "prompt", V)
        _check(hist, bits, record, V)


@pytest.mark.parametrize("temperature", [0.0, 0.8])
@pytest.mark.parametrize("dtype,V", [("bf16", 9000), ("bf16", 1003), ("f32", 5000)])
def test_filled_tokens_start_from_nothing(dtype, V, temperature):
    """The confidence call on emptied histories gives what it gives on zeros, the histories that it leaves among it.  Two
    tokens only are allowed, so a step fills several slots of a sequence with the same one."""
    B, W = 6, 40
    out = []
    for stale in (False, True):
        w, cfg, bits, record, _ = _fresh(B, V, seed=V, window=W, dtype=dtype, sample_temperature=temperature, sample_seed=99)
        cfg.tau = 50.0                                              # every mask is filled
        if not stale:
            record.zero_()
        on = np.zeros((1, V), bool)
        on[0, [3, V // 2]] = True
        rules = w.make_adjust(bits, record, *[torch.full((B,), x, device="cuda") for x in (1.3, 0.5, 0.2)], _i32(adj.pack_bits(on)),
                              torch.zeros(B, W, dtype=torch.int32, device="cuda"))
        g = torch.Generator().manual_seed(V)
        step = w.DecodeStep(cfg)
        tok = torch.full((B, W), V - 1, dtype=torch.int32, device="cuda")
        filled = torch.zeros(B, W, dtype=torch.uint8, device="cuda")
        prefix = torch.full((B,), 7, dtype=torch.int32, device="cuda")
        per_step = []
        for _ in range(2):                                          # the second step reads what the first has counted
            filled.zero_()
            step.reorder(filled, tok, prefix)
            logits = torch.randn(B, W, V, generator=g).cuda().to(cfg.torch_dtype)
            step.confidence_commit(logits, tok, filled, prefix, adjust=rules)
            assert (step.filled_count == W).all()
            per_step.append([t.clone() for t in (tok, step.argmax, step.maxprob, step.entropy, step.lse)])
        assert int(step.status.item()) == 0
        live = torch.as_tensor(np.unpackbits(bits.cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool), device="cuda")
        assert live.sum() <= 2 * B
        assert (record[..., 0][live] >= 2).all() and int(record[..., 0][live].sum()) == 2 * 2 * B * W
        out.append(per_step + [[bits.clone(), torch.where(live[..., None], record, 0)]])
    for x, y in zip(out[0], out[1]):
        for s, t in zip(x, y):
            assert torch.equal(s, t)
