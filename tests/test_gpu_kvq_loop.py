"""Norms of queries and keys, scaled rotations and the 8-bit cache run together through the decoding loop."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import kvq_oracle as kq
from oracle import model_oracle as mo
from oracle import wedlm_oracle as orc
from workloads.model import TINY, ModelConfig, make_model, make_prompts_and_targets

pytestmark = pytest.mark.gpu

NORMED = dataclasses.replace(TINY, name="tiny_normed", qk_norm=True)
SMALL = ModelConfig(name="small_normed", vocab=600, hidden=256, n_layers=2, n_q_heads=4, n_kv_heads=1, head_dim=128, ffn=256, dtype="bf16",
                    rope_theta=1.0e4, init_std=0.08, qk_norm=True)


@pytest.mark.parametrize("W,tilt,tau,rope", [(4, 8.0, 0.55, None), (8, 14.0, 0.35, dict(scaling="yarn", factor=4.0, original_len=16)),
                                             (5, 6.0, 2.05, dict(rotary_dim=16, scaling="linear", factor=2.0))])
def test_normed_model_text_is_token_exact(W, tilt, tau, rope):
    """Cache in the model's type: fp32 kernels against the cache-free fp64 model."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, P, N = 3, 21, 20
    wts = make_model(NORMED)
    pt = make_prompts_and_targets(NORMED, B, P, N)
    dec = StreamingDecoder(NORMED, wts, batch=B, window=W, max_total_len=P + N, tau=tau, lam=0.1, tilt=tilt, target=pt["target"], rope=rope)
    dec.prefill(pt["prompt"])
    got = dec.generate(N, use_graph=W == 8)
    assert int(dec.step_bufs.status.item()) == 0
    kw = dict(rope or {})
    table = kq.rope_frequencies(NORMED.rope_theta, kw.pop("rotary_dim", NORMED.head_dim), **kw)
    for b in range(B):
        prompt, target = [int(t) for t in pt["prompt"][b]], pt["target"][b]

        def forward(y, toks, pos):
            lg = mo.forward_window(wts, NORMED, prompt + y, toks, pos, rope=table)
            for r, p in enumerate(pos):
                lg[r, int(target[min(p, len(target) - 1)])] += tilt
            return lg
        ref = orc.decode_loop(forward, prefix_len=P, window=W, max_new_tokens=N, conf_mode="entropy", tau=tau, lam=0.1, maxprob_thr=0.9,
                              mask_token_id=NORMED.mask_token_id)
        assert got["y"][b] == ref["y"], b


@pytest.mark.parametrize("model,W,use_graph,group", [(NORMED, 4, False, None), (TINY, 8, True, None), (SMALL, 8, True, None), (SMALL, 1, False, None),
                                                     (SMALL, 6, True, [0, 0, -1])])
def test_generation_over_the_8_bit_cache(model, W, use_graph, group):
    """A tilt far above the logits decides the text, whatever the cache rounds; the windows, commits, pages and graphs around it are
    what is tested.  The same run as one graph a step and eagerly."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, P, N = 3, 37, 24
    wts = make_model(model)
    pt = make_prompts_and_targets(model, B, P, N)
    prompt, target = pt["prompt"].copy(), pt["target"].copy()
    if group is not None:
        prompt[1] = prompt[0]
    dec = StreamingDecoder(model, wts, batch=B, window=W, max_total_len=P + N, tau=0.35, lam=0.1, tilt=60.0, target=target, kv_cache="e4m3",
                           group=None if group is None else np.array(group))
    dec.prefill(prompt)
    got = dec.generate(N, use_graph=use_graph)
    assert int(dec.step_bufs.status.item()) == 0
    for b in range(B):
        assert got["y"][b] == target[b, P:P + N].tolist()
    if W >= 4:
        assert got["steps"] < N


@pytest.mark.parametrize("model", [NORMED, SMALL])
def test_a_step_over_the_8_bit_cache_is_what_its_inputs_say(model):
    """Replay of one layer in the middle of a generation: what the step stored and the attention over it, from the captured inputs."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, P, N, W = 2, 30, 12, 8
    wts = make_model(model)
    pt = make_prompts_and_targets(model, B, P, N)
    dec = StreamingDecoder(model, wts, batch=B, window=W, max_total_len=P + N, tau=2.05, lam=0.1, tilt=4.0, target=pt["target"], kv_cache="e4m3")
    dec.prefill(pt["prompt"])
    dec.start(N)
    dec.step()
    _, _, cap = dec.step(capture_layer=1)
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    table, prefix = dec.block_table.cpu().numpy(), cap["prefix_len"].cpu().numpy()
    cache = {}
    for i, x in enumerate("kv"):
        codes, scale, slots = kq.append(f64(cap[x]), cap[x + "_codes"].cpu().numpy(), cap[x + "_scale"].cpu().numpy(), table, prefix, None, 16)
        assert np.array_equal(slots, cap["kv_slot_idx"].cpu().numpy())
        assert np.array_equal(codes, dec.caches[1][2 * i].cpu().numpy()) and np.array_equal(scale, f64(dec.caches[1][2 * i + 1]))
        cache[x] = (codes, scale)
    out, size = kq.attention(f64(cap["q"]), *cache["k"], *cache["v"], table, prefix, model.head_dim ** -0.5)
    # half a step of the output, and 2^-9 of the average |v| for the weights (fp16 weights 2^-11, split queries and sums below 2^-11
    # at scores of normed queries and keys, |s| < 20)
    half = 2.0 ** -8 if model.dtype == "bf16" else 2.0 ** -24
    assert (np.abs(f64(cap["out"]) - out) <= half * np.abs(out) + 2.0 ** -9 * size).all()


def test_refusals():
    from paper_2512_22737_b200.loop import StreamingDecoder
    wts = make_model(TINY)
    with pytest.raises(ValueError, match="kv_cache"):
        StreamingDecoder(TINY, wts, batch=1, window=4, max_total_len=20, kv_cache="int4")
    with pytest.raises(ValueError, match="scaling"):
        StreamingDecoder(TINY, wts, batch=1, window=4, max_total_len=20, rope=dict(scaling="other"))
