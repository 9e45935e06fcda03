"""Masks that belong to places of the answer rather than to window slots: a caller that steps by itself rewrites mask_index after
every step, and gets what the cache-free fp64 model gives under a mask per position."""
import numpy as np
import pytest
import torch

from oracle import adjust_oracle as adj
from oracle import model_oracle as mo
from oracle import wedlm_oracle as orc
from workloads.model import TINY, make_model, make_prompts_and_targets

pytestmark = pytest.mark.gpu


def test_masks_of_positions():
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, P, W, N, tau, tilt = 3, 21, 6, 20, 0.55, 8.0
    wts = make_model(TINY)
    pt = make_prompts_and_targets(TINY, B, P, N)
    g = np.random.default_rng(4)
    allowed = g.random((5, TINY.vocab)) < 0.6
    allowed[:, TINY.mask_token_id] = False
    state = np.full((B, N + W), -1, dtype=np.int32)                 # mask of every place of the answers
    state[:, :N] = g.integers(0, 5, (B, N))
    state_dev = torch.from_numpy(state.astype(np.int64)).cuda()

    dec = StreamingDecoder(TINY, wts, batch=B, window=W, max_total_len=P + N, tau=tau, lam=0.1, tilt=tilt, target=pt["target"],
                           rules=dict(allowed=allowed, mask_index=state[:, :W]))
    dec.prefill(pt["prompt"])
    dec.start(N)
    got, moved = [[] for _ in range(B)], 0
    index = dec.adjust.tensors["mask_index"]
    for _ in range(200):
        if int(dec.window_len.sum()) == 0:
            break
        count, tokens = dec.step()
        for b in range(B):
            got[b].extend(tokens[b, : int(count[b])].tolist())
        at = (dec.prefix_len.long() - P)[:, None] + torch.arange(W, device="cuda")     # place of each slot, as it stands now
        index.copy_(state_dev.gather(1, at))
        moved += int(count.sum())
    assert moved == B * N and int(dec.step_bufs.status.item()) == 0

    for b in range(B):
        prompt = [int(t) for t in pt["prompt"][b]]

        def forward(y, toks, pos):
            rows = mo.forward_window(wts, TINY, prompt + y, toks, pos)
            for r, p in enumerate(pos):
                rows[r, int(pt["target"][b][min(p, P + N - 1)])] += tilt
            return np.stack([adj.adjusted_logits(row, None, allowed=allowed[state[b, p - P]]) for row, p in zip(rows, pos)])

        ref = orc.decode_loop(forward, prefix_len=P, window=W, max_new_tokens=N, conf_mode="entropy", tau=tau, lam=0.1,
                              maxprob_thr=0.9, mask_token_id=TINY.mask_token_id)
        assert got[b] == ref["y"]
        assert all(allowed[state[b, k], t] for k, t in enumerate(got[b]))
