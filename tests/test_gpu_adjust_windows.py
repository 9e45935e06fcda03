"""The confidence call under rules with short windows, budgets, both selections and both commit modes: every output, the window's
state and the histories against the oracle, with nothing left out.  The inputs are made on the CPU and keep every decision
away from its border (asserted), so that all of them have one right answer."""
import numpy as np
import pytest
import torch

from oracle import adjust_oracle as adj
from oracle import wedlm_oracle as orc

TAU, LAM, THR = 2.2, 0.5, 0.6


def _case(B, W, V, dtype, seed, *, lens=None, budgets=None, conf_mode="entropy", commit_mode="streaming"):
    g = np.random.default_rng(seed)
    c = dict(B=B, W=W, V=V, dtype=dtype, conf_mode=conf_mode, commit_mode=commit_mode)
    hist = [adj.History() for _ in range(B)]
    for h in hist:
        h.add((g.random(V // 20 + 3) ** 3 * V).astype(int), True, V)
        h.add((g.random(V // 20 + 3) ** 3 * V).astype(int), False, V)
        h.set_bias(g.integers(0, V, 5), np.float32(g.normal(0, 2, 5)), V)
    pen = np.float32(np.stack([1 + 0.4 * g.random(B), g.random(B) * 0.5, g.random(B) * 0.3]))
    masks = np.stack([np.zeros(V, bool), g.random(V) < 0.5, np.arange(V) < V // 3, g.random(V) < 0.97])
    which = np.where(g.random((B, W)) < 0.6, g.integers(0, 4, (B, W)), -1)
    # leading filled slots, so that most sequences commit, and some behind them
    lead = g.integers(0, W + 1, B)
    lead[0] = min(2, W)
    filled = ((np.arange(W) < lead[:, None]) | (g.random((B, W)) < 0.3)).astype(np.uint8)
    tokens = np.where(filled, g.integers(0, V - 1, (B, W)), V - 1).astype(np.int32)
    lens_np = np.full(B, W) if lens is None else np.asarray(lens)
    ro = orc.reorder(filled, np.zeros(B, np.int64), None if lens is None else lens_np, block_commit=commit_mode == "block")
    # a clear favourite among what the row may write (nearly certain), or noise (far from certain): nothing between
    x = g.normal(0, 1, (B, W, V))
    for b in range(B):
        for i in range(W):
            m = which[b, ro["perm"][b, i]]
            may = np.flatnonzero(masks[m]) if m >= 0 else np.arange(V)
            untouched = np.setdiff1d(may, list(hist[b].touched()))
            if len(untouched) and g.random() < 0.5:
                x[b, i, g.choice(untouched)] = 30.0
    logits = torch.as_tensor(x, dtype=torch.float32).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    stats, want = {}, []
    prefix = 11 * np.arange(B) + 5
    for b in range(B):
        L, nf = int(lens_np[b]), int(ro["n_filled"][b])
        am, ent, mp = [], [], []
        for i in range(nf, L):
            m = which[b, ro["perm"][b, i]]
            r, p, f = (float(v) for v in pen[:, b])
            y = adj.adjusted_logits(logits[b, i].double().numpy(), hist[b], r, p, f, masks[m] if m >= 0 else None)
            s = adj.row_statistics(y)
            stats[b, i] = s
            if s["argmax"] >= 0:
                # the winner is clear, or equal to others that no rule has touched
                top = np.flatnonzero(y > y.max() - 1e-4)
                assert len(top) == 1 or (len(set(y[top])) == 1 and not set(top) & hist[b].touched())
            am.append(s["argmax"])
            ent.append(s["entropy"] if s["argmax"] >= 0 else np.inf)
            mp.append(s["maxprob"])
        some = any(a >= 0 for a in am)
        budget = None if budgets is None else int(budgets[b])
        o = orc.select_commit_refill(tokens[b], filled[b], L, int(prefix[b]), am, ent, mp, conf_mode=conf_mode, tau=TAU, lam=LAM,
                                     maxprob_thr=THR, mask_token_id=V - 1, remaining_budget=budget, fallback=some,
                                     block_commit=commit_mode == "block")
        sc = np.array([s for s, a in zip(o["scores"], am) if a >= 0])
        border = TAU if conf_mode == "entropy" else -THR
        assert not (np.abs(sc - border) < 1e-2).any()
        if len(sc) > 1 and not (sc <= border).any():
            assert np.diff(np.sort(sc))[0] > (1e-2 if conf_mode == "entropy" else 1e-6)
        want.append(o)
    c.update(hist=hist, pen=pen, masks=masks, which=which, filled=filled, tokens=tokens, lens=lens, budgets=budgets, ro=ro, logits=logits,
             stats=stats, want=want, prefix=prefix)
    return c


CASES = {
    "one_row": dict(B=1, W=1, V=40, dtype="f32", seed=1),
    "one_request": dict(B=1, W=16, V=9000, dtype="bf16", seed=2),
    "one_request_odd": dict(B=1, W=9, V=1001, dtype="bf16", seed=3),
    "one_request_f32": dict(B=1, W=12, V=5003, dtype="f32", seed=4),
    "short_windows": dict(B=6, W=8, V=9000, dtype="bf16", seed=5, lens=[8, 5, 1, 0, 7, 3]),
    "short_windows_and_budgets": dict(B=6, W=8, V=2003, dtype="bf16", seed=6, lens=[8, 5, 1, 0, 7, 3], budgets=[9, 0, 1, 3, 2, 1]),
    "budgets": dict(B=5, W=33, V=8200, dtype="bf16", seed=7, budgets=[0, 1, 2, 40, 5]),
    "budgets_f32": dict(B=4, W=8, V=4100, dtype="f32", seed=8, lens=[8, 8, 6, 2], budgets=[1, 50, 2, 0]),
    "certainty": dict(B=6, W=8, V=9000, dtype="bf16", seed=9, lens=[8, 5, 8, 0, 7, 3], budgets=[9, 0, 1, 3, 2, 1], conf_mode="maxprob"),
    "blocks": dict(B=8, W=4, V=3000, dtype="bf16", seed=10, lens=[4, 4, 2, 1, 4, 0, 3, 4], budgets=[9, 0, 1, 3, 2, 1, 0, 7], commit_mode="block"),
}


@pytest.mark.parametrize("name", CASES)
def test_the_inputs_have_one_right_answer(name):
    c = _case(**CASES[name])
    if c["lens"] is not None or c["budgets"] is not None:
        assert any(o["committed_count"] for o in c["want"]) and any(o["filled_count"] for o in c["want"])


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_everything_that_a_step_writes(name):
    import paper_2512_22737_b200 as w
    c = _case(**CASES[name])
    B, W, V = c["B"], c["W"], c["V"]
    dev = lambda x, dt=torch.int32: torch.as_tensor(np.asarray(x), device="cuda").to(dt).contiguous()  # noqa: E731
    cfg = w.make_config(batch=B, window=W, vocab=V, dtype=c["dtype"], mask_token_id=V - 1, tau=TAU, lam=LAM, maxprob_thr=THR,
                        conf_mode=c["conf_mode"], commit_mode=c["commit_mode"])
    bits, record = np.zeros((B, V), bool), np.zeros((B, V, 2), np.int32)
    for b, h in enumerate(c["hist"]):
        for v in h.touched():
            bits[b, v] = True
            record[b, v] = 2 * h.generated.get(v, 0) + (v in h.prompt), np.float32(h.bias.get(v, 0.0)).view(np.int32)
    before = record[..., 0].sum(1)
    bits_d, record_d = dev(adj.pack_bits(bits)), dev(record)
    rules = w.make_adjust(bits_d, record_d, *[dev(p, torch.float32) for p in c["pen"]], dev(adj.pack_bits(c["masks"])), dev(c["which"]))
    tok, fil, pre = dev(c["tokens"]), dev(c["filled"], torch.uint8), dev(c["prefix"])
    wl = None if c["lens"] is None else dev(c["lens"])
    left = None if c["budgets"] is None else dev(c["budgets"])
    step = w.DecodeStep(cfg)
    step.reorder(fil, tok, pre, wl)
    for key in ("perm", "n_filled", "n_commit"):
        np.testing.assert_array_equal(getattr(step, key).cpu().numpy(), c["ro"][key])
    step.confidence_commit(c["logits"].cuda(), tok, fil, pre, wl, left, adjust=rules)
    empty = any(s["argmax"] < 0 for s in c["stats"].values())
    assert int(step.status.item()) == (w.binding.WEDLM_STATUS_EMPTY_ROW if empty else 0)
    argmax, maxprob, entropy, lse = (getattr(step, k).double().cpu().numpy() for k in ("argmax", "maxprob", "entropy", "lse"))
    for b in range(B):
        for i in range(W):
            s = c["stats"].get((b, i))
            if s is None:                                           # not an active mask row
                assert argmax[b, i] == -1 and np.isnan([maxprob[b, i], entropy[b, i], lse[b, i]]).all()
                continue
            assert argmax[b, i] == s["argmax"]
            if s["argmax"] < 0:
                assert maxprob[b, i] == 0 and entropy[b, i] == 0 and lse[b, i] == -np.inf
                continue
            # the logits carry up to five half steps of fp32 at magnitudes below 64
            assert abs(lse[b, i] - s["lse"]) <= 1e-5 + 1e-6 * abs(s["lse"])
            assert abs(maxprob[b, i] - s["maxprob"]) <= 2e-5 * s["maxprob"]
            assert abs(entropy[b, i] - s["entropy"]) <= 1e-5 + 1e-5 * s["entropy"]
        o = c["want"][b]
        assert tok[b].tolist() == o["window_tokens"] and fil[b].tolist() == o["filled"]
        assert int(pre[b]) == o["prefix_len"]
        assert int(step.committed_count[b]) == o["committed_count"] and int(step.filled_count[b]) == o["filled_count"]
        assert step.committed_tokens[b].tolist() == list(o["committed_tokens"]) + [-1] * (W - o["committed_count"])
        if wl is not None:
            assert int(wl[b]) == o["window_len"]
        if left is not None:
            assert int(left[b]) == o["remaining_budget"]
        # the filled tokens, and they alone, joined the history
        h, nf = c["hist"][b], int(c["ro"]["n_filled"][b])
        new = [c["stats"][b, nf + o["mask_slots"].index(j)]["argmax"] for j in o["filled_slots"]]
        h.add(new, False, V)
        got = record_d[b].cpu().numpy()
        touched = np.zeros(V, bool)
        touched[list(h.touched())] = True
        np.testing.assert_array_equal(bits_d[b].cpu().numpy(), adj.pack_bits(touched))
        assert int(got[:, 0].sum()) - int(before[b]) == 2 * len(new)
        for v in h.touched():
            assert got[v].tolist() == [2 * h.generated.get(v, 0) + (v in h.prompt), int(np.float32(h.bias.get(v, 0.0)).view(np.int32))]
