"""Several answers to one prompt under the rules of each request: shared-prefix attention, adjusted confidence and the
histories run together through the decoding loop, against the cache-free fp64 model with the rules written from their
formulas."""
import numpy as np
import pytest
import torch

from oracle import adjust_oracle as adj
from oracle import model_oracle as mo
from oracle import wedlm_oracle as orc
from workloads.model import TINY, ModelConfig, make_model, make_prompts_and_targets

pytestmark = pytest.mark.gpu

GROUPS = [0, -1, 0, 3, 3, 0]            # three answers, one alone, two answers


def _prompts(model, B, P, N, group):
    pt = make_prompts_and_targets(model, B, P, N)
    prompt = pt["prompt"].copy()
    for b in range(B):
        if 0 <= group[b] < B:
            prompt[b] = prompt[list(group).index(group[b])]
    return prompt, pt["target"]


def _rules(model, B, W, seed):
    g = np.random.default_rng(seed)
    allowed = g.random((2, model.vocab)) < 0.7
    allowed[:, model.mask_token_id] = False                     # so that a slot with the mask token is an unfilled one
    index = np.broadcast_to(np.array([b % 2 for b in range(B)], dtype=np.int32)[:, None], (B, W))
    f32 = np.float32
    return dict(repetition=g.uniform(1.0, 1.5, B).astype(f32), presence=g.uniform(0.0, 1.0, B).astype(f32),
                frequency=g.uniform(0.0, 0.5, B).astype(f32), allowed=allowed, mask_index=index)


def _reference(wts, model, prompt, target, rules, b, *, tilt, W, N, tau):
    prompt = [int(t) for t in prompt]

    def forward(y, toks, pos):
        lg = mo.forward_window(wts, model, prompt + y, toks, pos)
        for r, p in enumerate(pos):
            lg[r, int(target[min(p, len(target) - 1)])] += tilt
        hist = adj.History()
        hist.add(prompt, True, model.vocab)
        hist.add(y + [t for t in toks if t != model.mask_token_id], False, model.vocab)
        return np.stack([adj.adjusted_logits(row, hist, float(rules["repetition"][b]), float(rules["presence"][b]),
                                             float(rules["frequency"][b]), rules["allowed"][rules["mask_index"][b, 0]])
                         for row in lg])

    return orc.decode_loop(forward, prefix_len=len(prompt), window=W, max_new_tokens=N, conf_mode="entropy", tau=tau,
                           lam=0.1, maxprob_thr=0.9, mask_token_id=model.mask_token_id)


@pytest.mark.parametrize("P,W,tilt,tau,use_graph", [(21, 4, 8.0, 0.55, False), (37, 8, 14.0, 0.35, True), (64, 5, 6.0, 2.05, True)])
def test_answers_under_rules_are_token_exact(P, W, tilt, tau, use_graph):
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, N = len(GROUPS), 18
    wts = make_model(TINY)
    prompt, target = _prompts(TINY, B, P, N, GROUPS)
    rules = _rules(TINY, B, W, seed=P)
    dec = StreamingDecoder(TINY, wts, batch=B, window=W, max_total_len=P + N, tau=tau, lam=0.1, tilt=tilt, target=target,
                           group=np.array(GROUPS), rules=rules)
    dec.prefill(prompt)
    table = dec.block_table.cpu().numpy()
    full = P // dec.cfg.page_size
    assert (table[2, :full] == table[0, :full]).all() and (table[4, :full] == table[3, :full]).all()
    assert not (table[2, full:] == table[0, full:]).any()
    got = dec.generate(N, use_graph=use_graph)
    assert int(dec.step_bufs.status.item()) == 0
    record = dec.adjust.tensors["token_record"].cpu().numpy()
    for b in range(B):
        ref = _reference(wts, TINY, prompt[b], target[b], rules, b, tilt=tilt, W=W, N=N, tau=tau)
        assert got["y"][b] == ref["y"], (b, got["y"][b], ref["y"])
        assert len(ref["y"]) == N
        hist = adj.History()
        hist.add(prompt[b], True, TINY.vocab)
        hist.add(ref["y"], False, TINY.vocab)                  # at the end everything filled is committed
        want = np.zeros(TINY.vocab, dtype=np.int64)
        for v in hist.touched():
            want[v] = 2 * hist.generated.get(v, 0) + (v in hist.prompt)
        assert np.array_equal(record[b, :, 0], want)


def test_bf16_answers_follow_a_strong_tilt():
    """The tensor-core attention over shared pages, as a captured step: the tilt is far above what rounding can turn."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    m = ModelConfig(name="tiny_bf16", vocab=2000, hidden=256, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, ffn=512,
                    dtype="bf16", rope_theta=1.0e6, init_std=0.03)
    B, P, N, W = len(GROUPS), 75, 40, 16
    wts = make_model(m)
    prompt, target = _prompts(m, B, P, N, GROUPS)
    dec = StreamingDecoder(m, wts, batch=B, window=W, max_total_len=P + N, tau=0.35, lam=0.1, tilt=40.0, target=target,
                           group=np.array(GROUPS), rules=dict(presence=np.full(B, 0.5, dtype=np.float32)))
    dec.prefill(prompt)
    got = dec.generate(N, use_graph=True)
    assert int(dec.step_bufs.status.item()) == 0
    for b in range(B):
        assert got["y"][b] == target[b, P:P + N].tolist()


def test_drawn_answers_replayed_equal_the_eager_ones():
    """At a temperature the draws come from the logits under the rules; a captured step draws what an eager one draws."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    B, P, N, W = len(GROUPS), 37, 18, 8
    wts = make_model(TINY)
    prompt, target = _prompts(TINY, B, P, N, GROUPS)
    rules = _rules(TINY, B, W, seed=3)
    texts, records = [], []
    for use_graph in (False, True):
        dec = StreamingDecoder(TINY, wts, batch=B, window=W, max_total_len=P + N, tau=0.55, lam=0.1, tilt=6.0, target=target,
                               temperature=0.8, sample_seed=1234, group=np.array(GROUPS), rules=rules)
        dec.prefill(prompt)
        texts.append(dec.generate(N, use_graph=use_graph)["y"])
        records.append(dec.adjust.tensors["token_record"].clone())
        assert int(dec.step_bufs.status.item()) == 0
    assert texts[0] == texts[1] and torch.equal(records[0], records[1])
    for b in range(B):
        on = rules["allowed"][rules["mask_index"][b, 0]]
        assert len(texts[0][b]) == N and all(on[t] for t in texts[0][b])
        counts = np.bincount(texts[0][b], minlength=TINY.vocab)
        assert np.array_equal(records[0][b, :, 0].cpu().numpy() // 2, counts)
    assert texts[0][0] != texts[0][2]                           # answers to one prompt, drawn apart


def test_an_empty_batch_does_nothing():
    from paper_2512_22737_b200 import binding as w
    c = w.make_config(batch=0, window=4, n_q_heads=4, n_kv_heads=2, head_dim=128, vocab=64, max_pages_per_seq=4, num_pages=4,
                      mask_token_id=63, max_prefix_len=48)
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    rules = w.make_adjust(token_bits=torch.zeros(0, 4, **i32), token_record=torch.zeros(0, 64, 2, **i32))
    step = w.DecodeStep(c)
    cache = [torch.zeros(4, 2, 16, 128, **bf16) for _ in range(2)]
    q, kv = torch.zeros(0, 4, 4, 128, **bf16), torch.zeros(0, 4, 2, 128, **bf16)
    none = torch.zeros(0, **i32)
    step.shared_attention(none, q, kv, kv, *cache, torch.zeros(0, 4, **i32), none)
    w.wedlm_history_add(c, rules, torch.zeros(0, 3, **i32), none)
    step.confidence_commit(torch.zeros(0, 4, 64, **bf16), torch.zeros(0, 4, **i32), torch.zeros(0, 4, dtype=torch.uint8, device="cuda"),
                           none, adjust=rules)
    torch.cuda.synchronize()
    assert int(step.status.item()) == 0


def test_what_the_loop_refuses():
    from paper_2512_22737_b200.loop import StreamingDecoder
    wts = make_model(TINY)
    kw = dict(batch=2, window=4, max_total_len=60)
    with pytest.raises(ValueError, match="group must have shape"):
        StreamingDecoder(TINY, wts, group=np.zeros(3, dtype=np.int32), **kw)
    with pytest.raises(ValueError, match="fused LM head"):
        StreamingDecoder(TINY, wts, rules={}, fused_lm_head=True, **kw)
    with pytest.raises(ValueError, match="unknown rule"):
        StreamingDecoder(TINY, wts, rules=dict(temperature=np.ones(2)), **kw)
    with pytest.raises(ValueError, match="allowed must have shape"):
        StreamingDecoder(TINY, wts, rules=dict(allowed=np.ones((1, 5), dtype=bool)), **kw)
    dec = StreamingDecoder(TINY, wts, group=np.zeros(2, dtype=np.int32), **kw)
    with pytest.raises(ValueError, match="its prompt is another"):
        dec.prefill(np.array([[1, 2, 3], [1, 2, 4]], dtype=np.int32))


def test_a_decoder_with_groups_takes_one_prompt():
    """A second prompt would follow answers that differ, so its pages cannot be shared."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    dec = StreamingDecoder(TINY, make_model(TINY), batch=2, window=4, max_total_len=60, group=np.zeros(2, dtype=np.int32))
    prompt = np.tile(np.arange(20, dtype=np.int32), (2, 1))
    dec.prefill(prompt)
    with pytest.raises(ValueError, match="takes one prompt"):
        dec.prefill(prompt)


@pytest.mark.parametrize("use_graph", [False, True])
def test_rules_that_leave_nothing_end_the_loop(use_graph):
    """One sequence may still write, the other's mask is empty: the first finishes, then the loop says why it stops."""
    from paper_2512_22737_b200.loop import StreamingDecoder
    allowed = np.stack([np.ones(TINY.vocab, dtype=bool), np.zeros(TINY.vocab, dtype=bool)])
    rules = dict(allowed=allowed, mask_index=np.array([[0] * 4, [1] * 4], dtype=np.int32))
    dec = StreamingDecoder(TINY, make_model(TINY), batch=2, window=4, max_total_len=60, rules=rules)
    dec.prefill(np.tile(np.arange(20, dtype=np.int32), (2, 1)))
    with pytest.raises(RuntimeError, match="leave no token"):
        dec.generate(12, max_steps=200, use_graph=use_graph)
    assert int(dec.prefix_len[0]) == 32 and int(dec.prefix_len[1]) == 20


def _step_inputs(seed):
    from paper_2512_22737_b200 import binding as w
    from workloads import StepConfig, make_step
    cfg = StepConfig(name="answers", batch=4, window=8, n_q_heads=4, n_kv_heads=2, head_dim=128, vocab=5003, dtype="bf16",
                     prefix_lo=90, prefix_hi=130, obs_prob_lo=0.3, obs_prob_hi=0.3, boost=8.0, boost_prob=0.7, spare_pages=4 * 12)
    d = make_step(cfg, seed=seed)
    table = np.full((4, 12), -1, dtype=np.int32)                # room for what three steps commit
    table[:, :d["block_table"].shape[1]] = d["block_table"]
    free = np.setdiff1d(np.arange(d["k_cache"].shape[0]), d["block_table"])
    table[table < 0] = free[:(table < 0).sum()]
    d["block_table"] = table
    d["block_table"][1, :4] = d["block_table"][0, :4]           # two sequences with 64 tokens in common
    dev = {k: w.to_device(v) for k, v in d.items()}
    c = w.config_for(cfg, max_pages_per_seq=d["block_table"].shape[1], num_pages=d["k_cache"].shape[0], max_prefix_len=12 * 16 - 8)
    words = w.wedlm_token_bits_words(cfg.vocab)
    i32 = dict(dtype=torch.int32, device="cuda")
    rules = w.make_adjust(token_bits=torch.zeros(4, words, **i32), token_record=torch.zeros(4, cfg.vocab, 2, **i32),
                          repetition=torch.full((4,), 1.2, device="cuda"), presence=torch.full((4,), 0.4, device="cuda"))
    return c, dev, rules, torch.tensor([0, 0, -1, -1], **i32)


def _snapshot(step, d, rules):
    names = ("window_tokens", "filled", "prefix_len")
    return ([step.out.clone(), step.committed_tokens.clone(), step.committed_count.clone(), step.argmax.clone()]
            + [d[k].clone() for k in names] + [t.clone() for t in rules.tensors.values() if t is not None])


def test_two_captured_steps_of_one_workspace():
    """Graphs of two batches that share the step's buffers and workspaces, replayed in turn, give what each gives alone,
    on the capture's stream and on another one."""
    from paper_2512_22737_b200 import binding as w
    alone = []
    for seed in (5, 6):
        c, d, rules, group = _step_inputs(seed)
        step = w.DecodeStep(c)
        for _ in range(3):
            step.run(d, group=group, adjust=rules)
        alone.append(_snapshot(step, d, rules))
    sets = [_step_inputs(seed) for seed in (5, 6)]
    step = w.DecodeStep(sets[0][0])
    graphs = []
    for c, d, rules, group in sets:
        step.cfg = c
        graphs.append(step.capture_graph(d, group=group, adjust=rules))   # the first of three steps is eager
    graphs[0].replay()
    graphs[1].replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for k, (c, d, rules, group) in enumerate(sets):
        with torch.cuda.stream(side):
            graphs[k].replay()
            got = _snapshot(step, d, rules)
        side.synchronize()
        for x, y in zip(got, alone[k]):
            assert torch.equal(x, y)
    assert int(step.status.item()) == 0
