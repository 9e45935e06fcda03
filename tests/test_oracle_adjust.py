"""Pins of the adjustment oracle by hand-worked values and by its own definitions, and the host-side refusals of the
calls that take rules.  No GPU."""
import ctypes

import numpy as np
import pytest

from oracle import adjust_oracle as adj


def test_rules_in_their_order_by_hand():
    h = adj.History()
    h.add([1, 2, 2], False, 8)          # 1 once, 2 twice
    h.add([2, 3, 3, 9, -1], True, 8)    # 2 and 3 in the prompt; ids outside the vocabulary are skipped
    h.set_bias([4, 3, 4], [1.0, 0.5, 2.0], 8)
    x = np.array([1.0, 2.0, -2.0, 4.0, 0.0, 3.0, 3.0, 3.0])
    allowed = np.array([1, 1, 1, 1, 1, 1, 0, 1], bool)
    y = adj.adjusted_logits(x, h, repetition=2.0, presence=0.25, frequency=0.5, allowed=allowed)
    assert y[0] == 1.0
    assert y[1] == 2.0 / 2 - 0.25 - 0.5                  # generated once
    assert y[2] == -2.0 * 2 - 0.25 - 1.0                 # negative: multiplied; generated twice
    assert y[3] == 4.0 / 2 + 0.5                         # prompt only: no presence, no frequency; bias
    assert y[4] == 2.0                                   # bias alone; of equal ids the last counts
    assert y[5] == 3.0 and y[6] == -np.inf and y[7] == 3.0


def test_statistics_of_a_row():
    x = np.array([0.0, np.log(3.0), -np.inf, np.log(3.0)])
    s = adj.row_statistics(x)
    p = np.array([1, 3, 3]) / 7
    assert s["argmax"] == 1
    np.testing.assert_allclose([s["lse"], s["maxprob"], s["entropy"]], [np.log(7), 3 / 7, -(p * np.log(p)).sum()], rtol=1e-14)
    assert adj.row_statistics(np.full(5, -np.inf)) == dict(argmax=-1, lse=-np.inf, maxprob=0.0, entropy=0.0)


@pytest.mark.parametrize("v", [1, 31, 32, 33, 127, 128, 129, 1001])
def test_bit_packing(v):
    import paper_2512_22737_b200 as w
    on = np.random.default_rng(v).random((3, v)) < 0.4
    words = adj.pack_bits(on)
    assert words.shape == (3, w.wedlm_token_bits_words(v))
    u = words.view(np.uint32)
    for t in range(v):
        assert (((u[:, t // 32] >> (t % 32)) & 1) == on[:, t]).all()


def _adjust(**kw):
    import paper_2512_22737_b200 as w
    a = w.WedlmAdjust()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


GOOD = dict(token_bits=4096, token_record=8192, repetition=4096, allowed=4096, mask_index=4096, n_masks=1)


@pytest.mark.parametrize("change", [dict(token_bits=None), dict(token_record=None), dict(allowed=None), dict(mask_index=None),
                                    dict(n_masks=-1), dict(token_bits=4100), dict(token_record=8200), dict(allowed=4104),
                                    dict(token_bits=None, token_record=None, count_fills=1)])
def test_rules_that_do_not_fit_together_are_refused(change):
    import paper_2512_22737_b200 as w
    lib = w.load_library()
    cfg = w.make_config(batch=2, window=4, vocab=100)
    a = _adjust(**{**GOOD, **change})
    p = ctypes.c_void_p(4096)       # never read: the call is refused before anything is launched
    assert lib.wedlm_logits_adjust(ctypes.byref(cfg), ctypes.byref(a), p, p, p, p, None, None, None) == -1
    assert lib.wedlm_confidence_commit_adjusted(ctypes.byref(cfg), ctypes.byref(a), *([p] * 17), 1 << 20, None, None) == -1
    if "allowed" not in change and "mask_index" not in change:
        assert lib.wedlm_history_add(ctypes.byref(cfg), ctypes.byref(a), 4, p, p, 0, None, None) == -1
        assert lib.wedlm_history_bias(ctypes.byref(cfg), ctypes.byref(a), 4, p, p, None, None) == -1


def test_refusals_of_single_arguments():
    import paper_2512_22737_b200 as w
    lib = w.load_library()
    cfg = w.make_config(batch=2, window=4, vocab=100)
    a = _adjust(**GOOD)
    p, q, c, r = ctypes.c_void_p(4096), ctypes.c_void_p(1 << 20), ctypes.byref(cfg), ctypes.byref(a)
    assert lib.wedlm_logits_adjust(c, None, p, q, p, p, None, None, None) == -1
    for args in ((None, q, p, p), (p, None, p, p), (p, q, None, p), (p, q, p, None)):
        assert lib.wedlm_logits_adjust(c, r, *args, None, None, None) == -1
    # buffers that overlap without being the same
    assert lib.wedlm_logits_adjust(c, r, p, ctypes.c_void_p(4096 + 16), p, p, None, None, None) == -1
    assert lib.wedlm_logits_adjust(c, r, ctypes.c_void_p(4096 + 16), p, p, p, None, None, None) == -1
    # logits between two elements
    assert lib.wedlm_logits_adjust(c, r, ctypes.c_void_p(4097), q, p, p, None, None, None) == -1
    assert lib.wedlm_logits_adjust(c, r, p, ctypes.c_void_p((1 << 20) + 1), p, p, None, None, None) == -1
    assert lib.wedlm_confidence_commit_adjusted(c, r, ctypes.c_void_p(4097), *([p] * 16), 1 << 20, None, None) == -1
    assert lib.wedlm_history_add(c, r, -1, p, p, 0, None, None) == -1
    assert lib.wedlm_history_add(c, r, 4, None, p, 0, None, None) == -1
    assert lib.wedlm_history_add(c, r, 4, p, None, 0, None, None) == -1
    assert lib.wedlm_history_bias(c, r, -1, p, p, None, None) == -1
    assert lib.wedlm_history_bias(c, r, 5000, p, p, None, None) == -2
    assert lib.wedlm_history_bias(c, r, 4, None, p, None, None) == -1
    assert lib.wedlm_history_bias(c, r, 4, p, None, None, None) == -1
    args = [p] * 17
    assert lib.wedlm_confidence_commit_adjusted(c, r, *args, 16, None, None) == -3           # workspace too small
    for k in (0, 1, 2, 3, 4, 5, 6, 16):
        bad = list(args)
        bad[k] = None
        assert lib.wedlm_confidence_commit_adjusted(c, r, *bad, 1 << 20, None, None) == -1
    none = w.make_config(batch=2, window=4, vocab=0)
    assert lib.wedlm_logits_adjust(ctypes.byref(none), r, p, q, p, p, None, None, None) == -1
    assert lib.wedlm_history_add(ctypes.byref(none), r, 4, p, p, 0, None, None) == -1
    # nothing to do
    empty = w.make_config(batch=0, window=4, vocab=100)
    assert lib.wedlm_logits_adjust(ctypes.byref(empty), r, None, None, None, None, None, None, None) == 0
    assert lib.wedlm_history_add(ctypes.byref(cfg), r, 0, None, None, 0, None, None) == 0
    assert lib.wedlm_history_bias(ctypes.byref(cfg), r, 0, None, None, None, None) == 0


def test_shared_prefix_attention_refusals():
    import paper_2512_22737_b200 as w
    lib = w.load_library()
    kw = dict(batch=2, window=8, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_seq=8, num_pages=16, max_prefix_len=100)
    cfg = w.make_config(**kw)
    need = w.wedlm_shared_prefix_attn_workspace_bytes(cfg)
    assert need > 0
    p, c = ctypes.c_void_p(4096), ctypes.byref(cfg)
    args = [p] * 12                     # group, q, k, v, k_cache, v_cache, table, prefix, pos, out, slots, workspace
    assert lib.wedlm_shared_prefix_attn(c, *args, need - 1, None, None) == -3
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 11):
        bad = list(args)
        bad[i] = None
        assert lib.wedlm_shared_prefix_attn(c, *bad, need, None, None) == -1
    for i in (1, 2, 3, 4, 5, 9, 11):
        bad = list(args)
        bad[i] = ctypes.c_void_p(4104)
        assert lib.wedlm_shared_prefix_attn(c, *bad, need, None, None) == -1
    assert lib.wedlm_shared_prefix_attn(ctypes.byref(w.make_config(**{**kw, "n_q_heads": 7})), *args, need, None, None) == -1
    assert w.wedlm_shared_prefix_attn_workspace_bytes(w.make_config(**{**kw, "max_prefix_len": 200})) == 0
    assert lib.wedlm_shared_prefix_attn(ctypes.byref(w.make_config(**{**kw, "head_dim": 64, "attn_impl": "tensor"})), *args, need,
                                        None, None) == -2
    assert lib.wedlm_shared_prefix_attn(ctypes.byref(w.make_config(**{**kw, "batch": 0})), *([None] * 12), 0, None, None) == 0
