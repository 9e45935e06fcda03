"""Window attention of groups that share their leading cache pages, against the float64 oracle and the plain call."""
import numpy as np
import pytest
import torch

from oracle import wedlm_oracle as orc
from workloads import get_config, make_step

pytestmark = pytest.mark.gpu


def _inputs(prefix, group, pages, *, W=16, heads=(8, 2), D=128, dtype="bf16", seed=0):
    """Inputs of a step in which the members of a group have `pages[group]` leading pages in common."""
    cfg = get_config("cfg2_qwen_b1").replace(batch=len(prefix), window=W, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, vocab=64,
                                             dtype=dtype, name="shared")
    inp = make_step(cfg, seed=seed, prefix_len=np.asarray(prefix), with_logits=False)
    first = {}
    for b, g in enumerate(group):
        a = first.setdefault(g, b)
        n = pages.get(g, 0) if isinstance(pages, dict) else pages
        n = min(n, prefix[a] // cfg.page_size, prefix[b] // cfg.page_size)
        inp["block_table"][b, :n] = inp["block_table"][a, :n]
    return cfg, inp


def _call(cfg, inp, group, *, impl="auto", stream=None, plain=False, max_prefix=None, status=None):
    import paper_2512_22737_b200 as w
    import parity_util as pu
    d = pu.device_inputs(inp)
    W = cfg.window
    top = inp["block_table"].shape[1] * cfg.page_size - W
    c = w.config_for(cfg, max_pages_per_seq=inp["block_table"].shape[1], num_pages=inp["k_cache"].shape[0], attn_impl=impl,
                     max_prefix_len=top if max_prefix is None else max_prefix)
    ro = orc.reorder(inp["filled"], inp["prefix_len"])
    pos = torch.tensor(ro["pos_ids"], dtype=torch.int32, device="cuda")
    out = torch.full(tuple(d["q"].shape), 5.0, dtype=d["q"].dtype, device="cuda")
    slots = torch.zeros(cfg.batch, W, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
    args = (d["q"], d["k"], d["v"], d["k_cache"], d["v_cache"], d["block_table"], d["prefix_len"], pos, out, slots)
    if plain:
        ws = torch.empty(w.wedlm_window_attn_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        w.wedlm_window_attn(c, *args, ws, st)
    else:
        n = w.wedlm_shared_prefix_attn_workspace_bytes(c)
        ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")       # any contents; guard bytes behind
        g = torch.tensor(group, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        w.wedlm_shared_prefix_attn(c, g, *args, ws[:n], st, stream)
        torch.cuda.synchronize()
        assert (ws[n:] == 0xA5).all()
    torch.cuda.synchronize()
    return dict(out=out, slots=slots, k_cache=d["k_cache"], v_cache=d["v_cache"], status=int(st.item()))


def _check(cfg, inp, group, **kw):
    import parity_util as pu
    got = _call(cfg, inp, group, **kw)
    assert got["status"] == 0
    ro = orc.reorder(inp["filled"], inp["prefix_len"])
    ref = orc.window_attention(inp["q"], inp["k"], inp["v"], inp["k_cache"], inp["v_cache"], inp["block_table"], inp["prefix_len"],
                               ro["pos_ids"], theta=cfg.rope_theta)
    o = pu.bf16_from_device(got["out"])
    assert np.isfinite(o).all()
    err = pu.attn_vector_error(o, ref["out"])
    assert err.max() <= (pu.ATTN_REL_TOL if cfg.dtype == "bf16" else 1e-4), (err.max(), np.unravel_index(err.argmax(), err.shape))
    plain = _call(cfg, inp, group, plain=True)
    for name in ("slots", "k_cache", "v_cache"):
        assert torch.equal(got[name].view(torch.uint8), plain[name].view(torch.uint8)), name     # staging is the plain call's
    return got


@pytest.mark.parametrize("prefix,group,pages", [
    ([600, 640, 610, 900], [0, 0, 0, 0], 37),                           # one group, shared part ends inside a tile
    ([600, 640, 610, 900], [0, 1, 0, 1], {0: 30, 1: 37}),               # interleaved
    ([600, 640, 610, 900, 333], [0, 0, -7, 1000, 2], 30),               # values outside [0, B): alone
    ([700, 700, 700], [2, 2, 2], 43),
    ([700], [0], 10),                                                   # a single sequence
    ([300, 0, 17, 290], [0, 0, 0, 0], 18),                              # a member without a prefix: nothing is shared
    ([300, 310, 330, 290], [1, 1, 1, 1], 3),                            # less than a tile
    ([257, 4000, 256, 300], [3, 3, 3, 3], 16),                          # one far longer than the others
    ([64, 64, 64, 64], [0, 0, 0, 0], 4),                                # exactly a tile
    ([256, 256, 256], [0, 0, 0], 16),                                   # all of the prefix is shared
])
def test_groups(prefix, group, pages):
    cfg, inp = _inputs(prefix, group, pages, seed=len(prefix) * 100 + prefix[0])
    _check(cfg, inp, group)


@pytest.mark.parametrize("W", [1, 2, 5, 16, 31, 32, 33, 70])
@pytest.mark.parametrize("heads", [(8, 2), (4, 4), (16, 2)])
def test_windows_and_heads(W, heads):
    """Row tiles that hold several sequences, parts of them, exactly one, or that one sequence fills twice."""
    prefix = [520, 530, 650, 517, 601]
    group = [0, 0, 1, 0, 1]
    cfg, inp = _inputs(prefix, group, {0: 32, 1: 37}, W=W, heads=heads, seed=W * 10 + heads[0])
    _check(cfg, inp, group)


def test_many_sequences_of_single_tokens():
    g = np.random.default_rng(5)
    prefix = (400 + g.integers(0, 300, 300)).tolist()
    group = g.integers(0, 7, 300).tolist()
    cfg, inp = _inputs(prefix, group, 24, W=1, heads=(8, 2), seed=5)
    _check(cfg, inp, group)


def test_more_sequences_than_threads_plan():
    """Over 1024 sequences: the planner walks its tables in several steps."""
    prefix = [70 + (b % 5) * 3 for b in range(1100)]
    prefix[7] = prefix[500] = prefix[1099] = 600
    group = [b % 3 if b % 50 else b for b in range(1100)]
    group[7] = group[500] = group[1099] = 900
    cfg, inp = _inputs(prefix, group, {0: 4, 1: 4, 2: 4, 900: 37}, W=2, heads=(2, 1), seed=6)
    _check(cfg, inp, group)


def test_long_prefix_is_cut_into_many_pieces():
    prefix = [20000, 20100, 20033]
    cfg, inp = _inputs(prefix, [0, 0, 0], 1250, W=40, heads=(4, 1), seed=7)
    _check(cfg, inp, [0, 0, 0])


def test_long_prefix_in_chunks_over_row_tiles():
    g = np.random.default_rng(8)
    prefix = (6000 + g.integers(0, 200, 24)).tolist()
    cfg, inp = _inputs(prefix, [0] * 24, 375, W=16, heads=(8, 1), seed=8)
    _check(cfg, inp, [0] * 24)


@pytest.mark.parametrize("dtype,D,page", [("f32", 64, 16), ("f32", 128, 16), ("bf16", 64, 16), ("bf16", 256, 16), ("bf16", 32, 16)])
def test_other_types_and_head_sizes(dtype, D, page):
    cfg, inp = _inputs([200, 210, 333], [0, 0, 0], 12, W=6, heads=(4, 2), D=D, dtype=dtype, seed=D)
    _check(cfg, inp, [0, 0, 0])


def test_cuda_core_path_on_request():
    cfg, inp = _inputs([300, 310, 330], [0, 0, 0], 18, W=6, heads=(4, 2), seed=9)
    _check(cfg, inp, [0, 0, 0], impl="generic")


def test_groups_that_share_nothing_or_less_than_they_say():
    """Grouping is a hint: what is shared is read from the tables, page by page."""
    cfg, inp = _inputs([800, 800, 800, 800], [0, 0, 0, 0], 50, seed=10)
    own = _inputs([800, 800, 800, 800], [0, 1, 2, 3], 0, seed=10)[1]["block_table"]
    inp["block_table"][2, 20:] = own[2, 20:]                            # one member leaves after 20 pages
    _check(cfg, inp, [0, 0, 0, 0])
    inp["block_table"][:] = own
    _check(cfg, inp, [0, 0, 0, 0])


def test_rows_past_the_prefix_and_foreign_pages_cannot_leak():
    cfg, inp = _inputs([523, 540, 531], [0, 0, 0], 32, W=7, seed=11)
    for b in range(3):
        P = int(inp["prefix_len"][b])
        for t in range(P + 7, -(-(P + 7) // 16) * 16):
            pg = inp["block_table"][b, t // 16]
            inp["k_cache"][pg, :, t % 16] = 0x7FC0
            inp["v_cache"][pg, :, t % 16] = 0x7F80
    used = set(inp["block_table"][inp["block_table"] >= 0].tolist())
    for pg in set(range(inp["k_cache"].shape[0])) - used:
        inp["k_cache"][pg] = 0x7FC0
        inp["v_cache"][pg] = 0x7FC0
    _check(cfg, inp, [0, 0, 0])


@pytest.mark.parametrize("factor", [6.0, 40.0])
@pytest.mark.parametrize("page", [0, 10, 31, 33])
def test_outlier_keys(page, factor):
    """Scores far above all others in the shared part, at its end, or in a sequence's own part: the accumulator is rescaled
    and the parts are joined across many powers of two.  The plain call rounds the same rotated queries, so it is the
    measure (two bf16 paths: each within the stated tolerance)."""
    import parity_util as pu
    from workloads import bf16_bits, bf16_to_f32
    cfg, inp = _inputs([600, 640, 610], [0, 0, 0], 32, seed=int(page + factor))
    pg = inp["block_table"][1, page]
    inp["k_cache"][pg] = bf16_bits(bf16_to_f32(inp["k_cache"][pg].reshape(-1)) * np.float32(factor)).reshape(inp["k_cache"][pg].shape)
    got, ref = _call(cfg, inp, [0, 0, 0]), _call(cfg, inp, [0, 0, 0], plain=True)
    err = pu.attn_vector_error(pu.bf16_from_device(got["out"]), pu.bf16_from_device(ref["out"]))
    assert err.max() <= pu.ATTN_REL_TOL


def test_bad_pages_and_lengths_are_flagged_and_fault_nothing():
    import paper_2512_22737_b200 as w
    cfg, inp = _inputs([600, 640, 610, 300], [0, 0, 0, 1], 30, seed=12)
    good = _call(cfg, inp, [0, 0, 0, 1])
    inp["block_table"][:3, 5] = inp["k_cache"].shape[0] + 9             # in the shared part
    bad = _call(cfg, inp, [0, 0, 0, 1])
    assert bad["status"] & w.binding.WEDLM_STATUS_BAD_PAGE
    assert torch.isfinite(bad["out"].float()).all()
    assert torch.equal(bad["out"][3], good["out"][3]) or torch.allclose(bad["out"][3].float(), good["out"][3].float(), atol=2e-2)
    cfg, inp = _inputs([600, 640, 610, 300], [0, 0, 0, 1], 30, seed=12)
    over = _call(cfg, inp, [0, 0, 0, 1], max_prefix=620)                # 640 lies beyond what the caller planned for
    assert over["status"] & w.binding.WEDLM_STATUS_BAD_LENGTH
    assert torch.isfinite(over["out"].float()).all()
    inp["prefix_len"][3] = -5
    neg = _call(cfg, inp, [0, 0, 0, 1])
    assert neg["status"] & w.binding.WEDLM_STATUS_BAD_LENGTH
    assert torch.isfinite(neg["out"][:3].float()).all()


def test_same_bits_every_time_on_any_stream_and_from_a_graph():
    import paper_2512_22737_b200 as w
    import parity_util as pu
    cfg, inp = _inputs([900, 940, 1000, 915, 903], [0, 0, 1, 0, 1], {0: 55, 1: 50}, seed=13)
    group = [0, 0, 1, 0, 1]
    ref = _call(cfg, inp, group)
    for stream in (None, torch.cuda.Stream()):
        assert torch.equal(_call(cfg, inp, group, stream=stream)["out"], ref["out"])
    d = pu.device_inputs(inp)
    c = w.config_for(cfg, max_pages_per_seq=inp["block_table"].shape[1], num_pages=inp["k_cache"].shape[0],
                     max_prefix_len=inp["block_table"].shape[1] * 16 - cfg.window)
    ro = orc.reorder(inp["filled"], inp["prefix_len"])
    pos = torch.tensor(ro["pos_ids"], dtype=torch.int32, device="cuda")
    out, g = torch.zeros_like(d["q"]), torch.tensor(group, dtype=torch.int32, device="cuda")
    ws = torch.empty(w.wedlm_shared_prefix_attn_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    call = lambda: w.wedlm_shared_prefix_attn(c, g, d["q"], d["k"], d["v"], d["k_cache"], d["v_cache"], d["block_table"],  # noqa: E731
                                              d["prefix_len"], pos, out, None, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref["out"])
    # the captured call reads lengths and groups from device memory: other values, same graph
    d["prefix_len"].copy_(torch.tensor([880, 900, 1000, 915, 850], dtype=torch.int32))
    g.copy_(torch.tensor([0, 0, 0, 0, 1], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    inp["prefix_len"][:] = [880, 900, 1000, 915, 850]
    ro2 = orc.reorder(inp["filled"], np.asarray([900, 940, 1000, 915, 903]))
    fresh = orc.window_attention(inp["q"], inp["k"], inp["v"], orc.to_f64(pu.bf16_from_device(d["k_cache"])),
                                 orc.to_f64(pu.bf16_from_device(d["v_cache"])), inp["block_table"], inp["prefix_len"], ro2["pos_ids"],
                                 theta=cfg.rope_theta)
    assert pu.attn_vector_error(pu.bf16_from_device(out), fresh["out"]).max() <= pu.ATTN_REL_TOL
