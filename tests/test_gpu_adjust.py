"""Rules of single requests (penalties, biases, masks) on a GPU against the float64 oracle: histories, logits alone, and
the confidence pass with its window update."""
import numpy as np
import pytest
import torch

from oracle import adjust_oracle as adj
from oracle import wedlm_oracle as orc

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24          # half a step of fp32 and of bf16, relative
U16 = 2.0 ** -8


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _f32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32), device="cuda")


class Case:
    """A batch with histories, biases, penalties and masks, on both sides."""

    def __init__(self, B, W, V, dtype="bf16", seed=0, length=40, n_bias=6, masked=0.6, fill=0.4, cfg=None):
        import paper_2512_22737_b200 as w
        g = np.random.default_rng(seed)
        self.w, self.B, self.W, self.V, self.g = w, B, W, V, g
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.cfg = w.make_config(batch=B, window=W, vocab=V, dtype=dtype, mask_token_id=V - 1, **{**dict(tau=0.35, lam=0.1), **(cfg or {})})
        self.bits = torch.zeros(B, w.wedlm_token_bits_words(V), dtype=torch.int32, device="cuda")
        self.record = torch.zeros(B, V, 2, dtype=torch.int32, device="cuda")
        self.hist = [adj.History() for _ in range(B)]
        self.pen = np.float32(np.stack([1 + 0.4 * g.random(B), g.random(B) - 0.3, g.random(B) * 0.5]))
        self.pen[:, 0] = (1, 0, 0)
        kinds = [np.zeros(V, bool), np.ones(V, bool), g.random(V) < min(1.0, 3 / V), g.random(V) < 0.5, np.arange(V) >= V - max(1, V // 3),
                 np.arange(V) < max(1, V // 9)]
        self.allowed_np = np.stack(kinds)
        self.mask_np = np.where(g.random((B, W)) < masked, g.integers(0, len(kinds), (B, W)), -g.integers(1, 9, (B, W)))
        self.allowed, self.mask_index = _i32(adj.pack_bits(self.allowed_np)), _i32(self.mask_np)
        self.rules = w.make_adjust(self.bits, self.record, *[_f32(p) for p in self.pen], self.allowed, self.mask_index)
        self.plain = w.make_adjust(self.bits, self.record)
        for in_prompt in (True, False):
            toks = (g.random((B, length)) ** 3 * V).astype(np.int64)
            count = g.integers(0, length + 1, B)
            w.wedlm_history_add(self.cfg, self.rules, _i32(toks), _i32(count), in_prompt)
            for b in range(B):
                self.hist[b].add(toks[b, :count[b]], in_prompt, V)
        if n_bias:
            ids = g.integers(0, V, (B, n_bias))
            val = np.float32(g.normal(0, 3, (B, n_bias)))
            w.wedlm_history_bias(self.cfg, self.rules, _i32(ids), _f32(val))
            for b in range(B):
                self.hist[b].set_bias(ids[b], val[b], V)
        self.filled_np = (g.random((B, W)) < fill).astype(np.uint8)
        self.ro = orc.reorder(self.filled_np, np.zeros(B, np.int64))
        x = torch.randn(B, W, V, generator=torch.Generator().manual_seed(seed)) * 3
        top = torch.as_tensor(g.integers(0, V, (B, W, 1)))
        x.scatter_add_(2, top, torch.as_tensor(np.where(g.random((B, W, 1)) < 0.5, 16.0, 0.0), dtype=torch.float32))
        self.logits = x.cuda().to(self.dt)
        self.perm, self.n_filled = _i32(self.ro["perm"]), _i32(self.ro["n_filled"])

    def expect_row(self, b, i, hist=None):
        m = int(self.mask_np[b, self.ro["perm"][b, i]])
        x = self.logits[b, i].double().cpu().numpy()
        r, p, f = (float(v) for v in self.pen[:, b])
        return adj.adjusted_logits(x, (hist or self.hist)[b], r, p, f, self.allowed_np[m] if m >= 0 else None)


def _check_history(case, bits, record):
    b_np, r_np = bits.cpu().numpy(), record.cpu().numpy()
    for b, h in enumerate(case.hist):
        touched = np.zeros(case.V, bool)
        want = np.zeros((case.V, 2), np.int32)
        for v in h.touched():
            touched[v] = True
            want[v, 0] = 2 * h.generated.get(v, 0) + (v in h.prompt)
            want[v, 1] = np.float32(h.bias.get(v, 0.0)).view(np.int32)
        np.testing.assert_array_equal(b_np[b], adj.pack_bits(touched))
        np.testing.assert_array_equal(r_np[b], want)


@pytest.mark.parametrize("B,V,length,n_bias", [(1, 1, 3, 1), (3, 40, 300, 20), (5, 1001, 700, 64), (2, 151936, 5000, 300), (9, 129, 1, 0)])
def test_histories(B, V, length, n_bias):
    c = Case(B, 4, V, seed=V + length, length=length, n_bias=n_bias)
    _check_history(c, c.bits, c.record)


def test_history_ids_outside_the_vocabulary_are_skipped_and_flagged():
    c = Case(2, 4, 50, seed=3, length=5)
    w, st = c.w, torch.zeros(1, dtype=torch.int32, device="cuda")
    w.wedlm_history_add(c.cfg, c.rules, _i32([[1, 2], [3, 4]]), _i32([2, 7]), False, st)       # count beyond length: clamped
    assert st.item() == 0
    c.hist[0].add([1, 2], False, 50), c.hist[1].add([3, 4], False, 50)
    w.wedlm_history_add(c.cfg, c.rules, _i32([[50, 7], [-1, 2 ** 31 - 1]]), _i32([2, 2]), True, st)
    assert st.item() == w.binding.WEDLM_STATUS_BAD_TOKEN
    c.hist[0].add([7], True, 50)
    st.zero_()
    w.wedlm_history_bias(c.cfg, c.rules, _i32([[5, -3, 5], [-1, -1, -1]]), _f32([[1, 2, 4], [1, 1, 1]]), st)
    assert st.item() == 0                                          # negative ids are unused entries
    c.hist[0].set_bias([5], [4.0], 50)
    w.wedlm_history_bias(c.cfg, c.rules, _i32([[50, 6], [6, 99]]), _f32([[1, 2], [3, 4]]), st)
    assert st.item() == w.binding.WEDLM_STATUS_BAD_TOKEN
    c.hist[0].set_bias([6], [2.0], 50), c.hist[1].set_bias([6], [3.0], 50)
    _check_history(c, c.bits, c.record)


def test_negative_counts_add_nothing():
    c = Case(2, 4, 50, seed=4, length=5)
    c.w.wedlm_history_add(c.cfg, c.rules, _i32([[1, 2], [3, 4]]), _i32([-1, 0]), False)
    _check_history(c, c.bits, c.record)


SHAPES = [(2, 5, 1, "bf16"), (1, 3, 7, "bf16"), (3, 4, 100, "f32"), (2, 8, 1001, "f32"), (2, 8, 1001, "bf16"), (2, 6, 8192, "bf16"),
          (2, 6, 8200, "bf16"), (1, 5, 16385, "bf16"), (70, 8, 24601, "bf16"), (40, 16, 18006, "bf16"), (60, 9, 12001, "f32"),
          (3, 9, 8191, "bf16"), (3, 9, 8193, "bf16"), (3, 9, 16390, "bf16"), (5, 5, 4093, "f32"), (5, 5, 8197, "f32"), (2, 3, 20000, "f32"), (1, 4, 4100, "f32"), (2, 4, 151936, "bf16")]


def test_buffers_off_16_byte_boundaries():
    """A logits tensor that begins two bytes (bf16) or four (f32) into an allocation: the token-by-token kernels."""
    for dtype, V in (("bf16", 9000), ("bf16", 2003), ("f32", 5000)):
        c = Case(2, 6, V, dtype, seed=61)
        ref, ref_out = _confidence(c), torch.zeros_like(c.logits)
        c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, ref_out, c.perm, c.n_filled)
        moved = torch.empty(c.logits.numel() + 1, dtype=c.dt, device="cuda")[1:].view(c.logits.shape)
        moved.copy_(c.logits)
        c.logits = moved
        got, out = _confidence(c), torch.zeros_like(ref_out)
        c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled)
        assert torch.equal(out, ref_out)
        for name in ("argmax", "tok", "fil", "record"):
            assert torch.equal(got[name], ref[name]), name
        for name in ("entropy", "lse", "maxprob"):
            torch.testing.assert_close(got[name], ref[name], rtol=1e-5, atol=1e-5, equal_nan=True)


def _adjust_bound(c, b, i, want):
    """Four fp32 operations, each off by half a step of a value no larger than |x r| + |p| + |f c| + |bias|, one rounding
    to the storage type."""
    x = c.logits[b, i].double().cpu().numpy()
    x = np.where(np.isfinite(x), x, 0)
    r, p, f = (abs(float(v)) for v in c.pen[:, b])
    most = np.zeros(c.V)
    for v in c.hist[b].touched():
        most[v] = abs(x[v]) * max(r, 1 / r) + p + f * c.hist[b].generated.get(v, 0) + abs(c.hist[b].bias.get(v, 0.0))
    small = 2.0 ** -133                                            # half of the smallest bf16 step, subnormal
    return 5 * U32 * most + (U16 if c.dt == torch.bfloat16 else U32) * (np.abs(np.where(np.isfinite(want), want, 0)) + 5 * U32 * most) + small


@pytest.mark.parametrize("B,W,V,dtype", SHAPES)
def test_adjusted_logits(B, W, V, dtype):
    c = Case(B, W, V, dtype, seed=V)
    out = torch.full_like(c.logits, 7.0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = c.logits.clone()
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled, None, st)
    assert st.item() == 0
    assert torch.equal(before, c.logits)
    got = out.double().cpu().numpy()
    for b in range(B):
        nf = int(c.ro["n_filled"][b])
        assert (got[b, :nf] == 7.0).all()                          # rows that are no masks are left alone
        for i in range(nf, W):
            want = c.expect_row(b, i)
            gone = np.isneginf(want)
            assert (np.isneginf(got[b, i]) == gone).all()
            off = np.abs(got[b, i][~gone] - want[~gone])
            assert (off <= _adjust_bound(c, b, i, want)[~gone]).all(), off.max()
    # in place: the same bits
    place = c.logits.clone()
    c.w.wedlm_logits_adjust(c.cfg, c.rules, place, place, c.perm, c.n_filled)
    for b in range(B):
        nf = int(c.ro["n_filled"][b])
        assert torch.equal(place[b, nf:], out[b, nf:])
        assert torch.equal(place[b, :nf], before[b, :nf])


@pytest.mark.parametrize("dtype,V", [("bf16", 9000), ("bf16", 9001), ("f32", 5000)])
def test_short_windows_and_missing_rules(dtype, V):
    c = Case(3, 8, V, dtype, seed=11)
    wl = _i32([8, 3, 0])
    out = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled, wl)
    for b, n in enumerate((8, 3, 0)):
        assert (out[b, n:] == 0).all()
    full = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, full, c.perm, c.n_filled)
    for b, n in enumerate((8, 3, 0)):
        nf = int(c.ro["n_filled"][b])
        assert torch.equal(out[b, nf:n], full[b, nf:n])
    # no rules at all: a copy of the mask rows
    none = c.w.make_adjust()
    out.fill_(1)
    c.w.wedlm_logits_adjust(c.cfg, none, c.logits, out, c.perm, c.n_filled)
    for b in range(3):
        nf = int(c.ro["n_filled"][b])
        assert torch.equal(out[b, nf:], c.logits[b, nf:]) and (out[b, :nf] == 1).all()
    # masks alone, and a history without penalties
    masks = c.w.make_adjust(allowed=c.allowed, mask_index=c.mask_index)
    c.w.wedlm_logits_adjust(c.cfg, masks, c.logits, out, c.perm, c.n_filled)
    hist = c.w.make_adjust(c.bits, c.record, presence=_f32([0.5, 0.5, 0.5]))
    out2 = torch.zeros_like(out)
    c.w.wedlm_logits_adjust(c.cfg, hist, c.logits, out2, c.perm, c.n_filled)
    for b in range(3):
        for i in range(int(c.ro["n_filled"][b]), 8):
            m = int(c.mask_np[b, c.ro["perm"][b, i]])
            x = c.logits[b, i].double().cpu().numpy()
            want = adj.adjusted_logits(x, None, allowed=c.allowed_np[m] if m >= 0 else None)
            np.testing.assert_array_equal(out[b, i].double().cpu().numpy(), want)
            want = adj.adjusted_logits(x, c.hist[b], presence=0.5)
            got = out2[b, i].double().cpu().numpy()
            # two fp32 operations on values below 64 in magnitude, one rounding to the storage type
            assert np.abs(got - want).max() <= 2 * U32 * 64 + (U16 if dtype == "bf16" else U32) * 64


@pytest.mark.parametrize("dtype,V", [("bf16", 9000), ("bf16", 9001), ("f32", 5000)])
def test_excluded_logits_are_not_looked_at(dtype, V):
    """NaN, infinities and the type's lowest value at tokens that a mask excludes."""
    c = Case(2, 6, V, dtype, seed=13, masked=1.0, fill=0.3)
    clean = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, clean, c.perm, c.n_filled)
    bad = [float("nan"), float("inf"), float("-inf"), torch.finfo(c.dt).min]
    ref = _confidence(c)
    for b in range(2):
        for i in range(6):
            m = int(c.mask_np[b, c.ro["perm"][b, i]])
            off = np.flatnonzero(~c.allowed_np[m])
            c.logits[b, i, torch.as_tensor(off, device="cuda")] = torch.tensor([bad[k % 4] for k in range(len(off))], device="cuda").to(c.dt)
    out = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled)
    assert torch.equal(out, clean)
    got = _confidence(c)
    for name in ref:
        assert torch.equal(torch.nan_to_num(got[name].double(), nan=-7.0), torch.nan_to_num(ref[name].double(), nan=-7.0)), name


def test_mask_index_beyond_the_table_is_flagged_and_constrains_nothing():
    c = Case(1, 4, 9000, seed=17, fill=0.0)
    c.mask_index.fill_(-1)
    free = torch.zeros_like(c.logits)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, free, c.perm, c.n_filled, None, st)
    assert st.item() == 0
    c.mask_index.fill_(c.allowed.shape[0])
    out = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled, None, st)
    assert st.item() == c.w.binding.WEDLM_STATUS_BAD_TOKEN
    assert torch.equal(out, free)
    st.zero_()
    _confidence(c, status=st)
    assert st.item() == c.w.binding.WEDLM_STATUS_BAD_TOKEN


# ---------------------------------------------------------------------------------------------- confidence
def _confidence(c, rules=None, status=None, window_len=None, budget=None, stream=None, state=None):
    """One call on fresh copies of the window and of the histories.  Returns everything it wrote."""
    w, B, W = c.w, c.B, c.W
    step = w.DecodeStep(c.cfg)
    tok = state["tok"].clone() if state else torch.where(torch.as_tensor(c.filled_np, device="cuda") > 0, 3 % c.V, c.V - 1).to(torch.int32)
    fil = torch.as_tensor(c.filled_np, device="cuda").clone()
    pre = torch.arange(B, dtype=torch.int32, device="cuda") * 11 + 5
    bits, record = c.bits.clone(), c.record.clone()
    r = rules or c.rules
    mine = w.make_adjust(bits if r.tensors["token_bits"] is not None else None, record if r.tensors["token_bits"] is not None else None,
                         r.tensors["repetition"], r.tensors["presence"], r.tensors["frequency"], r.tensors["allowed"],
                         r.tensors["mask_index"], bool(r.count_fills))
    n_commit = _i32(c.ro["n_commit"])
    wl = None if window_len is None else _i32(window_len)
    bud = None if budget is None else _i32(budget)
    n = w.wedlm_confidence_adjusted_workspace_bytes(c.cfg)
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")                # any contents; guard bytes behind
    torch.cuda.synchronize()
    w.wedlm_confidence_commit_adjusted(c.cfg, mine, c.logits, c.perm, c.n_filled, n_commit, tok, fil, pre, wl, bud, step.argmax,
                                       step.maxprob, step.entropy, step.lse, step.committed_tokens, step.committed_count,
                                       step.filled_count, ws[:n], status, stream)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xA5).all()
    return dict(argmax=step.argmax, maxprob=step.maxprob, entropy=step.entropy, lse=step.lse, committed_tokens=step.committed_tokens,
                committed_count=step.committed_count, filled_count=step.filled_count, tok=tok, fil=fil, pre=pre, bits=bits, record=record)


def _check_confidence(c, got, temperature=0.0):
    """Against the oracle.  Rows whose decision lies within 1e-3 of a border are excluded, as everywhere in these tests."""
    B, W, V = c.B, c.W, c.V
    skipped = 0
    for b in range(B):
        nf = int(c.ro["n_filled"][b])
        rows = [c.expect_row(b, i) for i in range(nf, W)]
        stats = [adj.row_statistics(x) for x in rows]
        am, near = [], False
        for k, (x, s) in enumerate(zip(rows, stats)):
            i = nf + k
            a = int(got["argmax"][b, i])
            ent, mp, lse = (float(got[n][b, i]) for n in ("entropy", "maxprob", "lse"))
            if s["argmax"] < 0:
                assert a == -1 and ent == 0 and mp == 0 and lse == -np.inf
            else:
                if temperature == 0.0:
                    # the logits carry up to five half steps of fp32 at magnitudes below 64
                    assert x[a] >= x[s["argmax"]] - 10 * U32 * 64
                    near |= a != s["argmax"]
                assert abs(ent - s["entropy"]) <= 1e-5 + 1e-5 * s["entropy"], (ent, s)
                assert abs(lse - s["lse"]) <= 1e-5 + 1e-6 * abs(s["lse"])
                assert abs(mp - s["maxprob"]) <= 2e-5 * s["maxprob"]
            am.append(a)
        ent = [s["entropy"] if s["argmax"] >= 0 else np.inf for s in stats]
        mp = [s["maxprob"] for s in stats]
        some = any(s["argmax"] >= 0 for s in stats)
        tok0 = [3 % V if f else V - 1 for f in c.filled_np[b]]
        r = orc.select_commit_refill(tok0, c.filled_np[b], W, b * 11 + 5, am, ent, mp, conf_mode="entropy", tau=float(np.float32(0.35)),
                                     lam=float(np.float32(0.1)), maxprob_thr=0.9, mask_token_id=V - 1, fallback=some)
        sc = np.array([s for s in r["scores"] if np.isfinite(s)])
        tie = len(sc) > 0 and (np.abs(sc - 0.35) < 1e-3).any()
        if len(sc) > 1 and not (sc <= 0.35).any():
            srt = np.sort(sc)
            tie |= srt[1] - srt[0] < 1e-3
        if tie:
            skipped += 1
            continue
        if temperature == 0.0:
            assert got["tok"][b].tolist() == r["window_tokens"]
        assert got["fil"][b].tolist() == r["filled"]
        assert int(got["filled_count"][b]) == r["filled_count"]
        assert int(got["committed_count"][b]) == r["committed_count"]
        assert int(got["pre"][b]) == r["prefix_len"]
        # filled tokens joined the history
        masks = r["mask_slots"]
        new = [int(got["argmax"][b, nf + masks.index(j)]) for j in r["filled_slots"]]
        c.hist[b].add(new, False, V)
        assert int(got["record"][b, :, 0].sum() - c.record[b, :, 0].sum()) == 2 * len(new)
        h = c.hist[b]
        for v in set(new):
            assert int(got["record"][b, v, 0]) == 2 * h.generated[v] + (v in h.prompt)
            assert (int(got["bits"][b, v // 32]) >> (v % 32)) & 1
    return skipped


@pytest.mark.parametrize("B,W,V,dtype", SHAPES)
@pytest.mark.parametrize("masked", [0.0, 0.6])
def test_confidence_on_adjusted_logits(B, W, V, dtype, masked):
    c = Case(B, W, V, dtype, seed=V + 1, masked=masked)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _confidence(c, status=st)
    empty = any(int(c.mask_np[b, c.ro["perm"][b, i]]) >= 0 and not c.allowed_np[c.mask_np[b, c.ro["perm"][b, i]]].any()
                for b in range(B) for i in range(int(c.ro["n_filled"][b]), W))
    assert st.item() == (c.w.binding.WEDLM_STATUS_EMPTY_ROW if empty else 0)
    assert _check_confidence(c, got) <= max(1, B // 3)


@pytest.mark.parametrize("dtype,V,length", [("bf16", 8192, 60000), ("bf16", 9000, 9000), ("bf16", 9000, 2500), ("f32", 4096, 60000),
                                            ("bf16", 8191, 60000)])
@pytest.mark.parametrize("masked", [0.0, 0.7])
def test_dense_histories(dtype, V, length, masked):
    """Most tokens of a chunk have a record: more than a list holds, more than fit beside the logits, or just below."""
    c = Case(2, 6, V, dtype, seed=V + length, length=length, masked=masked)
    got = _confidence(c)
    out = torch.zeros_like(c.logits)
    c.w.wedlm_logits_adjust(c.cfg, c.rules, c.logits, out, c.perm, c.n_filled)
    o = out.double().cpu().numpy()
    for b in range(2):
        for i in range(int(c.ro["n_filled"][b]), 6):
            want = c.expect_row(b, i)
            gone = np.isneginf(want)
            assert (np.isneginf(o[b, i]) == gone).all()
            assert (np.abs(o[b, i][~gone] - want[~gone]) <= _adjust_bound(c, b, i, want)[~gone]).all()
    assert _check_confidence(c, got) <= 1          # (last: it adds the filled tokens to the histories)


@pytest.mark.parametrize("dtype,V", [("bf16", 8192 * 2), ("bf16", 5001), ("f32", 4096 + 4)])
def test_without_rules_it_is_the_plain_call(dtype, V):
    c = Case(4, 16, V, dtype, seed=23)
    got = _confidence(c, rules=c.w.make_adjust())
    w, step = c.w, c.w.DecodeStep(c.cfg)
    tok = torch.where(torch.as_tensor(c.filled_np, device="cuda") > 0, 3 % c.V, c.V - 1).to(torch.int32)
    fil, pre = torch.as_tensor(c.filled_np, device="cuda").clone(), torch.arange(4, dtype=torch.int32, device="cuda") * 11 + 5
    w.wedlm_confidence_commit(c.cfg, c.logits, c.perm, c.n_filled, _i32(c.ro["n_commit"]), tok, fil, pre, None, None, step.argmax,
                              step.maxprob, step.entropy, step.lse, step.committed_tokens, step.committed_count, step.filled_count,
                              step.conf_ws)
    assert torch.equal(got["argmax"], step.argmax)
    for a, b in ((got["tok"], tok), (got["fil"], fil), (got["pre"], pre), (got["committed_tokens"], step.committed_tokens),
                 (got["filled_count"], step.filled_count)):
        assert torch.equal(a, b)
    for a, b in ((got["entropy"], step.entropy), (got["lse"], step.lse), (got["maxprob"], step.maxprob)):
        torch.testing.assert_close(a, b, rtol=1e-5, atol=1e-5, equal_nan=True)
    assert torch.equal(got["bits"], c.bits) and torch.equal(got["record"], c.record)


@pytest.mark.parametrize("dtype,V", [("bf16", 20000), ("bf16", 2003), ("f32", 6000)])
def test_rows_without_a_token_are_never_filled(dtype, V):
    c = Case(3, 6, V, dtype, seed=29, fill=0.0, length=4, n_bias=0)
    # entropies far above tau: one slot falls back
    c.logits.copy_(torch.randn(c.logits.shape, generator=torch.Generator().manual_seed(V)).to(c.dt))
    c.mask_np[:] = -1
    c.mask_np[0] = 0                                                    # nothing allowed anywhere
    c.mask_np[1, :4] = 0                                                # the first rows only
    c.mask_index.copy_(_i32(c.mask_np))
    c.logits[2, 1] = float("-inf")                                      # the logits themselves leave nothing
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _confidence(c, status=st)
    assert st.item() == c.w.binding.WEDLM_STATUS_EMPTY_ROW
    assert got["filled_count"].tolist() == [0, 1, 1]
    assert got["fil"][0].sum() == 0 and (got["tok"][0] == V - 1).all()
    assert got["fil"][1].tolist() == [0, 0, 0, 0, 1, 0]
    assert got["argmax"][0].tolist() == [-1] * 6 and got["argmax"][2, 1] == -1 and (got["argmax"][2, [0, 2, 3, 4, 5]] >= 0).all()
    assert torch.equal(got["record"][0], c.record[0])
    assert _check_confidence(c, got) <= 1


@pytest.mark.parametrize("dtype,V", [("bf16", 16384 + 8), ("bf16", 3001), ("bf16", 20001), ("f32", 6000), ("f32", 9003)])
def test_very_low_and_tied_logits(dtype, V):
    """Rows at the type's lowest value throughout are uniform; ties go to the lowest token, across chunks and lanes; a
    touched token that ties with an untouched one counts like any other."""
    c = Case(1, 6, V, dtype, seed=31, fill=0.0, masked=0.0, length=6, n_bias=0)
    low = torch.finfo(c.dt).min
    c.pen[:, 0] = (1, 0, 0)
    c.rules = c.w.make_adjust(c.bits, c.record, allowed=c.allowed, mask_index=c.mask_index)
    x = torch.zeros(6, V)
    x[0] = low
    x[1] = low
    x[1, V - 1] = 1.0
    x[2] = -5.0                                                          # all equal
    x[3] = -5.0
    touched = min(c.hist[0].touched())
    x[3, [touched, V - 2, V // 2]] = 2.0
    x[4] = float("-inf")
    x[4, V - 3] = low
    x[5] = -1e25
    x[5, 5] = -1.5e25
    c.logits[0] = x.to(c.dt)
    got = _confidence(c)
    want = [0, V - 1, 0, min(touched, V // 2), V - 3, 0]
    assert got["argmax"][0].tolist() == want
    ent, mp = got["entropy"][0].double().cpu().numpy(), got["maxprob"][0].double().cpu().numpy()
    np.testing.assert_allclose(ent[[0, 2]], np.log(V), rtol=1e-6)
    np.testing.assert_allclose(mp[[0, 2]], 1 / V, rtol=1e-6)
    np.testing.assert_allclose(ent[[1, 4]], 0, atol=1e-6)
    np.testing.assert_allclose(mp[[1, 4]], 1, rtol=1e-6)
    np.testing.assert_allclose(mp[5], 1 / (V - 1), rtol=1e-6)
    np.testing.assert_allclose(ent[5], np.log(V - 1), rtol=1e-6)


@pytest.mark.parametrize("dtype,V", [("bf16", 4096), ("bf16", 1003), ("f32", 2000)])
def test_drawn_tokens_come_from_the_adjusted_logits(dtype, V):
    seed = (1 << 33) + 77
    c = Case(4, 8, V, dtype, seed=37, masked=0.7, cfg=dict(tau=50.0, sample_temperature=0.7, sample_seed=seed))
    got = _confidence(c)
    drawn = 0
    for b in range(4):
        nf = int(c.ro["n_filled"][b])
        new = []
        for i in range(nf, 8):
            x = c.expect_row(b, i)
            a = int(got["argmax"][b, i])
            if not (x > -np.inf).any():
                assert a == -1
                continue
            j = int(c.ro["perm"][b, i])
            with np.errstate(divide="ignore"):
                tok, margin = orc.sample_token(x, 0.7, (seed & 0xFFFFFFFF, seed >> 32), b, b * 11 + 5 + j)
            if margin > 1e-3:
                assert a == tok
                drawn += 1
            new.append(a)
            dst = j - int(c.ro["n_commit"][b])
            assert int(got["tok"][b, dst]) == a and int(got["fil"][b, dst]) == 1
        c.hist[b].add(new, False, V)
    assert drawn > 6
    _check_history(c, got["bits"], got["record"])


def test_histories_stay_as_they_are_without_count_fills():
    c = Case(3, 8, 9000, seed=41)
    r = c.w.make_adjust(c.bits, c.record, *[_f32(p) for p in c.pen], c.allowed, c.mask_index, count_fills=False)
    got, ref = _confidence(c, rules=r), _confidence(c)
    assert torch.equal(got["bits"], c.bits) and torch.equal(got["record"], c.record)
    assert torch.equal(got["tok"], ref["tok"]) and torch.equal(got["argmax"], ref["argmax"])


def test_short_windows_and_budgets():
    c = Case(4, 8, 9000, seed=43, fill=0.3)
    got = _confidence(c, window_len=[8, 5, 1, 0], budget=[9, 0, 1, 3])
    for b, n in enumerate((8, 5, 1, 0)):
        assert (got["argmax"][b, n:] == -1).all() and torch.isnan(got["entropy"][b, n:]).all()
    assert int(got["filled_count"][3]) == 0


def test_same_result_every_time_and_on_another_stream():
    c = Case(6, 16, 30000, seed=47, length=4000, masked=0.4)
    ref = _confidence(c)
    side = torch.cuda.Stream()
    for stream in (None, side):
        got = _confidence(c, stream=stream)
        for name in ref:
            assert torch.equal(torch.nan_to_num(got[name].double(), nan=-7.0), torch.nan_to_num(ref[name].double(), nan=-7.0)), name


def test_shapes_of_the_rules_are_checked():
    c = Case(2, 4, 300, seed=53)
    w = c.w
    out = torch.zeros_like(c.logits)
    for kw in (dict(repetition=_f32([1.0])), dict(allowed=c.allowed[:, :4].contiguous(), mask_index=c.mask_index),
               dict(allowed=c.allowed, mask_index=c.mask_index[:, :2].contiguous()), dict(token_bits=c.bits, token_record=c.record[:1])):
        with pytest.raises(ValueError):
            w.wedlm_logits_adjust(c.cfg, w.make_adjust(**kw), c.logits, out, c.perm, c.n_filled)
    with pytest.raises(TypeError):
        w.make_adjust(c.bits.float(), c.record)
    with pytest.raises(ValueError):
        w.wedlm_history_add(c.cfg, c.rules, torch.zeros(3, 4, dtype=torch.int32, device="cuda"), _i32([1, 1]))
    with pytest.raises(ValueError):
        w.wedlm_history_bias(c.cfg, c.rules, torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, device="cuda"))
