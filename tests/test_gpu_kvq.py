"""The 8-bit cache: staging bit by bit, and attention over it, against the fp64 oracle.

Tolerances of the attention.  A weight p is off by a relative delta that the queries' and scores' roundings give, the sum of
  scale * 2^-18 * max|q| * max_j sum_d |k_jd|      the two-part split of q (tensor cores; exact for most elements of a bf16 row)
  scale * D * 2^-24 * max_j sum_d |q_d k_jd|       fp32 products and sums
  2^-21 * (1 + max|s|)                             the exponent's fp32 argument and 2^x
and by 2^-11 where it is rounded to fp16 (tensor cores); a sum over n keys adds n * 2^-24.  An output is an average: it is off by at
most (2 delta + 2^-11 + n * 2^-24) * average(|v|), and its rounding by half a step."""
import numpy as np
import pytest
import torch

from oracle import kvq_oracle as kq

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _f64(t):
    return t.detach().double().cpu().numpy()


def _cache(n_pages, Hkv, page, D, g, spread=1.0):
    """Pages as a program has them: codes and power-of-two scales of normal values, pages and heads of different size."""
    out = []
    for _ in range(2):
        x = g.standard_normal((n_pages, Hkv, page, D)) * np.exp(spread * g.standard_normal((n_pages, Hkv, 1, 1)))
        e = np.ceil(np.log2(np.abs(x).max((2, 3)) / kq.TOP))
        out += [kq.to_code(x * 2.0 ** -e[:, :, None, None]), (2.0 ** e).astype(np.float32)]
    return out


def _tables(prefix, W, page, g, spare=3):
    need = [-(-(p + W) // page) for p in prefix]
    pool = g.permutation(sum(need) + spare).astype(np.int32)
    table = np.zeros((len(prefix), max(need)), dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    return table, sum(need) + spare


def _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages, **kw):
    return w.make_config(batch=len(prefix), window=W, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_size=page, dtype=dtype,
                         max_pages_per_seq=table.shape[1], num_pages=n_pages, max_prefix_len=table.shape[1] * page - W, **kw)


def _run_attention(w, cfg, q, cache, table, prefix, status=None):
    kc, ks, vc, vs = (torch.from_numpy(x).cuda() for x in cache)
    out = torch.full(q.shape, 3.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(w.wedlm_kvq_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    w.wedlm_kvq_attn(cfg, q, kc, ks, vc, vs, torch.from_numpy(table).cuda(), torch.tensor(prefix, dtype=torch.int32, device="cuda"), out, ws, status)
    torch.cuda.synchronize()
    return out


def _tolerance(q, cache, table, prefix, scale, size, dtype, tensor):
    page = cache[0].shape[2]
    B, W, Hq, D = q.shape
    Hkv = cache[0].shape[1]
    tol = np.zeros(size.shape)
    for b in range(B):
        n = prefix[b] + W
        pages = table[b, : -(-n // page)].astype(np.int64)
        k = (kq.VALUES[cache[0][pages]] * cache[1][pages].astype(np.float64)[:, :, None, None]).transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n]
        for h in range(Hq):
            ak = np.abs(k[h * Hkv // Hq])
            for i in range(W):
                aq = np.abs(q[b, i, h])
                dots = ak @ aq
                delta = scale * D * 2.0 ** -24 * dots.max() + 2.0 ** -21 * (1 + scale * dots.max())
                if tensor:
                    delta += scale * 2.0 ** -18 * aq.max() * ak.sum(-1).max()
                tol[b, i, h] = (2 * delta + (2.0 ** -11 if tensor else 0) + n * 2.0 ** -24) * size[b, i, h]
    return tol


def _check_attention(dtype, prefix, W, Hq, Hkv, D, page, impl="auto", seed=0, spread=1.0, qsize=1.0, edit=None, softmax_scale=0.0):
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(seed)
    table, n_pages = _tables(prefix, W, page, g)
    cache = _cache(n_pages, Hkv, page, D, g, spread)
    if edit:
        edit(cache, table)
    q = torch.from_numpy(g.standard_normal((len(prefix), W, Hq, D)).astype(np.float32) * qsize).cuda().to(_dt(dtype))
    cfg = _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages, attn_impl=impl, softmax_scale=softmax_scale)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = _run_attention(w, cfg, q, cache, table, prefix, status)
    assert int(status.item()) == 0
    scale = softmax_scale if softmax_scale else D ** -0.5
    ref, size = kq.attention(_f64(q), *cache, table, prefix, scale)
    tensor = dtype == "bf16" and D == 128 and page == 16 and impl != "generic"
    tol = _tolerance(_f64(q), cache, table, prefix, scale, size, dtype, tensor) + HALF[dtype] * np.abs(ref)
    err = np.abs(_f64(out) - ref)
    assert (err <= tol).all(), float((err / tol).max())
    return out


@pytest.mark.parametrize("prefix,W,Hq,Hkv", [
    ([0], 1, 4, 1), ([1], 1, 4, 1), ([127], 1, 4, 1), ([128, 500, 3], 1, 32, 8),                # N = 16: single tokens
    ([255, 0, 16], 4, 4, 1), ([130, 700], 3, 20, 4),                                            # 16 rows, and 15 in 16
    ([64, 1000], 8, 8, 2), ([300], 7, 12, 4),                                                   # N = 32, head groups of 3
    ([0, 77, 1200], 16, 4, 1), ([513], 9, 14, 2),                                               # N = 64, groups of 7
    ([5, 640], 32, 8, 2), ([1000], 33, 3, 3), ([90], 128, 1, 1),                                # N = 128
    ([200, 0], 64, 4, 1), ([33], 70, 6, 2), ([17], 5, 128, 1), ([40], 3, 50, 1),                # several row tiles
])
def test_attention_tensor_cores(prefix, W, Hq, Hkv):
    _check_attention("bf16", prefix, W, Hq, Hkv, 128, 16, impl="tensor", seed=W)


@pytest.mark.parametrize("prefix,W,Hq,Hkv", [([300, 17], 2, 8, 2), ([129], 1, 14, 2), ([700, 2], 8, 1, 1), ([513, 40], 1, 9, 1), ([64], 3, 6, 2)])
def test_attention_of_about_eight_rows(prefix, W, Hq, Hkv):
    _check_attention("bf16", prefix, W, Hq, Hkv, 128, 16, impl="tensor", seed=40 + W)


@pytest.mark.parametrize("dtype,prefix,W,Hq,Hkv,D,page", [
    ("f32", [0, 330, 64], 8, 4, 2, 64, 16), ("f32", [1], 1, 2, 1, 32, 8), ("f32", [100, 31], 5, 6, 2, 128, 32), ("f32", [70], 3, 2, 2, 256, 16),
    ("bf16", [500, 7], 9, 8, 2, 64, 16), ("bf16", [65], 20, 4, 4, 32, 32), ("bf16", [129, 12], 4, 4, 1, 128, 8), ("bf16", [200], 2, 8, 1, 256, 8),
])
def test_attention_cuda_cores(dtype, prefix, W, Hq, Hkv, D, page):
    _check_attention(dtype, prefix, W, Hq, Hkv, D, page, seed=D)


def test_attention_both_paths_on_the_same_cache():
    for prefix, W in (([700, 20], 4), ([513], 16)):
        a = _check_attention("bf16", prefix, W, 8, 2, 128, 16, impl="tensor", seed=3)
        b = _check_attention("bf16", prefix, W, 8, 2, 128, 16, impl="generic", seed=3)
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -6 * b.float().abs().max()


@pytest.mark.parametrize("W", [1, 4, 16, 32])
def test_scores_that_grow_move_the_references(W):
    """Keys further on are ever larger, so that references move in almost every tile and accumulators follow."""
    def grow(cache, table):
        order = table[0]
        for j, page in enumerate(order):
            cache[1][page] *= np.float32(2.0) ** (j // 8)
    _check_attention("bf16", [1150], W, 4, 1, 128, 16, impl="tensor", seed=5, spread=0.3, edit=grow)


@pytest.mark.parametrize("W", [1, 16, 32])
def test_values_of_very_different_size(W):
    """The page that holds nearly all of the weight has values far below the others'."""
    def sink(cache, table):
        cache[1][table[0, 0]] *= np.float32(16.0)
        cache[3][table[0, 0]] *= np.float32(2.0 ** -20)
        cache[3][table[0, 7]] *= np.float32(2.0 ** 30)
    _check_attention("bf16", [600], W, 4, 1, 128, 16, impl="tensor", seed=6, spread=0.1, edit=sink)


def test_scales_need_not_be_powers_of_two_and_pages_may_be_zero():
    def odd(cache, table):
        cache[1][:] *= np.float32(1.37)
        cache[3][:] *= np.float32(0.77)
        cache[2][table[0, 1]] = 0
        cache[0][table[0, 2]] = 0
    _check_attention("bf16", [300, 40], 4, 8, 2, 128, 16, impl="tensor", seed=7, edit=odd)
    _check_attention("f32", [300, 40], 4, 8, 2, 64, 16, seed=7, edit=odd)


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_softmax_scale(scale):
    _check_attention("bf16", [400], 2, 8, 2, 128, 16, impl="tensor", seed=8, spread=0.2, softmax_scale=scale)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_rows_behind_the_window_may_hold_anything(dtype, D):
    """Codes of NaN in the rest of the last page, and in pages that no table entry in use names."""
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(9)
    prefix, W, Hq, Hkv, page = [37, 250], 4, 4, 1, 16
    table, n_pages = _tables(prefix, W, page, g)
    cache = _cache(n_pages, Hkv, page, D, g)
    q = torch.from_numpy(g.standard_normal((2, W, Hq, D)).astype(np.float32)).cuda().to(_dt(dtype))
    cfg = _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages)
    clean = _run_attention(w, cfg, q, cache, table, prefix)
    used = {(int(table[b, t // page]), t % page) for b in range(2) for t in range(prefix[b] + W)}
    for p in range(n_pages):
        for r in range(page):
            if (p, r) not in used:
                cache[0][p, :, r] = 0x7F
                cache[2][p, :, r] = 0xFF
    for p in set(range(n_pages)) - {p for p, _ in used}:
        cache[1][p] = np.nan
        cache[3][p] = np.inf
    table[0, -(-(prefix[0] + W) // page):] = -5                                  # entries behind the sequence are not looked at
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert torch.equal(_run_attention(w, cfg, q, cache, table, prefix, status), clean) and int(status.item()) == 0


@pytest.mark.parametrize("dtype,D,W", [("bf16", 128, 4), ("bf16", 128, 7), ("bf16", 128, 40), ("f32", 64, 12)])
def test_rows_of_a_padded_window_may_hold_anything(dtype, D, W):
    """Fewer rows stored than the window has, into pages of NaN codes and scales that are no scales: the stored rows' results are
    those of a cache without any of that."""
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(12)
    Hq, Hkv, page = 4, 1, 16
    prefix, count = [0, 31, 125, 256], [1, W - 1, 3, 2]
    table, n_pages = _tables(prefix, W, page, g)
    clean = _cache(n_pages, Hkv, page, D, g)
    dirty = [x.copy() for x in clean]
    for b, (P, n) in enumerate(zip(prefix, count)):
        for t in range(P + n, P + W):
            dirty[0][table[b, t // page], :, t % page] = 0xFF
            dirty[2][table[b, t // page], :, t % page] = 0x7F
        for j in range(-(-(P + n) // page), -(-(P + W) // page)):                # pages without a stored row
            dirty[1][table[b, j]] = [np.nan, 0.0, -2.0, np.inf][(b + j) % 4]
            dirty[3][table[b, j]] = [0.0, np.nan, np.inf, -1.0][(b + j) % 4]
    q = torch.from_numpy(g.standard_normal((4, W, Hq, D)).astype(np.float32)).cuda().to(_dt(dtype))
    cfg = _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages)
    want, got = (_run_attention(w, cfg, q, c, table, prefix) for c in (clean, dirty))
    for b, n in enumerate(count):
        assert torch.equal(got[b, :n], want[b, :n]), b


@pytest.mark.parametrize("W", [3, 33])
def test_nan_and_infinite_queries_of_short_and_long_windows(W):
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(13)
    prefix, Hq, Hkv, D, page = [300], 4, 1, 128, 16
    table, n_pages = _tables(prefix, W, page, g)
    cache = _cache(n_pages, Hkv, page, D, g)
    q = torch.from_numpy(g.standard_normal((1, W, Hq, D)).astype(np.float32)).cuda().to(torch.bfloat16)
    cfg = _config(w, "bf16", prefix, W, Hq, Hkv, D, page, table, n_pages)
    clean = _run_attention(w, cfg, q, cache, table, prefix)
    q[0, 0, 1, 5], q[0, 1, 0, 3], q[0, W - 1, 3, 0] = float("nan"), float("-inf"), float("inf")
    out = _run_attention(w, cfg, q, cache, table, prefix)
    same = (out == clean).all(-1)
    assert torch.isnan(out[0, 0, 1]).all() and torch.isnan(out[0, 1, 0]).all() and torch.isnan(out[0, W - 1, 3]).all()
    assert int((~same).sum()) == 3


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_nan_and_infinite_queries_stay_in_their_row(dtype, D):
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(10)
    prefix, W, Hq, Hkv, page = [300], 8, 4, 1, 16
    table, n_pages = _tables(prefix, W, page, g)
    cache = _cache(n_pages, Hkv, page, D, g)
    q = torch.from_numpy(g.standard_normal((1, W, Hq, D)).astype(np.float32)).cuda().to(_dt(dtype))
    cfg = _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages)
    clean = _run_attention(w, cfg, q, cache, table, prefix)
    q[0, 2, 1, 5], q[0, 6, 3, 0] = float("nan"), float("inf")
    out = _run_attention(w, cfg, q, cache, table, prefix)
    same = (out == clean).all(-1)
    assert torch.isnan(out[0, 2, 1]).all() and torch.isnan(out[0, 6, 3]).all()
    assert int((~same).sum()) == 2


def test_bad_pages_and_lengths_are_reported():
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(11)
    prefix, W, Hq, Hkv, page = [40, 300], 2, 4, 1, 16
    for dtype, D in (("bf16", 128), ("f32", 64)):
        table, n_pages = _tables(prefix, W, page, g)
        cache = _cache(n_pages, Hkv, page, D, g)
        q = torch.from_numpy(g.standard_normal((2, W, Hq, D)).astype(np.float32)).cuda().to(_dt(dtype))
        cfg = _config(w, dtype, prefix, W, Hq, Hkv, D, page, table, n_pages)
        clean = _run_attention(w, cfg, q, cache, table, prefix)
        table[1, 3] = n_pages + 7
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = _run_attention(w, cfg, q, cache, table, prefix, status)
        assert int(status.item()) == 1 and torch.equal(out[0], clean[0]) and torch.isfinite(out).all()
        # keys of the missing page are left out
        keep = [j for j in range(-(-(prefix[1] + W) // page)) if j != 3]
        short = np.zeros_like(table)
        short[0], short[1, : len(keep)] = table[0], table[1, keep]
        less = _run_attention(w, cfg, q, cache, short, [prefix[0], prefix[1] - page])
        assert (out[1].float() - less[1].float()).abs().max() <= 2.0 ** -6 * less[1].float().abs().max()
        table[1, 3] = 0
        status.zero_()
        _run_attention(w, cfg, q, cache, table, [-3, table.shape[1] * page], status)
        assert int(status.item()) == 2


@pytest.mark.parametrize("B,W", [(300, 1), (1500, 1), (260, 9)])
def test_many_sequences(B, W):
    """More sequences than a block of the plan has threads, and than it keeps in shared memory."""
    g = np.random.default_rng(B)
    prefix = g.integers(0, 200, B).tolist()
    import paper_2512_22737_b200 as w
    table, n_pages = _tables(prefix, W, 16, g)
    cache = _cache(n_pages, 1, 16, 128, g)
    q = torch.from_numpy(g.standard_normal((B, W, 4, 128)).astype(np.float32)).cuda().bfloat16()
    cfg = _config(w, "bf16", prefix, W, 4, 1, 128, 16, table, n_pages)
    out = _f64(_run_attention(w, cfg, q, cache, table, prefix))
    for b in list(range(0, B, 97)) + [B - 1]:
        one = lambda x: x[b:b + 1]  # noqa: E731
        ref, size = kq.attention(_f64(q[b:b + 1]), *cache, one(table), prefix[b:b + 1], 128 ** -0.5)
        tol = _tolerance(_f64(q[b:b + 1]), cache, one(table), prefix[b:b + 1], 128 ** -0.5, size, "bf16", True) + HALF["bf16"] * np.abs(ref)
        assert (np.abs(out[b:b + 1] - ref) <= tol).all()


@pytest.mark.parametrize("W,Hq", [(1, 4), (16, 4)])
def test_a_unit_in_more_pieces_than_a_warp_has_lanes(W, Hq):
    _check_attention("bf16", [20000], W, Hq, 1, 128, 16, impl="tensor", seed=13, spread=0.2)


def test_pools_beyond_32_bit_offsets():
    """Pages that begin beyond 2^31 bytes, in both paths and in the staging."""
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(14)
    Hkv, page, D, W, prefix = 8, 16, 128, 4, [60, 200]
    n_pages = 140_000                                              # 16 KB a page
    small, _ = _tables(prefix, W, page, g)
    used = sorted({int(x) for x in small.reshape(-1)})
    where = {p: n_pages - 1 - 3 * i for i, p in enumerate(used)}
    table = np.vectorize(lambda x: where[int(x)])(small).astype(np.int32)
    part = _cache(max(used) + 1, Hkv, page, D, g)
    pools = [torch.zeros((n_pages, *x.shape[1:]), dtype=torch.uint8 if x.dtype == np.uint8 else torch.float32, device="cuda") for x in part]
    at = torch.tensor([where[p] for p in used], device="cuda")
    for pool, x in zip(pools, part):
        pool[at] = torch.from_numpy(x[used]).cuda()
    q = torch.from_numpy(g.standard_normal((2, W, 8, D)).astype(np.float32)).cuda().bfloat16()
    lens = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    for impl in ("tensor", "generic"):
        want = None
        for tb, cache, n in ((small, [torch.from_numpy(x).cuda() for x in part], part[0].shape[0]), (table, pools, n_pages)):
            cfg = _config(w, "bf16", prefix, W, 8, Hkv, D, page, tb, n, attn_impl=impl)
            out = torch.empty_like(q)
            ws = torch.empty(w.wedlm_kvq_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            w.wedlm_kvq_attn(cfg, q, *cache, torch.from_numpy(tb).cuda(), lens, out, ws)
            k = torch.from_numpy(np.random.default_rng(1).standard_normal((2, W, Hkv, D)).astype(np.float32)).cuda().bfloat16()
            if impl == "generic":
                w.wedlm_kvq_append(cfg, k, k, *cache, torch.from_numpy(tb).cuda(), lens)
                after = torch.empty_like(q)
                w.wedlm_kvq_attn(cfg, q, *cache, torch.from_numpy(tb).cuda(), lens, after, ws)
                out = torch.stack([out, after])
            if want is None:
                want = out
        assert torch.equal(out, want)


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own."""
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(15)
    jobs = []
    for W, prefix in ((1, [3000, 100, 700]), (16, [1500, 40])):
        table, n_pages = _tables(prefix, W, 16, g)
        cache = [torch.from_numpy(x).cuda() for x in _cache(n_pages, 2, 16, 128, g)]
        cfg = _config(w, "bf16", prefix, W, 8, 2, 128, 16, table, n_pages)
        q = torch.from_numpy(g.standard_normal((len(prefix), W, 8, 128)).astype(np.float32)).cuda().bfloat16()
        ws = torch.empty(w.wedlm_kvq_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        jobs.append((cfg, q, cache, torch.from_numpy(table).cuda(), torch.tensor(prefix, dtype=torch.int32, device="cuda"), torch.empty_like(q), ws,
                     torch.cuda.Stream()))
    want = []
    for cfg, q, cache, table, lens, out, ws, _ in jobs:
        w.wedlm_kvq_attn(cfg, q, *cache, table, lens, out, ws)
        torch.cuda.synchronize()
        want.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(30):
        for cfg, q, cache, table, lens, out, ws, st in jobs:
            w.wedlm_kvq_attn(cfg, q, *cache, table, lens, out, ws, None, st)
    torch.cuda.synchronize()
    assert all(torch.equal(j[5], x) for j, x in zip(jobs, want))


def test_attention_under_a_graph_on_another_stream_and_with_shared_buffers():
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(12)
    prefix, W, Hq, Hkv, D, page = [900, 100, 2000], 4, 8, 2, 128, 16
    table, n_pages = _tables(prefix, W, page, g)
    cache = [torch.from_numpy(x).cuda() for x in _cache(n_pages, Hkv, page, D, g)]
    cfg = _config(w, "bf16", prefix, W, Hq, Hkv, D, page, table, n_pages)
    q = torch.from_numpy(g.standard_normal((3, W, Hq, D)).astype(np.float32)).cuda().bfloat16()
    table, lens = torch.from_numpy(table).cuda(), torch.tensor(prefix, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(w.wedlm_kvq_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    call = lambda o=out: w.wedlm_kvq_attn(cfg, q, *cache, table, lens, o, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    lens -= 60                                                   # a replay reads the lengths as they are then
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    moved = out.clone()
    call()
    assert torch.equal(moved, out) and not torch.equal(moved, want)
    lens += 60
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            ws.fill_(255)                                        # nothing is taken over from an earlier call
            call()
    side.synchronize()
    assert torch.equal(out, want)


# ---------------------------------------------------------------------------------------------- staging
def _append(w, cfg, k, v, cache, table, prefix, count, status=None, slots=True):
    dev = [torch.from_numpy(x).cuda() for x in cache]
    idx = torch.full((cfg.batch, cfg.window), 99, dtype=torch.int32, device="cuda") if slots else None
    w.wedlm_kvq_append(cfg, k, v, *dev, torch.from_numpy(table).cuda(), torch.tensor(prefix, dtype=torch.int32, device="cuda"),
                       None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda"), idx, status)
    return [x.cpu().numpy() for x in dev], None if idx is None else idx.cpu().numpy()


def _same_codes(a, b):
    nan = (a & 127) == 127
    return np.array_equal(nan, (b & 127) == 127) and np.array_equal(a[~nan], b[~nan])


@pytest.mark.parametrize("dtype,prefix,W,count,Hkv,D,page", [
    ("bf16", [0, 5, 15, 16, 100], 1, None, 8, 128, 16),
    ("bf16", [3, 64, 31], 40, [40, 0, 17], 2, 128, 16),
    ("bf16", [9], 100, [1000], 1, 64, 8), ("bf16", [30, 7], 6, [-4, 6], 3, 32, 32), ("bf16", [11], 70, None, 2, 256, 32),
    ("f32", [0, 14], 5, None, 2, 64, 16), ("f32", [40], 33, [30], 1, 256, 32), ("f32", [7, 8], 3, None, 4, 32, 8), ("f32", [1], 9, None, 2, 128, 16),
])
def test_append(dtype, prefix, W, count, Hkv, D, page):
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(D + W)
    table, n_pages = _tables(prefix, W, page, g)
    cache = _cache(n_pages, Hkv, page, D, g)
    B = len(prefix)
    size = np.exp(2 * g.standard_normal((B, W, Hkv, 1)))
    k = torch.from_numpy((g.standard_normal((B, W, Hkv, D)) * size).astype(np.float32)).cuda().to(_dt(dtype))
    fused = torch.from_numpy(g.standard_normal((B, W, 3 * Hkv * D)).astype(np.float32)).cuda().to(_dt(dtype))
    v = fused[..., Hkv * D: 2 * Hkv * D].unflatten(-1, (Hkv, D))
    cfg = _config(w, dtype, prefix, W, Hkv, Hkv, D, page, table, n_pages)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, slots = _append(w, cfg, k, v, cache, table, prefix, count, status)
    assert int(status.item()) == 0
    for i, rows in ((0, k), (2, v)):
        codes, scale, want_slots = kq.append(_f64(rows), cache[i], cache[i + 1], table, prefix, count, page)
        assert np.array_equal(got[i], codes) and np.array_equal(got[i + 1], scale.astype(np.float32)) and np.array_equal(slots, want_slots)
    again, _ = _append(w, cfg, k, v, got, table, prefix, count)                  # staged anew, nothing moves
    assert all(np.array_equal(a, b) for a, b in zip(again, got))


def test_append_of_odd_values():
    """Zeros, infinities, NaN, values below the lowest scale and near the largest float."""
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(20)
    for dtype in ("bf16", "f32"):
        table, n_pages = _tables([0] * 5, 16, 16, g)
        cache = _cache(n_pages, 1, 16, 64, g)
        k = g.standard_normal((5, 16, 1, 64)).astype(np.float32)
        k[0] = 0
        k[1, 3, 0, 7], k[1, 4, 0, 0], k[1, 5, 0, 9] = np.inf, -np.inf, np.nan
        k[2] *= np.float32(1e-30)
        k[3] *= np.float32(2.0 ** 125)
        k[4] = np.nan
        kt = torch.from_numpy(k).cuda().to(_dt(dtype))
        cfg = _config(w, dtype, [0] * 5, 16, 1, 1, 64, 16, table, n_pages)
        got, _ = _append(w, cfg, kt, kt, cache, table, [0] * 5, None)
        x = _f64(kt)
        for i in (0, 2):
            codes, scale, _ = kq.append(x, cache[i], cache[i + 1], table, [0] * 5, None, 16)
            assert _same_codes(got[i], codes) and np.array_equal(got[i + 1], scale.astype(np.float32))


def test_append_to_bad_pages_and_lengths():
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(21)
    prefix, W = [10, 20], 20
    table, n_pages = _tables(prefix, W, 16, g)
    cache = _cache(n_pages, 2, 16, 64, g)
    k = torch.randn(2, W, 2, 64, device="cuda")
    cfg = _config(w, "f32", prefix, W, 2, 2, 64, 16, table, n_pages)
    bad = table.copy()
    bad[0, 1] = n_pages
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, slots = _append(w, cfg, k, k, cache, bad, prefix, None, status)
    codes, scale, want = kq.append(_f64(k), cache[0], cache[1], bad, prefix, None, 16)
    assert int(status.item()) == 1 and np.array_equal(got[0], codes) and np.array_equal(slots, want) and (want[0, 6:] == -1).any()
    status.zero_()
    got, slots = _append(w, cfg, k, k, cache, table, [2 ** 31 - 5, 2 ** 31 - 16], None, status)
    assert int(status.item()) == 2 and np.array_equal(got[0], cache[0]) and (slots == -1).all()
    status.zero_()
    got, slots = _append(w, cfg, k, k, cache, table, [-1, table.shape[1] * 16 - 4], None, status)
    codes, _, want = kq.append(_f64(k)[1:], cache[0], cache[1], table[1:], [table.shape[1] * 16 - 4], None, 16)
    assert int(status.item()) == 2 and np.array_equal(got[0], codes) and (slots[0] == -1).all() and np.array_equal(slots[1:], want)


def test_refusals():
    import paper_2512_22737_b200 as w
    g = np.random.default_rng(22)
    table, n_pages = _tables([20], 4, 16, g)
    cache = [torch.from_numpy(x).cuda() for x in _cache(n_pages, 2, 16, 64, g)]
    cfg = _config(w, "bf16", [20], 4, 4, 2, 64, 16, table, n_pages)
    q = torch.zeros(1, 4, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    tb, lens = torch.from_numpy(table).cuda(), torch.tensor([20], dtype=torch.int32, device="cuda")
    ws = torch.empty(w.wedlm_kvq_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="k_scale"):
        w.wedlm_kvq_append(cfg, k, k, cache[0], cache[1][:1], cache[2], cache[3], tb, lens)
    with pytest.raises(TypeError, match="k_codes"):
        w.wedlm_kvq_append(cfg, k, k, cache[0].float(), *cache[1:], tb, lens)
    with pytest.raises(ValueError, match="shape"):
        w.wedlm_kvq_attn(cfg, q[:, :2], *cache, tb, lens, q, ws)
    with pytest.raises(w.WedlmError):
        w.wedlm_kvq_attn(cfg, q, *cache, tb, lens, torch.empty_like(q), ws[:16])
    tensor = _config(w, "bf16", [20], 4, 4, 2, 64, 16, table, n_pages, attn_impl="tensor")
    with pytest.raises(w.WedlmError):                                            # head_dim 64 is not the tensor cores'
        w.wedlm_kvq_attn(tensor, q, *cache, tb, lens, torch.empty_like(q), ws)
    w.wedlm_kvq_append(cfg, k, k, cache[0].view(torch.float8_e4m3fn), cache[1], cache[2].view(torch.float8_e4m3fn), cache[3], tb, lens)
    empty = w.make_config(batch=0, window=4, n_q_heads=4, n_kv_heads=2, head_dim=64, max_pages_per_seq=table.shape[1], num_pages=n_pages)
    w.wedlm_kvq_attn(empty, q[:0], *cache, tb[:0], lens[:0], torch.empty_like(q[:0]), ws)
    w.wedlm_kvq_append(empty, k[:0], k[:0], *cache, tb[:0], lens[:0])
