"""Cases of the operators that carry a layer's queries, keys and values through a cache held in 8 bits:

rope       norms of queries and keys for each head, with the position rotation in the same pass
rope_back  its gradients
append     keys and values of a window into pages of 8-bit codes, with one scale for each page and head
attention  attention of the windows over that cache, down to one token per sequence

Each is given in a plain form (elementary torch operations) and, where `own` is true, through this package's calls.
"""
import math
import random

import torch

own = False

HEADS = {"hq": 32, "hkv": 8, "d": 128}                     # heads of the serving configurations
THETA = 1.0e6
EPS = 1.0e-6
PAGE = 16
TOP = 448.0                                                # the largest e4m3 value
LOWEST = -64                                               # no page's scale is below 2^-64
YARN = {"factor": 4.0, "length": 32768, "fast": 32.0, "slow": 1.0}


def listed():
    bf = dict(dtype="bf16", hq=HEADS["hq"], hkv=HEADS["hkv"], d=HEADS["d"])
    rope = dict(op="rope", style=0, rotary=128, scaling="none", far=9000)
    return [
        # one request's window in one layer: the call's latency
        dict(bf, **rope, name="rope_one_window", batch=1, window=16),
        # a prefill chunk of a batch of long texts, context stretched fourfold
        dict(bf, **dict(rope, scaling="yarn", far=131072), name="rope_prefill", batch=16, window=1024),
        # the fp32 configuration, half of the head rotated, neighbouring pairs
        dict(op="rope", name="rope_fp32", dtype="f32", hq=4, hkv=2, d=64, style=1, rotary=32, scaling="linear", far=900, batch=2, window=37),
        # one training step's rows: both streams of eight sequences
        dict(bf, **dict(rope, op="rope_back", far=4096), name="rope_back_training", batch=16, window=512),
        # the same on a few rows
        dict(bf, **dict(rope, op="rope_back", far=600), name="rope_back_few", batch=3, window=33),
        # what one step of a serving batch stages
        dict(bf, op="append", name="append_step", batch=64, window=16, prefix=8192, layout=1),
        # prefill of a batch in chunks
        dict(bf, op="append", name="append_prefill", batch=8, window=1024, prefix=6000, layout=2),
        # one request: the call's latency
        dict(bf, op="attention", name="attention_one_request", batch=1, window=16, prefix=2048, layout=3),
        # plain decoding, one token per sequence, a full batch with ragged lengths
        dict(bf, op="attention", name="attention_single_tokens", batch=128, window=1, prefix=16000, layout=4),
        # the batched serving configuration
        dict(bf, op="attention", name="attention_serving", batch=64, window=32, prefix=8192, layout=5),
        # the long-context configuration
        dict(bf, op="attention", name="attention_long", batch=8, window=64, prefix=32768, layout=6),
        # the fp32 configuration
        dict(op="attention", name="attention_fp32", dtype="f32", hq=4, hkv=2, d=64, batch=6, window=8, prefix=330, layout=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope_back", "append", "attention", "attention", "attention"])
    layout = rng.randrange(100, 1 << 20)
    hq, hkv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 2), (8, 1), (12, 4)])
    case = dict(op=op, dtype="bf16", hq=hq, hkv=hkv, d=128)
    small = rng.random() < 0.2
    if small:
        case.update(dtype=rng.choice(["f32", "bf16"]), hq=4, hkv=2, d=rng.choice([32, 64]))
    if op in ("rope", "rope_back"):
        while True:
            batch, window = _log(rng, 1, 64), _log(rng, 1, 1024)
            if batch * window <= (2048 if small else 8192 if op == "rope_back" else 16384):
                break
        scaling = rng.choice(["none", "linear", "yarn"])
        return dict(case, style=rng.randrange(2), rotary=rng.choice([case["d"], case["d"], case["d"] // 2]), scaling=scaling,
                    far=_log(rng, 1100, 32768 if scaling == "none" else 131072), batch=batch, window=window)
    while True:
        batch, window = _log(rng, 1, 128), _log(rng, 1, 1024 if op == "append" else 64)
        prefix = _log(rng, 1, 32768)
        if small:
            batch, window, prefix = min(batch, 8), min(window, 16), min(prefix, 1024)
        if op == "append" and batch * window <= 8192 and batch * (prefix + window) <= 64 * 8300:
            break
        if op == "attention" and batch * prefix <= 64 * 8192 and batch * prefix * window <= 64 * 8192 * 16:
            break
    return dict(case, batch=batch, window=window, prefix=prefix, layout=layout)


# ---------------------------------------------------------------------------------------------- shapes that a case stands for
def _lengths(case):
    """Prefix length of each sequence: the longest first, the others ragged below it."""
    rng = random.Random(case["layout"])
    lens = [case["prefix"]] + [rng.randint(case["prefix"] // 8, case["prefix"]) for _ in range(case["batch"] - 1)]
    rng.shuffle(lens)
    return lens


def _counts(case):
    """Rows that an append stages: mostly the whole window, in some sequences a part of it or nothing."""
    rng = random.Random(case["layout"] + 1)
    return [case["window"] if rng.random() < 0.8 else rng.randint(0, case["window"]) for _ in range(case["batch"])]


def _inv_freq(case):
    """(f64 [rotary / 2] frequencies, factor on the rotated pairs), the scaled kinds by their published formulas."""
    r = case["rotary"]
    base = torch.pow(torch.tensor(THETA, dtype=torch.float64), -2 * torch.arange(r // 2, dtype=torch.float64) / r)
    if case["scaling"] == "linear":
        return base / 8.0, 1.0
    if case["scaling"] == "yarn":
        turns = YARN["length"] * base / (2 * math.pi)
        keep = ((turns - YARN["slow"]) / (YARN["fast"] - YARN["slow"])).clamp(0, 1)
        return base / YARN["factor"] * (1 - keep) + base * keep, 0.1 * math.log(YARN["factor"]) + 1
    return base, 1.0


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = _gen(seed)
    s = (_prepare_rope if case["op"] in ("rope", "rope_back") else _prepare_cache)(case, g)
    s["case"] = case
    if own:
        _make_handles(case, s)
    return s


def _split(case, x):
    """q, k and v of a fused projection [B, W, (Hq + 2 Hkv) D], as views."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    return [x[..., a * d: b * d].unflatten(-1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]


def _prepare_rope(case, g):
    n, w, d, dt = case["batch"], case["window"], case["d"], _dtype(case)
    width = (case["hq"] + 2 * case["hkv"]) * d
    s = {"qkv": (torch.randn(n, w, width, generator=g, device="cuda") * 1.7).to(dt)}
    s["q"], s["k"], _ = _split(case, s["qkv"])
    start = torch.randint(0, max(1, case["far"] - w), (n, 1), generator=g, device="cuda")
    order = torch.sort(torch.rand(n, w, generator=g, device="cuda"), dim=1).indices            # a reordered window
    s["pos_ids"] = (start + order).int()
    s["q_gain"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
    s["k_gain"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
    freq, s["factor"] = _inv_freq(case)
    s["freq"] = freq.cuda()
    if case["op"] == "rope_back":
        s["dq_out"] = torch.randn(n, w, case["hq"], d, generator=g, device="cuda").to(dt)
        s["dk_out"] = torch.randn(n, w, case["hkv"], d, generator=g, device="cuda").to(dt)
    return s


def _quantised(x):
    """(codes, scale) of pages x [..., page, d]: the smallest power of two that holds the page."""
    top = torch.where(x.isfinite(), x.abs(), 0).amax((-2, -1))
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (m > TOP / 512).int(), LOWEST).clamp(min=LOWEST)
    scale = torch.ldexp(torch.ones_like(top), e)
    return (x / scale[..., None, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn), scale


def _prepare_cache(case, g):
    n, w, hq, hkv, d, dt = case["batch"], case["window"], case["hq"], case["hkv"], case["d"], _dtype(case)
    prefix = _lengths(case)
    per = [-(-(p + w) // PAGE) for p in prefix]
    max_pages, total = max(per), sum(per)
    first = [sum(per[:b]) for b in range(n)]
    table = torch.tensor(first)[:, None] + torch.arange(max_pages)
    table = torch.where(torch.arange(max_pages) < torch.tensor(per)[:, None], table, 0)
    pool = torch.randperm(total + 3, generator=g, device="cuda")
    s = {"block_table": pool[table.cuda()].int(), "prefix_len": torch.tensor(prefix, dtype=torch.int32, device="cuda")}
    for x in ("k", "v"):
        size = torch.exp(0.5 * torch.randn(total + 3, hkv, 1, 1, generator=g, device="cuda"))     # some pages and heads are larger
        s[x + "_codes"], s[x + "_scale"] = _quantised(torch.randn(total + 3, hkv, PAGE, d, generator=g, device="cuda") * size)
    if case["op"] == "append":
        fused = torch.randn(n, w, (hq + 2 * hkv) * d, generator=g, device="cuda").to(dt)
        s["k"] = torch.randn(n, w, hkv, d, generator=g, device="cuda").to(dt)
        s["v"] = _split(case, fused)[2]
        s["count"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda")
    else:
        s["q"] = torch.randn(n, w, hq, d, generator=g, device="cuda").to(dt)
    return s


def _make_handles(case, s):
    """What a user's program keeps: the configuration, the frequencies, output buffers and the workspace."""
    import paper_2512_22737_b200 as wedlm
    s["lib"] = wedlm
    n, w, hq, hkv, d = case["batch"], case["window"], case["hq"], case["hkv"], case["d"]
    dims = dict(batch=n, window=w, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=PAGE, dtype=case["dtype"], rope_theta=THETA)
    empty = lambda *shape, dtype=_dtype(case): torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if case["op"] in ("rope", "rope_back"):
        s["cfg"] = wedlm.make_config(**dims, rope_style=case["style"])
        how = {"none": {}, "linear": dict(scaling="linear", factor=8.0),
               "yarn": dict(scaling="yarn", factor=YARN["factor"], original_len=YARN["length"], beta_fast=YARN["fast"], beta_slow=YARN["slow"])}
        s["rope"] = wedlm.make_rope(s["cfg"], rotary_dim=case["rotary"], **how[case["scaling"]])
        s["q_out"], s["k_out"] = empty(n, w, hq, d), empty(n, w, hkv, d)
        if case["op"] == "rope_back":
            s["dq_gain"], s["dk_gain"] = empty(d, dtype=torch.float32), empty(d, dtype=torch.float32)
            s["workspace"] = empty(wedlm.wedlm_norm_rope_backward_workspace_bytes(s["cfg"]), dtype=torch.uint8)
        return
    pages = s["block_table"].shape[1]
    s["cfg"] = wedlm.make_config(**dims, max_pages_per_seq=pages, num_pages=s["k_codes"].shape[0], max_prefix_len=pages * PAGE - w)
    if case["op"] == "append":
        s["slots"] = empty(n, w, dtype=torch.int32)
    else:
        s["out"] = empty(n, w, hq, d)
        s["workspace"] = empty(wedlm.wedlm_kvq_attn_workspace_bytes(s["cfg"]), dtype=torch.uint8)


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"rope": _run_rope, "rope_back": _run_rope_back, "append": _run_append, "attention": _run_attention}[s["case"]["op"]](s)


def _turns(s):
    """cos and sin of each row's angles, [B, W, 1, rotary / 2]; angles in 64 bits."""
    ang = s["pos_ids"].double()[..., None] * s["freq"]
    return (torch.cos(ang) * s["factor"]).float()[:, :, None], (torch.sin(ang) * s["factor"]).float()[:, :, None]


def _pairs(case, x):
    """The first and second members of the rotated pairs, and what is not rotated."""
    r = case["rotary"]
    if case["style"] == 0:
        return x[..., : r // 2], x[..., r // 2: r], x[..., r:]
    return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]


def _joined(case, a, b, rest):
    turned = torch.cat([a, b], -1) if case["style"] == 0 else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _run_rope(s):
    if own:
        s["lib"].wedlm_norm_rope(s["cfg"], s["rope"], s["q"], s["k"], s["pos_ids"], s["q_gain"], s["k_gain"], EPS, s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    return _turned(s, s["q"], s["q_gain"]), _turned(s, s["k"], s["k_gain"])


def _turned(s, x, gain):
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.float()
    cs, sn = _turns(s)
    a, b, rest = _pairs(s["case"], y)
    return _joined(s["case"], a * cs - b * sn, b * cs + a * sn, rest).to(x.dtype)


def _run_rope_back(s):
    if own:
        s["lib"].wedlm_norm_rope_backward(s["cfg"], s["rope"], s["q"], s["k"], s["pos_ids"], s["q_gain"], s["k_gain"], EPS, s["dq_out"], s["dk_out"],
                                          s["q_out"], s["k_out"], s["dq_gain"], s["dk_gain"], s["workspace"])
        return s["q_out"], s["k_out"], s["dq_gain"], s["dk_gain"]
    dq, dq_gain = _turned_back(s, s["q"], s["q_gain"], s["dq_out"])
    dk, dk_gain = _turned_back(s, s["k"], s["k_gain"], s["dk_out"])
    return dq, dk, dq_gain, dk_gain


def _turned_back(s, x, gain, dy):
    cs, sn = _turns(s)
    a, b, rest = _pairs(s["case"], dy.float())
    dn = _joined(s["case"], a * cs + b * sn, b * cs - a * sn, rest)
    y = x.float()
    r = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    hat = y * r
    dgain = (dn * hat).sum((0, 1, 2), dtype=torch.float64).float()
    dhat = dn * gain.float()
    return (r * (dhat - hat * (dhat * hat).mean(-1, keepdim=True))).to(x.dtype), dgain


def _run_append(s):
    if own:
        s["lib"].wedlm_kvq_append(s["cfg"], s["k"], s["v"], s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"], s["block_table"], s["prefix_len"],
                                  s["count"], s["slots"])
        return s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"], s["slots"]
    n, w = s["k"].shape[:2]
    first, count = s["prefix_len"].long()[:, None], s["count"].long()[:, None]
    span = (w + PAGE - 2) // PAGE + 1                                              # pages that a window can touch
    page_at = first // PAGE + torch.arange(span, device="cuda")
    used = (page_at * PAGE < first + count) & (count > 0)
    page = s["block_table"].long().gather(1, page_at.clamp(max=s["block_table"].shape[1] - 1))
    at = page_at[..., None] * PAGE + torch.arange(PAGE, device="cuda")             # [B, span, page] positions
    old, new = at < first[..., None], (at >= first[..., None]) & (at < (first + count)[..., None])
    row = (at - first[..., None]).clamp(0, w - 1)
    _stage(s["k"], s["k_codes"], s["k_scale"], page, used, old, new, row)
    _stage(s["v"], s["v_codes"], s["v_scale"], page, used, old, new, row)
    t = first + torch.arange(w, device="cuda")
    slots = s["block_table"].long().gather(1, t // PAGE) * PAGE + t % PAGE
    slots = torch.where(torch.arange(w, device="cuda") < count, slots, -1).int()
    return s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"], slots


def _stage(x, codes, scale, page, used, old, new, row):
    n = x.shape[0]
    come = x.float()[torch.arange(n, device="cuda")[:, None, None], row].transpose(2, 3)       # [B, span, Hkv, page, D]
    had = codes.view(torch.uint8)[page].view(torch.float8_e4m3fn)
    there = had.float() * scale[page][..., None, None]
    fresh, size = _quantised(torch.where(new[:, :, None, :, None], come, torch.where(old[:, :, None, :, None], there, 0)))
    fresh = torch.where((old | new)[:, :, None, :, None], fresh.view(torch.uint8), had.view(torch.uint8))
    codes.view(torch.uint8)[page[used]] = fresh[used]
    scale[page[used]] = size[used]


def _run_attention(s):
    if own:
        s["lib"].wedlm_kvq_attn(s["cfg"], s["q"], s["k_codes"], s["k_scale"], s["v_codes"], s["v_scale"], s["block_table"], s["prefix_len"], s["out"],
                                s["workspace"])
        return s["out"]
    n, w, hq, d = s["q"].shape
    hkv = s["k_codes"].shape[1]
    keys = _read(s, "k")
    score = torch.einsum("nwhgd,nhsd->nwhgs", s["q"].float().view(n, w, hkv, hq // hkv, d), keys) / math.sqrt(d)
    del keys
    last = s["prefix_len"][:, None] + torch.arange(w, device="cuda")
    seen = torch.arange(score.shape[-1], device="cuda") <= last[:, :, None]
    score = score.masked_fill(~seen[:, :, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    p = torch.exp(score)
    del score
    p /= p.sum(-1, keepdim=True)
    out = torch.einsum("nwhgs,nhsd->nwhgd", p, _read(s, "v"))
    return out.reshape(n, w, hq, d).to(s["q"].dtype)


def _read(s, x):
    """f32 [B, Hkv, max_pages * page, D]: each sequence's pages laid out one after the other."""
    page = s["block_table"].long()
    y = s[x + "_codes"].view(torch.uint8)[page].view(torch.float8_e4m3fn).float() * s[x + "_scale"][page][..., None, None]
    return y.transpose(1, 2).flatten(2, 3)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    n, w, hq, hkv, d = case["batch"], case["window"], case["hq"], case["hkv"], case["d"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        return {"bytes": n * w * ((hq + hkv) * d * size * 2 + 4), "flops": 8.0 * n * w * (hq + hkv) * d}
    if case["op"] == "rope_back":
        return {"bytes": n * w * ((hq + hkv) * d * size * 3 + 4) + 8 * d, "flops": 16.0 * n * w * (hq + hkv) * d}
    if case["op"] == "append":
        rows = sum(_counts(case))
        old = sum(p % PAGE for p, c in zip(_lengths(case), _counts(case)) if c)            # rows that share the first page
        return {"bytes": 2 * hkv * (rows * d * (size + 1) + old * d) + n * 8 + n * w * 4, "flops": 4.0 * rows * hkv * d}
    keys = sum(p + w for p in _lengths(case))
    pairs = sum(w * p + w * (w + 1) // 2 for p in _lengths(case))
    return {"bytes": keys * 2 * hkv * (d + 4 / PAGE) + n * w * hq * d * size * 2, "flops": 4.0 * pairs * hq * d}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "rope_back": _exact_rope_back, "append": _exact_append, "attention": _exact_attention}[case["op"]](case, s)


def _angle(case, s):
    """e^(i angle) of each row and pair, with the factor on it."""
    i = torch.arange(case["rotary"] // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(-2 * i / case["rotary"] * math.log(THETA))
    size = 1.0
    if case["scaling"] == "linear":
        f = f / 8
    elif case["scaling"] == "yarn":
        wave = 2 * math.pi / f
        gamma = torch.clamp((YARN["length"] / wave - YARN["slow"]) / (YARN["fast"] - YARN["slow"]), 0, 1)
        f = (1 - gamma) * f / YARN["factor"] + gamma * f
        size = 1 + math.log(YARN["factor"]) / 10
    a = s["pos_ids"].double()[:, :, None, None] * f
    return torch.polar(torch.full_like(a, size), a)


def _as_complex(case, x):
    r = case["rotary"]
    z = x[..., :r].reshape(*x.shape[:-1], *((2, r // 2) if case["style"] == 0 else (r // 2, 2)))
    return torch.complex(*z.unbind(-2 if case["style"] == 0 else -1))


def _as_real(case, z, rest):
    return torch.cat([torch.stack([z.real, z.imag], -2 if case["style"] == 0 else -1).flatten(-2), rest], -1)


def _exact_rope(case, s):
    out = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        x = x.double()
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.double()
        out.append(_as_real(case, _as_complex(case, y) * _angle(case, s), y[..., case["rotary"]:]))
    return tuple(out)


def _exact_rope_back(case, s):
    dx, dgain = [], []
    for x, gain, dy in ((s["q"], s["q_gain"], s["dq_out"]), (s["k"], s["k_gain"], s["dk_out"])):
        x, gain, dy = x.double(), gain.double(), dy.double()
        d = x.shape[-1]
        dn = _as_real(case, _as_complex(case, dy) * _angle(case, s).conj(), dy[..., case["rotary"]:])
        norm = torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
        dgain.append((dn * x / norm).sum((0, 1, 2)))
        along = (dn * gain * x).sum(-1, keepdim=True)
        dx.append(dn * gain / norm - x * along / (d * norm ** 3))
    return (*dx, *dgain)


def _exact_append(case, s):
    """Page by page: what it holds after the call, divided by the power of two that its largest value asks for, on the e4m3 grid.
    (log2 may miss a whole number by an ulp; 1e-9 is below the distance of the next fp32 value.)"""
    out = []
    for x in ("k", "v"):
        codes, scale = s[x + "_codes"].double(), s[x + "_scale"].double()
        for b in range(case["batch"]):
            first, count = int(s["prefix_len"][b]), int(s["count"][b])
            for j in range(first // PAGE, -(-(first + count) // PAGE) if count else 0):
                page, t0 = int(s["block_table"][b, j]), j * PAGE
                lo, hi = max(first - t0, 0), min(first + count - t0, PAGE)
                held = codes[page, :, :hi] * scale[page][:, None, None]
                held[:, lo:] = s[x][b, t0 + lo - first: t0 + hi - first].double().transpose(0, 1)
                top = held.abs().flatten(1).amax(1)
                scale[page] = torch.exp2(torch.ceil(torch.log2(top / TOP) - 1e-9).clamp(min=LOWEST))
                z = held / scale[page][:, None, None]
                step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6)) + 1e-9) - 3)
                codes[page, :, :hi] = torch.round(z / step) * step
        out += [codes, scale]
    return (*out, None)


def _pages(codes, pages):
    return torch.index_select(codes.view(torch.int8), 0, pages).view(torch.float8_e4m3fn).double()


def _exact_attention(case, s):
    n, w, hq, hkv, d = case["batch"], case["window"], case["hq"], case["hkv"], case["d"]
    out = torch.empty(n, w, hq, d, dtype=torch.float64, device="cuda")
    for b in range(n):
        p = int(s["prefix_len"][b])
        pages = s["block_table"][b, : -(-(p + w) // PAGE)].long()
        k, v = (_pages(s[x + "_codes"], pages) * s[x + "_scale"][pages].double()[:, :, None, None] for x in ("k", "v"))
        k = k.permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, : p + w]
        v = v.permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, : p + w]
        for h in range(hkv):
            group = slice(h * hq // hkv, (h + 1) * hq // hkv)
            score = s["q"][b, :, group].double() @ k[h].T / d ** 0.5
            for j in range(w):
                score[j, :, p + j + 1:] = -math.inf
            out[b, :, group] = torch.softmax(score, -1) @ v[h]
    return out
