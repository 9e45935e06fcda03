"""Cases of the operators that serve a batch whose requests share a prompt and differ in their rules:

attention   window attention of groups of sequences that share their leading cache pages
confidence  confidence and commit on logits with penalties, biases and allowed-token masks
adjust      the same adjustment of logits alone, for callers with a sampler of their own
history     upkeep of the token histories that the penalties read

Each is given in a plain form (elementary torch operations) and, where `own` is true, through this package's calls.
"""
import math
import random

import torch

own = False

QWEN = {"hq": 32, "hkv": 8, "d": 128, "theta": 1.0e6, "vocab": 151936}   # heads and vocabulary of the serving configurations
PAGE = 16
TAU, LAM = 0.35, 0.1


def listed():
    att = dict(op="attention", dtype="bf16", hq=QWEN["hq"], hkv=QWEN["hkv"], d=QWEN["d"])
    voc = dict(dtype="bf16", vocab=QWEN["vocab"])
    return [
        # four answers drawn side by side from one prompt: the call's latency
        dict(att, name="attention_four_answers", batch=4, window=8, groups=1, shared=1040, own_len=40, layout=1),
        # a serving batch with three system prompts, ragged answers
        dict(att, name="attention_three_prompts", batch=32, window=16, groups=3, shared=4099, own_len=700, layout=2),
        # a full batch of answers over one long document
        dict(att, name="attention_long_document", batch=64, window=16, groups=1, shared=16384, own_len=1024, layout=3),
        # one token per sequence: plain decoding on two prompts, an odd batch
        dict(att, name="attention_single_tokens", batch=61, window=1, groups=2, shared=8200, own_len=512, layout=4),
        # the fp32 configuration
        dict(op="attention", name="attention_fp32", dtype="f32", hq=4, hkv=2, d=64, batch=6, window=8, groups=2, shared=330, own_len=50, layout=5),
        # one request with penalties
        dict(voc, op="confidence", name="confidence_one_request", batch=1, window=16, history=500, masked=0.0, layout=6),
        # a serving batch with penalties and biases
        dict(voc, op="confidence", name="confidence_penalties", batch=64, window=32, history=8192, masked=0.0, layout=7),
        # structured output: most rows under a grammar
        dict(voc, op="confidence", name="confidence_grammars", batch=48, window=32, history=2000, masked=0.9, layout=8),
        # the fp32 configuration with its odd vocabulary
        dict(op="adjust", name="adjust_fp32", dtype="f32", vocab=1001, batch=2, window=8, history=90, masked=0.5, layout=9),
        # a serving batch whose sampler is the caller's
        dict(voc, op="adjust", name="adjust_batch", batch=64, window=32, history=3000, masked=0.4, layout=10),
        # what one step adds
        dict(op="history", name="history_step", vocab=QWEN["vocab"], batch=64, length=32, prompt=False, layout=11),
        # admission of a batch of prompts
        dict(op="history", name="history_prompts", vocab=QWEN["vocab"], batch=64, length=8192, prompt=True, layout=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "confidence", "confidence", "adjust", "history"])
    layout = rng.randrange(100, 1 << 20)
    if op == "attention":
        while True:
            batch, window = _log(rng, 2, 64), _log(rng, 1, 33)
            shared, own_len = _log(rng, 33, 16384), _log(rng, 1, 1024)
            if batch * (shared + own_len) * max(window, 8) <= 64 * 17408 * 16:
                break
        case = dict(op=op, batch=batch, window=window, groups=rng.randint(1, max(1, batch // 4)), shared=shared, own_len=own_len, layout=layout)
        if rng.random() < 0.8:
            hq, hkv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 2), (8, 1)])
            return dict(case, dtype="bf16", hq=hq, hkv=hkv, d=128)
        case.update(batch=min(batch, 8), window=min(window, 16), shared=min(shared, 1024), own_len=min(own_len, 200), groups=min(case["groups"], 2))
        return dict(case, dtype=rng.choice(["f32", "bf16"]), hq=4, hkv=2, d=rng.choice([32, 64]))
    if op == "history":
        return dict(op=op, vocab=_log(rng, 1000, 151936), batch=_log(rng, 1, 64), length=_log(rng, 1, 8192), prompt=rng.random() < 0.5, layout=layout)
    batch, window = _log(rng, 1, 64), _log(rng, 1, 32)
    vocab = rng.choice([_log(rng, 100, 151936), 8 * _log(rng, 100, 18992), 151936])
    return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), vocab=vocab, batch=batch, window=window, history=_log(rng, 1, 8192),
                masked=rng.choice([0.0, 0.3, 0.9]), layout=layout)


# ---------------------------------------------------------------------------------------------- shapes that a case stands for
def _attention_layout(case):
    """(group of each sequence, shared pages of each group, prefix length of each sequence)."""
    rng = random.Random(case["layout"])
    n, g = case["batch"], min(case["groups"], case["batch"])
    group = [i if i < g else rng.randrange(g) for i in range(n)]
    rng.shuffle(group)
    pages = [max(1, int(case["shared"] * (1.0 if j == 0 else rng.uniform(0.3, 1.0))) // PAGE) for j in range(g)]
    prefix = [pages[group[b]] * PAGE + rng.randint(0, case["own_len"]) for b in range(n)]
    return group, pages, prefix


def _filled_slots(case):
    """Which window slots are filled, in logical order: the first is a mask, so that this step commits nothing."""
    rng = random.Random(case["layout"] + 1)
    p = [rng.uniform(0.1, 0.6) for _ in range(case["batch"])]
    return [[0] + [int(rng.random() < p[b]) for _ in range(case["window"] - 1)] for b in range(case["batch"])]


MASKS = ["empty", "narrow", "narrow", "some", "half", "wide", "wide"]      # what a grammar allows in a state
SHARE = {"empty": 0.0, "narrow": 64.0, "some": 0.01, "half": 0.3, "wide": 0.998}


def _mask_rows(case):
    """Row of the mask table for each slot, -1 where the slot is free."""
    rng = random.Random(case["layout"] + 2)
    return [[rng.randrange(len(MASKS)) if rng.random() < case["masked"] else -1 for _ in range(case["window"])] for _ in range(case["batch"])]


def _share(kind, vocab):
    s = SHARE[kind]
    return min(0.5, s / vocab) if kind == "narrow" else s


def _words(vocab):
    return -(-vocab // 128) * 4


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _pack_bits(on):
    """bool [..., words * 32] -> i32 words, token v in bit v % 32 of word v / 32."""
    w = on.reshape(*on.shape[:-1], -1, 32).to(torch.int64) << torch.arange(32, device=on.device)
    w = w.sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _unpack_bits(words, vocab):
    on = (words[..., None] >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return on.reshape(*words.shape[:-1], -1)[..., :vocab].bool()


def _tokens(shape, vocab, g):
    """Token ids as text has them: a few frequent ones, a long tail."""
    return (torch.rand(shape, generator=g, device="cuda", dtype=torch.float64) ** 3 * vocab).long().clamp_(max=vocab - 1)


def _stable_order(filled):
    """Physical order of the slots: filled ones first, masks last."""
    return torch.sort(1 - filled.int(), dim=1, stable=True).indices.int()


def prepare(case, seed):
    g = _gen(seed)
    s = _prepare_attention(case, g) if case["op"] == "attention" else _prepare_tokens(case, g)
    s["case"] = case
    if own:
        _make_handles(case, s)
    return s


def _prepare_attention(case, g):
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    group, pages, prefix = _attention_layout(case)
    n, w, hq, hkv, d = case["batch"], case["window"], case["hq"], case["hkv"], case["d"]
    max_pages = -(-(max(prefix) + w) // PAGE)
    first, at = [], 0
    for p in pages:
        first.append(at)
        at += p
    table = torch.zeros(n, max_pages, dtype=torch.int64)
    for b in range(n):
        p, need = pages[group[b]], -(-(prefix[b] + w) // PAGE)
        table[b, :p] = torch.arange(p) + first[group[b]]
        table[b, p:need] = torch.arange(need - p) + at
        at += need - p
    pool = torch.randperm(at + 3, generator=g, device="cuda")
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    s = {
        "group": torch.tensor(group, dtype=torch.int32, device="cuda"),
        "block_table": pool[table.cuda()].int(),
        "prefix_len": torch.tensor(prefix, dtype=torch.int32, device="cuda"),
        "q": normal(n, w, hq, d), "k": normal(n, w, hkv, d), "v": normal(n, w, hkv, d),
        "k_cache": normal(at + 3, hkv, PAGE, d), "v_cache": normal(at + 3, hkv, PAGE, d),
    }
    order = _stable_order(torch.rand(n, w, generator=g, device="cuda") < 0.35)
    s["pos_ids"] = (s["prefix_len"][:, None] + order).int()
    return s


def _prepare_tokens(case, g):
    n, vocab = case["batch"], case["vocab"]
    s = {"token_bits": torch.zeros(n, _words(vocab), dtype=torch.int32, device="cuda"),
         "token_record": torch.zeros(n, vocab, 2, dtype=torch.int32, device="cuda")}
    rng = random.Random(case["layout"])
    if case["op"] == "history":
        s["tokens"] = _tokens((n, case["length"]), vocab, g).int()
        s["count"] = torch.tensor([rng.randint((case["length"] + 1) // 2 if case["prompt"] else 0, case["length"]) for _ in range(n)],
                                  dtype=torch.int32, device="cuda")
        return s
    w, length = case["window"], case["history"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    # histories: the first half of each is the prompt; a few tokens carry a bias
    toks = _tokens((n, length), vocab, g)
    lens = torch.tensor([rng.randint((length + 1) // 2, length) for _ in range(n)], device="cuda")
    col = torch.arange(length, device="cuda")
    out = ((col >= length // 2) & (col < lens[:, None])).int() * 2
    rec = s["token_record"][..., 0]
    rec.scatter_add_(1, toks, out)
    seen = torch.zeros(n, vocab, dtype=torch.int32, device="cuda")
    seen.scatter_add_(1, toks, (col < min(length // 2, length)).int().expand(n, -1).contiguous())
    rec += (seen > 0).int()
    ids = torch.randint(0, vocab, (n, 16), generator=g, device="cuda")
    bias = torch.randn(n, 16, generator=g, device="cuda") * 2
    s["token_record"].view(torch.float32)[..., 1].scatter_(1, ids, bias)
    on = torch.zeros(n, _words(vocab) * 32, dtype=torch.bool, device="cuda")
    on[:, :vocab] = rec != 0
    on.scatter_(1, ids, True)
    s["token_bits"].copy_(_pack_bits(on))
    even = torch.rand(n, 3, generator=g, device="cuda")
    even[::5] = 0
    s["repetition"], s["presence"], s["frequency"] = (1 + 0.3 * even[:, 0]).contiguous(), (0.5 * even[:, 1]).contiguous(), (0.3 * even[:, 2]).contiguous()
    share = torch.tensor([_share(k, vocab) for k in MASKS], device="cuda")
    on = torch.zeros(len(MASKS), _words(vocab) * 32, dtype=torch.bool, device="cuda")
    on[:, :vocab] = torch.rand(len(MASKS), vocab, generator=g, device="cuda") < share[:, None]
    s["allowed"] = _pack_bits(on)
    s["mask_index"] = torch.tensor(_mask_rows(case), dtype=torch.int32, device="cuda")
    # logits: noise, and a clear favourite in half of the rows
    logits = torch.empty(n, w, vocab, dtype=dt, device="cuda")
    for b in range(n):
        logits[b] = torch.randn(w, vocab, generator=g, device="cuda") * 2
    top = torch.randint(0, vocab, (n, w, 1), generator=g, device="cuda")
    lift = (torch.rand(n, w, 1, generator=g, device="cuda") < 0.5).float() * 19
    logits.scatter_(2, top, (logits.gather(2, top).float() + lift).to(dt))
    s["logits"] = logits
    filled = torch.tensor(_filled_slots(case), dtype=torch.uint8, device="cuda")
    s["filled"], s["perm"] = filled, _stable_order(filled).contiguous()
    s["n_filled"] = filled.sum(1).int()
    if case["op"] == "adjust":
        s["out"] = torch.zeros_like(logits)
        return s
    s["n_commit"] = torch.zeros(n, dtype=torch.int32, device="cuda")
    s["window_tokens"] = torch.where(filled.bool(), _tokens((n, w), vocab, g), vocab - 1).int()
    s["prefix_len"] = torch.tensor([rng.randint(0, 8192) for _ in range(n)], dtype=torch.int32, device="cuda")
    return s


def _make_handles(case, s):
    """What a user's program keeps: the configuration, output buffers and the workspace."""
    import paper_2512_22737_b200 as wedlm
    n = case["batch"]
    if case["op"] == "attention":
        cfg = wedlm.make_config(batch=n, window=case["window"], n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["d"], page_size=PAGE,
                                max_pages_per_seq=s["block_table"].shape[1], num_pages=s["k_cache"].shape[0], dtype=case["dtype"],
                                rope_theta=QWEN["theta"], max_prefix_len=s["block_table"].shape[1] * PAGE - case["window"])
        s["out"], s["slots"] = torch.empty_like(s["q"]), torch.empty_like(s["pos_ids"])
        s["workspace"] = torch.empty(wedlm.wedlm_shared_prefix_attn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    else:
        cfg = wedlm.make_config(batch=n, window=case.get("window", 1), vocab=case["vocab"], dtype=case.get("dtype", "bf16"), tau=TAU, lam=LAM,
                                mask_token_id=case["vocab"] - 1)
        s["rules"] = wedlm.make_adjust(s["token_bits"], s["token_record"], s.get("repetition"), s.get("presence"), s.get("frequency"),
                                       s.get("allowed"), s.get("mask_index"))
    if case["op"] == "confidence":
        s["step"] = wedlm.DecodeStep(cfg)
        s["step"].perm, s["step"].n_filled, s["step"].n_commit = s["perm"], s["n_filled"], s["n_commit"]
    s["cfg"], s["lib"] = cfg, wedlm


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"attention": _run_attention, "confidence": _run_confidence, "adjust": _run_adjust, "history": _run_history}[s["case"]["op"]](s)


def _run_attention(s):
    if own:
        s["lib"].wedlm_shared_prefix_attn(s["cfg"], s["group"], s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"],
                                          s["prefix_len"], s["pos_ids"], s["out"], s["slots"], s["workspace"])
        return s["out"], s["k_cache"], s["v_cache"], s["slots"]
    n, w, hq, d = s["q"].shape
    hkv = s["k"].shape[2]
    dt = s["q"].dtype
    at = s["prefix_len"].long()[:, None] + torch.arange(w, device="cuda")
    page = s["block_table"].long().gather(1, at // PAGE)
    s["k_cache"][page, :, at % PAGE] = _rotate(s["k"], s["pos_ids"]).to(dt)
    s["v_cache"][page, :, at % PAGE] = s["v"]
    keys = s["k_cache"][s["block_table"].long()].transpose(2, 3).reshape(n, -1, hkv, d).float()
    q = _rotate(s["q"], s["pos_ids"]).view(n, w, hkv, hq // hkv, d)
    score = torch.einsum("nwhgd,nshd->nwhgs", q, keys) / math.sqrt(d)
    del keys
    visible = torch.arange(score.shape[-1], device="cuda") <= at[:, :, None]
    score = score.masked_fill(~visible[:, :, None, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    del score
    values = s["v_cache"][s["block_table"].long()].transpose(2, 3).reshape(n, -1, hkv, d).float()
    out = torch.einsum("nwhgs,nshd->nwhgd", p, values) / p.sum(-1, keepdim=True)
    return out.reshape(n, w, hq, d).to(dt), s["k_cache"], s["v_cache"], (page * PAGE + at % PAGE).int()


def _rotate(x, pos):
    """RoPE in the pairs (i, i + d/2), angles in 64 bits."""
    half = x.shape[-1] // 2
    freq = QWEN["theta"] ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    ang = pos.double()[..., None] * freq
    c, sn = torch.cos(ang).float()[..., None, :], torch.sin(ang).float()[..., None, :]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * sn, b * c + a * sn], -1)


def _adjusted(s, x):
    """Rules in their order: repetition, presence, frequency, bias, mask.  x: f32 [B, W, V]."""
    vocab = x.shape[-1]
    touched = _unpack_bits(s["token_bits"], vocab)[:, None]
    rec = s["token_record"][..., 0][:, None]
    count = (rec >> 1).float()
    rep = torch.where(touched & (rec > 0), s["repetition"][:, None, None], 1.0)
    y = torch.where(x > 0, x / rep, x * rep)
    y = torch.where(touched & (count > 0), y - s["presence"][:, None, None], y)
    y = torch.where(touched, y - s["frequency"][:, None, None] * count, y)
    y = torch.where(touched, y + s["token_record"].view(torch.float32)[..., 1][:, None], y)
    return y.masked_fill(~_allowed(s, vocab), -math.inf)


def _allowed(s, vocab):
    row = s["mask_index"].long().gather(1, s["perm"].long())
    return _unpack_bits(s["allowed"], vocab)[row.clamp(min=0)] | (row < 0)[..., None]


def _active(s):
    """Rows of the window that are masks, in physical order."""
    return torch.arange(s["perm"].shape[1], device="cuda") >= s["n_filled"][:, None]


def _run_adjust(s):
    if own:
        s["lib"].wedlm_logits_adjust(s["cfg"], s["rules"], s["logits"], s["out"], s["perm"], s["n_filled"])
        return s["out"]
    y = _adjusted(s, s["logits"].float()).to(s["logits"].dtype)
    s["out"] = torch.where(_active(s)[..., None], y, s["out"])
    return s["out"]


def _run_confidence(s):
    if own:
        st = s["step"]
        st.confidence_commit(s["logits"], s["window_tokens"], s["filled"], s["prefix_len"], adjust=s["rules"])
        return (st.argmax, st.maxprob, st.entropy, st.lse, st.committed_tokens, st.committed_count, st.filled_count, s["window_tokens"],
                s["filled"], s["prefix_len"], s["token_bits"], s["token_record"])
    x = _adjusted(s, s["logits"].float())
    n, w, vocab = x.shape
    top = x.amax(-1)
    some, live = top > -math.inf, _active(s)
    index = torch.arange(vocab, device="cuda", dtype=torch.int32)
    best = torch.where(x == top[..., None], index, vocab).amin(-1)
    x -= torch.where(some, top, 0)[..., None]
    e = torch.exp(x)
    mass = e.sum(-1, dtype=torch.float64)
    tilt = torch.where(e > 0, x * e, 0).sum(-1, dtype=torch.float64)
    entropy = torch.where(some, torch.log(mass) - tilt / mass, 0)
    maxprob = torch.where(some, 1 / mass, 0)
    lse = torch.where(some, top.double() + torch.log(mass), -math.inf)
    best = torch.where(some, best, -1)
    # selection: entropy with the distance to the leftmost mask, or the best row where none passes
    slot = s["perm"].long()
    far = slot - slot.gather(1, s["n_filled"].long()[:, None])
    score = torch.where(live & some, entropy + torch.tensor(LAM, dtype=torch.float32).double() * far, math.inf)
    take = score <= torch.tensor(TAU, dtype=torch.float32).double()
    least = score.amin(1, keepdim=True)
    first = torch.where((score == least) & (least < math.inf), torch.arange(w, device="cuda"), w).amin(1, keepdim=True)
    take = torch.where(take.any(1, keepdim=True), take, torch.arange(w, device="cuda") == first)
    by_slot = torch.zeros_like(take).scatter(1, slot, take)
    token = torch.zeros_like(best).scatter(1, slot, best)
    tokens = torch.where(by_slot, token, s["window_tokens"])
    filled = torch.where(by_slot, 1, s["filled"])
    # a filled token joins its sequence's history
    s["token_record"][..., 0].scatter_add_(1, best.clamp(min=0).long(), take.int() * 2)
    on = _unpack_bits(s["token_bits"], s["token_bits"].shape[1] * 32)
    on |= torch.zeros(on.shape, dtype=torch.int32, device="cuda").scatter_add_(1, best.clamp(min=0).long(), take.int()) > 0
    s["token_bits"].copy_(_pack_bits(on))
    # commit, shift, refill
    gone = s["n_commit"][:, None]
    at = torch.arange(w, device="cuda") + gone
    shifted = lambda v, empty: torch.where(at < w, v.gather(1, at.clamp(max=w - 1)), empty)  # noqa: E731
    committed = torch.where(torch.arange(w, device="cuda") < gone, tokens, -1)
    s["window_tokens"].copy_(shifted(tokens, vocab - 1))
    s["filled"].copy_(shifted(filled, 0))
    s["prefix_len"] += s["n_commit"]
    stat = lambda v: torch.where(live, v, math.nan).float()  # noqa: E731
    return (torch.where(live, best, -1), stat(maxprob), stat(entropy), stat(lse), committed, s["n_commit"].clone(), take.sum(1).int(),
            s["window_tokens"], s["filled"], s["prefix_len"], s["token_bits"], s["token_record"])


def _run_history(s):
    prompt = s["case"]["prompt"]
    if own:
        s["lib"].wedlm_history_add(s["cfg"], s["rules"], s["tokens"], s["count"], prompt)
        return s["token_bits"], s["token_record"]
    n, vocab = s["token_record"].shape[:2]
    live = (torch.arange(s["tokens"].shape[1], device="cuda") < s["count"][:, None]).int()
    new = torch.zeros(n, _words(vocab) * 32, dtype=torch.int32, device="cuda").scatter_add_(1, s["tokens"].long(), live)
    rec = s["token_record"][..., 0]
    if prompt:
        rec |= (new[:, :vocab] > 0).int()
    else:
        rec += 2 * new[:, :vocab]
    s["token_bits"] |= _pack_bits(new > 0)
    return s["token_bits"], s["token_record"]


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 2 if case.get("dtype", "bf16") == "bf16" else 4
    n = case["batch"]
    if case["op"] == "attention":
        group, pages, prefix = _attention_layout(case)
        w, hq, hkv, d = case["window"], case["hq"], case["hkv"], case["d"]
        keys = sum(pages[j] * PAGE for j in set(group)) + sum(p - pages[j] * PAGE for p, j in zip(prefix, group))
        rows = n * w
        pairs = sum(w * p + w * (w + 1) // 2 for p in prefix)
        return {"bytes": (keys * 2 * hkv + rows * 4 * hkv + rows * 2 * hq) * d * size, "flops": 4.0 * pairs * hq * d}
    if case["op"] == "history":
        rng = random.Random(case["layout"])
        total = sum(rng.randint((case["length"] + 1) // 2 if case["prompt"] else 0, case["length"]) for _ in range(n))
        return {"bytes": total * (4 + 8 + 8 + 8), "flops": 0}      # a token, its record and its word of bits read and written
    vocab = case["vocab"]
    filled, mask = _filled_slots(case), _mask_rows(case)
    full = sum(not f for row in filled for f in row)
    # slots of a row are in logical order on both sides; a masked row needs the logits that its mask allows
    part = sum((1.0 if m < 0 else _share(MASKS[m], vocab)) for fr, mr in zip(filled, mask) for f, m in zip(fr, mr) if not f)
    tables = n * (vocab / 8 + min(case["history"], vocab) * 8) + len(MASKS) * vocab / 8
    if case["op"] == "adjust":
        return {"bytes": (part + full) * vocab * size + tables, "flops": 4.0 * full * vocab}
    return {"bytes": part * vocab * size + tables + n * case["window"] * 32, "flops": 6.0 * part * vocab}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["op"] == "history":
        return None
    s = prepare(case, seed)
    return {"attention": _exact_attention, "confidence": _exact_confidence, "adjust": _exact_adjust}[case["op"]](case, s)


def _exact_attention(case, s):
    n, w, hq, hkv, d = case["batch"], case["window"], case["hq"], case["hkv"], case["d"]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    out = torch.empty(n, w, hq, d, dtype=torch.float64, device="cuda")
    turned = []
    for b in range(n):
        turn = torch.exp(1j * s["pos_ids"][b].double()[:, None] * torch.pow(torch.tensor(QWEN["theta"], dtype=torch.float64, device="cuda"), -2 * i / d))

        def rope(x):
            z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double()) * turn[:, None]
            return torch.cat([z.real, z.imag], -1)
        turned.append(rope(s["q"][b]))
        k = rope(s["k"][b]).to(s["k"].dtype).double()               # stored in the cache's type
        for j in range(w):
            t = int(s["prefix_len"][b]) + j
            p = int(s["block_table"][b, t // PAGE])
            kc[p, :, t % PAGE], vc[p, :, t % PAGE] = k[j], s["v"][b, j].double()
    for b in range(n):
        length = int(s["prefix_len"][b])
        pages = s["block_table"][b, : -(-(length + w) // PAGE)].long()
        k = kc[pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, : length + w]
        v = vc[pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, : length + w]
        for h in range(hkv):
            q = turned[b][:, h * hq // hkv: (h + 1) * hq // hkv]
            sc = q.reshape(-1, d) @ k[h].T / d ** 0.5
            sc = sc.view(w, -1, length + w)
            for j in range(w):
                sc[j, :, length + j + 1:] = -math.inf
            out[b, :, h * hq // hkv: (h + 1) * hq // hkv] = torch.softmax(sc, -1) @ v[h]
    return out, kc, vc, None


def _exact_rows(s, b):
    """Adjusted logits of one sequence's window in 64 bits."""
    vocab = s["logits"].shape[-1]
    x = s["logits"][b].double().clone()
    bit = torch.arange(vocab, device="cuda")
    touched = ((s["token_bits"][b].long() & 0xFFFFFFFF)[bit // 32] >> (bit % 32)) & 1
    rec, bias = s["token_record"][b, :, 0].long(), s["token_record"][b, :, 1].contiguous().view(torch.float32).double()
    ids = torch.nonzero(touched).flatten()
    r, a, f = (s[k][b].double() for k in ("repetition", "presence", "frequency"))
    z, c = x[:, ids], (rec[ids] // 2).double()
    seen = rec[ids] != 0
    z = torch.where(seen & (z > 0), z / r, torch.where(seen, z * r, z))
    x[:, ids] = z - a * (c > 0) - f * c + bias[ids]
    for i in range(x.shape[0]):
        m = int(s["mask_index"][b, int(s["perm"][b, i])])
        if m >= 0:
            ok = ((s["allowed"][m].long() & 0xFFFFFFFF)[bit // 32] >> (bit % 32)) & 1
            x[i, ok == 0] = -math.inf
    return x


def _exact_adjust(case, s):
    out = s["out"].double()
    for b in range(case["batch"]):
        first = int(s["n_filled"][b])
        out[b, first:] = _exact_rows(s, b)[first:]
    return out


def _exact_confidence(case, s):
    n, w = case["batch"], case["window"]
    stat = torch.full((3, n, w), math.nan, dtype=torch.float64, device="cuda")
    for b in range(n):
        first = int(s["n_filled"][b])
        x = _exact_rows(s, b)[first:]
        lse = torch.logsumexp(x, -1)
        p = torch.where(x > -math.inf, torch.exp(x - lse[:, None]), 0)
        some = lse > -math.inf
        stat[0, b, first:] = torch.where(some, p.amax(-1), 0)
        stat[1, b, first:] = torch.where(some, -torch.where(p > 0, p * (x - lse[:, None]), 0).sum(-1), 0)
        stat[2, b, first:] = lse
    return (None, stat[0], stat[1], stat[2]) + (None,) * 8
