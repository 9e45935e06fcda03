"""Norms of queries and keys with the rotation, and their gradients, against the fp64 oracle.

Tolerances.  A turned pair (a, c) is off by at most 2^-19 of its length: 16 squares a lane and 5 more additions of the mean (half of
21 * 2^-24 on the root), 2^-22 of rsqrt, three products (3 * 2^-24), the angle rounded to fp32 after its reduction (pi * 2^-24),
2^-23 of sin and cos; together below 1.9e-6.  Results are then rounded once, by half a step at most."""
import numpy as np
import pytest
import torch

from oracle import kvq_oracle as kq

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
NEAR = 2.0 ** -19


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _f64(t):
    return t.detach().double().cpu().numpy()


def _length(y, rotary, style):
    """Length of the pair that each element belongs to; its own size behind the rotated ones."""
    z = np.abs(y).copy()
    a, c = kq._members(rotary, style)
    z[..., a] = z[..., c] = np.hypot(y[..., a], y[..., c])
    return z


def _case(dtype, B, W, Hq, Hkv, D, rotary, style, kw, seed, far=200000, fused=True):
    import paper_2512_22737_b200 as w
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dt(dtype)
    cfg = w.make_config(batch=B, window=W, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, dtype=dtype, rope_style=style, rope_theta=1.0e4)
    rope = w.make_rope(cfg, rotary_dim=rotary, **kw)
    x = (torch.randn(B, W, (Hq + 2 * Hkv) * D, generator=g, device="cuda") * 3).to(dt)
    q = x[..., : Hq * D].unflatten(-1, (Hq, D))
    k = x[..., Hq * D: (Hq + Hkv) * D].unflatten(-1, (Hkv, D))
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    pos = torch.randint(0, far, (B, W), generator=g, device="cuda", dtype=torch.int32)
    gq = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt)
    gk = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt)
    freq, factor = kq.rope_frequencies(1.0e4, rotary, **kw)
    return w, cfg, rope, q, k, pos, gq, gk, freq, float(np.float32(factor)), g


SHAPES = [
    ("bf16", 1, 1, 32, 8, 128, 128, 0, {}),
    ("bf16", 3, 37, 32, 8, 128, 64, 0, dict(scaling="yarn", factor=4.0, original_len=4096)),
    ("bf16", 2, 700, 4, 1, 128, 128, 1, dict(scaling="linear", factor=8.0)),
    ("bf16", 5, 7, 3, 1, 64, 16, 1, {}),
    ("bf16", 2, 9, 5, 5, 256, 240, 0, {}),
    ("bf16", 4, 3, 2, 1, 32, 32, 0, {}),
    ("f32", 1, 1, 4, 2, 64, 64, 0, {}),
    ("f32", 2, 33, 4, 2, 32, 16, 1, dict(scaling="yarn", factor=2.0, original_len=100)),
    ("f32", 3, 500, 2, 2, 128, 48, 0, {}),
    ("f32", 2, 5, 3, 1, 256, 256, 1, {}),
]


@pytest.mark.parametrize("dtype,B,W,Hq,Hkv,D,rotary,style,kw", SHAPES)
@pytest.mark.parametrize("norm", [True, False])
def test_forward(dtype, B, W, Hq, Hkv, D, rotary, style, kw, norm):
    w, cfg, rope, q, k, pos, gq, gk, freq, factor, _ = _case(dtype, B, W, Hq, Hkv, D, rotary, style, kw, seed=D + W)
    qo, ko = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
    w.wedlm_norm_rope(cfg, rope, q, k, pos, gq if norm else None, gk if norm else None, 1e-5, qo, ko)
    for x, gain, got in ((q, gq, qo), (k, gk, ko)):
        ref = kq.norm_rope(_f64(x), _f64(gain) if norm else None, float(np.float32(1e-5)), pos.cpu().numpy(), freq, factor, style)
        assert (np.abs(_f64(got) - ref) <= NEAR * _length(ref, rotary, style) + HALF[dtype] * np.abs(ref)).all()


@pytest.mark.parametrize("dtype,B,W,Hq,Hkv,D,rotary,style,kw", SHAPES)
def test_backward(dtype, B, W, Hq, Hkv, D, rotary, style, kw):
    w, cfg, rope, q, k, pos, gq, gk, freq, factor, g = _case(dtype, B, W, Hq, Hkv, D, rotary, style, kw, seed=D + W)
    dt = _dt(dtype)
    dqo = torch.randn(B, W, Hq, D, generator=g, device="cuda").to(dt)
    dko = torch.randn(B, W, Hkv, D, generator=g, device="cuda").to(dt)
    fused = torch.full((B, W, (Hq + 2 * Hkv) * D), 7.0, dtype=dt, device="cuda")
    dq, dk = fused[..., : Hq * D].unflatten(-1, (Hq, D)), fused[..., Hq * D: (Hq + Hkv) * D].unflatten(-1, (Hkv, D))
    dgq, dgk = torch.full((D,), 5.0, device="cuda"), torch.full((D,), 5.0, device="cuda")
    ws = torch.empty(w.wedlm_norm_rope_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    w.wedlm_norm_rope_backward(cfg, rope, q, k, pos, gq, gk, 1e-5, dqo, dko, dq, dk, dgq, dgk, ws)
    assert (fused[..., (Hq + Hkv) * D:] == 7).all()                                  # the slice of v is not touched
    eps = float(np.float32(1e-5))
    for x, gain, dy, got, dgain in ((q, gq, dqo, dq, dgq), (k, gk, dko, dk, dgk)):
        x, gain, dy = _f64(x), _f64(gain), _f64(dy)
        ref, ref_gain = kq.norm_rope_backward(x, gain, eps, pos.cpu().numpy(), freq, factor, style, dy)
        # sizes of the two terms of dx, whose difference may be far smaller
        root = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        dn = _length(dy, rotary, style) * factor
        term = dn * np.abs(gain) / root + np.abs(x) / root ** 2 * (dn * np.abs(gain * x) / root).mean(-1, keepdims=True)
        assert (np.abs(_f64(got) - ref) <= 2 * NEAR * term + HALF[dtype] * np.abs(ref)).all()
        # sums: below 2^7 additions in a row in each thread, block and over the blocks at these sizes
        rows = (dn * np.abs(x) / root).reshape(-1, D).sum(0)
        assert (np.abs(_f64(dgain) - ref_gain) <= 2.0 ** -17 * rows).all()
    first = (dq.clone(), dgq.clone(), dgk.clone())
    w.wedlm_norm_rope_backward(cfg, rope, q, k, pos, gq, gk, 1e-5, dqo, dko, dq, dk, dgq, dgk, ws)
    assert torch.equal(first[0], dq) and torch.equal(first[1], dgq) and torch.equal(first[2], dgk)


def test_only_one_of_the_two_and_in_place():
    w, cfg, rope, q, k, pos, gq, gk, freq, factor, _ = _case("bf16", 2, 5, 8, 2, 128, 128, 0, {}, seed=9, fused=False)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    w.wedlm_norm_rope(cfg, rope, q, k, pos, gq, gk, 1e-6, qo, ko)
    only = torch.empty_like(k)
    w.wedlm_norm_rope(cfg, rope, None, k, pos, None, gk, 1e-6, None, only)
    assert torch.equal(only, ko)
    w.wedlm_norm_rope(cfg, rope, q, k, pos, gq, gk, 1e-6, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    dq, dgq = torch.empty_like(q), torch.empty(128, device="cuda")
    ws = torch.empty(w.wedlm_norm_rope_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    w.wedlm_norm_rope_backward(cfg, rope, q, None, pos, gq, None, 1e-6, qo, None, dq, None, dgq, None, ws)
    ref, ref_gain = kq.norm_rope_backward(_f64(q), _f64(gq), 1e-6, pos.cpu().numpy(), freq, factor, 0, _f64(qo))
    assert np.abs(_f64(dq) - ref).max() < 0.05 * np.abs(ref).max() and np.abs(_f64(dgq) - ref_gain).max() < 1e-4 * np.abs(ref_gain).max()


def test_rows_of_zeros_and_of_huge_values():
    w, cfg, rope, q, k, pos, gq, gk, freq, factor, _ = _case("f32", 1, 4, 2, 1, 64, 64, 0, {}, seed=4, fused=False)
    q[0, 0] = 0
    q[0, 1] *= 1e15
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    w.wedlm_norm_rope(cfg, rope, q, k, pos, gq, gk, 1e-6, qo, ko)
    ref = kq.norm_rope(_f64(q), _f64(gq), 1e-6, pos.cpu().numpy(), freq, factor, 0)
    assert (qo[0, 0] == 0).all()
    assert (np.abs(_f64(qo) - ref) <= NEAR * _length(ref, 64, 0) + HALF["f32"] * np.abs(ref)).all()
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    ws = torch.empty(w.wedlm_norm_rope_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    w.wedlm_norm_rope_backward(cfg, rope, q, k, pos, gq, gk, 1e-6, qo, ko, dq, dk, None, None, ws)
    assert torch.isfinite(dq).all()


def test_a_captured_call_reads_new_positions():
    w, cfg, rope, q, k, pos, gq, gk, _, _, _ = _case("bf16", 2, 8, 8, 2, 128, 128, 0, {}, seed=5)
    qo, ko = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
    call = lambda: w.wedlm_norm_rope(cfg, rope, q, k, pos, gq, gk, 1e-6, qo, ko)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    pos += 17
    graph.replay()
    torch.cuda.synchronize()
    got = qo.clone()
    call()
    assert torch.equal(got, qo)


def test_refusals():
    w, cfg, rope, q, k, pos, gq, gk, _, _, _ = _case("bf16", 2, 4, 4, 2, 64, 64, 0, {}, seed=6)
    qo, ko = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
    with pytest.raises(ValueError, match="shape"):
        w.wedlm_norm_rope(cfg, rope, q[:, :2], k, pos, gq, gk, 1e-6, qo, ko)
    with pytest.raises(TypeError, match="dtype"):
        w.wedlm_norm_rope(cfg, rope, q.float(), k, pos, gq, gk, 1e-6, qo, ko)
    with pytest.raises(ValueError, match="strides"):
        w.wedlm_norm_rope(cfg, rope, q.transpose(0, 1).contiguous().transpose(0, 1), k, pos, gq, gk, 1e-6, qo, ko)
    with pytest.raises(w.WedlmError):
        w.wedlm_norm_rope(cfg, rope, q, k, pos, gq, gk, -1.0, qo, ko)
    with pytest.raises(w.WedlmError):
        w.wedlm_norm_rope(cfg, rope, None, None, pos, None, None, 1e-6, None, None)
    odd = torch.zeros(2, 4, 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[..., 4:].unflatten(-1, (4, 64))
    with pytest.raises(w.WedlmError):                                                 # rows off the 16-byte grid
        w.wedlm_norm_rope(cfg, rope, odd, k, pos, gq, gk, 1e-6, qo, ko)
    with pytest.raises(w.WedlmError):
        w.wedlm_norm_rope_backward(cfg, rope, q, k, pos, gq, gk, 1e-6, qo, ko, qo, ko, None, None, torch.empty(8, dtype=torch.uint8, device="cuda"))
