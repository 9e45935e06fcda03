"""What the calls of the 8-bit cache and of the norms with rotation refuse on the host, before anything is launched (no device needed)."""
import ctypes

import pytest

import paper_2512_22737_b200 as w

OK, INVALID, UNSUPPORTED, SMALL = 0, -1, -2, -3
P = ctypes.c_void_p(1 << 20)               # an aligned address that is never read: every call below is refused first
ODD = ctypes.c_void_p((1 << 20) + 4)


def _cfg(**kw):
    return w.make_config(**{**dict(batch=2, window=4, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, max_pages_per_seq=8, num_pages=20,
                                   max_prefix_len=100), **kw})


def _norm_rope(cfg, rope, q=P, qs=1024, k=P, ks=256, pos=P, gq=P, gk=P, eps=1e-6, qo=P, ko=P):
    return w.load_library().wedlm_norm_rope(ctypes.byref(cfg), rope, q, qs, k, ks, pos, gq, gk, eps, qo, ko, None)


def test_norm_rope():
    cfg = _cfg()
    rope = w.make_rope(cfg)
    r = ctypes.byref(rope)
    assert _norm_rope(cfg, None) == INVALID
    assert _norm_rope(cfg, r, q=None) == INVALID                        # an output without its input
    assert _norm_rope(cfg, r, q=None, qo=None, k=None, ko=None) == INVALID
    assert _norm_rope(cfg, r, pos=None) == INVALID
    assert _norm_rope(cfg, r, qs=1020) == INVALID and _norm_rope(cfg, r, ks=252) == INVALID        # rows that overlap
    assert _norm_rope(cfg, r, qs=1028) == INVALID and _norm_rope(cfg, r, q=ODD) == INVALID         # off the 16-byte grid
    assert _norm_rope(cfg, r, gq=ODD) == INVALID and _norm_rope(cfg, r, ko=ODD) == INVALID
    assert _norm_rope(cfg, r, eps=-1.0) == INVALID and _norm_rope(cfg, r, eps=float("nan")) == INVALID
    assert _norm_rope(_cfg(head_dim=80), r) == UNSUPPORTED and _norm_rope(_cfg(rope_style=2), r) == INVALID
    rope.rotary_dim = 144
    assert _norm_rope(cfg, r) == INVALID
    rope.rotary_dim = 24
    assert _norm_rope(cfg, r) == UNSUPPORTED
    assert _norm_rope(_cfg(batch=0), ctypes.byref(w.make_rope(cfg))) == OK


def test_norm_rope_backward():
    cfg = _cfg()
    rope = w.make_rope(cfg)
    need = w.wedlm_norm_rope_backward_workspace_bytes(cfg)
    assert need > 0 and w.wedlm_norm_rope_backward_workspace_bytes(_cfg(head_dim=48)) == 0

    def call(q=P, k=P, gq=P, gk=P, dqo=P, dko=P, dq=P, dqs=1024, dk=P, dks=256, dgq=P, dgk=P, ws=P, n=need):
        return w.load_library().wedlm_norm_rope_backward(ctypes.byref(cfg), ctypes.byref(rope), q, 1024, k, 256, P, gq, gk, 1e-6, dqo, dko, dq, dqs, dk,
                                                         dks, dgq, dgk, ws, n, None)
    assert call(dq=None) == INVALID and call(dko=None) == INVALID and call(ws=None) == INVALID
    assert call(dqs=1000) == INVALID and call(dk=ODD) == INVALID
    assert call(gq=None) == INVALID                                     # a gradient of a gain that there is not
    assert call(n=need - 1) == SMALL


@pytest.mark.parametrize("rotary,kind,factor,length,fast,slow,rc", [
    (128, 0, 0.0, 0, 0.0, 0.0, OK), (8, 0, 1.0, 1, 32.0, 1.0, INVALID), (24, 0, 1.0, 1, 32.0, 1.0, UNSUPPORTED), (144, 0, 1.0, 1, 32.0, 1.0, INVALID),
    (64, 3, 1.0, 1, 32.0, 1.0, INVALID), (64, 1, 0.5, 1, 32.0, 1.0, INVALID), (64, 1, float("nan"), 1, 32.0, 1.0, INVALID),
    (64, 2, 4.0, 0, 32.0, 1.0, INVALID), (64, 2, 4.0, 100, 1.0, 1.0, INVALID), (64, 2, 4.0, 100, 2.0, -1.0, INVALID), (64, 2, 4.0, 100, 2.0, 1.0, OK),
])
def test_rope_tables(rotary, kind, factor, length, fast, slow, rc):
    rope = w.WedlmRope()
    assert w.load_library().wedlm_rope_init(ctypes.byref(_cfg()), rotary, kind, factor, length, fast, slow, ctypes.byref(rope)) == rc


def test_append():
    def call(cfg, k=P, ks=256, v=P, vs=256, kc=P, kscale=P, vc=P, vscale=P, table=P, prefix=P):
        return w.load_library().wedlm_kvq_append(ctypes.byref(cfg), k, ks, v, vs, kc, kscale, vc, vscale, table, prefix, None, None, None, None)
    cfg = _cfg()
    for name in ("k", "v", "kc", "kscale", "vc", "vscale", "table", "prefix"):
        assert call(cfg, **{name: None}) == INVALID, name
    assert call(cfg, ks=255) == INVALID and call(cfg, vs=260) == INVALID and call(cfg, v=ODD) == INVALID and call(cfg, kc=ODD) == INVALID
    assert call(_cfg(page_size=64)) == UNSUPPORTED and call(_cfg(head_dim=16)) == UNSUPPORTED and call(_cfg(max_prefix_len=125)) == INVALID
    assert call(_cfg(batch=0), k=None) == OK


def test_attention():
    def call(cfg, q=P, kc=P, out=P, ws=P, n=1 << 40):
        return w.load_library().wedlm_kvq_attn(ctypes.byref(cfg), q, kc, P, P, P, P, P, out, ws, n, None, None)
    cfg = _cfg()
    need = w.wedlm_kvq_attn_workspace_bytes(cfg)
    assert need > 0 and w.wedlm_kvq_attn_workspace_bytes(_cfg(n_q_heads=7)) == 0
    assert call(cfg, q=None) == INVALID and call(cfg, kc=None) == INVALID and call(cfg, ws=None) == INVALID and call(cfg, out=ODD) == INVALID
    assert call(cfg, n=need - 1) == SMALL and call(_cfg(dtype="f32"), n=16) == SMALL
    assert call(_cfg(head_dim=64, attn_impl="tensor")) == UNSUPPORTED
    assert call(_cfg(page_size=8, max_pages_per_seq=16, attn_impl="tensor")) == UNSUPPORTED
    assert call(_cfg(n_q_heads=129, n_kv_heads=1, attn_impl="tensor")) == UNSUPPORTED
    assert call(_cfg(batch=0), q=None) == OK
