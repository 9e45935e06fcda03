"""Shared-prefix attention of shapes whose plan would pass 32-bit positions: computed sequence by sequence, as every shape that
the tensor-core kernel does not take."""
import ctypes

import numpy as np
import pytest
import torch

KW = dict(batch=4, window=8, n_q_heads=16, n_kv_heads=16, head_dim=128, num_pages=16)
PAGES = 1 << 26                                 # of a sequence's table: prefixes of up to 2^30 tokens, in 64-key tiles of 112 units


def _config(**kw):
    import paper_2512_22737_b200 as w
    kw = {**KW, "max_pages_per_seq": PAGES, "max_prefix_len": PAGES * 16 - 64, **kw}
    return w.make_config(**kw)


def test_the_size_query_and_the_call_agree():
    import paper_2512_22737_b200 as w
    lib = w.load_library()
    large = _config()
    need = w.wedlm_shared_prefix_attn_workspace_bytes(large)
    assert need == w.wedlm_shared_prefix_attn_workspace_bytes(_config(attn_impl="generic")) > 0
    args = [ctypes.c_void_p(4096)] * 12
    assert lib.wedlm_shared_prefix_attn(ctypes.byref(large), *args, need - 1, None, None) == -3       # too small, not unsupported
    # the tensor-core kernel by name is refused, as for its other shapes
    assert lib.wedlm_shared_prefix_attn(ctypes.byref(_config(attn_impl="tensor")), *args, 1 << 40, None, None) == -2
    # a table of an ordinary length goes to the tensor-core kernel
    usual = dict(max_pages_per_seq=8, max_prefix_len=100)
    assert w.wedlm_shared_prefix_attn_workspace_bytes(_config(**usual)) != w.wedlm_shared_prefix_attn_workspace_bytes(
        _config(**usual, attn_impl="generic"))


@pytest.mark.gpu
def test_large_bounds_are_computed():
    """The bound is 2^30 tokens, the prefixes themselves are short: the result is that of a table of an ordinary length."""
    import paper_2512_22737_b200 as w
    g = torch.Generator().manual_seed(3)
    B, W, H, D = KW["batch"], KW["window"], KW["n_kv_heads"], KW["head_dim"]
    bf16 = lambda *s: torch.randn(s, generator=g).cuda().to(torch.bfloat16)  # noqa: E731
    q, k, v = bf16(B, W, H, D), bf16(B, W, H, D), bf16(B, W, H, D)
    caches = bf16(16, H, 16, D), bf16(16, H, 16, D)
    table = torch.tensor([[0, 1, 2, 3], [0, 1, 4, 5], [6, 7, 8, 9], [10, 11, 12, 13]], dtype=torch.int32, device="cuda")
    prefix = torch.tensor([40, 33, 0, 55], dtype=torch.int32, device="cuda")
    pos = prefix[:, None] + torch.arange(W, dtype=torch.int32, device="cuda")
    group = torch.tensor([0, 0, 1, 1], dtype=torch.int32, device="cuda")
    outs = []
    for pages in (4, PAGES):
        c = _config(max_pages_per_seq=pages, max_prefix_len=pages * 16 - (8 if pages == 4 else 64), attn_impl="generic" if pages == 4 else "auto")
        wide = torch.zeros(B, pages, dtype=torch.int32, device="cuda")
        wide[:, :4] = table
        kc, vc = caches[0].clone(), caches[1].clone()
        out, slots = torch.full_like(q, 5.0), torch.full((B, W), -1, dtype=torch.int32, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(w.wedlm_shared_prefix_attn_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        w.wedlm_shared_prefix_attn(c, group, q, k, v, kc, vc, wide, prefix, pos, out, slots, ws, st)
        assert int(st.item()) == 0
        outs.append((out.float(), slots, kc, vc))
    for x, y in zip(outs[0][1:], outs[1][1:]):
        assert torch.equal(x, y)
    # the two differ in how the keys are cut, fp32 sums of at most 64 terms, and in one rounding to bf16 of values below 8
    assert np.isfinite(outs[1][0].cpu().numpy()).all()
    assert (outs[0][0] - outs[1][0]).abs().max() <= 2 * 8 * 2.0 ** -8
