"""The shared-prefix call where it goes sequence by sequence: page sizes other than 16, group sizes that do not divide 128, fp32,
other head sizes, with prefixes around the borders of its 32-key chunks; against the float64 oracle and the plain call."""
import numpy as np
import pytest

from test_gpu_shared_prefix import _check
from workloads import get_config, make_step

pytestmark = pytest.mark.gpu


def _inputs(prefix, group, shared, *, W, heads, D, dtype, page, seed):
    cfg = get_config("cfg2_qwen_b1").replace(batch=len(prefix), window=W, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, vocab=64,
                                             dtype=dtype, page_size=page, name="shared")
    inp = make_step(cfg, seed=seed, prefix_len=np.asarray(prefix), with_logits=False)
    assert inp["k_cache"].shape[2] == page
    first = {}
    for b, g in enumerate(group):
        a = first.setdefault(g, b)
        n = min(shared // page, prefix[a] // page, prefix[b] // page)
        inp["block_table"][b, :n] = inp["block_table"][a, :n]
    return cfg, inp


@pytest.mark.parametrize("W", [1, 6, 17])
@pytest.mark.parametrize("dtype,D,page,heads", [("f32", 64, 8, (4, 2)), ("f32", 64, 32, (4, 2)), ("f32", 128, 8, (4, 4)),
                                                ("bf16", 64, 32, (4, 2)), ("bf16", 128, 8, (8, 2)), ("bf16", 128, 32, (8, 2)),
                                                ("bf16", 32, 8, (4, 1)), ("bf16", 256, 32, (2, 1)), ("bf16", 128, 16, (12, 4))])
def test_pages_and_head_groups(W, dtype, D, page, heads):
    prefix = [200, 33, 31, 0, 64, 257, 32]
    group = [0, 0, 1, 2, 1, 0, 1]
    cfg, inp = _inputs(prefix, group, 192, W=W, heads=heads, D=D, dtype=dtype, page=page, seed=D + page + W)
    _check(cfg, inp, group)


@pytest.mark.parametrize("dtype,page", [("f32", 8), ("bf16", 32)])
def test_many_chunks(dtype, page):
    prefix = [3000, 2999]
    cfg, inp = _inputs(prefix, [0, 0], 2048, W=3, heads=(2, 1), D=128, dtype=dtype, page=page, seed=page)
    _check(cfg, inp, [0, 0])
