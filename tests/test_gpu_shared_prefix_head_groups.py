"""Shared-prefix attention at the ends of the tensor-core kernel's range of query heads per KV head: a row tile then holds many
window slots, or only one."""
import pytest

from test_gpu_shared_prefix import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [1, 3, 9])
@pytest.mark.parametrize("heads", [(128, 1), (128, 2), (32, 1), (16, 1), (3, 3), (2, 1)])
def test_heads_per_kv_head(W, heads):
    prefix, group = [520, 530, 300, 517, 640], [0, 0, 1, 0, 0]
    cfg, inp = _inputs(prefix, group, {0: 32, 1: 0}, W=W, heads=heads, seed=W * 1000 + heads[0])
    _check(cfg, inp, group)
