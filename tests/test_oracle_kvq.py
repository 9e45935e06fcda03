"""Pins of the oracle for norms with rotation and the 8-bit cache."""
import math

import numpy as np
import pytest
import torch

from oracle import kvq_oracle as kq


def test_codes_are_torchs():
    g = np.random.default_rng(1)
    x = np.concatenate([g.standard_normal(4000) * 2.0 ** g.integers(-14, 9, 4000), kq.VALUES[:126],
                        (kq.VALUES[:126] + kq.VALUES[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(kq.to_code(x), want.view(torch.uint8).numpy())
    ok = [c for c in range(256) if c & 127 != 127]
    assert np.array_equal(kq.VALUES[ok], torch.tensor(ok, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.1, 1), (224.0, -1), (0.0, -64), (1e-30, -64), (3.3e38, 120), (7.0, -6), (7.0000005, -5)])
def test_page_exponents(top, e):
    assert kq.page_exponent(np.array([0.0, -top, np.nan, np.inf])) == e


@pytest.mark.parametrize("style", [0, 1])
def test_gradients_are_the_differences(style):
    g = np.random.default_rng(2)
    x, dy, gain = g.standard_normal((2, 3, 32)), g.standard_normal((2, 3, 32)), 1 + 0.2 * g.standard_normal(32)
    pos = np.array([3, 70000])
    freq, factor = kq.rope_frequencies(1e4, 16, "yarn", 4.0, 64)
    f = lambda x, gain: float((kq.norm_rope(x, gain, 1e-3, pos, freq, factor, style) * dy).sum())  # noqa: E731
    dx, dgain = kq.norm_rope_backward(x, gain, 1e-3, pos, freq, factor, style, dy)
    h = 1e-5
    for idx in [(0, 0, 0), (1, 2, 31), (0, 1, 9), (1, 0, 16)]:
        d = np.zeros_like(x)
        d[idx] = h
        assert abs((f(x + d, gain) - f(x - d, gain)) / (2 * h) - dx[idx]) < 1e-8
    for i in (0, 15, 20):
        d = np.zeros_like(gain)
        d[i] = h
        assert abs((f(x, gain + d) - f(x, gain - d)) / (2 * h) - dgain[i]) < 1e-8


def test_yarn_keeps_fast_pairs_and_interpolates_slow_ones():
    plain, _ = kq.rope_frequencies(1e6, 128)
    scaled, factor = kq.rope_frequencies(1e6, 128, "yarn", 4.0, 32768)
    assert scaled[0] == plain[0] and abs(scaled[-1] * 4 - plain[-1]) < 1e-18
    assert abs(factor - (0.1 * math.log(4) + 1)) < 1e-15


def test_library_tables_are_the_oracles():
    import paper_2512_22737_b200 as w
    cfg = w.make_config(batch=1, window=1, head_dim=128, rope_theta=1.0e6)
    for kw in (dict(), dict(scaling="linear", factor=8.0), dict(scaling="yarn", factor=4.0, original_len=32768)):
        for rotary in (16, 64, 128):
            rope = w.make_rope(cfg, rotary_dim=rotary, **kw)
            freq, factor = kq.rope_frequencies(1.0e6, rotary, **kw)
            assert np.allclose(np.array(rope.inv_freq[: rotary // 2]), freq, rtol=1e-14, atol=0)
            assert not any(rope.inv_freq[rotary // 2:]) and abs(rope.attention_factor - factor) < 1e-7


def test_a_moved_scale_rounds_only_small_values():
    """Rows that are there already follow a scale that moves by whole powers of two."""
    g = np.random.default_rng(3)
    D, page = 32, 16
    codes = np.zeros((1, 1, page, D), dtype=np.uint8)
    scale = np.ones((1, 1))
    table = np.zeros((1, 1), dtype=np.int32)
    first = g.standard_normal((1, 4, 1, D))
    codes, scale, _ = kq.append(first, codes, scale, table, [0], None, page)
    before = kq.VALUES[codes[0, 0, :4]] * scale[0, 0]
    codes, scale, slots = kq.append(np.full((1, 1, 1, D), 900.0), codes, scale, table, [4], None, page)
    after = kq.VALUES[codes[0, 0, :4]] * scale[0, 0]
    assert scale[0, 0] == 4.0 and slots[0, 0] == 4
    big = np.abs(before) >= 2.0 ** -6 * scale[0, 0]
    assert np.array_equal(before[big], after[big]) and np.abs(before - after).max() <= 2.0 ** -10 * scale[0, 0]
