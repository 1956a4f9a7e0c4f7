"""Pins of oracle/new_tokens.py: closed forms and brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import new_tokens as o


def test_turn_keeps_norms_and_adds_angles():
    r = np.random.default_rng(0)
    x = r.standard_normal(128)
    for inter in (False, True):
        for rot in (128, 64, 16):
            f = o.rope_frequencies(rot, 10000.0)
            turn = lambda v, p: o.rope_turn(v, np.cos(p * f), np.sin(p * f), inter)  # noqa: E731
            y = turn(x, 37)
            assert math.isclose(np.linalg.norm(y), np.linalg.norm(x), rel_tol=1e-12)
            assert (y[rot:] == x[rot:]).all()
            np.testing.assert_allclose(turn(turn(x, 30), 7), y, atol=1e-12)
            # scores depend on the distance alone
            z = r.standard_normal(128)
            assert math.isclose(turn(x, 105) @ turn(z, 100), turn(x, 25) @ turn(z, 20), rel_tol=1e-9, abs_tol=1e-9)


def test_frequency_scaling():
    f = o.rope_frequencies(128, 500000.0)
    assert f[0] == 1.0 and math.isclose(f[63], 500000.0 ** (-126 / 128))
    np.testing.assert_allclose(o.rope_frequencies(128, 500000.0, factor=4.0), f / 4)
    g = o.rope_frequencies(128, 500000.0, factor=8.0, low_turns=1.0, high_turns=4.0, original_len=8192)
    turns = 8192 * f / (2 * math.pi)
    assert (g[turns >= 4] == f[turns >= 4]).all() and np.allclose(g[turns <= 1], f[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and ((g[mid] > f[mid] / 8) & (g[mid] < f[mid])).all()


def test_e4m3_is_torchs():
    codes = torch.arange(127, dtype=torch.uint8)
    assert (codes.view(torch.float8_e4m3fn).double().numpy() == o.e4m3_values()).all()
    r = np.random.default_rng(1)
    x = np.concatenate([r.uniform(-448, 448, 4000), r.uniform(-0.1, 0.1, 4000), (o.e4m3_values()[1:] + o.e4m3_values()[:-1]) / 2])
    x = x.astype(np.float32).astype(np.float64)
    assert (o.nearest_value(x, "e4m3") == torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()).all()


@pytest.mark.parametrize("fmt,most", [("e4m3", 448.0), ("int8", 127.0)])
def test_scale_is_the_smallest_power_of_two(fmt, most):
    r = np.random.default_rng(2)
    for top in [most, np.nextafter(most, 0), np.nextafter(most, 1e9), 1.0, 2.0, 3.3e-30, 1e30, 2.0 ** -133]:
        x = r.uniform(-1, 1, (16, 128)) * top
        x[3, 5] = -top
        v, s = o.quantise_block(x, fmt)
        assert s == 2.0 ** round(math.log2(s)) and top <= most * s and (top > most * s / 2 or s == 2.0 ** -126)
        assert np.abs(v).max() <= most
    assert o.quantise_block(np.zeros((16, 128)), fmt)[1] == 1.0
    assert math.isnan(o.quantise_block(np.full((16, 128), np.inf), fmt)[1])


def test_attention_oracles_agree():
    r = np.random.default_rng(3)
    K, V, q = r.standard_normal((50, 128)), r.standard_normal((50, 128)), o.f64_to_bf16_bits(r.standard_normal(128))
    a = o.attn8(q, K[:31], V[:31], 0.1)
    b = o.prompt_attn(o.bf16_bits_to_f64(q), K, V, 30, 0, 31, 0.1)
    np.testing.assert_allclose(a[0], b[0], rtol=1e-12)
    assert math.isclose(a[2], b[1]) and math.isclose(a[1].sum(), 1.0)
    # a large cap and no slope change nothing; an empty range gives zeros
    np.testing.assert_allclose(o.prompt_attn(o.bf16_bits_to_f64(q), K, V, 30, 0, 31, 0.1, cap=1e6)[0], b[0], rtol=1e-6)
    out, lse = o.prompt_attn(o.bf16_bits_to_f64(q), K, V, 30, 20, 20, 0.1)
    assert (out == 0).all() and lse == -math.inf
    # a steep slope leaves the own row
    np.testing.assert_allclose(o.prompt_attn(o.bf16_bits_to_f64(q), K, V, 30, 0, 31, 0.1, slope=1e3)[0], V[30], rtol=1e-9)
